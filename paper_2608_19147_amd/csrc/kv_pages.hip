// Host code of the paged cache: pools, sequences, the layout of a step and the forward over sequences.
#include "runtime.h"
#include "paged.h"

#include <numeric>

// A pool's sequences and steps, which go with it.
struct Member {
    Member *before = nullptr, *after = nullptr;
    virtual ~Member() {
        if (before) before->after = after;
        if (after) after->before = before;
    }
    void join(Member& head) {
        before = &head;
        after = head.after;
        if (after) after->before = this;
        head.after = this;
    }
};

struct KVPages {
    Stage* stage = nullptr;
    Member members;
    PagedPool p{};
    int page_rows = 0, n_axes = 1;
    uint8_t* axis = nullptr;                       // device [D / 2], or null
    std::vector<int> refs;                         // sequences that hold a page
    std::vector<uint64_t> open;                    // a bit for each free page
    size_t low = 0;                                // no word before it has one
    int n_free = 0;
    KVStep* fwd = nullptr;                         // of stage_forward_paged
    KVStep* spare = nullptr;                       // steps that were freed, for the next ones
    uint8_t* ws = nullptr;                         // and its workspace, grown on need
    size_t ws_cap = 0;

    int take() {                                   // the lowest free page; the caller has checked n_free
        while (!open[low]) ++low;
        const int b = __builtin_ctzll(open[low]), page = (int)(64 * low) + b;
        open[low] &= ~(1ull << b);
        --n_free;
        refs[page] = 1;
        return page;
    }
    void give(int page) {
        if (--refs[page]) return;
        open[page / 64] |= 1ull << (page % 64);
        low = std::min<size_t>(low, page / 64);
        ++n_free;
    }
    int slot(const std::vector<int>& pages, int row) const { return (pages[row >> p.shift] << p.shift) + (row & (page_rows - 1)); }
    int pages_for(int rows) const { return (int)(((unsigned)rows + page_rows - 1) >> p.shift); }
};

struct KVSeq : Member {
    KVPages* pool = nullptr;
    std::vector<int> pages;
    int length = 0;
    std::vector<KVStep*> steps;                    // whose plans have rows of it
    void lose(int len);                            // rows from len on, or their pages
    ~KVSeq() override { lose(-1); }
};

struct KVStep : Member {
    struct Rows { KVSeq* seq; int begin, end; };   // the new rows of one of its sequences
    KVPages* pool = nullptr;
    KVStep* next = nullptr;                        // of the pool's spare ones
    uint8_t* dev = nullptr;
    size_t cap = 0;
    uint8_t* host[2] = {nullptr, nullptr};         // pinned
    size_t host_cap[2] = {0, 0};
    hipEvent_t ev[2] = {nullptr, nullptr};         // its upload has been read
    bool used[2] = {false, false};
    int ring = 0;
    // the plan
    bool planned = false, captured = false, turned = false, merge = false;
    bool many = false;
    int M = 0, n_items = 0;
    size_t parts = 0;
    size_t o_items = 0, o_rows = 0, o_list = 0, o_tables = 0, o_slots = 0, o_pos = 0, o_masks = 0;
    std::vector<Rows> of;

    size_t part_bytes() const {
        const StageConfig& c = pool->stage->cfg;
        return merge ? parts * c.n_q_heads * (size_t)(c.head_dim * 4 + 8) : 0;
    }
    void leave() {                                 // its sequences forget it
        for (Rows& x : of) x.seq->steps.erase(std::remove(x.seq->steps.begin(), x.seq->steps.end(), this), x.seq->steps.end());
        of.clear();
    }
    bool shared() const {                          // whether a page of its new rows is some other sequence's too
        for (const Rows& x : of)
            for (int t = x.begin >> pool->p.shift; t <= (x.end - 1) >> pool->p.shift; ++t)
                if (pool->refs[x.seq->pages[t]] > 1) return true;
        return false;
    }
    ~KVStep() override {
        leave();
        for (int i = 0; i < 2; ++i) {
            if (host[i]) (void)hipHostFree(host[i]);
            if (ev[i]) (void)hipEventDestroy(ev[i]);
        }
        if (dev) (void)hipFree(dev);
    }
};

// A plan with one of the rows is none: its pages may soon be another sequence's.
void KVSeq::lose(int len) {
    for (size_t i = 0; i < steps.size();) {
        KVStep* step = steps[i];
        const auto x = std::find_if(step->of.begin(), step->of.end(), [&](const KVStep::Rows& y) { return y.seq == this; });
        if (x->end <= len) {
            ++i;
            continue;
        }
        step->planned = false;
        step->leave();                             // (takes it out of `steps`)
    }
}

namespace {

constexpr size_t MAX_MASK_WORDS = (size_t)1 << 31;
constexpr int MAX_POOL_ROWS = INT_MAX;

// Pages that a call has taken and references that it holds, given back unless it comes to its end.
struct Taken {
    KVPages* pool;
    std::vector<int> held;
    explicit Taken(KVPages* p) : pool(p) {}
    Taken(const Taken&) = delete;
    Taken& operator=(const Taken&) = delete;
    void reserve(size_t n) { held.reserve(held.size() + n); }
    int page() {                                   // room has been reserved: no exception between taking and noting
        held.push_back(pool->take());
        return held.back();
    }
    void share(int page) {
        held.push_back(page);
        ++pool->refs[page];
    }
    void keep() { held.clear(); }
    ~Taken() {
        for (int page : held) pool->give(page);
    }
};

// A call's place in the stage's order: the tensors' device, the previous call waited for, a capturing stream refused.
#define PAGED_BEGIN(st, s)              \
    DeviceGuard dev_((st)->device);     \
    HIP_TRY(dev_.err);                  \
    if (int rc_ = not_captured(s)) return rc_

// Metadata of a call to the device, as meta_upload sends it, but up to 64 KB by a kernel that reads the pinned copy: a copy
// command between two kernels takes some 15 us of the stream, such a kernel 4.
constexpr size_t SEND_BYTES = 64 << 10;
int send(Stage* st, const void* host, size_t bytes, hipStream_t s, const uint8_t** dev) {
    if (bytes > SEND_BYTES) return meta_upload(st, host, bytes, s, dev);
    if (int rc = ensure_meta(st, std::max<size_t>(bytes, 16))) return rc;
    const int slot = st->ring_i;
    st->ring_i = (st->ring_i + 1) % META_RING;
    if (st->meta_ev_used[slot]) HIP_TRY(hipEventSynchronize(st->meta_ev[slot]));
    std::memcpy(st->meta_host[slot], host, bytes);
    HIP_TRY(launch_paged_send(st->meta_host[slot], st->meta_dev, bytes, s, st->meta_ev[slot]));
    st->meta_ev_used[slot] = true;
    *dev = st->meta_dev;
    return STAGE_OK;
}

int no_room(const KVPages* pool, size_t need) {
    return fail(STAGE_E_CAPACITY, std::to_string(need) + " pages needed, " + std::to_string(pool->n_free) + " free");
}

// Whether two arrays of m rows (row and ld bytes) share memory; rows of one stride may lie between each other.
bool overlap(const void* a, int64_t row_a, int64_t ld_a, const void* b, int64_t row_b, int64_t ld_b, int m) {
    const int64_t d = (int64_t)((uintptr_t)b - (uintptr_t)a);
    if (d >= (m - 1) * ld_a + row_a || -d >= (m - 1) * ld_b + row_b) return false;
    if (m == 1 || ld_a != ld_b) return true;
    const int64_t at = ((d % ld_a) + ld_a) % ld_a;
    return at < row_a || at + row_b > ld_a;
}

// Whether n rows moved in every layer's pieces are one launch (paged.hip).
bool one_launch(const PagedPool& p, size_t n) { return (n + 63) / 64 * 2 * p.layers * p.Hkv < ((size_t)1 << 24) && n <= INT_MAX; }

// The bits of n bytes that are not zero.
void pack_bits(const uint8_t* m, int n, uint32_t* out) {
    for (int j = 0; j < n; j += 32) {
        uint32_t w = 0;
        if (j + 32 <= n) {
            for (int b = 0; b < 4; ++b) {
                uint64_t x;
                std::memcpy(&x, m + j + 8 * b, 8);
                x = ((((x & 0x7f7f7f7f7f7f7f7full) + 0x7f7f7f7f7f7f7f7full) | x) >> 7) & 0x0101010101010101ull;
                w |= (uint32_t)((x * 0x0102040810204080ull) >> 56) << (8 * b);
            }
        } else {
            for (int b = 0; j + b < n; ++b) w |= (m[j + b] ? 1u : 0u) << b;
        }
        out[j / 32] = w;
    }
}

// ---------------------------------------------------------------- the layout of a step

// A run of keys [k0, k1) and the rows of the step that see it.  A run that several sequences share comes before (is the
// parent of) theirs.
struct Run {
    int k0, k1, rows, n_rows, seq, parent;
    bool shared;
    int chunk = 0, splits = 1, slot = 0;
};

struct Layout {
    std::vector<PagedItem> items;
    std::vector<PagedRow> rows, list;
    std::vector<int> rowlist, tables, slots, pos;
    std::vector<uint32_t> masks;
    size_t parts = 0;
    bool merge = false, many = false;
};

// What a workgroup's start and end, and a partial result of a query vector, cost beside a step of 32 keys of a tile.
constexpr double START_STEPS = 6, PART_STEPS = 1.0 / 16;
constexpr int SPLIT_STEPS = 8;                     // fewest steps of a split
constexpr int SHARE_QUERIES = 128;                 // a sequence with more query vectors a kv head fills tiles alone

// The runs of a batch: sequences sorted by their whole pages, so that those that share pages are neighbours.  A common
// beginning becomes a run of them all where that saves more steps of tiles than its starts and partial results cost (12
// sequences of 5 rows that share 288 keys, and 2048 by fours: one run for the 288 38.9 us, none 35.6); what follows is laid
// out for each set with a common next page.  A sequence that fills tiles by itself keeps its keys in one run: shared rows
// save it no product, and partial results would be written and read for every one of its rows.
struct RunBuilder {
    const KVPages* pool;
    const std::vector<const std::vector<int>*>& pages;   // of each sequence
    const std::vector<int>&P, &n, &row0;
    std::vector<Run>& runs;
    std::vector<int>& rowlist;
    int gs;

    int whole(int s) const { return P[s] / pool->page_rows; }
    int add(const int* order, int cnt, int k0, int k1, int parent, bool shared) {
        Run r{k0, k1, (int)rowlist.size(), 0, order[0], parent, shared};
        for (int i = 0; i < cnt; ++i)
            for (int t = 0; t < n[order[i]]; ++t) rowlist.push_back(row0[order[i]] + t);
        r.n_rows = (int)rowlist.size() - r.rows;
        runs.push_back(r);
        return (int)runs.size() - 1;
    }
    void build(const int* order, int cnt, int from, int parent) {
        const int pr = pool->page_rows;
        for (;;) {
            if (cnt == 1) {
                add(order, 1, from * pr, P[order[0]] + n[order[0]], parent, false);
                return;
            }
            const std::vector<int>&a = *pages[order[0]], &b = *pages[order[cnt - 1]];
            const int lim = std::min(whole(order[0]), whole(order[cnt - 1]));
            int lcp = from;
            while (lcp < lim && a[lcp] == b[lcp]) ++lcp;
            // sets with the same page at lcp; a sequence that ends there is alone
            std::vector<int> ends;
            long rows = 0, set_rows = 0;
            double apart = 0;
            auto tiles = [&](long r) { return (r * gs + PAGED_MANY - 1) / PAGED_MANY; };
            // a tile's last queries take half a tile up to 64 of them (loads of rows bound a smaller one), so sets that fill
            // halves save no product (48 x 15 rows of 4 heads 73 us shared, 54 apart), and sets of 80 do (48 x 10 rows of 8 168
            // apart, 125 shared).  Two halves cost a little more than a whole: 48 x 8 rows of 8 behind 30000 to 60000 shared keys
            // are 6 to 10% slower apart, 12 x 8 rows behind 60000 11% faster.
            auto work = [&](long r) {
                const long q = r * gs, rest = q % PAGED_MANY;
                return q / PAGED_MANY + (rest == 0 ? 0.0 : rest <= 64 ? 0.5 : 1.0);
            };
            for (int j = 0; j < cnt; ++j) {
                rows += n[order[j]];
                set_rows += n[order[j]];
                const bool last = j + 1 == cnt || whole(order[j]) <= lcp || whole(order[j + 1]) <= lcp ||
                                  (*pages[order[j + 1]])[lcp] != (*pages[order[j]])[lcp];
                if (!last) continue;
                ends.push_back(j + 1);
                apart += work(set_rows);
                set_rows = 0;
            }
            const double steps = (lcp - from) * pr / 32.0;
            if (steps * (apart - work(rows)) > START_STEPS * tiles(rows) + PART_STEPS * rows * gs) {
                parent = add(order, cnt, from * pr, lcp * pr, parent, true);
                from = lcp;
            }
            // the last set goes on in this loop
            int i = 0;
            for (size_t e = 0; e + 1 < ends.size(); i = ends[e++]) build(order + i, ends[e] - i, from, parent);
            order += i;
            cnt -= i;
        }
    }
};

// Splits of the runs, their tiles as workgroups and each row's partial results.  A tile is up to 16 query vectors where no
// run has more (decoding rows), else up to 128; a split is a whole number of steps of 32 keys.  Splits are as long as leaves
// every place on the card a workgroup (four a CU; two of the larger tiles) and no more: what a split adds is a partial
// result of each of its query vectors, written and read.
void lay_out_items(const KVPages* pool, int n_cus, const std::vector<int>& table_off, std::vector<Run>& runs, Layout& L) {
    const StageConfig& c = pool->stage->cfg;
    const int gs = c.n_q_heads / c.n_kv_heads;
    auto steps = [](int k0, int k1) { return (k1 + 31) / 32 - k0 / 32; };
    for (const Run& r : runs) L.many = L.many || (long)r.n_rows * gs > PAGED_FEW;
    const int T = L.many ? PAGED_MANY : PAGED_FEW;
    const long places = (long)(L.many ? 2 : 4) * n_cus;
    auto tiles = [&](const Run& r) { return (r.n_rows * gs + T - 1) / T; };
    // the split after which the card should be done first: the places' share of all workgroups' steps, starts and partial
    // results, and the longest of them
    int longest = 0;
    for (const Run& r : runs) longest = std::max(longest, steps(r.k0, r.k1));
    int lo = longest;
    double best = 1e30;
    for (int C = std::min(SPLIT_STEPS, longest);; C = std::min(longest, C + std::max(1, C / 16))) {
        double all = 0;
        long wgs = 0;
        int most = 0;
        for (const Run& r : runs) {
            const int n = steps(r.k0, r.k1), S = (n + C - 1) / C, t = tiles(r), q = r.n_rows * gs;
            all += (double)t * (n + S * START_STEPS) + (S > 1 || r.parent >= 0 || r.shared ? (double)S * q * PART_STEPS : 0.0);
            most = std::max(most, (n + S - 1) / S);
            wgs += (long)t * S;
        }
        // (in more than one round the last ones leave places empty)
        const double time = std::max(all * c.n_kv_heads / places, (double)most + START_STEPS) + (wgs * c.n_kv_heads > places ? most * 0.5 : 0.0);
        if (time < best) {
            best = time;
            lo = C;
        }
        if (C == longest) break;
    }
    for (Run& r : runs) {
        const int n = steps(r.k0, r.k1), S = (n + lo - 1) / lo, st = (n + S - 1) / S;
        r.chunk = 32 * st;
        r.splits = (n + st - 1) / st;
        if (r.parent >= 0) r.slot = runs[r.parent].slot + runs[r.parent].splits;
    }
    std::vector<int> cost;
    for (const Run& r : runs) {
        const int a0 = r.k0 / 32 * 32;             // splits end at whole steps
        for (int q = 0; q < r.n_rows * gs; q += T) {
            const int nq = std::min(T, r.n_rows * gs - q);
            int low = INT_MAX, high = 0;
            bool masked = false;
            for (int i = q / gs; i <= (q + nq - 1) / gs; ++i) {
                const PagedRow& w = L.rows[L.rowlist[r.rows + i]];
                low = std::min(low, w.limit);
                high = std::max(high, w.limit);
                masked = masked || w.mask >= 0;
            }
            for (int j = 0; j < r.splits; ++j) {
                const int kb = std::max(r.k0, a0 + j * r.chunk), ke = std::min({r.k1, a0 + (j + 1) * r.chunk, high});
                if (ke <= kb) break;
                const bool two = r.shared || (long)r.n_rows * gs <= SHARE_QUERIES;   // of the row's own sequence: the same in all its runs
                L.items.push_back(PagedItem{r.rows, q, nq, kb, ke, table_off[r.seq], r.slot + j, (masked ? 2 : low >= ke) | (two ? 4 : 0)});
                cost.push_back(steps(kb, ke));
            }
        }
    }
    // the longest first
    std::vector<int> at(L.items.size());
    std::iota(at.begin(), at.end(), 0);
    std::stable_sort(at.begin(), at.end(), [&](int x, int y) { return cost[x] > cost[y]; });
    std::vector<PagedItem> sorted(L.items.size());
    for (size_t i = 0; i < at.size(); ++i) sorted[i] = L.items[at[i]];
    L.items.swap(sorted);
    // a row's partial results: its ancestors' splits, and those of its own run that begin before its limit
    for (const Run& r : runs) {
        if (r.shared) continue;                    // never a row's last
        const int a0 = r.k0 / 32 * 32;
        for (int i = 0; i < r.n_rows; ++i) {
            PagedRow& w = L.rows[L.rowlist[r.rows + i]];
            w.nparts = r.slot + (std::min(w.limit, r.k1) - a0 + r.chunk - 1) / r.chunk;
            if (w.nparts > 1) {
                w.part = (int)L.parts;
                L.parts += w.nparts;
                L.merge = true;
            }
        }
    }
    L.list.reserve(L.rowlist.size());
    for (int row : L.rowlist) L.list.push_back(L.rows[row]);
}

struct Planned {                                   // of one request
    KVSeq* seq;
    int P, n;
    bool copy_last;                                // its last page is shared and not full
    std::vector<int> pages;                        // as they will be
};

// Checks of a step's requests that need no memory; M.
int check_requests(const KVPages* pool, const KVStepRequest* reqs, int n_req, int max_rows, bool forward, int& M, size_t& mask_words) {
    const StageConfig& c = pool->stage->cfg;
    long total = 0;
    mask_words = 0;
    std::vector<const KVSeq*> seen;
    for (int r = 0; r < n_req; ++r) {
        const KVStepRequest& q = reqs[r];
        const std::string who = "request " + std::to_string(r) + ": ";
        if (!q.seq) return fail(STAGE_E_INVALID, who + "sequence is NULL");
        if (q.seq->pool != pool) return fail(STAGE_E_STATE_MISMATCH, who + "sequence belongs to another pool");
        if (q.n_tokens < 1) return fail(STAGE_E_INVALID, who + "n_tokens must be positive");
        if ((total += q.n_tokens) > max_rows) return fail(STAGE_E_CAPACITY, "more than " + std::to_string(max_rows) + " rows");
        if (q.seq->length > MAX_POOL_ROWS - q.n_tokens) return fail(STAGE_E_CAPACITY, who + "sequence too long");
        if (forward && !q.positions) return fail(STAGE_E_INVALID, who + "positions are required");
        if (!q.positions != !reqs[0].positions) return fail(STAGE_E_INVALID, who + "positions for some sequences only");
        if (q.positions)
            for (long i = 0; i < (long)pool->n_axes * q.n_tokens; ++i)
                if (q.positions[i] < 0 || q.positions[i] >= c.max_positions)
                    return fail(STAGE_E_CAPACITY, who + "position " + std::to_string(q.positions[i]) + " outside the rotary table");
        const size_t words = (size_t)(q.seq->length + q.n_tokens + 31) / 32;
        if (q.attention_mask_rows) mask_words += words * q.n_tokens;
        else if (q.attention_mask) mask_words += words;
        if (mask_words >= MAX_MASK_WORDS) return fail(STAGE_E_CAPACITY, "masks too large");
        if (forward && (q.attention_mask || q.attention_mask_rows)) {
            const int P = q.seq->length, n = q.n_tokens;
            for (int i = 0; i < n; ++i) {
                const uint8_t* rw = q.attention_mask_rows ? q.attention_mask_rows + (size_t)i * (P + n) : nullptr;
                bool any = false;
                for (int j = P + i; j >= 0 && !any; --j) any = (!rw || rw[j]) && (!q.attention_mask || q.attention_mask[j]);
                if (!any) return fail(STAGE_E_INVALID, who + "row " + std::to_string(i) + " sees no key");
            }
        }
        seen.push_back(q.seq);
    }
    std::sort(seen.begin(), seen.end());
    if (std::adjacent_find(seen.begin(), seen.end()) != seen.end()) return fail(STAGE_E_STATE_MISMATCH, "a sequence twice in one step");
    M = (int)total;
    return STAGE_OK;
}

// The bits of a request's masks: one row of words for all its new rows, or one each; none where nothing is hidden.
void lay_out_masks(const KVStepRequest& q, int P, int row0, Layout& L) {
    const int n = q.n_tokens, T = P + n, words = (T + 31) / 32;
    if (!q.attention_mask && !q.attention_mask_rows) return;
    std::vector<uint32_t> two;
    if (q.attention_mask) {
        two.resize(words);
        pack_bits(q.attention_mask, T, two.data());
    }
    auto open = [&](const uint32_t* w) {
        for (int i = 0; i < T / 32; ++i)
            if (w[i] != ~0u) return false;
        return T % 32 == 0 || (w[T / 32] | (~0u << (T % 32))) == ~0u;
    };
    if (!q.attention_mask_rows) {
        if (open(two.data())) return;
        for (int i = 0; i < n; ++i) L.rows[row0 + i].mask = (int)L.masks.size();
        L.masks.insert(L.masks.end(), two.begin(), two.end());
        return;
    }
    std::vector<uint32_t> w(words);
    for (int i = 0; i < n; ++i) {
        pack_bits(q.attention_mask_rows + (size_t)i * T, T, w.data());
        if (q.attention_mask)
            for (int j = 0; j < words; ++j) w[j] &= two[j];
        if (open(w.data())) continue;
        L.rows[row0 + i].mask = (int)L.masks.size();
        L.masks.insert(L.masks.end(), w.begin(), w.end());
    }
}

template <class T>
size_t place(size_t& at, const std::vector<T>& v) {
    const size_t o = at;
    at = (at + v.size() * sizeof(T) + 255) / 256 * 256;
    return o;
}

// Room on the device and a pinned copy (the other one of two may still be read) for a plan of `bytes`.
int step_room(KVStep* step, size_t bytes) {
    if (bytes > step->cap) {
        size_t cap = std::max<size_t>(2 * step->cap, std::max<size_t>(bytes, 1 << 14));
        step->planned = false;
        if (int rc = grow(&step->dev, &step->cap, cap)) return rc;
    }
    const int i = step->ring;
    if (step->used[i]) HIP_TRY(hipEventSynchronize(step->ev[i]));
    if (!step->ev[i]) HIP_TRY(hipEventCreateWithFlags(&step->ev[i], hipEventDisableTiming));
    if (bytes > step->host_cap[i]) {
        if (step->host[i]) HIP_TRY(hipHostFree(step->host[i]));
        step->host[i] = nullptr;
        step->host_cap[i] = 0;
        if (hipHostMalloc(&step->host[i], step->cap, hipHostMallocDefault) != hipSuccess) {
            (void)hipGetLastError();
            step->host[i] = nullptr;
            return fail(STAGE_E_OOM, "pinned metadata allocation failed");
        }
        step->host_cap[i] = step->cap;
    }
    return STAGE_OK;
}

// Plans the step on stream s, which order_on has ordered.
int plan(KVStep* step, const KVStepRequest* reqs, int n_req, int M, size_t mask_words, hipStream_t s) {
    KVPages* pool = step->pool;
    Stage* st = pool->stage;
    const StageConfig& c = st->cfg;
    const int pr = pool->page_rows;
    size_t need = 0, moves_n = 0, table_n = 0;
    std::vector<Planned> ps((size_t)n_req);
    for (int r = 0; r < n_req; ++r) {
        Planned& p = ps[r];
        p.seq = reqs[r].seq;
        p.P = p.seq->length;
        p.n = reqs[r].n_tokens;
        p.copy_last = p.P % pr && pool->refs[p.seq->pages.back()] > 1;
        p.pages = p.seq->pages;
        p.pages.reserve(pool->pages_for(p.P + p.n));
        need += pool->pages_for(p.P + p.n) - p.pages.size() + p.copy_last;
        if (p.copy_last) moves_n += p.P % pr;
        table_n += pool->pages_for(p.P + p.n);
    }
    if (need > (size_t)pool->n_free) return no_room(pool, need);
    if (table_n > INT_MAX || !one_launch(pool->p, moves_n)) return fail(STAGE_E_CAPACITY, "too many pages in one step");
    Taken taken(pool);
    taken.reserve(need);
    std::vector<int2> moves;
    moves.reserve(moves_n);
    for (Planned& p : ps) {
        if (p.copy_last) {
            const int page = taken.page(), old = p.pages.back();
            for (int i = 0; i < p.P % pr; ++i) moves.push_back(int2{(old << pool->p.shift) + i, (page << pool->p.shift) + i});
            p.pages.back() = page;
        }
        while ((int)p.pages.size() < pool->pages_for(p.P + p.n)) p.pages.push_back(taken.page());
    }

    Layout L;
    L.rows.resize(M);
    L.masks.reserve(mask_words);
    L.tables.reserve(table_n);
    L.slots.reserve(M);
    std::vector<int> P, n, row0, table_off, order((size_t)n_req);
    std::vector<const std::vector<int>*> pages;
    int row = 0;
    for (int r = 0; r < n_req; ++r) {
        const Planned& p = ps[r];
        P.push_back(p.P);
        n.push_back(p.n);
        row0.push_back(row);
        pages.push_back(&p.pages);
        table_off.push_back((int)L.tables.size());
        L.tables.insert(L.tables.end(), p.pages.begin(), p.pages.end());
        for (int i = 0; i < p.n; ++i) {
            L.rows[row + i] = PagedRow{row + i, p.P + i + 1, -1, 0, 1, {}};
            L.slots.push_back(pool->slot(p.pages, p.P + i));
        }
        lay_out_masks(reqs[r], p.P, row, L);
        row += p.n;
    }
    const bool turned = reqs[0].positions != nullptr;
    if (turned)
        for (int a = 0; a < pool->n_axes; ++a)
            for (int r = 0; r < n_req; ++r)
                L.pos.insert(L.pos.end(), reqs[r].positions + (size_t)a * n[r], reqs[r].positions + (size_t)(a + 1) * n[r]);
    std::vector<Run> runs;
    const int gs = c.n_q_heads / c.n_kv_heads;
    RunBuilder rb{pool, pages, P, n, row0, runs, L.rowlist, gs};
    std::iota(order.begin(), order.end(), 0);
    auto alone = std::stable_partition(order.begin(), order.end(), [&](int x) { return (long)n[x] * gs <= SHARE_QUERIES; });
    std::sort(order.begin(), alone, [&](int x, int y) {
        return std::lexicographical_compare(pages[x]->begin(), pages[x]->begin() + rb.whole(x), pages[y]->begin(), pages[y]->begin() + rb.whole(y));
    });
    if (alone != order.begin()) rb.build(order.data(), (int)(alone - order.begin()), 0, -1);
    for (auto i = alone; i != order.end(); ++i) rb.build(&*i, 1, 0, -1);
    lay_out_items(pool, st->n_cus, table_off, runs, L);
    if (L.items.size() * (size_t)c.n_kv_heads >= (1u << 24) || (size_t)M * c.n_q_heads >= (1u << 24) || L.parts > INT_MAX)
        return fail(STAGE_E_CAPACITY, "too many rows in one step");

    size_t bytes = 0;
    const size_t o_items = place(bytes, L.items), o_rows = place(bytes, L.rows), o_list = place(bytes, L.list),
                 o_tables = place(bytes, L.tables), o_slots = place(bytes, L.slots), o_pos = place(bytes, L.pos),
                 o_masks = place(bytes, L.masks), o_moves = place(bytes, moves);
    if (int rc = step_room(step, bytes)) return rc;
    uint8_t* hb = step->host[step->ring];
    auto put = [&](size_t o, const void* p, size_t b) {
        if (b) std::memcpy(hb + o, p, b);
    };
    put(o_items, L.items.data(), L.items.size() * sizeof(PagedItem));
    put(o_rows, L.rows.data(), L.rows.size() * sizeof(PagedRow));
    put(o_list, L.list.data(), L.list.size() * sizeof(PagedRow));
    put(o_tables, L.tables.data(), L.tables.size() * 4);
    put(o_slots, L.slots.data(), L.slots.size() * 4);
    put(o_pos, L.pos.data(), L.pos.size() * 4);
    put(o_masks, L.masks.data(), L.masks.size() * 4);
    put(o_moves, moves.data(), moves.size() * sizeof(int2));
    std::vector<KVStep::Rows> of;
    of.reserve(ps.size());
    for (const Planned& p : ps) {
        of.push_back(KVStep::Rows{p.seq, p.P, p.P + p.n});
        p.seq->steps.reserve(p.seq->steps.size() + 1);
    }
    step->planned = false;                         // until the new plan is there
    step->leave();
    if (bytes <= SEND_BYTES) {
        HIP_TRY(launch_paged_send(hb, step->dev, bytes, s, step->ev[step->ring]));
    } else {
        HIP_TRY(hipMemcpyAsync(step->dev, hb, bytes, hipMemcpyHostToDevice, s));
        HIP_TRY(hipEventRecord(step->ev[step->ring], s));
    }
    step->used[step->ring] = true;
    step->ring ^= 1;
    if (!moves.empty()) HIP_TRY(launch_paged_copy(pool->p, (const int2*)(step->dev + o_moves), (int)moves.size(), s, nullptr));

    // ---- nothing fails from here on
    taken.keep();
    for (Planned& p : ps) {
        if (p.copy_last) {
            p.seq->lose(p.P / pr * pr);            // other steps' plans with rows of the page that is replaced
            pool->give(p.seq->pages.back());
        }
        p.seq->pages.swap(p.pages);
        p.seq->length = p.P + p.n;
        p.seq->steps.push_back(step);
    }
    step->of.swap(of);
    step->planned = true;
    step->turned = turned;
    step->merge = L.merge;
    step->M = M;
    step->many = L.many;
    step->n_items = (int)L.items.size();
    step->parts = L.parts;
    step->o_items = o_items;
    step->o_rows = o_rows;
    step->o_list = o_list;
    step->o_tables = o_tables;
    step->o_slots = o_slots;
    step->o_pos = o_pos;
    step->o_masks = o_masks;
    return STAGE_OK;
}

PagedWrite write_args(const KVStep* step, int layer) {
    const KVPages* pool = step->pool;
    PagedWrite a{};
    a.kp = pool->p.k + layer * pool->p.layer_elems();
    a.vp = pool->p.v + layer * pool->p.layer_elems();
    a.slots = (const int*)(step->dev + step->o_slots);
    a.pos = step->turned ? (const int*)(step->dev + step->o_pos) : nullptr;
    a.M = step->M;
    a.axis = pool->axis;
    a.rope = pool->stage->rope;
    a.shift = pool->p.shift;
    a.Hq = pool->stage->cfg.n_q_heads;
    a.Hkv = pool->p.Hkv;
    a.kv_dt = pool->p.kv_dt;
    return a;
}

PagedAttend attend_args(const KVStep* step, int layer, float scale, void* ws) {
    const KVPages* pool = step->pool;
    const StageConfig& c = pool->stage->cfg;
    PagedAttend a{};
    a.k = pool->p.k + layer * pool->p.layer_elems();
    a.v = pool->p.v + layer * pool->p.layer_elems();
    a.shift = pool->p.shift;
    a.Hkv = c.n_kv_heads;
    a.gs = c.n_q_heads / c.n_kv_heads;
    a.items = (const PagedItem*)(step->dev + step->o_items);
    a.n_items = step->n_items;
    a.many = step->many;
    a.rows = (const PagedRow*)(step->dev + step->o_rows);
    a.M = step->M;
    a.list = (const PagedRow*)(step->dev + step->o_list);
    a.tables = (const int*)(step->dev + step->o_tables);
    a.masks = (const uint32_t*)(step->dev + step->o_masks);
    a.scale2 = (float)(1.4426950408889634 * (scale == 0.f ? 1.0 / std::sqrt((double)c.head_dim) : (double)scale));
    a.part_o = (float*)ws;
    a.part_ml = (float2*)((uint8_t*)ws + step->parts * c.n_q_heads * (size_t)c.head_dim * 4);
    a.merge = step->merge;
    return a;
}

// New pages for rows [P, P + n) of seq, a shared last page replaced: `pages` as they will be, the rows to copy, the new
// rows' slots.
int room_for(KVSeq* seq, int n, Taken& taken, std::vector<int>& pages, std::vector<int2>& moves, std::vector<int>& slots) {
    KVPages* pool = seq->pool;
    const int P = seq->length, pr = pool->page_rows;
    if (P > MAX_POOL_ROWS - n) return fail(STAGE_E_CAPACITY, "sequence too long");
    const bool copy_last = P % pr && pool->refs[seq->pages.back()] > 1;
    const size_t need = pool->pages_for(P + n) - seq->pages.size() + copy_last;
    if (need > (size_t)pool->n_free) return no_room(pool, need);
    if (!one_launch(pool->p, n)) return fail(STAGE_E_CAPACITY, "too many rows for one call");
    pages = seq->pages;
    pages.reserve(pool->pages_for(P + n));
    taken.reserve(need);
    if (copy_last) {
        const int page = taken.page(), old = pages.back();
        for (int i = 0; i < P % pr; ++i) moves.push_back(int2{(old << pool->p.shift) + i, (page << pool->p.shift) + i});
        pages.back() = page;
    }
    while ((int)pages.size() < pool->pages_for(P + n)) pages.push_back(taken.page());
    slots.reserve(n);
    for (int i = 0; i < n; ++i) slots.push_back(pool->slot(pages, P + i));
    return STAGE_OK;
}

// Rows of [layers][S][Hkv][cap][D] (row start .. of `slot`, through `table`) behind the sequence's own.
int fill(KVSeq* seq, const uint16_t* k, const uint16_t* v, const int16_t* table, int S, int slot, int cap, int start, int n, hipStream_t s) {
    KVPages* pool = seq->pool;
    Stage* st = pool->stage;
    PAGED_BEGIN(st, s);
    Taken taken(pool);
    std::vector<int> pages, slots;
    std::vector<int2> moves;
    if (int rc = room_for(seq, n, taken, pages, moves, slots)) return rc;
    std::vector<uint8_t> meta(moves.size() * sizeof(int2) + slots.size() * 4);
    if (!moves.empty()) std::memcpy(meta.data(), moves.data(), moves.size() * sizeof(int2));
    std::memcpy(meta.data() + moves.size() * sizeof(int2), slots.data(), slots.size() * 4);
    HIP_TRY(order_on(st, s));
    WorkOn work(st, s);
    const uint8_t* d = nullptr;
    if (int rc = send(st, meta.data(), meta.size(), s, &d)) return rc;
    if (!moves.empty()) HIP_TRY(launch_paged_copy(pool->p, (const int2*)d, (int)moves.size(), s, nullptr));
    HIP_TRY(launch_paged_fill(pool->p, k, v, table, S, slot, cap, start, (const int*)(d + moves.size() * sizeof(int2)), n, s, st->done_ev));
    work.launched();
    taken.keep();
    if (!moves.empty()) {
        seq->lose((int)(seq->pages.size() - 1) * pool->page_rows);   // plans with rows of the page that is replaced
        pool->give(seq->pages.back());
    }
    seq->pages.swap(pages);
    seq->length += n;
    return STAGE_OK;
}

}  // namespace

extern "C" {

int kv_pages_create(Stage* st, int n_pages, int page_rows, void* k, void* v, const uint8_t* pair_axis, int n_axes, KVPages** out) {
    return guarded([&]() -> int {
        if (!st || !k || !v || !out) return fail(STAGE_E_INVALID, "NULL argument");
        *out = nullptr;
        if (((uintptr_t)k | (uintptr_t)v) & 15) return fail(STAGE_E_INVALID, "pages must be 16-byte aligned");
        if (page_rows < 16 || page_rows > 256 || (page_rows & (page_rows - 1)))
            return fail(STAGE_E_UNSUPPORTED, "page_rows must be 16, 32, 64, 128 or 256");
        if (n_pages < 1 || n_pages > MAX_POOL_ROWS / page_rows) return fail(STAGE_E_CAPACITY, "n_pages must be in [1, (2^31 - 1) / page_rows]");
        if (n_axes < 1 || n_axes > STAGE_MAX_AXES) return fail(STAGE_E_CAPACITY, "n_axes must be in [1, STAGE_MAX_AXES]");
        const StageConfig& c = st->cfg;
        for (int i = 0; pair_axis && i < c.head_dim / 2; ++i)
            if (pair_axis[i] >= n_axes) return fail(STAGE_E_INVALID, "pair_axis names an axis that is not there");
        if (!pair_axis && n_axes != 1) return fail(STAGE_E_INVALID, "several axes need pair_axis");
        DeviceGuard dev(st->device);
        HIP_TRY(dev.err);
        auto pool = std::make_unique<KVPages>();
        pool->stage = st;
        int shift = 0;
        while ((1 << shift) < page_rows) ++shift;
        pool->p = PagedPool{(uint16_t*)k, (uint16_t*)v, c.n_layers, n_pages, shift, c.n_kv_heads, c.head_dim, dt_code(c.kv_dtype)};
        pool->page_rows = page_rows;
        pool->n_axes = n_axes;
        pool->refs.assign(n_pages, 0);
        pool->open.assign((n_pages + 63) / 64, ~0ull);
        if (n_pages % 64) pool->open.back() = (1ull << (n_pages % 64)) - 1;
        pool->n_free = n_pages;
        if (pair_axis) {
            if (hipMalloc(&pool->axis, c.head_dim / 2) != hipSuccess) {
                (void)hipGetLastError();
                return fail(STAGE_E_OOM, "device allocation failed");
            }
            const hipError_t e = hipMemcpy(pool->axis, pair_axis, c.head_dim / 2, hipMemcpyHostToDevice);
            if (e != hipSuccess) {
                (void)hipFree(pool->axis);
                return fail(STAGE_E_HIP, std::string("kv_pages_create: ") + hipGetErrorString(e));
            }
        }
        *out = pool.release();
        return STAGE_OK;
    });
}

int kv_pages_free(KVPages* pool) {
    return guarded([&]() -> int {
        if (!pool) return fail(STAGE_E_INVALID, "pool is NULL");
        DeviceGuard dev(pool->stage->device);
        (void)hipDeviceSynchronize();
        while (pool->members.after) delete pool->members.after;
        delete pool->fwd;
        if (pool->ws) (void)hipFree(pool->ws);
        if (pool->axis) (void)hipFree(pool->axis);
        delete pool;
        return STAGE_OK;
    });
}

int kv_pages_available(const KVPages* pool, int* free_pages) {
    if (!pool || !free_pages) return fail(STAGE_E_INVALID, "NULL argument");
    *free_pages = pool->n_free;
    return STAGE_OK;
}

int kv_seq_create(KVPages* pool, KVSeq** out) {
    return guarded([&]() -> int {
        if (!pool || !out) return fail(STAGE_E_INVALID, "NULL argument");
        *out = nullptr;
        KVSeq* q = new KVSeq();
        q->pool = pool;
        q->join(pool->members);
        *out = q;
        return STAGE_OK;
    });
}

int kv_seq_free(KVSeq* seq) {
    if (!seq) return fail(STAGE_E_INVALID, "sequence is NULL");
    for (int p : seq->pages) seq->pool->give(p);
    delete seq;
    return STAGE_OK;
}

int kv_seq_length(const KVSeq* seq, int* length_out) {
    if (!seq || !length_out) return fail(STAGE_E_INVALID, "NULL argument");
    *length_out = seq->length;
    return STAGE_OK;
}

int kv_seq_pages(const KVSeq* seq, int32_t* pages_out, int capacity, int* count_out) {
    if (!seq || !count_out) return fail(STAGE_E_INVALID, "NULL argument");
    *count_out = (int)seq->pages.size();
    for (int i = 0; pages_out && i < std::min(capacity, *count_out); ++i) pages_out[i] = seq->pages[i];
    return STAGE_OK;
}

int kv_seq_fork(KVSeq* const* seqs, const int32_t* lengths, const uint8_t* const* keep, int n, KVSeq** out, void* stream) {
    return guarded([&]() -> int {
        if (!seqs || !out || n < 1) return fail(STAGE_E_INVALID, "NULL argument or n < 1");
        for (int i = 0; i < n; ++i) {
            out[i] = nullptr;
            if (!seqs[i]) return fail(STAGE_E_INVALID, "sequence " + std::to_string(i) + " is NULL");
            if (seqs[i]->pool != seqs[0]->pool) return fail(STAGE_E_STATE_MISMATCH, "sequences of different pools");
            if (lengths && (lengths[i] < 0 || lengths[i] > seqs[i]->length))
                return fail(STAGE_E_INVALID, "length " + std::to_string(i) + " out of range");
        }
        KVPages* pool = seqs[0]->pool;
        Stage* st = pool->stage;
        const int pr = pool->page_rows;
        hipStream_t s = (hipStream_t)stream;
        PAGED_BEGIN(st, s);
        struct Child { int shared, kept; std::vector<int> rows; };   // whole pages shared; the rows behind them
        std::vector<Child> kids((size_t)n);
        size_t need = 0, moves_n = 0, held = 0;
        for (int i = 0; i < n; ++i) {
            const int len = lengths ? lengths[i] : seqs[i]->length;
            const uint8_t* kp = keep ? keep[i] : nullptr;
            Child& k = kids[i];
            int first = len;
            if (kp)
                for (first = 0; first < len && kp[first];) ++first;
            k.shared = first / pr;
            k.rows.reserve(len - k.shared * pr);
            for (int j = k.shared * pr; j < len; ++j)
                if (!kp || kp[j]) k.rows.push_back(j);
            k.kept = k.shared * pr + (int)k.rows.size();
            moves_n += k.rows.size();
            need += pool->pages_for((int)k.rows.size());
            held += pool->pages_for(k.kept);
        }
        if (need > (size_t)pool->n_free) return no_room(pool, need);
        if (!one_launch(pool->p, moves_n)) return fail(STAGE_E_CAPACITY, "too many rows copied in one call");
        Taken taken(pool);
        taken.reserve(held);
        std::vector<std::unique_ptr<KVSeq>> made((size_t)n);
        std::vector<int2> moves;
        moves.reserve(moves_n);
        for (int i = 0; i < n; ++i) {
            const Child& k = kids[i];
            made[i] = std::make_unique<KVSeq>();
            made[i]->pool = pool;
            made[i]->length = k.kept;
            std::vector<int>& pg = made[i]->pages;
            pg.reserve(pool->pages_for(k.kept));
            for (int t = 0; t < k.shared; ++t) {
                taken.share(seqs[i]->pages[t]);
                pg.push_back(seqs[i]->pages[t]);
            }
            for (int t = pool->pages_for((int)k.rows.size()); t > 0; --t) pg.push_back(taken.page());
            for (size_t j = 0; j < k.rows.size(); ++j)
                moves.push_back(int2{pool->slot(seqs[i]->pages, k.rows[j]), pool->slot(pg, k.shared * pr + (int)j)});
        }
        if (!moves.empty()) {
            HIP_TRY(order_on(st, s));
            WorkOn work(st, s);
            const uint8_t* d = nullptr;
            if (int rc = send(st, moves.data(), moves.size() * sizeof(int2), s, &d)) return rc;
            HIP_TRY(launch_paged_copy(pool->p, (const int2*)d, (int)moves.size(), s, st->done_ev));
            work.launched();
        }
        taken.keep();
        for (int i = 0; i < n; ++i) {
            made[i]->join(pool->members);
            out[i] = made[i].release();
        }
        return STAGE_OK;
    });
}

int kv_seq_compact(KVSeq* seq, const uint8_t* keep, void* stream) {
    return guarded([&]() -> int {
        if (!seq || !keep) return fail(STAGE_E_INVALID, "NULL argument");
        KVPages* pool = seq->pool;
        Stage* st = pool->stage;
        const int pr = pool->page_rows, P = seq->length;
        hipStream_t s = (hipStream_t)stream;
        PAGED_BEGIN(st, s);
        int first = 0;
        while (first < P && keep[first]) ++first;
        if (first == P) return STAGE_OK;
        const int t0 = first / pr;
        std::vector<int> rows;                     // kept, from page t0 on
        for (int j = t0 * pr; j < P; ++j)
            if (keep[j]) rows.push_back(j);
        const int kept = t0 * pr + (int)rows.size(), n_pages = pool->pages_for(kept);
        const bool moved = kept > first;           // else only a tail is dropped
        // into new pages where there are enough, all rows at once; else in place, in order, by one thread per 16 bytes of a row
        // (16 layers of 8 x 128: 64 rows 14 and 24 us, 1024 rows 33 and 215)
        const bool fresh = moved && n_pages - t0 <= pool->n_free && one_launch(pool->p, rows.size());
        size_t need = 0;
        if (moved)
            for (int t = t0; t < n_pages; ++t) need += fresh || pool->refs[seq->pages[t]] > 1;
        if (need > (size_t)pool->n_free) return no_room(pool, need);
        Taken taken(pool);
        taken.reserve(need);
        std::vector<int> pages(seq->pages.begin(), seq->pages.begin() + n_pages), gone;
        gone.reserve(seq->pages.size());
        if (moved)
            for (int t = t0; t < n_pages; ++t)
                if (fresh || pool->refs[pages[t]] > 1) {
                    gone.push_back(pages[t]);
                    pages[t] = taken.page();
                }
        gone.insert(gone.end(), seq->pages.begin() + n_pages, seq->pages.end());
        std::vector<int2> moves;
        for (size_t j = 0; moved && j < rows.size(); ++j) {
            const int2 m{pool->slot(seq->pages, rows[j]), pool->slot(pages, t0 * pr + (int)j)};
            if (m.x != m.y) moves.push_back(m);
        }
        if (!moves.empty()) {
            HIP_TRY(order_on(st, s));
            WorkOn work(st, s);
            const uint8_t* d = nullptr;
            if (int rc = send(st, moves.data(), moves.size() * sizeof(int2), s, &d)) return rc;
            HIP_TRY(fresh ? launch_paged_copy(pool->p, (const int2*)d, (int)moves.size(), s, st->done_ev)
                          : launch_paged_slide(pool->p, (const int2*)d, (int)moves.size(), s, st->done_ev));
            work.launched();
        }
        taken.keep();
        // from the first row of a replaced page on: its plans would write and read what may be another sequence's
        seq->lose(moved && pages[t0] != seq->pages[t0] ? t0 * pr : first);
        for (int p : gone) pool->give(p);
        seq->pages.swap(pages);
        seq->length = kept;
        return STAGE_OK;
    });
}

int kv_seq_truncate(KVSeq* seq, int new_len) {
    if (!seq) return fail(STAGE_E_INVALID, "sequence is NULL");
    if (new_len < 0 || new_len > seq->length) return fail(STAGE_E_INVALID, "new_len must be in [0, length]");
    seq->lose(new_len);
    const size_t n = seq->pool->pages_for(new_len);
    while (seq->pages.size() > n) {
        seq->pool->give(seq->pages.back());
        seq->pages.pop_back();
    }
    seq->length = new_len;
    return STAGE_OK;
}

int kv_seq_append(KVSeq* seq, const void* k, const void* v, int n, void* stream) {
    return guarded([&]() -> int {
        if (!seq || !k || !v) return fail(STAGE_E_INVALID, "NULL argument");
        if (n < 1) return fail(STAGE_E_INVALID, "n must be positive");
        if (((uintptr_t)k | (uintptr_t)v) & 15) return fail(STAGE_E_INVALID, "rows must be 16-byte aligned");
        return fill(seq, (const uint16_t*)k, (const uint16_t*)v, nullptr, 1, 0, n, 0, n, (hipStream_t)stream);
    });
}

int kv_seq_load(KVSeq* seq, KVState* kv, int slot, int start, int n, void* stream) {
    return guarded([&]() -> int {
        if (!seq || !kv) return fail(STAGE_E_INVALID, "NULL argument");
        if (kv->stage != seq->pool->stage) return fail(STAGE_E_STATE_MISMATCH, "state belongs to another stage");
        if (n < 1) return fail(STAGE_E_INVALID, "n must be positive");
        if (slot < 0 || slot >= kv->S || start < 0 || start > kv->P - n) return fail(STAGE_E_INVALID, "slot or rows out of range");
        return fill(seq, kv->kc, kv->vc, kv->table[kv->cur], kv->S, slot, kv->cap, start, n, (hipStream_t)stream);
    });
}

int kv_seq_read(KVSeq* seq, int layer, int start, int count, void* k_out, void* v_out, void* stream) {
    return guarded([&]() -> int {
        if (!seq || !k_out || !v_out) return fail(STAGE_E_INVALID, "NULL argument");
        KVPages* pool = seq->pool;
        Stage* st = pool->stage;
        if (layer < 0 || layer >= st->cfg.n_layers) return fail(STAGE_E_INVALID, "layer out of range");
        if (start < 0 || count < 0 || start > seq->length - count) return fail(STAGE_E_INVALID, "row range exceeds the length");
        if (count == 0) return STAGE_OK;
        hipStream_t s = (hipStream_t)stream;
        PAGED_BEGIN(st, s);
        std::vector<int> slots;
        slots.reserve(count);
        for (int i = 0; i < count; ++i) slots.push_back(pool->slot(seq->pages, start + i));
        HIP_TRY(order_on(st, s));
        WorkOn work(st, s);
        const uint8_t* d = nullptr;
        if (int rc = send(st, slots.data(), slots.size() * 4, s, &d)) return rc;
        HIP_TRY(launch_paged_read(pool->p, layer, (const int*)d, count, (uint16_t*)k_out, (uint16_t*)v_out, s, st->done_ev));
        work.launched();
        return STAGE_OK;
    });
}

int kv_step_create(KVPages* pool, KVStep** out) {
    return guarded([&]() -> int {
        if (!pool || !out) return fail(STAGE_E_INVALID, "NULL argument");
        *out = nullptr;
        KVStep* step = pool->spare;
        if (step) {
            pool->spare = step->next;
        } else {
            step = new KVStep();
            step->pool = pool;
            step->join(pool->members);
        }
        *out = step;
        return STAGE_OK;
    });
}

int kv_step_free(KVStep* step) {
    if (!step) return fail(STAGE_E_INVALID, "step is NULL");
    if (step->captured) return STAGE_OK;           // a graph may still read its metadata: it goes with the pool
    // Queued work may still read its metadata, and to wait for that would end a capture of any thread.  The next step of the
    // pool takes it over: its plan is sent behind the work that is queued.
    step->planned = false;
    step->leave();
    step->next = step->pool->spare;
    step->pool->spare = step;
    return STAGE_OK;
}

int kv_step_plan(KVStep* step, const KVStepRequest* reqs, int n_req, void* stream) {
    return guarded([&]() -> int {
        if (!step || !reqs || n_req < 1) return fail(STAGE_E_INVALID, "NULL argument or n_req < 1");
        int M = 0;
        size_t words = 0;
        if (int rc = check_requests(step->pool, reqs, n_req, STAGE_MAX_STEP_ROWS, false, M, words)) return rc;
        Stage* st = step->pool->stage;
        hipStream_t s = (hipStream_t)stream;
        PAGED_BEGIN(st, s);
        if (step->captured) return fail(STAGE_E_UNSUPPORTED, "a graph holds this step's plan");
        HIP_TRY(order_on(st, s));
        WorkOn work(st, s);                        // marked behind its last work as it ends
        return plan(step, reqs, n_req, M, words, s);
    });
}

int kv_step_write(KVStep* step, int layer, const void* q, int64_t ldq, const void* k, int64_t ldk, const void* v, int64_t ldv, int dtype,
                  void* q_out, int64_t ldqo, int q_out_dtype, void* stream) {
    return guarded([&]() -> int {
        if (!step || !q || !k || !v || !q_out) return fail(STAGE_E_INVALID, "NULL argument");
        if (!step->planned) return fail(STAGE_E_INVALID, "the step has no plan");
        Stage* st = step->pool->stage;
        const StageConfig& c = st->cfg;
        if (layer < 0 || layer >= c.n_layers) return fail(STAGE_E_INVALID, "layer out of range");
        if (!dtype_ok(dtype) || !dtype_ok(q_out_dtype)) return fail(STAGE_E_INVALID, "dtypes must be F32, F16 or BF16");
        const int64_t nq = (int64_t)c.n_q_heads * c.head_dim, nk = (int64_t)c.n_kv_heads * c.head_dim;
        if (ldq < nq || ldqo < nq || ldk < nk || ldv < nk) return fail(STAGE_E_SHAPE, "row stride below the row length");
        const int e = dtype == STAGE_DTYPE_F32 ? 4 : 2, eo = q_out_dtype == STAGE_DTYPE_F32 ? 4 : 2;
        const bool in_place = q_out == q && q_out_dtype == dtype && ldqo == ldq;
        if ((!in_place && overlap(q, nq * e, ldq * e, q_out, nq * eo, ldqo * eo, step->M)) ||
            overlap(k, nk * e, ldk * e, q_out, nq * eo, ldqo * eo, step->M) || overlap(v, nk * e, ldv * e, q_out, nq * eo, ldqo * eo, step->M))
            return fail(STAGE_E_INVALID, "q_out overlaps q, k or v (it may be q itself, in its dtype and stride)");
        if (step->shared()) return fail(STAGE_E_INVALID, "a page of the step's new rows is shared since they were planned");
        DeviceGuard dev(st->device);
        HIP_TRY(dev.err);
        hipStream_t s = (hipStream_t)stream;
        bool graph = false;
        if (int rc = captured(s, graph)) return rc;
        PagedWrite a = write_args(step, layer);
        a.q = q;
        a.k = k;
        a.v = v;
        a.dt = any_dt(dtype);
        a.ldq = (size_t)ldq;
        a.ldk = (size_t)ldk;
        a.ldv = (size_t)ldv;
        a.q_out = q_out;
        a.q_out_dt = any_dt(q_out_dtype);
        a.ldqo = (size_t)ldqo;
        if (graph) {
            step->captured = true;
            HIP_TRY(launch_paged_write(a, c.head_dim, s, nullptr));
            return STAGE_OK;
        }
        HIP_TRY(order_on(st, s));
        WorkOn work(st, s);
        HIP_TRY(launch_paged_write(a, c.head_dim, s, st->done_ev));
        work.launched();
        return STAGE_OK;
    });
}

int kv_step_workspace(const KVStep* step, int64_t* bytes_out) {
    if (!step || !bytes_out) return fail(STAGE_E_INVALID, "NULL argument");
    if (!step->planned) return fail(STAGE_E_INVALID, "the step has no plan");
    *bytes_out = (int64_t)step->part_bytes();
    return STAGE_OK;
}

int kv_step_attend(KVStep* step, int layer, const void* q, int q_dtype, int64_t ldq, void* out, int out_dtype, int64_t ldo, float scale,
                   void* workspace, int64_t workspace_bytes, void* stream) {
    return guarded([&]() -> int {
        if (!step || !q || !out) return fail(STAGE_E_INVALID, "NULL argument");
        if (!step->planned) return fail(STAGE_E_INVALID, "the step has no plan");
        Stage* st = step->pool->stage;
        const StageConfig& c = st->cfg;
        if (layer < 0 || layer >= c.n_layers) return fail(STAGE_E_INVALID, "layer out of range");
        if (q_dtype != STAGE_DTYPE_F32 && q_dtype != c.kv_dtype) return fail(STAGE_E_INVALID, "q must be F32 or in kv_dtype");
        if (!dtype_ok(out_dtype)) return fail(STAGE_E_INVALID, "out must be F32, F16 or BF16");
        if (!(scale >= 0.f) || !std::isfinite(scale)) return fail(STAGE_E_INVALID, "scale must be finite and not negative");
        const int64_t nq = (int64_t)c.n_q_heads * c.head_dim;
        if (ldq < nq || ldo < nq) return fail(STAGE_E_SHAPE, "row stride below the row length");
        const int e = q_dtype == STAGE_DTYPE_F32 ? 4 : 2, eo = out_dtype == STAGE_DTYPE_F32 ? 4 : 2;
        if (overlap(q, nq * e, ldq * e, out, nq * eo, ldo * eo, step->M)) return fail(STAGE_E_INVALID, "out overlaps q");
        if (step->merge && (!workspace || ((uintptr_t)workspace & 15) || workspace_bytes < (int64_t)step->part_bytes()))
            return fail(STAGE_E_INVALID, "workspace too small (kv_step_workspace) or not aligned to 16 bytes");
        DeviceGuard dev(st->device);
        HIP_TRY(dev.err);
        hipStream_t s = (hipStream_t)stream;
        bool graph = false;
        if (int rc = captured(s, graph)) return rc;
        PagedAttend a = attend_args(step, layer, scale, workspace);
        a.q = q;
        a.q_dt = any_dt(q_dtype);
        a.ldq = (size_t)ldq;
        a.out = out;
        a.out_dt = any_dt(out_dtype);
        a.ldo = (size_t)ldo;
        if (graph) {
            step->captured = true;
            HIP_TRY(launch_paged_attend(a, c.head_dim, step->pool->p.kv_dt, s, nullptr));
            return STAGE_OK;
        }
        HIP_TRY(order_on(st, s));
        WorkOn work(st, s);
        HIP_TRY(launch_paged_attend(a, c.head_dim, step->pool->p.kv_dt, s, st->done_ev));
        work.launched();
        return STAGE_OK;
    });
}

int stage_forward_paged(Stage* st, const KVStepRequest* reqs, int n_req, const void* hidden_in, void* hidden_out, void* stream) {
    return guarded([&]() -> int {
        if (!st || !reqs || !hidden_in || !hidden_out || n_req < 1) return fail(STAGE_E_INVALID, "NULL argument or n_req < 1");
        if (!reqs[0].seq) return fail(STAGE_E_INVALID, "request 0: sequence is NULL");
        KVPages* pool = reqs[0].seq->pool;
        if (pool->stage != st) return fail(STAGE_E_STATE_MISMATCH, "request 0: sequence belongs to another stage");
        const StageConfig& c = st->cfg;
        int M = 0;
        size_t words = 0;
        if (int rc = check_requests(pool, reqs, n_req, STAGE_MAX_ROWS, true, M, words)) return rc;
        const size_t bytes = (size_t)M * c.hidden * 2;
        if ((const uint8_t*)hidden_in < (const uint8_t*)hidden_out + bytes && (const uint8_t*)hidden_out < (const uint8_t*)hidden_in + bytes)
            return fail(STAGE_E_INVALID, "hidden_in and hidden_out overlap");
        hipStream_t s = (hipStream_t)stream;
        PAGED_BEGIN(st, s);
        if (!pool->fwd) {
            pool->fwd = new KVStep();
            pool->fwd->pool = pool;
        }
        HIP_TRY(order_on(st, s));
        WorkOn work(st, s);                        // marked behind its last work as it ends
        KVStep* step = pool->fwd;
        if (int rc = plan(step, reqs, n_req, M, words, s)) return rc;
        struct Back {                              // a forward that fails leaves the sequences as long as they were
            const KVStepRequest* reqs;
            int n_req;
            ~Back() {
                for (int r = 0; r < n_req; ++r) (void)kv_seq_truncate(reqs[r].seq, reqs[r].seq->length - reqs[r].n_tokens);
            }
        } back{reqs, n_req};
        if (int rc = grow(&pool->ws, &pool->ws_cap, step->part_bytes())) return rc;

        // rotary and the rows' write, in place on the q part; attention; the o product's prepared input
        struct PagesAttention : LayerAttention {
            Stage* st;
            const KVStep* step;
            hipStream_t s;
            hipError_t run(int l, uint16_t* bp, float* bc) override {
                const StageConfig& c = st->cfg;
                const int D = c.head_dim, nq = c.n_q_heads * D, nk = c.n_kv_heads * D, ld = nq + 2 * nk;
                PagedWrite w = write_args(step, l);
                w.q = st->qkv;
                w.k = st->qkv + nq;
                w.v = st->qkv + nq + nk;
                w.dt = w.q_out_dt = DT_F32;
                w.ldq = w.ldk = w.ldv = w.ldqo = ld;
                w.q_out = st->qkv;
                if (hipError_t e = launch_paged_write(w, D, s, nullptr)) return e;
                PagedAttend a = attend_args(step, l, 0.f, step->pool->ws);
                a.q = st->qkv;
                a.q_dt = a.out_dt = DT_F32;
                a.ldq = ld;
                a.out = st->attn;
                a.ldo = nq;
                if (hipError_t e = launch_paged_attend(a, D, step->pool->p.kv_dt, s, nullptr)) return e;
                return bp ? launch_bprep_plain(st->attn, nq, step->M, bp, bc, st->kp, s) : hipSuccess;
            }
        } attention;
        attention.st = st;
        attention.step = step;
        attention.s = s;
        if (int rc = run_layers(st, M, hidden_in, hidden_out, s, attention)) return rc;
        back.n_req = 0;
        return STAGE_OK;
    });
}

}  // extern "C"
