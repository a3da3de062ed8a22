// Sampling from logits rows, and the walk of a drafted tree.
//
// The tokens of a row are ranked highest logit first, lowest index first among
// equal logits.  Temperature, top-k, top-p and min-p each keep a run of that
// ranking from its start, so what is kept is its first C tokens, and the token
// drawn is the first whose running weight passes u times the kept weight.  Every
// step is then a search for a place in the ranking by count, by weight or by
// value, and none needs the row sorted: a histogram over bins of the scaled
// logit says which bin holds the place, and only that bin's tokens are ranked.
//
// Bins: x = logit * 32 / T, q = floor(x), bin = q_max - q, weight exp((x - x_max)
// / 32) up to a common factor: exp(d) E[bin], d = (x - q) / 32, E[b] = exp(-b / 32).
// exp(d) goes into a bin's sum as an integer in units of 2^-43 (sums are then
// the same in any order, below 2^64 for 2^20 tokens), the bins' sums are joined
// in 64-bit floating point.  Bins from 1024 on (weights below e^-31.97 of the
// largest, together less than 2^20 e^-31.97 = 1.4e-8 of the kept weight) are left
// out: neither u nor top_p, 24-bit numbers below 1, come nearer to 1 than 6e-8,
// so no draw and no cut falls there.
#include "device.h"

namespace stg {

constexpr int SB_BINS = 1024;        // bins of 1/32 of a unit of logit / T
constexpr int SB_CAP = 2048;         // tokens of one bin that are ranked in LDS
constexpr int SB_THREADS = 1024;
constexpr double SB_UNIT = 8796093022208.0;        // 2^43

// Order of finite logits as unsigned integers; NaN and -inf are not ranked (0), +inf ranks as the largest finite value, -0 as 0.
__device__ __forceinline__ uint32_t rank_key(float l) {
    if (!(l >= -3.402823466e38f)) return 0u;
    const uint32_t u = __float_as_uint(fminf(l, 3.402823466e38f) + 0.0f);
    return (u & 0x80000000u) ? ~u : (u | 0x80000000u);
}
__device__ __forceinline__ float key_logit(uint32_t k) { return __uint_as_float((k & 0x80000000u) ? (k & 0x7fffffffu) : ~k); }

// exp(d) 2^43 as an integer, d in [0, 1/32]: Taylor to d^7, the rest below 3e-17.
__device__ __forceinline__ unsigned long long exp_units(double d) {
    double p = 1.0 / 5040.0;
    p = fma(p, d, 1.0 / 720.0);
    p = fma(p, d, 1.0 / 120.0);
    p = fma(p, d, 1.0 / 24.0);
    p = fma(p, d, 1.0 / 6.0);
    p = fma(p, d, 0.5);
    p = fma(p, d, 1.0);
    p = fma(p, d, 1.0);
    return (unsigned long long)(p * SB_UNIT + 0.5);
}

struct RowBins {                      // the scaled logit of a row's tokens
    double per_t;                     // 32 / T
    double qmax;                      // floor(x) of the largest
    __device__ __forceinline__ double x(uint32_t key) const { return (double)key_logit(key) * per_t; }
    __device__ __forceinline__ double bin(double xv) const { return qmax - floor(xv); }
    __device__ __forceinline__ unsigned long long units(double xv) const { return exp_units((xv - floor(xv)) * (1.0 / 32.0)); }
};

// Tokens of one row with lo <= key <= hi in bin `bin`: a part of the ranking
// without gaps.
struct Part {
    int bin;
    uint32_t lo, hi;
    int n;
};

enum Want : int { BY_COUNT = 0, BY_MASS = 1, BY_VALUE = 2 };

struct Place { int count; unsigned long long units; uint32_t key; int index; };   // the first `count` of a part: their units, the last one

struct SampleShared {
    unsigned long long list[SB_CAP];           // key << 32 | ~index
    unsigned long long mass[SB_BINS];
    unsigned cnt[SB_BINS];
    unsigned long long wave_u[SB_THREADS / 64];
    unsigned wave_c[SB_THREADS / 64];
    double wave_d[SB_THREADS / 64];
    uint32_t klo, khi;
    unsigned fill;
    unsigned bin_c0;
    int found;
    unsigned long long bin_u0;
    Place place;
};

struct RowArgs {
    const void* logits; int dt; size_t base; int V;
};

// Inclusive sums over the workgroup's threads, in thread order.
template <class S>
__device__ __forceinline__ S scan_block(S v, S* wave, S* total) {
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6, nw = blockDim.x >> 6;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
        const S u = __shfl_up(v, o);
        if (lane >= o) v += u;
    }
    __syncthreads();                            // earlier readers of wave[] are done
    if (lane == 63) wave[w] = v;
    __syncthreads();
    S b = S(0), t = S(0);
    for (int i = 0; i < nw; ++i) {
        if (i < w) b += wave[i];
        t += wave[i];
    }
    *total = t;
    return v + b;
}

// The place in `part` that `want` asks for: its first `t` tokens (BY_COUNT), the
// fewest whose units together reach `t`, all of them if none do (BY_MASS), or
// those of at least `t` units each (BY_VALUE).  Whole workgroup; every thread
// gets the result.
__device__ Place find_place(const RowArgs& r, const RowBins& rb, Part part, Want want, unsigned long long t, SampleShared& sh) {
    const int tid = threadIdx.x;
    int c0 = 0;                                 // tokens and units of the part ahead of the piece looked at
    unsigned long long u0 = 0;
    auto key_of = [&](int i) {
        const uint32_t k = rank_key(load_val(r.logits, r.dt, r.base + i));
        return k != 0u && k >= part.lo && k <= part.hi && rb.bin(rb.x(k)) == (double)part.bin ? k : 0u;
    };
    while (part.n > SB_CAP) {
        // the keys' range, then a histogram over it
        if (tid == 0) { sh.klo = 0xffffffffu; sh.khi = 0u; }
        for (int i = tid; i < SB_BINS; i += SB_THREADS) { sh.mass[i] = 0; sh.cnt[i] = 0; }
        __syncthreads();
        uint32_t lo = 0xffffffffu, hi = 0u;
        for (int i = tid; i < r.V; i += SB_THREADS) {
            const uint32_t k = key_of(i);
            if (k) { lo = min(lo, k); hi = max(hi, k); }
        }
        if (hi) { atomicMin(&sh.klo, lo); atomicMax(&sh.khi, hi); }
        __syncthreads();
        part.lo = sh.klo;
        part.hi = sh.khi;
        if (part.lo == part.hi) {               // all equal: ranked by index alone
            const unsigned long long e = rb.units(rb.x(part.lo));
            unsigned long long q;
            if (want == BY_COUNT) q = t - (unsigned)c0;
            else if (want == BY_VALUE) q = e >= t ? (unsigned)part.n : 0u;
            else q = t > u0 ? (t - u0 + e - 1) / e : 1u;
            const int k = q < (unsigned)part.n ? (int)q : part.n;
            // the k-th by index: each thread counts a run of the row
            const int run = (r.V + SB_THREADS - 1) / SB_THREADS, b = min(r.V, tid * run), e1 = min(r.V, b + run);
            unsigned mine = 0, tot;
            for (int i = b; i < e1; ++i) mine += key_of(i) != 0u;
            const unsigned upto = scan_block<unsigned>(mine, sh.wave_c, &tot);
            if (tid == 0) sh.place.index = -1;
            __syncthreads();
            if (k > 0 && upto >= (unsigned)k && upto - mine < (unsigned)k) {
                unsigned at = upto - mine;
                for (int i = b; i < e1; ++i)
                    if (key_of(i) != 0u && ++at == (unsigned)k) { sh.place.index = i; break; }
            }
            __syncthreads();
            const Place p{c0 + k, u0 + (unsigned long long)k * e, part.lo, sh.place.index};
            __syncthreads();
            return p;
        }
        int shift = 0;
        while (((part.hi - part.lo) >> shift) >= (uint32_t)SB_BINS) ++shift;
        for (int i = tid; i < r.V; i += SB_THREADS) {
            const uint32_t k = key_of(i);
            if (k) {
                const uint32_t s = (part.hi - k) >> shift;
                atomicAdd(&sh.cnt[s], 1u);
                atomicAdd(&sh.mass[s], rb.units(rb.x(k)));
            }
        }
        __syncthreads();
        if (tid == 0) {                         // the first piece that holds the place, else the last one
            int s = 0, last = 0;
            int cc = c0, lc = c0;
            unsigned long long uu = u0, lu = u0;
            for (; s < SB_BINS; ++s) {
                if (!sh.cnt[s]) continue;
                last = s; lc = cc; lu = uu;
                const int c1 = cc + (int)sh.cnt[s];
                const unsigned long long u1 = uu + sh.mass[s];
                bool here;
                if (want == BY_COUNT) here = (unsigned long long)c1 >= t;
                else if (want == BY_MASS) here = u1 >= t;
                else here = rb.units(rb.x(max(part.lo, part.hi - (((uint32_t)s + 1) << shift) + 1))) < t;   // its least token fails
                if (here) break;
                cc = c1;
                uu = u1;
            }
            sh.found = last;
            sh.bin_c0 = (unsigned)lc;
            sh.bin_u0 = lu;
        }
        __syncthreads();
        const int s = sh.found;
        const uint32_t nhi = part.hi - ((uint32_t)s << shift);
        const uint32_t span = (1u << shift) - 1u;
        part.lo = max(part.lo, nhi >= span ? nhi - span : 0u);
        part.hi = nhi;
        part.n = (int)sh.cnt[s];
        c0 = (int)sh.bin_c0;
        u0 = sh.bin_u0;
        __syncthreads();
    }
    // few enough: into LDS, ranked, summed
    if (tid == 0) sh.fill = 0;
    int n2 = 64;
    while (n2 < part.n) n2 <<= 1;
    for (int i = tid; i < n2; i += SB_THREADS) sh.list[i] = 0;
    __syncthreads();
    for (int i = tid; i < r.V; i += SB_THREADS) {
        const uint32_t k = key_of(i);
        if (k) {
            const unsigned at = atomicAdd(&sh.fill, 1u);
            if (at < SB_CAP) sh.list[at] = ((unsigned long long)k << 32) | (uint32_t)~i;
        }
    }
    __syncthreads();
    for (int size = 2; size <= n2; size <<= 1)
        for (int step = size >> 1; step > 0; step >>= 1) {
            for (int i = tid; i < n2 / 2; i += SB_THREADS) {
                const int a = 2 * i - (i & (step - 1)), b = a + step;
                const bool down = (a & size) == 0;
                const unsigned long long va = sh.list[a], vb = sh.list[b];
                if ((va < vb) == down) { sh.list[a] = vb; sh.list[b] = va; }
            }
            __syncthreads();
        }
    constexpr int PER = SB_CAP / SB_THREADS;    // neighbours in rank a thread
    unsigned long long e[PER], mine = 0, tot;
#pragma unroll
    for (int j = 0; j < PER; ++j) {
        const int i = tid * PER + j;
        e[j] = i < part.n && i < n2 ? rb.units(rb.x((uint32_t)(sh.list[i] >> 32))) : 0ull;
        mine += e[j];
    }
    if (tid == 0) sh.place.count = 0;
    const unsigned long long upto = scan_block<unsigned long long>(mine, sh.wave_u, &tot);
    unsigned long long run = upto - mine;
#pragma unroll
    for (int j = 0; j < PER; ++j) {
        const int i = tid * PER + j;
        const unsigned long long was = run;
        run += e[j];
        if (i >= part.n) continue;
        bool here;                              // true at one i: the last of the place
        if (want == BY_COUNT) here = (unsigned long long)(c0 + i + 1) == t || (i == part.n - 1 && (unsigned long long)(c0 + part.n) < t);
        else if (want == BY_MASS) here = (u0 + run >= t || i == part.n - 1) && (u0 + was < t || i == 0);
        else here = e[j] >= t && (i == part.n - 1 || rb.units(rb.x((uint32_t)(sh.list[i + 1] >> 32))) < t);
        if (here) sh.place = Place{c0 + i + 1, u0 + run, (uint32_t)(sh.list[i] >> 32), (int)~(uint32_t)sh.list[i]};
    }
    __syncthreads();
    Place p = sh.place;
    if (p.count == 0) p = Place{c0, u0, 0u, -1};   // BY_VALUE: none
    __syncthreads();
    return p;
}

// One workgroup a row.
__global__ __launch_bounds__(SB_THREADS) void sample_kernel(SampleArgs a) {
    __shared__ SampleShared sh;
    __shared__ double cum[SB_BINS];             // weight of the bins up to and with this one
    __shared__ unsigned cumc[SB_BINS];
    const int row = blockIdx.x, tid = threadIdx.x;
    const RowArgs r{a.logits, a.dt, (size_t)row * a.ld, a.V};
    const SampleRow p = a.rows[row];
    // the largest
    if (tid == 0) sh.khi = 0u;
    __syncthreads();
    uint32_t top = 0;
    for (int i = tid; i < r.V; i += SB_THREADS) top = max(top, rank_key(load_val(r.logits, r.dt, r.base + i)));
    atomicMax(&sh.khi, top);
    __syncthreads();
    top = sh.khi;
    if (!top) {                                 // nothing to draw from
        if (tid == 0) {
            a.token[row] = -1;
            a.p[row] = 0.0f;
            if (a.top) a.top[row] = -INFINITY;
        }
        return;
    }
    RowBins rb{p.per_t, 0.0};
    const double xtop = rb.x(top);
    rb.qmax = floor(xtop);
    for (int i = tid; i < SB_BINS; i += SB_THREADS) { sh.mass[i] = 0; sh.cnt[i] = 0; }
    __syncthreads();
    for (int i = tid; i < r.V; i += SB_THREADS) {
        const uint32_t k = rank_key(load_val(r.logits, r.dt, r.base + i));
        if (!k) continue;
        const double x = rb.x(k), b = rb.bin(x);
        if (b < (double)SB_BINS) {
            atomicAdd(&sh.cnt[(int)b], 1u);
            atomicAdd(&sh.mass[(int)b], rb.units(x));
        }
    }
    __syncthreads();
    // E[b] and the bins' sums; one bin a thread
    const double E = exp((double)tid * (-1.0 / 32.0));
    double all;
    unsigned nall;
    const unsigned bc = sh.cnt[tid];
    const unsigned long long bu = sh.mass[tid];
    cum[tid] = scan_block<double>((double)bu * E, sh.wave_d, &all);
    cumc[tid] = scan_block<unsigned>(bc, sh.wave_c, &nall);
    __shared__ unsigned bins_c[SB_BINS];
    __shared__ unsigned long long bins_u[SB_BINS];
    bins_c[tid] = bc;
    bins_u[tid] = bu;
    __syncthreads();
    auto before = [&](int b) { return b ? cum[b - 1] : 0.0; };
    auto cbefore = [&](int b) { return b ? cumc[b - 1] : 0u; };
    auto E_of = [&](int b) { return exp((double)b * (-1.0 / 32.0)); };
    // first bin with pred, by the lowest thread that has it
    auto first_bin = [&](bool pred) {
        __syncthreads();
        if (tid == 0) sh.found = SB_BINS;
        __syncthreads();
        if (pred) atomicMin(&sh.found, tid);
        __syncthreads();
        return sh.found;
    };
    auto part_of = [&](int b) { return Part{b, 0u, 0xffffffffu, (int)bins_c[b]}; };
    // kept: the first C tokens, of weight W; W0: the units of those in bin 0, where the largest is (E[0] = 1)
    int C = (int)nall;
    double W = all;
    unsigned long long W0 = bins_u[0];
    auto cut = [&](int b, const Place& pl) {
        const int c = (int)cbefore(b) + pl.count;
        if (c >= C) return;
        C = c;
        W = before(b) + (double)pl.units * E_of(b);
        if (b == 0) W0 = pl.units;
    };
    // share * kept weight, in units of bin b and less what is ahead of it, rounded down or up.  Where all that is
    // kept is in bin 0 the product is exact: equal logits have no other way to agree with u or top_p times their number.
    auto target = [&](float share, int b, bool up) {
        if (C <= (int)cumc[0]) {
            const unsigned long long f = (unsigned long long)((double)share * 18446744073709551616.0);
            return __umul64hi(W0, f) + (up && W0 * f != 0ull ? 1ull : 0ull);
        }
        const double t = fmax(0.0, ((double)share * W - before(b)) / E_of(b));
        return (unsigned long long)(up ? ceil(t) : floor(t));
    };
    auto bin_of = [&](float share) {            // the bin in which the running weight reaches share * W
        const double t = (double)share * W;
        const int b = first_bin(bc != 0u && cum[tid] >= t), last = first_bin(bc != 0u && cumc[tid] >= (unsigned)C);
        return C <= (int)cumc[0] ? 0 : min(b, last);
    };
    if (p.top_k > 0 && (unsigned)p.top_k < nall) {
        const int b = first_bin(cumc[tid] >= (unsigned)p.top_k);
        cut(b, find_place(r, rb, part_of(b), BY_COUNT, (unsigned)p.top_k - cbefore(b), sh));
    }
    if (p.top_p < 1.0f) {
        const int b = bin_of(p.top_p);
        cut(b, find_place(r, rb, part_of(b), BY_MASS, target(p.top_p, b, true), sh));
    }
    if (p.min_p > 0.0f) {
        // exp(d) E[bin] >= min_p exp(d_max), exp(d) in [1, e^(1/32)): the first bin whose least weight fails may hold
        // some that pass, those behind it none
        const double thr = (double)p.min_p * (double)rb.units(xtop);
        const int b = first_bin(bc != 0u && E * SB_UNIT < thr);
        if (b < SB_BINS) cut(b, find_place(r, rb, part_of(b), BY_VALUE, (unsigned long long)ceil(thr / E_of(b)), sh));
    }
    const float u = a.u ? fminf(fmaxf(a.u[row], 0.0f), 0.99999994f) : 0.0f;
    const int b = bin_of(u);
    Place pl = find_place(r, rb, part_of(b), BY_MASS, target(u, b, false) + 1ull, sh);
    if ((int)cbefore(b) + pl.count > C) pl = find_place(r, rb, part_of(b), BY_COUNT, (unsigned)C - cbefore(b), sh);
    if (tid == 0) {
        a.token[row] = pl.index;
        a.p[row] = (float)((double)rb.units(rb.x(pl.key)) * E_of(b) / W);
        if (a.top) a.top[row] = key_logit(top);
    }
}

hipError_t launch_sample(const SampleArgs& a, int m, hipStream_t st) {
    sample_kernel<<<dim3((unsigned)m), dim3(SB_THREADS), 0, st>>>(a);
    return hipGetLastError();
}

// ------------------------------------------------------------------ drafted tree

// One wave a slot, one lane a node.  A node is reached if its parent is and it
// is the parent's first child whose token is the one sampled there; node 0 is.
// Each step takes the lowest such child, so it goes to a later node and the walk
// ends after at most n steps.
__global__ __launch_bounds__(64) void tree_accept_kernel(const int32_t* __restrict__ parents, const int32_t* __restrict__ tokens,
                                                         const int32_t* __restrict__ sampled, int n, int32_t* __restrict__ count,
                                                         int32_t* __restrict__ path, int32_t* __restrict__ next,
                                                         uint8_t* __restrict__ keep) {
    const int i = threadIdx.x;
    const size_t base = (size_t)blockIdx.x * n;
    const int par = i > 0 && i < n ? parents[base + i] : -1;
    const int tok = i < n ? tokens[base + i] : 0;
    const int smp = i < n ? sampled[base + i] : 0;
    const bool child = par >= 0 && par < i;
    const int asked = __shfl(smp, child ? par : 0);                // by every lane: a lane that is not in step has no value to give
    const bool hit = child && asked == tok;
    unsigned long long kept = 1ull;
    int cur = 0;
    for (;;) {
        const unsigned long long next_of = __ballot(hit && par == cur);
        if (!next_of) break;
        cur = __ffsll(next_of) - 1;
        kept |= 1ull << cur;
    }
    const int c = __popcll(kept);
    const int last = __shfl(smp, cur);
    const bool in = (kept >> i) & 1ull;
    if (in) path[base + __popcll(kept & ((1ull << i) - 1ull))] = i;
    if (i < n) {
        if (i >= c) path[base + i] = -1;
        keep[base + i] = in ? 1 : 0;
    }
    if (i == 0) {
        count[blockIdx.x] = c;
        next[blockIdx.x] = last;
    }
}

hipError_t launch_tree_accept(const int32_t* parents, const int32_t* tokens, const int32_t* sampled, int S, int n, int32_t* count,
                              int32_t* path, int32_t* next, uint8_t* keep, hipStream_t st) {
    if (n < 1 || n > 64) return hipErrorInvalidValue;
    tree_accept_kernel<<<dim3((unsigned)S), dim3(64), 0, st>>>(parents, tokens, sampled, n, count, path, next, keep);
    return hipGetLastError();
}

}  // namespace stg
