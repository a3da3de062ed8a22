// Kernels of the paged cache: attention over runs of pages that rows share, the write of rotated rows, and the moves of
// rows between pages.
#include "paged.h"
#include "device.h"

namespace stg {

namespace {

typedef __bf16 bf16x8_t __attribute__((ext_vector_type(8)));
typedef _Float16 half8_t __attribute__((ext_vector_type(8)));
typedef float f32x16_t __attribute__((ext_vector_type(16)));
typedef float f32x4_t __attribute__((ext_vector_type(4)));
typedef f32x4_t __attribute__((aligned(1))) f32x4_any;
typedef uint16_t u16x4 __attribute__((ext_vector_type(4)));

// Loads whose address is the same in every lane, of memory that no kernel running beside writes: scalar loads, which do
// not queue behind the cache rows on their way to LDS.
template <class T>
__device__ __forceinline__ T uniform_load(const T* p, size_t i) {
    const auto* w = (const __attribute__((address_space(4))) uint32_t*)(uintptr_t)(p + i);
    uint32_t b[sizeof(T) / 4];
#pragma unroll
    for (size_t j = 0; j < sizeof(T) / 4; ++j) b[j] = w[j];
    return __builtin_bit_cast(T, b);
}

template <int KVDT>
__device__ __forceinline__ f32x16_t mma32(const u32x4& a, const u32x4& b, f32x16_t c) {
    if constexpr (KVDT == DT_BF16)
        return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8_t, a), __builtin_bit_cast(bf16x8_t, b), c, 0, 0, 0);
    else
        return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(half8_t, a), __builtin_bit_cast(half8_t, b), c, 0, 0, 0);
}
template <int KVDT>
__device__ __forceinline__ f32x4_t mma16(const u32x4& a, const u32x4& b, f32x4_t c) {
    if constexpr (KVDT == DT_BF16)
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, a), __builtin_bit_cast(bf16x8_t, b), c, 0, 0, 0);
    else
        return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(half8_t, a), __builtin_bit_cast(half8_t, b), c, 0, 0, 0);
}
template <int KVDT>
__device__ __forceinline__ float kv_float(uint16_t b) { return KVDT == DT_BF16 ? bf16_to_f32(b) : f16_to_f32(b); }
// Two floats rounded to the cache dtype and packed, low half first.
template <int KVDT>
__device__ __forceinline__ uint32_t pack2(float lo, float hi) {
    if constexpr (KVDT == DT_BF16) {
        typedef __bf16 bf16x2_t __attribute__((ext_vector_type(2)));
        const bf16x2_t v = {(__bf16)lo, (__bf16)hi};
        return __builtin_bit_cast(uint32_t, v);
    } else {
        return pack_f16x2(lo, hi);
    }
}
// The value of this lane and of lane ^ 32, the lower lane's first.
__device__ __forceinline__ void halves(float v, float& lo, float& hi) {
    const uint32_t u = __float_as_uint(v);
    const auto r = __builtin_amdgcn_permlane32_swap(u, u, false, false);
    lo = __uint_as_float(r[0]);
    hi = __uint_as_float(r[1]);
}
__device__ __forceinline__ void quarters(float v, float& lo, float& hi) {   // and of lane ^ 16
    const uint32_t u = __float_as_uint(v);
    const auto r = __builtin_amdgcn_permlane16_swap(u, u, false, false);
    lo = __uint_as_float(r[0]);
    hi = __uint_as_float(r[1]);
}
// Over the lanes of a query vector: 2 (32 apart) or 4 (16 apart).
template <int LANES>
__device__ __forceinline__ float lanes_max(float v) {
    float lo, hi;
    halves(v, lo, hi);
    v = fmaxf(lo, hi);
    if constexpr (LANES == 4) {
        quarters(v, lo, hi);
        v = fmaxf(lo, hi);
    }
    return v;
}
__device__ __forceinline__ float lanes_sum4(float v) {
    float lo, hi;
    halves(v, lo, hi);
    v = lo + hi;
    quarters(v, lo, hi);
    return lo + hi;
}

// ------------------------------------------------------------------ attention
//
// o = sum_j w_j v_j / sum_j w_j, w_j = exp(s_j - max), in one pass over the keys with the running maximum and sum.  A
// workgroup takes a tile of the query vectors of one kv head (rows x heads of the group) and a run of keys.  Scores are
// S^T = K Q^T, so that a lane holds scores of one query vector and P^T is, as it lies, the second operand of
// O^T += V^T P^T; V^T comes from LDS transpose reads.  Rows go from the pages to LDS by direct loads; 16-byte chunk c of a
// row lies at c ^ f(row), so that neither read meets a bank more often than it has to.
// Queries of the cache's type enter as they are, fp32 ones as two terms of it (QT = 2).


template <int D>
__device__ __forceinline__ int swz_k(int row) { return D == 128 ? row & 15 : (row >> 1) & 7; }
template <int D>
__device__ __forceinline__ int swz_v(int row) { return D == 128 ? 2 * (row & 7) : 2 * ((row >> 1) & 3); }

// The value, as one that is only known here: what is computed from it is not kept in registers through a loop.
__device__ __forceinline__ uint32_t here(uint32_t v) {
    asm volatile("" : "+v"(v));
    return v;
}

// This lane's part of the direct loads of 16 rows of a page, a kilobyte (1024 / (2 D) rows) an instruction: byte offsets
// into the rows, for K and V.
template <int D>
__device__ __forceinline__ uint32_t lane_k() { const int l = threadIdx.x & 63, r = l / (D / 8); return r * 2 * D + 16 * (l % (D / 8) ^ swz_k<D>(r)); }
template <int D>
__device__ __forceinline__ uint32_t lane_v() { const int l = threadIdx.x & 63, r = l / (D / 8); return r * 2 * D + 16 * (l % (D / 8) ^ swz_v<D>(r)); }
// 16 rows at src (the same in every lane) to LDS.  The instruction's offset moves both places; a later kilobyte's swizzle is
// the first's with one bit turned.
template <int D, bool ISV>
__device__ __forceinline__ void load_rows16(const uint8_t* src, uint32_t lane_off, uint8_t* lds) {
    lane_off = here(lane_off);
    constexpr auto turn = [](int u) { return ISV ? (D == 128 ? 128 * (u & 1) : 0) : 64 * u; };
#define PAGED_LOAD(U)                                                                                                             \
    __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)(src + (lane_off ^ turn(U))),                \
                                     (__attribute__((address_space(3))) void*)lds, 16, 1024 * U, 0)
    PAGED_LOAD(0);
    PAGED_LOAD(1);
    if constexpr (D == 128) {
        PAGED_LOAD(2);
        PAGED_LOAD(3);
    }
#undef PAGED_LOAD
}
__device__ __forceinline__ uint32_t lds_addr(const void* p) { return (uint32_t)(uintptr_t)(const __attribute__((address_space(3))) void*)p; }

template <int N>
__device__ __forceinline__ void wait_loads() { asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory"); }
__device__ __forceinline__ void bare_barrier() { asm volatile("s_barrier" ::: "memory"); }

// LDS reads with the wait for them: with reads of the compiler's own it would also wait for the loads to LDS in flight.
// Fragment t of K lies at k ^ (S t), fragments of V (transposed: one lane, four keys) at v ^ (S t).
template <int D>
__device__ __forceinline__ void read_k16(uint32_t k, u32x4* f) {
    if constexpr (D == 128)
        asm volatile("ds_read_b128 %0, %4\n\tds_read_b128 %1, %5\n\tds_read_b128 %2, %6\n\tds_read_b128 %3, %7\n\ts_waitcnt lgkmcnt(0)"
                     : "=&v"(f[0]), "=&v"(f[1]), "=&v"(f[2]), "=&v"(f[3])
                     : "v"(k), "v"(k ^ 64u), "v"(k ^ 128u), "v"(k ^ 192u)
                     : "memory");
    else
        asm volatile("ds_read_b128 %0, %2\n\tds_read_b128 %1, %3\n\ts_waitcnt lgkmcnt(0)"
                     : "=&v"(f[0]), "=&v"(f[1])
                     : "v"(k), "v"(k ^ 64u)
                     : "memory");
}
__device__ __forceinline__ void read_v16(uint32_t v, u32x2* f) {   // 64 dims
    asm volatile(
        "ds_read_b64_tr_b16 %0, %4\n\tds_read_b64_tr_b16 %1, %5\n\tds_read_b64_tr_b16 %2, %6\n\tds_read_b64_tr_b16 %3, %7\n\t"
        "s_waitcnt lgkmcnt(0)"
        : "=&v"(f[0]), "=&v"(f[1]), "=&v"(f[2]), "=&v"(f[3])
        : "v"(v), "v"(v ^ 32u), "v"(v ^ 64u), "v"(v ^ 96u)
        : "memory");
}
__device__ __forceinline__ void read_k32(uint32_t k, u32x4* f, bool upper) {
    const uint32_t x = upper ? k ^ 128u : k;
    asm volatile("ds_read_b128 %0, %4\n\tds_read_b128 %1, %5\n\tds_read_b128 %2, %6\n\tds_read_b128 %3, %7\n\ts_waitcnt lgkmcnt(0)"
                 : "=&v"(f[0]), "=&v"(f[1]), "=&v"(f[2]), "=&v"(f[3])
                 : "v"(x), "v"(x ^ 32u), "v"(x ^ 64u), "v"(x ^ 96u)
                 : "memory");
}
// Two 32-dim fragments (at v and v ^ 64) of 32 keys: four reads each, 8 keys apart (RB bytes a row).
template <int RB>
__device__ __forceinline__ void read_v32(uint32_t v, u32x2* f) {
    asm volatile(
        "ds_read_b64_tr_b16 %0, %8\n\tds_read_b64_tr_b16 %1, %8 offset:%10\n\tds_read_b64_tr_b16 %2, %8 offset:%11\n\t"
        "ds_read_b64_tr_b16 %3, %8 offset:%12\n\tds_read_b64_tr_b16 %4, %9\n\tds_read_b64_tr_b16 %5, %9 offset:%10\n\t"
        "ds_read_b64_tr_b16 %6, %9 offset:%11\n\tds_read_b64_tr_b16 %7, %9 offset:%12\n\ts_waitcnt lgkmcnt(0)"
        : "=&v"(f[0]), "=&v"(f[1]), "=&v"(f[2]), "=&v"(f[3]), "=&v"(f[4]), "=&v"(f[5]), "=&v"(f[6]), "=&v"(f[7])
        : "v"(v), "v"(v ^ 64u), "n"(8 * RB), "n"(16 * RB), "n"(24 * RB)
        : "memory");
}

// Bits 15 and 31: the halves of x whose exponent is all ones (no number).
template <int KVDT>
__device__ __forceinline__ uint32_t not_numbers(uint32_t x) {
    constexpr uint32_t E = KVDT == DT_BF16 ? 0x7f807f80u : 0x7c007c00u, A = KVDT == DT_BF16 ? 0x00800080u : 0x04000400u;
    return ((x & E) + A) & 0x80008000u;
}

// A query vector's fragments: values first + stride t .. + 7.  fp32 ones are divided by a power of two that brings the
// vector's largest magnitude to [1, 2), which is returned: no term leaves the range of 16-bit floats, whatever its size.
template <int KVDT, int QT, int NT, int LANES>
__device__ __forceinline__ float load_query(const PagedAttend& a, size_t at, int stride, u32x4 (&qf)[QT][NT]) {
    if constexpr (QT == 1) {
        const uint16_t* q = (const uint16_t*)a.q + at;
#pragma unroll
        for (int t = 0; t < NT; ++t) qf[0][t] = *(const u32x4_any*)(q + stride * t);
        return 1.f;
    } else {
        const float* q = (const float*)a.q + at;
        float x[NT][8], top = 0.f;
#pragma unroll
        for (int t = 0; t < NT; ++t) {
            *(f32x4_t*)&x[t][0] = *(const f32x4_any*)(q + stride * t);
            *(f32x4_t*)&x[t][4] = *(const f32x4_any*)(q + stride * t + 4);
        }
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
            for (int e = 0; e < 8; ++e) top = fmaxf(top, fabsf(x[t][e]));
        top = lanes_max<LANES>(top);
        const int e = (int)((__float_as_uint(top) >> 23) & 255) - 127, ec = e > 126 ? 126 : e < -126 ? -126 : e;
        const float inv = __uint_as_float((uint32_t)(127 - ec) << 23);
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
            for (int w = 0; w < 4; ++w) {
                const float x0 = x[t][2 * w] * inv, x1 = x[t][2 * w + 1] * inv;
                const uint32_t b = pack2<KVDT>(x0, x1);
                qf[0][t][w] = b;
                qf[QT - 1][t][w] = pack2<KVDT>(x0 - kv_float<KVDT>((uint16_t)b), x1 - kv_float<KVDT>((uint16_t)(b >> 16)));
            }
        return __uint_as_float((uint32_t)(127 + ec) << 23);
    }
}

// Four neighbouring dims of a query vector's result: a partial one, or times inv to out.
template <int D>
__device__ __forceinline__ void put_result(const PagedAttend& a, const PagedRow& r, size_t part, int head, int d, const f32x4_t& v, float inv) {
    if (r.nparts > 1) {
        *(f32x4_t*)(a.part_o + part * D + d) = v;
        return;
    }
    const size_t at = (size_t)r.row * a.ldo + (size_t)head * D + d;
    if (a.out_dt == DT_F32) {
        *(f32x4_any*)((float*)a.out + at) = v * inv;
    } else {
        const f32x4_t x = v * inv;
        *(u32x2_any*)((uint16_t*)a.out + at) = a.out_dt == DT_BF16 ? u32x2{pack2<DT_BF16>(x[0], x[1]), pack2<DT_BF16>(x[2], x[3])}
                                                                   : u32x2{pack2<DT_F16>(x[0], x[1]), pack2<DT_F16>(x[2], x[3])};
    }
}

// The bits of a step of AK keys from key k0 on that lie in the item's run, and of those the ones below `limit`.
template <int AK>
__device__ __forceinline__ uint32_t run_bits(int kb, int ke, int k0) {
    const int lo = max(kb - k0, 0), hi = min(ke - k0, AK);
    return hi <= lo ? 0u : (~0u >> (32 - (hi - lo))) << lo;
}
__device__ __forceinline__ uint32_t bits_below(int n) { return n <= 0 ? 0u : n >= 32 ? ~0u : ~0u >> (32 - n); }

// ---- tiles of up to 64 query vectors
//
// Decoding rows, verifies, and what they share.  The four waves are NQT tiles of 16 query vectors by KG = 4 / NQT key
// groups, which take alternate steps and are merged through LDS.  A step is 16 keys (one page's), or 32 where the four
// waves share it: what a step costs beside its products is then half.  Bound by memory: what counts is bytes in flight, so
// a wave holds at most 128 registers and a workgroup 33 KB of LDS, and four workgroups share a CU (16 x 8 KB under way).
// A wave with a buffer of one step (NQT = 1, D = 128) reads all of it into registers before it asks for the next;
// otherwise each key group has a ring of NB steps.  A probability enters as its rounded part and the residual (2^-17 in
// bf16), in one product: the second operand's 32 k slots hold 16 keys twice, those of V^T repeat them.
template <int D, int KVDT, int QT, int NQT>
__device__ __forceinline__ void few_item(const PagedAttend& a, const PagedItem& it, int g, uint8_t* lds, float2* sml) {
    constexpr int H = NQT == 4 ? 2 : 1, AK = 16 * H;   // 16-key parts of a step
    constexpr int RB = 2 * D, SB = AK * RB, KT = D / 32, MB = D / 16;
    constexpr int KG = 4 / NQT, NB = 128 * 256 / (KG * 2 * SB);   // key groups; steps that a group's ring holds
    constexpr int NL = (NQT == 1 ? 2 : 1) * 16 * RB / 1024;   // loads of a wave and step
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int qt = wave % NQT, kg = wave / NQT, ql = lane & 15, lg = lane >> 4;
    const int Hq = a.Hkv * a.gs, pmask = (1 << a.shift) - 1;
    const int s0 = it.kb / AK, s1 = (it.ke + AK - 1) / AK, turns = (s1 - s0 + KG - 1) / KG;
    uint8_t* ring = lds + kg * NB * 2 * SB;

    const int c0 = it.q0 + 16 * qt + ql;
    int limit, mask;                               // of the lane's row
    {
        const PagedRow* r = a.list + it.rows + min(c0, it.q0 + it.nq - 1) / a.gs;
        limit = r->limit;
        mask = r->mask;
    }

    // Step i of the group: with one tile the wave loads K and V; of two waves one K, one V; of four, of 16 rows each.  Every
    // row of a page may be read.
    const size_t head_at = ((size_t)g << a.shift) * RB, page_bytes = ((size_t)a.Hkv << a.shift) * RB;
    const uint32_t lk = lane_k<D>(), lv = lane_v<D>();
    const bool loads_v = NQT == 1 || (NQT == 2 ? qt == 1 : qt >= 2), loads_k = NQT == 1 || !loads_v;
    const int part16 = NQT == 4 ? qt & 1 : 0;
    auto issue = [&](int i) {
        const int key = AK * (s0 + kg + KG * i) + 16 * part16;
        const int page = uniform_load(a.tables, (size_t)it.table + (min(key, it.ke - 1) >> a.shift));
        const size_t at = (size_t)page * page_bytes + head_at + (size_t)(key & pmask) * RB;
        uint8_t* buf = ring + (NB > 1 ? i % NB : 0) * 2 * SB + part16 * 16 * RB;
        if (loads_k) load_rows16<D, false>((const uint8_t*)a.k + at, lk, buf);
        if (loads_v) load_rows16<D, true>((const uint8_t*)a.v + at, lv, buf + SB);
    };
#pragma unroll
    for (int i = 0; i < (NB > 1 ? NB - 1 : 1); ++i)
        if (i < turns) issue(i);

    u32x4 qf[QT][KT];
    float sc = a.scale2;
    {
        const int cq = min(c0, it.q0 + it.nq - 1);
        sc *= load_query<KVDT, QT, KT, 4>(a, (size_t)a.list[it.rows + cq / a.gs].row * a.ldq + (size_t)(g * a.gs + cq % a.gs) * D + 8 * lg, 32, qf);
    }

    const uint32_t ka = lds_addr(ring) + ql * RB + 16 * (lg ^ swz_k<D>(ql));
    const int vkey = 4 * lg + (ql >> 2);
    const uint32_t va = lds_addr(ring) + SB + vkey * RB + 16 * (swz_v<D>(vkey) + ((ql & 3) >> 1)) + 8 * (ql & 1);

    float base = -INFINITY, lsum = 0.f;            // the largest score so far (before scaling), the sum of the probabilities
    f32x4_t o[MB];
#pragma unroll
    for (int mb = 0; mb < MB; ++mb) o[mb] = f32x4_t{0.f, 0.f, 0.f, 0.f};

    for (int i = 0; i < turns; ++i) {
        const int k0 = AK * (s0 + kg + KG * i);
        if constexpr (NB > 1) {
            if (i + NB - 2 < turns) wait_loads<(NB - 2) * NL>();   // this wave's loads of step i are there
            else wait_loads<0>();
            if constexpr (NQT > 1) bare_barrier();                 // every wave's are, and the buffer of step i - 1 has been read
            if (i + NB - 1 < turns) issue(i + NB - 1);
        } else {
            wait_loads<0>();
        }
        const bool whole = it.open && k0 >= it.kb && k0 + AK <= it.ke;
        uint32_t in = ~0u, see = ~0u;              // keys of the step in the run; those that this lane's query vector sees
        bool work = true;
        if (!whole) {
            in = run_bits<AK>(it.kb, it.ke, k0);
            see = in & bits_below(limit - k0);
            if (mask >= 0 && see) see &= a.masks[(size_t)mask + k0 / 32] >> (H == 1 ? k0 & 16 : 0);
            work = __any(see != 0u);
        }
        f32x4_t s[H];
        u32x2 vf[MB];
        const uint32_t off = NB > 1 ? i % NB * (2 * SB) : 0;
        auto read_v = [&](int h) {
            const uint32_t v = here(va + off + h * 16 * RB);
            read_v16(v, vf);
            if constexpr (MB == 8) read_v16(v ^ 128u, vf + 4);
        };
        if (work) {
#pragma unroll
            for (int h = 0; h < H; ++h) {
                u32x4 kf[KT];
                read_k16<D>(here(ka + off + h * 16 * RB), kf);
                s[h] = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int t = 0; t < KT; ++t) {
                    s[h] = mma16<KVDT>(kf[t], qf[0][t], s[h]);
                    if constexpr (QT == 2) s[h] = mma16<KVDT>(kf[t], qf[1][t], s[h]);
                }
            }
            if constexpr (H == 1) read_v(0);
        }
        if constexpr (NB == 1) {
            if (i + 1 < turns) issue(i + 1);       // the buffer is read
        }
        if (!work) continue;
        if (!whole) {
#pragma unroll
            for (int h = 0; h < H; ++h)
#pragma unroll
                for (int j = 0; j < 4; ++j) s[h][j] = (see >> (16 * h + 4 * lg + j)) & 1u ? s[h][j] : -INFINITY;
        }
        float mx = fmaxf(fmaxf(s[0][0], s[0][1]), fmaxf(s[0][2], s[0][3]));
        if constexpr (H == 2) mx = fmaxf(mx, fmaxf(fmaxf(s[1][0], s[1][1]), fmaxf(s[1][2], s[1][3])));
        if (__any(mx > base)) {
            const float top = fmaxf(base, lanes_max<4>(mx));
            const float corr = base == -INFINITY ? 0.f : __builtin_amdgcn_exp2f((base - top) * sc);
            base = top;
            lsum *= corr;
#pragma unroll
            for (int mb = 0; mb < MB; ++mb)
#pragma unroll
                for (int j = 0; j < 4; ++j) o[mb][j] *= corr;
        }
        const float nb = base == -INFINITY ? 0.f : -base * sc;
        uint32_t bad = 0u;
#pragma unroll
        for (int h = 0; h < H; ++h) {
#pragma unroll
            for (int j = 0; j < 4; ++j) s[h][j] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[h][j], sc, nb));   // the probabilities
            lsum += (s[h][0] + s[h][1]) + (s[h][2] + s[h][3]);
            if constexpr (H == 2) read_v(h);
            if (!whole) {
                // Rows outside the run enter as zeros: what they hold is nobody's.  Of the others, a value that is no number
                // must reach the query vectors that see it and no other (0 times it is no number either): it is taken out
                // of the products and added where it is seen.
                uint32_t m[2];
#pragma unroll
                for (int w = 0; w < 2; ++w) {
                    const uint32_t bits = in >> (16 * h + 4 * lg + 2 * w);
                    m[w] = (bits & 1u ? 0xFFFFu : 0u) | (bits & 2u ? 0xFFFF0000u : 0u);
                }
#pragma unroll
                for (int mb = 0; mb < MB; ++mb)
#pragma unroll
                    for (int w = 0; w < 2; ++w) {
                        const uint32_t x = vf[mb][w] & m[w], no = not_numbers<KVDT>(x);
                        vf[mb][w] = x & ~((no >> 15) * 0xFFFFu);
                        bad |= no;
                    }
            }
            u32x4 pb;
#pragma unroll
            for (int w = 0; w < 2; ++w) {
                const float p0 = s[h][2 * w], p1 = s[h][2 * w + 1];
                pb[w] = pack2<KVDT>(p0, p1);
                pb[2 + w] = pack2<KVDT>(p0 - kv_float<KVDT>((uint16_t)pb[w]), p1 - kv_float<KVDT>((uint16_t)(pb[w] >> 16)));
            }
#pragma unroll
            for (int mb = 0; mb < MB; ++mb) o[mb] = mma16<KVDT>(u32x4{vf[mb][0], vf[mb][1], vf[mb][0], vf[mb][1]}, pb, o[mb]);
        }
        if (!whole && __any(bad != 0u)) {
#pragma unroll 1
            for (int key = 0; key < AK; ++key) {
                if (!((in >> key) & 1u)) continue;
                float p = 0.f;
#pragma unroll
                for (int j = 0; j < 4 * H; ++j) p = (key & 3) + key / 16 * 4 == j ? s[j / 4][j % 4] : p;
                p = __shfl(p, 16 * ((key >> 2) & 3) + ql);
                const int page = uniform_load(a.tables, (size_t)it.table + ((k0 + key) >> a.shift));
                const uint16_t* vr = a.v + ((((size_t)page * a.Hkv + g) << a.shift) + ((k0 + key) & pmask)) * D + here(4 * lg);
                if ((see >> key) & 1u) {
#pragma unroll
                    for (int mb = 0; mb < MB; ++mb) {
                        const u16x4 x = *(const u16x4*)(vr + 16 * mb);
#pragma unroll
                        for (int e = 0; e < 4; ++e)
                            if (not_numbers<KVDT>(x[e])) o[mb][e] += p * kv_float<KVDT>(x[e]);
                    }
                }
            }
        }
    }

    // ---- results: dims 16 mb + 4 lg .. + 3 of the lane's query vector
    lsum = lanes_sum4(lsum);
    base = base == -INFINITY ? base : base * sc;
    int cq = min(c0, it.q0 + it.nq - 1);
    asm volatile("" : "+v"(cq));                   // its row is read again: it need not stay in registers through the loop
    const PagedRow ri = a.list[it.rows + cq / a.gs];
    const int head = g * a.gs + cq % a.gs;
    const bool mine = c0 < it.q0 + it.nq && it.slot < ri.nparts;   // (a row that ends before this run has no part of it)
    const size_t part = ((size_t)(ri.part + it.slot) * Hq + head);
    if constexpr (KG == 1) {
        if (!mine) return;
        if (ri.nparts > 1 && lg == 0) a.part_ml[part] = float2{base, lsum};
        const float inv = lsum == 0.f ? 0.f : 1.0f / lsum;
#pragma unroll
        for (int mb = 0; mb < MB; ++mb) put_result<D>(a, ri, part, head, 16 * mb + 4 * lg, o[mb], inv);
    } else {
        __syncthreads();                           // every wave has read its last step
        f32x4_t* so = (f32x4_t*)lds;               // [wave][MB][64]
        if (lg == 0) sml[wave * 16 + ql] = float2{base, lsum};
#pragma unroll
        for (int mb = 0; mb < MB; ++mb) so[(wave * MB + mb) * 64 + lane] = o[mb];
        __syncthreads();
        if (!mine) return;
        float top = -INFINITY, sum = 0.f, f[KG];
#pragma unroll
        for (int k = 0; k < KG; ++k) top = fmaxf(top, sml[(k * NQT + qt) * 16 + ql].x);
#pragma unroll
        for (int k = 0; k < KG; ++k) {
            const float2 ml = sml[(k * NQT + qt) * 16 + ql];
            f[k] = ml.x == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(ml.x - top);
            sum += ml.y * f[k];
        }
        if (ri.nparts > 1 && lg == 0 && kg == 0) a.part_ml[part] = float2{top, sum};
        const float inv = sum == 0.f ? 0.f : 1.0f / sum;
#pragma unroll
        for (int u = 0; u < MB / KG; ++u) {        // the tile's waves share its dims
            const int mb = kg + KG * u;
            f32x4_t v = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int k = 0; k < KG; ++k) v += so[((k * NQT + qt) * MB + mb) * 64 + lane] * f[k];
            put_result<D>(a, ri, part, head, 16 * mb + 4 * lg, v, inv);
        }
    }
}

template <int D, int KVDT, int QT>
__global__ __launch_bounds__(256, 4) void paged_few_kernel(PagedAttend a) {
    __shared__ __attribute__((aligned(1024))) uint8_t lds[128 * 256];
    __shared__ float2 sml[64];
    const int b = __builtin_amdgcn_readfirstlane(blockIdx.x / a.Hkv), g = __builtin_amdgcn_readfirstlane(blockIdx.x % a.Hkv);
    const PagedItem it = uniform_load(a.items, b);
    if (it.nq <= 16) few_item<D, KVDT, QT, 1>(a, it, g, lds, sml);
    else if (it.nq <= 32) few_item<D, KVDT, QT, 2>(a, it, g, lds, sml);
    else few_item<D, KVDT, QT, 4>(a, it, g, lds, sml);
}

// ---- tiles of up to 128 query vectors
//
// Prompts.  A wave takes 32 query vectors and every key of the run, on 32 x 32 x 16 products; the four waves share steps of
// 32 keys in a ring of four.  Bound by the matrix cores and, as much, by LDS (a wave reads a step for 32 query vectors) and
// the exponentials.  P: terms of a probability (1: rounded to the cache's type, while the sum keeps it whole).
template <int D, int KVDT, int QT, int PT>
__global__ __launch_bounds__(256, 2) void paged_many_kernel(PagedAttend a) {
    constexpr int AK = 32, RB = 2 * D, SB = AK * RB, KT = D / 16, MB = D / 32, NB = 4;
    constexpr int NL = 2 * SB / 1024 / 4;          // kilobytes of a step that a wave loads
    __shared__ __attribute__((aligned(1024))) uint8_t ring[NB * 2 * SB];
    const int b = __builtin_amdgcn_readfirstlane(blockIdx.x / a.Hkv), g = __builtin_amdgcn_readfirstlane(blockIdx.x % a.Hkv);
    const PagedItem it = uniform_load(a.items, a.n_few + b);
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int ql = lane & 31, h = lane >> 5;
    const int Hq = a.Hkv * a.gs, pmask = (1 << a.shift) - 1;
    const int s0 = it.kb / AK, turns = (it.ke + AK - 1) / AK - s0;

    const int c0 = it.q0 + 32 * wave + ql;
    int limit, mask;
    {
        const PagedRow* r = a.list + it.rows + min(c0, it.q0 + it.nq - 1) / a.gs;
        limit = r->limit;
        mask = r->mask;
    }

    const size_t head_at = ((size_t)g << a.shift) * RB, page_bytes = ((size_t)a.Hkv << a.shift) * RB;
    const uint32_t lane_at = wave < 2 ? lane_k<D>() : lane_v<D>();
    auto issue = [&](int i) {                      // waves 0, 1: 16 rows of K each; 2, 3: of V
        const int key = AK * (s0 + i) + (wave & 1) * 16;
        const int page = uniform_load(a.tables, (size_t)it.table + (min(key, it.ke - 1) >> a.shift));
        const size_t at = (size_t)page * page_bytes + head_at + (size_t)(key & pmask) * RB;
        uint8_t* buf = ring + i % NB * 2 * SB + (wave & 1) * 16 * RB;
        if (wave < 2) load_rows16<D, false>((const uint8_t*)a.k + at, lane_at, buf);
        else load_rows16<D, true>((const uint8_t*)a.v + at, lane_at, buf + SB);
    };
#pragma unroll
    for (int i = 0; i < NB - 1; ++i)
        if (i < turns) issue(i);

    u32x4 qf[QT][KT];
    float sc = a.scale2;
    {
        const int cq = min(c0, it.q0 + it.nq - 1);
        sc *= load_query<KVDT, QT, KT, 2>(a, (size_t)a.list[it.rows + cq / a.gs].row * a.ldq + (size_t)(g * a.gs + cq % a.gs) * D + 8 * h, 16, qf);
    }

    const uint32_t ka = lds_addr(ring) + ql * RB + 16 * (h ^ swz_k<D>(ql));
    const int j16 = lane & 15, vkey = 4 * h + (j16 >> 2);   // keys 8 apart have the same place
    const uint32_t va = lds_addr(ring) + SB + vkey * RB + 16 * ((2 * ((lane >> 4) & 1)) ^ swz_v<D>(vkey)) + 16 * ((j16 & 3) >> 1) + 8 * (j16 & 1);

    float base = -INFINITY, lsum = 0.f;
    f32x16_t o[MB];
#pragma unroll
    for (int mb = 0; mb < MB; ++mb)
#pragma unroll
        for (int r = 0; r < 16; ++r) o[mb][r] = 0.f;

    for (int i = 0; i < turns; ++i) {
        const int k0 = AK * (s0 + i);
        if (i + NB - 2 < turns) wait_loads<(NB - 2) * NL>();
        else wait_loads<0>();
        bare_barrier();
        if (i + NB - 1 < turns) issue(i + NB - 1);
        uint32_t in = ~0u, see = ~0u;
        bool whole = it.open && k0 >= it.kb && k0 + AK <= it.ke, work = true;
        if (!whole) {
            in = run_bits<AK>(it.kb, it.ke, k0);
            see = in & bits_below(limit - k0);
            if (mask >= 0 && see) see &= a.masks[(size_t)mask + k0 / 32];
            work = __any(see != 0u);
            whole = !__any(see != ~0u);            // a prompt's rows see whole steps well before their own keys
        }
        if (!work) continue;
        const uint32_t off = i % NB * (2 * SB);
        u32x4 kf[KT];
        f32x16_t s;
#pragma unroll
        for (int r = 0; r < 16; ++r) s[r] = 0.f;
#pragma unroll
        for (int t = 0; t < KT; t += 4) {
            read_k32(here(ka + off), kf + t, t != 0);
#pragma unroll
            for (int u = t; u < t + 4; ++u) {
                s = mma32<KVDT>(kf[u], qf[0][u], s);
                if constexpr (QT == 2) s = mma32<KVDT>(kf[u], qf[1][u], s);
            }
        }
        u32x4 vf[MB][2];
#pragma unroll
        for (int mb = 0; mb < MB; mb += 2) {
            u32x2 p[8];
            read_v32<RB>(here((va + off) ^ (64u * mb)), p);
#pragma unroll
            for (int e = 0; e < 4; ++e) vf[mb + e / 2][e % 2] = u32x4{p[2 * e][0], p[2 * e][1], p[2 * e + 1][0], p[2 * e + 1][1]};
        }
        if (!whole) {
            const uint32_t x = see >> (4 * h);
#pragma unroll
            for (int r = 0; r < 16; ++r) s[r] = (x >> (8 * (r / 4) + r % 4)) & 1u ? s[r] : -INFINITY;
        }
        float mx = s[0];
#pragma unroll
        for (int r = 1; r < 16; ++r) mx = fmaxf(mx, s[r]);
        if (__any(mx > base)) {
            const float top = fmaxf(base, lanes_max<2>(mx));
            const float corr = base == -INFINITY ? 0.f : __builtin_amdgcn_exp2f((base - top) * sc);
            base = top;
            lsum *= corr;
#pragma unroll
            for (int mb = 0; mb < MB; ++mb)
#pragma unroll
                for (int r = 0; r < 16; ++r) o[mb][r] *= corr;
        }
        const float nb = base == -INFINITY ? 0.f : -base * sc;
        float pv[16];
#pragma unroll
        for (int r = 0; r < 16; ++r) pv[r] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[r], sc, nb));
        lsum += (((pv[0] + pv[1]) + (pv[2] + pv[3])) + ((pv[4] + pv[5]) + (pv[6] + pv[7]))) +
                (((pv[8] + pv[9]) + (pv[10] + pv[11])) + ((pv[12] + pv[13]) + (pv[14] + pv[15])));
        uint32_t bad = 0u;
        if (!whole) {                              // as in few_item
#pragma unroll
            for (int t = 0; t < 2; ++t)
#pragma unroll
                for (int w = 0; w < 4; ++w) {
                    const uint32_t bits = in >> (16 * t + 8 * (w >> 1) + 4 * h + 2 * (w & 1));
                    const uint32_t m = (bits & 1u ? 0xFFFFu : 0u) | (bits & 2u ? 0xFFFF0000u : 0u);
#pragma unroll
                    for (int mb = 0; mb < MB; ++mb) {
                        const uint32_t x = vf[mb][t][w] & m, no = not_numbers<KVDT>(x);
                        vf[mb][t][w] = x & ~((no >> 15) * 0xFFFFu);
                        bad |= no;
                    }
                }
        }
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            u32x4 pb, pr;
#pragma unroll
            for (int w = 0; w < 4; ++w) {
                const float p0 = pv[8 * t + 2 * w], p1 = pv[8 * t + 2 * w + 1];
                pb[w] = pack2<KVDT>(p0, p1);
                if constexpr (PT == 2)
                    pr[w] = pack2<KVDT>(p0 - kv_float<KVDT>((uint16_t)pb[w]), p1 - kv_float<KVDT>((uint16_t)(pb[w] >> 16)));
            }
#pragma unroll
            for (int mb = 0; mb < MB; ++mb) {
                o[mb] = mma32<KVDT>(vf[mb][t], pb, o[mb]);
                if constexpr (PT == 2) o[mb] = mma32<KVDT>(vf[mb][t], pr, o[mb]);
            }
        }
        if (!whole && __any(bad != 0u)) {
#pragma unroll 1
            for (int key = 0; key < AK; ++key) {
                if (!((in >> key) & 1u)) continue;
                float p = 0.f;
#pragma unroll
                for (int r = 0; r < 16; ++r) p = 4 * (key / 8) + key % 4 == r ? pv[r] : p;
                p = __shfl(p, 32 * ((key >> 2) & 1) + ql);
                const int page = uniform_load(a.tables, (size_t)it.table + ((k0 + key) >> a.shift));
                const uint16_t* vr = a.v + ((((size_t)page * a.Hkv + g) << a.shift) + ((k0 + key) & pmask)) * D + here(4 * h);
                if ((see >> key) & 1u) {
#pragma unroll
                    for (int mb = 0; mb < MB; ++mb)
#pragma unroll
                        for (int r4 = 0; r4 < 4; ++r4) {
                            const u16x4 x = *(const u16x4*)(vr + 32 * mb + 8 * r4);
#pragma unroll
                            for (int e = 0; e < 4; ++e)
                                if (not_numbers<KVDT>(x[e])) o[mb][4 * r4 + e] += p * kv_float<KVDT>(x[e]);
                        }
                }
            }
        }
    }

    // ---- results: dims 32 mb + 8 r4 + 4 h .. + 3 of the lane's query vector
    {
        float lo, hi;
        halves(lsum, lo, hi);
        lsum = lo + hi;
    }
    base = base == -INFINITY ? base : base * sc;
    int cq = min(c0, it.q0 + it.nq - 1);
    asm volatile("" : "+v"(cq));
    const PagedRow ri = a.list[it.rows + cq / a.gs];
    const int head = g * a.gs + cq % a.gs;
    if (c0 >= it.q0 + it.nq || it.slot >= ri.nparts) return;
    const size_t part = ((size_t)(ri.part + it.slot) * Hq + head);
    if (ri.nparts > 1 && h == 0) a.part_ml[part] = float2{base, lsum};
    const float inv = lsum == 0.f ? 0.f : 1.0f / lsum;
#pragma unroll
    for (int mb = 0; mb < MB; ++mb)
#pragma unroll
        for (int r4 = 0; r4 < 4; ++r4)
            put_result<D>(a, ri, part, head, 32 * mb + 8 * r4 + 4 * h, f32x4_t{o[mb][4 * r4], o[mb][4 * r4 + 1], o[mb][4 * r4 + 2], o[mb][4 * r4 + 3]}, inv);
}

// Rows with several partial results: m = max m_r, o = sum o_r 2^(m_r - m) / sum l_r 2^(m_r - m), added in the order of the
// runs.  One wave per row and head; the first eight results are under way before their weights are known.
template <int D>
__global__ __launch_bounds__(256) void paged_merge_kernel(PagedAttend a) {
    constexpr int E = D / 64, U = 8;
    const int lane = threadIdx.x & 63, Hq = a.Hkv * a.gs;
    const int id = __builtin_amdgcn_readfirstlane(4 * blockIdx.x + (threadIdx.x >> 6));
    if (id >= a.M * Hq) return;
    const int row = id / Hq, head = id % Hq;
    const PagedRow ri = uniform_load(a.rows, row);
    const int n = ri.nparts;
    if (n < 2) return;
    const float* po = a.part_o + ((size_t)ri.part * Hq + head) * D + E * lane;
    const float2* pm = a.part_ml + (size_t)ri.part * Hq + head;
    float x[U][E];
    auto load = [&](int p) {
#pragma unroll
        for (int u = 0; u < U; ++u) __builtin_memcpy(x[u], po + (size_t)min(p + u, n - 1) * Hq * D, 4 * E);
    };
    const float2 first = pm[(size_t)min(lane, n - 1) * Hq];
    load(0);
    float top = -INFINITY;
    for (int p0 = 0; p0 < n; p0 += 64) {
        float m = p0 + lane < n ? (p0 ? pm[(size_t)(p0 + lane) * Hq].x : first.x) : -INFINITY;
#pragma unroll
        for (int s = 1; s < 64; s <<= 1) m = fmaxf(m, __shfl_xor(m, s));
        top = fmaxf(top, m);
    }
    float acc[E] = {}, sum = 0.f;
    for (int p0 = 0; p0 < n; p0 += 64) {
        const float2 ml = p0 + lane < n ? (p0 ? pm[(size_t)(p0 + lane) * Hq] : first) : float2{-INFINITY, 0.f};
        const float w = ml.x == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(ml.x - top), l = w * ml.y;
        const int cnt = min(64, n - p0);
        for (int p = 0; p < cnt; p += U) {
            if (p0 + p) load(p0 + p);
#pragma unroll
            for (int u = 0; u < U; ++u) {
                if (p + u >= cnt) break;
                const float wu = __shfl(w, p + u);
                sum += __shfl(l, p + u);
#pragma unroll
                for (int e = 0; e < E; ++e) acc[e] += wu * x[u][e];
            }
        }
    }
    const float inv = sum == 0.f ? 0.f : 1.0f / sum;
    const size_t at = (size_t)row * a.ldo + (size_t)head * D + E * lane;
    if (a.out_dt == DT_F32) {
#pragma unroll
        for (int e = 0; e < E; ++e) ((float*)a.out)[at + e] = acc[e] * inv;
    } else {
#pragma unroll
        for (int e = 0; e < E; ++e) ((uint16_t*)a.out)[at + e] = to_half_bits(acc[e] * inv, a.out_dt);
    }
}

// ------------------------------------------------------------------ the write of new rows
//
// Pair (i, i + D/2) of a q or k head turns by p[axis(i)] theta^(-2i/D) (cos and sin from the stage's table, computed in 64
// bits); k and v go to their rows of the pages.  Bound by memory.  A thread takes four neighbouring pairs, so 16 (or 8)
// threads a head; the angles of a row are read once per thread and reused for the heads that it walks.
template <int D>
__global__ __launch_bounds__(256) void paged_write_kernel(PagedWrite a) {
    constexpr int TPH = D / 8, HPB = 256 / TPH;    // threads a head, heads a step
    const int m = blockIdx.x, i0 = 4 * (threadIdx.x % TPH), heads = a.Hq + 2 * a.Hkv;
    const int stride = HPB * gridDim.y, first = HPB * blockIdx.y + threadIdx.x / TPH;
    const int slot = a.slots[m], page = slot >> a.shift, r = slot & ((1 << a.shift) - 1);
    float2 cs[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) cs[e] = float2{1.f, 0.f};
    if (a.pos) {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const int ax = a.axis ? a.axis[i0 + e] : 0;
            cs[e] = a.rope[(size_t)a.pos[(size_t)ax * a.M + m] * (D / 2) + i0 + e];
        }
    }
    auto load4 = [&](const void* p, size_t at, float (&x)[4]) {
        if (a.dt == DT_F32) {
            *(f32x4_t*)x = *(const f32x4_any*)((const float*)p + at);
        } else {
            const u32x2 b = *(const u32x2_any*)((const uint16_t*)p + at);
#pragma unroll
            for (int e = 0; e < 4; ++e) x[e] = half_bits_to_f32((uint16_t)(b[e >> 1] >> (16 * (e & 1))), a.dt);
        }
    };
    auto store4 = [&](void* p, int dt, size_t at, const float (&x)[4]) {
        if (dt == DT_F32) {
            *(f32x4_any*)((float*)p + at) = *(const f32x4_t*)x;
        } else {
            u32x2 b;
#pragma unroll
            for (int e = 0; e < 2; ++e) b[e] = (uint32_t)to_half_bits(x[2 * e], dt) | ((uint32_t)to_half_bits(x[2 * e + 1], dt) << 16);
            *(u32x2_any*)((uint16_t*)p + at) = b;
        }
    };
    for (int hd = first; hd < heads; hd += stride) {
        const bool isq = hd < a.Hq, isv = hd >= a.Hq + a.Hkv;
        const int g = isq ? hd : isv ? hd - a.Hq - a.Hkv : hd - a.Hq;
        const void* src = isq ? a.q : isv ? a.v : a.k;
        const size_t at = (size_t)m * (isq ? a.ldq : isv ? a.ldv : a.ldk) + (size_t)g * D + i0;
        float x[4], y[4];
        load4(src, at, x);
        load4(src, at + D / 2, y);
        if (!isv) {
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const float u = x[e], w = y[e];
                x[e] = u * cs[e].x - w * cs[e].y;
                y[e] = u * cs[e].y + w * cs[e].x;
            }
        }
        if (isq) {
            const size_t to = (size_t)m * a.ldqo + (size_t)g * D + i0;
            store4(a.q_out, a.q_out_dt, to, x);
            store4(a.q_out, a.q_out_dt, to + D / 2, y);
        } else {
            const size_t to = ((((size_t)page * a.Hkv + g) << a.shift) + r) * D + i0;
            uint16_t* dst = isv ? a.vp : a.kp;
            store4(dst, a.kv_dt, to, x);
            store4(dst, a.kv_dt, to + D / 2, y);
        }
    }
}

// ------------------------------------------------------------------ moves of rows
//
// Bound by memory: a row of one layer, kv head and K or V is D values in one piece, 16 bytes a thread; a workgroup moves
// up to 64 rows of it, four loads a thread in flight.

constexpr int MOVE_ROWS = 64;

// Piece pc of [2 (K, V)][layers][Hkv]: where it begins in the pool's K or V.
__device__ __forceinline__ uint16_t* piece(const PagedPool& p, int pc, size_t& head) {
    const int per = p.layers * p.Hkv, in = pc % per;
    head = in % p.Hkv;
    return (pc < per ? p.k : p.v) + (size_t)(in / p.Hkv) * p.layer_elems();
}
__device__ __forceinline__ size_t slot_at(const PagedPool& p, int slot, size_t head) {
    const int page = slot >> p.shift, r = slot & ((1 << p.shift) - 1);
    return ((((size_t)page * p.Hkv + head) << p.shift) + r) * p.D;
}

__global__ __launch_bounds__(256) void paged_copy_kernel(PagedPool p, const int2* moves, int n, int chunks) {
    const int nch = p.D / 8, rows = 256 / nch, c = threadIdx.x % nch, r0 = (blockIdx.x % chunks) * MOVE_ROWS;
    size_t head;
    uint16_t* base = piece(p, blockIdx.x / chunks, head) + 8 * c;
    const int last = min(r0 + MOVE_ROWS, n);
    for (int r = r0 + threadIdx.x / nch; r < last; r += 4 * rows) {
        int2 mv[4];
        u32x4 x[4];
#pragma unroll
        for (int u = 0; u < 4; ++u) mv[u] = moves[min(r + u * rows, last - 1)];
#pragma unroll
        for (int u = 0; u < 4; ++u) x[u] = *(const u32x4*)(base + slot_at(p, mv[u].x, head));
#pragma unroll
        for (int u = 0; u < 4; ++u)
            if (r + u * rows < last) *(u32x4*)(base + slot_at(p, mv[u].y, head)) = x[u];
    }
}

// One thread moves one 16-byte column of every row, 16 rows at a time: what it has not read yet lies behind what it writes.
__global__ __launch_bounds__(256) void paged_slide_kernel(PagedPool p, const int2* moves, int n, int columns) {
    const int id = blockIdx.x * 256 + threadIdx.x, nch = p.D / 8;
    if (id >= columns) return;
    size_t head;
    uint16_t* base = piece(p, id / nch, head) + 8 * (id % nch);
    for (int r = 0; r < n; r += 16) {
        u32x4 x[16];
#pragma unroll
        for (int u = 0; u < 16; ++u) x[u] = *(const u32x4*)(base + slot_at(p, moves[min(r + u, n - 1)].x, head));
#pragma unroll
        for (int u = 0; u < 16; ++u)
            if (r + u < n) *(u32x4*)(base + slot_at(p, moves[r + u].y, head)) = x[u];
    }
}

__global__ __launch_bounds__(256) void paged_fill_kernel(PagedPool p, const uint16_t* k, const uint16_t* v, const int16_t* table, int S, int slot,
                                                         int cap, int start, const int* slots, int n, int chunks) {
    const int nch = p.D / 8, rows = 256 / nch, c = threadIdx.x % nch, r0 = (blockIdx.x % chunks) * MOVE_ROWS;
    const int pc = blockIdx.x / chunks, per = p.layers * p.Hkv, l = pc % per / p.Hkv;
    size_t head;
    uint16_t* base = piece(p, pc, head) + 8 * c;
    const uint16_t* src = (pc < per ? k : v) + 8 * c;
    const int last = min(r0 + MOVE_ROWS, n);
    for (int r = r0 + threadIdx.x / nch; r < last; r += rows) {
        const int j = start + r, s = table ? table[(size_t)slot * cap + j] : slot;
        *(u32x4*)(base + slot_at(p, slots[r], head)) = *(const u32x4*)(src + ((((size_t)l * S + s) * p.Hkv + head) * cap + j) * p.D);
    }
}

__global__ __launch_bounds__(256) void paged_read_kernel(PagedPool p, int layer, const int* slots, int n, uint16_t* k, uint16_t* v, int chunks) {
    const int nch = p.D / 8, rows = 256 / nch, c = threadIdx.x % nch, r0 = (blockIdx.x % chunks) * MOVE_ROWS;
    const int pc = blockIdx.x / chunks, head = pc % p.Hkv;
    const uint16_t* base = (pc < p.Hkv ? p.k : p.v) + (size_t)layer * p.layer_elems() + 8 * c;
    uint16_t* dst = (pc < p.Hkv ? k : v) + (size_t)head * n * p.D + 8 * c;
    const int last = min(r0 + MOVE_ROWS, n);
    for (int r = r0 + threadIdx.x / nch; r < last; r += rows)
        *(u32x4_any*)(dst + (size_t)r * p.D) = *(const u32x4*)(base + slot_at(p, slots[r], head));
}

// Grid of a move of n rows in `pieces` pieces.
bool move_grid(int n, int pieces, int& chunks, dim3& grid) {
    chunks = (n + MOVE_ROWS - 1) / MOVE_ROWS;
    const size_t g = (size_t)chunks * pieces;
    grid = dim3((unsigned)g);
    return n > 0 && g < (1u << 24);                // a launch has fewer than 2^32 threads
}

}  // namespace

hipError_t launch_paged_attend(const PagedAttend& a, int D, int kv_dt, hipStream_t st, hipEvent_t done) {
    const size_t few = (size_t)a.n_few * a.Hkv, many = (size_t)a.n_many * a.Hkv, waves = (size_t)a.M * a.Hkv * a.gs;
    if (a.n_few < 0 || a.n_many < 0 || few + many < 1 || few + many >= (1u << 24) || waves >= (1u << 24)) return hipErrorInvalidValue;
    const bool f32 = a.q_dt == DT_F32, bf = kv_dt == DT_BF16;
    if ((!f32 && a.q_dt != kv_dt) || (D != 64 && D != 128)) return hipErrorInvalidValue;
    const dim3 block(256);
    hipError_t e = hipSuccess;
#define PAGED_PICK(D_, KERNEL, F32_, H16_, GRID, DONE)                                                            \
    (f32 ? bf ? launch_done(KERNEL<D_, DT_BF16, F32_>, GRID, block, 0, st, DONE, a)                               \
              : launch_done(KERNEL<D_, DT_F16, F32_>, GRID, block, 0, st, DONE, a)                                \
         : bf ? launch_done(KERNEL<D_, DT_BF16, H16_>, GRID, block, 0, st, DONE, a)                               \
              : launch_done(KERNEL<D_, DT_F16, H16_>, GRID, block, 0, st, DONE, a))
    if (few) {
        const dim3 grid((unsigned)few);
        const hipEvent_t d = a.merge || many ? nullptr : done;
        e = D == 128 ? PAGED_PICK(128, paged_few_kernel, 2, 1, grid, d) : PAGED_PICK(64, paged_few_kernel, 2, 1, grid, d);
        if (e != hipSuccess) return e;
    }
#define PAGED_TWO 2, 2
#define PAGED_ONE 1, 1
    if (many) {
        const dim3 grid((unsigned)many);
        const hipEvent_t d = a.merge ? nullptr : done;
        e = D == 128 ? PAGED_PICK(128, paged_many_kernel, PAGED_TWO, PAGED_ONE, grid, d)
                     : PAGED_PICK(64, paged_many_kernel, PAGED_TWO, PAGED_ONE, grid, d);
        if (e != hipSuccess) return e;
    }
    if (!a.merge) return e;
    const dim3 mg((unsigned)((waves + 3) / 4));
    return D == 128 ? launch_done(paged_merge_kernel<128>, mg, block, 0, st, done, a)
                    : launch_done(paged_merge_kernel<64>, mg, block, 0, st, done, a);
}

hipError_t launch_paged_write(const PagedWrite& a, int D, hipStream_t st, hipEvent_t done) {
    if (a.M < 1 || (D != 64 && D != 128)) return hipErrorInvalidValue;
    const int heads = a.Hq + 2 * a.Hkv, steps = (heads + 2048 / D - 1) / (2048 / D);
    const dim3 grid(a.M, a.M >= 512 ? 1 : steps);  // few rows: a step of heads a workgroup
    return D == 128 ? launch_done(paged_write_kernel<128>, grid, dim3(256), 0, st, done, a)
                    : launch_done(paged_write_kernel<64>, grid, dim3(256), 0, st, done, a);
}

hipError_t launch_paged_copy(const PagedPool& p, const int2* moves, int n, hipStream_t st, hipEvent_t done) {
    int chunks;
    dim3 grid;
    if (!move_grid(n, 2 * p.layers * p.Hkv, chunks, grid)) return hipErrorInvalidValue;
    return launch_done(paged_copy_kernel, grid, dim3(256), 0, st, done, p, moves, n, chunks);
}

hipError_t launch_paged_slide(const PagedPool& p, const int2* moves, int n, hipStream_t st, hipEvent_t done) {
    const int columns = 2 * p.layers * p.Hkv * (p.D / 8);
    if (n < 1) return hipErrorInvalidValue;
    return launch_done(paged_slide_kernel, dim3((columns + 255) / 256), dim3(256), 0, st, done, p, moves, n, columns);
}

hipError_t launch_paged_fill(const PagedPool& p, const uint16_t* k, const uint16_t* v, const int16_t* table, int S, int slot, int cap,
                             int start, const int* slots, int n, hipStream_t st, hipEvent_t done) {
    int chunks;
    dim3 grid;
    if (!move_grid(n, 2 * p.layers * p.Hkv, chunks, grid)) return hipErrorInvalidValue;
    return launch_done(paged_fill_kernel, grid, dim3(256), 0, st, done, p, k, v, table, S, slot, cap, start, slots, n, chunks);
}

hipError_t launch_paged_read(const PagedPool& p, int layer, const int* slots, int n, uint16_t* k, uint16_t* v, hipStream_t st, hipEvent_t done) {
    int chunks;
    dim3 grid;
    if (!move_grid(n, 2 * p.Hkv, chunks, grid)) return hipErrorInvalidValue;
    return launch_done(paged_read_kernel, grid, dim3(256), 0, st, done, p, layer, slots, n, k, v, chunks);
}

}  // namespace stg
