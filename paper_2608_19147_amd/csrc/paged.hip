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

// ------------------------------------------------------------------ attention
//
// o = sum_j w_j v_j / sum_j w_j, w_j = exp(s_j - max), in one pass over the keys with the running maximum and sum.  A
// workgroup takes up to 128 query vectors of one kv head (rows x heads of the group, in tiles of 32) and a run of keys; its
// four waves are NQT tiles by KG = 4 / NQT key groups, which take alternate steps of 32 keys and are merged through LDS.
// Scores are S^T = K Q^T on 32 x 32 x 16 products: a lane then holds 16 scores of one query vector, and P^T is the second
// operand of O^T += V^T P^T as it lies (lane half h holds keys 8 i + 4 h .. + 3, and V^T is read in that order, by LDS
// transpose reads).  Rows go from the pages to LDS by direct loads, NQT steps per key group in flight: with one tile the
// wave's whole step goes to registers before the next is asked for, so that one buffer is enough.  16-byte chunk c of a
// row lies at c ^ f(row), so that neither read meets a bank twice.
// Probabilities enter as P terms of the cache's type (PT = 2: rounded part and residual, 2^-17 in bf16); queries of that
// type as they are, fp32 ones as two terms (QT).

constexpr int AK = 32;                             // keys a step

template <int D>
__device__ __forceinline__ int swz_k(int row) { return D == 128 ? row & 15 : (row >> 1) & 7; }
template <int D>
__device__ __forceinline__ int swz_v(int row) { return D == 128 ? 2 * (row & 7) : 2 * ((row >> 1) & 3); }

__device__ __forceinline__ void dma16(const void* src, void* lds) {
    __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)src, (__attribute__((address_space(3))) void*)lds, 16, 0, 0);
}
__device__ __forceinline__ uint32_t lds_addr(const void* p) { return (uint32_t)(uintptr_t)(const __attribute__((address_space(3))) void*)p; }

// Four 16-byte LDS reads and the wait for them (with reads of the compiler's own it would wait for the loads to LDS in flight).
__device__ __forceinline__ void lds_read4(u32x4* v, uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3) {
    asm volatile(
        "ds_read_b128 %0, %4\n\tds_read_b128 %1, %5\n\tds_read_b128 %2, %6\n\tds_read_b128 %3, %7\n\ts_waitcnt lgkmcnt(0)"
        : "=&v"(v[0]), "=&v"(v[1]), "=&v"(v[2]), "=&v"(v[3])
        : "v"(a0), "v"(a1), "v"(a2), "v"(a3)
        : "memory");
}
__device__ __forceinline__ void lds_read8(u32x4* v, const uint32_t* a) {
    asm volatile(
        "ds_read_b128 %0, %8\n\tds_read_b128 %1, %9\n\tds_read_b128 %2, %10\n\tds_read_b128 %3, %11\n\t"
        "ds_read_b128 %4, %12\n\tds_read_b128 %5, %13\n\tds_read_b128 %6, %14\n\tds_read_b128 %7, %15\n\ts_waitcnt lgkmcnt(0)"
        : "=&v"(v[0]), "=&v"(v[1]), "=&v"(v[2]), "=&v"(v[3]), "=&v"(v[4]), "=&v"(v[5]), "=&v"(v[6]), "=&v"(v[7])
        : "v"(a[0]), "v"(a[1]), "v"(a[2]), "v"(a[3]), "v"(a[4]), "v"(a[5]), "v"(a[6]), "v"(a[7])
        : "memory");
}
// The value fragments of 32 dims: four transposed reads, 8 keys apart (RB bytes a row), and the wait for them.
template <int RB>
__device__ __forceinline__ void lds_read_v(u32x2* v, uint32_t a) {
    asm volatile(
        "ds_read_b64_tr_b16 %0, %4\n\tds_read_b64_tr_b16 %1, %4 offset:%5\n\tds_read_b64_tr_b16 %2, %4 offset:%6\n\t"
        "ds_read_b64_tr_b16 %3, %4 offset:%7\n\ts_waitcnt lgkmcnt(0)"
        : "=&v"(v[0]), "=&v"(v[1]), "=&v"(v[2]), "=&v"(v[3])
        : "v"(a), "n"(8 * RB), "n"(16 * RB), "n"(24 * RB)
        : "memory");
}
template <int N>
__device__ __forceinline__ void wait_loads() { asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory"); }
__device__ __forceinline__ void bare_barrier() { asm volatile("s_barrier" ::: "memory"); }

// Bits 15 and 31: the halves of x whose exponent is all ones (no number).
template <int KVDT>
__device__ __forceinline__ uint32_t not_numbers(uint32_t x) {
    constexpr uint32_t E = KVDT == DT_BF16 ? 0x7f807f80u : 0x7c007c00u, A = KVDT == DT_BF16 ? 0x00800080u : 0x04000400u;
    return ((x & E) + A) & 0x80008000u;
}

template <int D, int KVDT, int QT, int PT, int NQT>
__device__ __forceinline__ void attend_item(const PagedAttend& a, const PagedItem& it, int g, uint8_t* lds, float2* sml) {
    constexpr int RB = 2 * D, SB = AK * RB, NCH = D / 8, KT = D / 16, MB = D / 32;
    constexpr int KG = 4 / NQT, NB = NQT;          // key groups; steps of a group that LDS holds
    constexpr int NP = SB / 1024;                  // kilobytes (one load of a wave) of a step's K, and of its V
    constexpr int NL = 2 * NP / NQT;               // of both, a wave's
    constexpr int RPP = 1024 / RB;                 // rows of a kilobyte
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int qt = wave % NQT, kg = wave / NQT, ql = lane & 31, h = lane >> 5;
    const int Hq = a.Hkv * a.gs, pmask = (1 << a.shift) - 1;
    const int s0 = it.kb / AK, s1 = (it.ke + AK - 1) / AK, turns = (s1 - s0 + KG - 1) / KG;
    uint8_t* ring = lds + kg * NB * 2 * SB;

    // ---- this wave's loads of step st: kilobytes qt NL .. of K's, then V's; every row of a page may be read
    const int prow = lane / NCH, ppos = lane % NCH;
    auto issue = [&](int st, int buf) {
        int page[2];
#pragma unroll
        for (int i = 0; i < 2; ++i)                // 16 rows never span pages
            page[i] = uniform_load(a.tables, (size_t)it.table + (min(AK * st + 16 * i, it.ke - 1) >> a.shift));
#pragma unroll
        for (int u = 0; u < NL; ++u) {
            const int p = qt * NL + u;             // the same in every lane
            const bool isv = p >= NP;
            const int r0 = (isv ? p - NP : p) * RPP, row = r0 + prow;
            const int c = ppos ^ (isv ? swz_v<D>(row) : swz_k<D>(row));
            const size_t at = ((size_t)((size_t)(r0 < 16 ? page[0] : page[1]) * a.Hkv + g) << a.shift) + ((AK * st + r0) & pmask);
            const uint8_t* src = (const uint8_t*)((isv ? a.v : a.k) + at * D) + prow * RB + 16 * c;
            dma16(src, ring + buf * 2 * SB + p * 1024);
        }
    };
#pragma unroll
    for (int i = 0; i < (NB > 1 ? NB - 1 : 1); ++i)
        if (i < turns) issue(s0 + kg + KG * i, i);

    // ---- this wave's query vectors
    const int c0 = it.q0 + 32 * qt + ql, cq = min(c0, it.q0 + it.nq - 1);
    bool mine = c0 < it.q0 + it.nq;
    const int row = a.rowlist[it.rows + cq / a.gs], head = g * a.gs + cq % a.gs;
    const PagedRow ri = a.rows[row];
    mine = mine && it.slot < ri.nparts;          // (a row that ends before this run has no part of it)
    const bool full = it.form & 8;
    u32x4 qf[QT][KT];
    float qscale = 1.f;                            // fp32 queries: the power of two that they are divided by
    if constexpr (QT == 1) {
        const uint16_t* qr = (const uint16_t*)a.q + (size_t)row * a.ldq + (size_t)head * D + 8 * h;
#pragma unroll
        for (int t = 0; t < KT; ++t) qf[0][t] = *(const u32x4_any*)(qr + 16 * t);
    } else {
        const float* qr = (const float*)a.q + (size_t)row * a.ldq + (size_t)head * D + 8 * h;
        float x[KT][8], top = 0.f;
#pragma unroll
        for (int t = 0; t < KT; ++t) {
            *(f32x4_t*)&x[t][0] = *(const f32x4_any*)(qr + 16 * t);
            *(f32x4_t*)&x[t][4] = *(const f32x4_any*)(qr + 16 * t + 4);
        }
#pragma unroll
        for (int t = 0; t < KT; ++t)
#pragma unroll
            for (int e = 0; e < 8; ++e) top = fmaxf(top, fabsf(x[t][e]));
        float lo, hi;
        halves(top, lo, hi);
        top = fmaxf(lo, hi);
        // the largest magnitude in [1, 2): no term leaves the range of 16-bit floats, whatever the query's size
        const int e = (int)((__float_as_uint(top) >> 23) & 255) - 127;
        const int ec = e > 126 ? 126 : e < -126 ? -126 : e;
        qscale = __uint_as_float((uint32_t)(127 + ec) << 23);
        const float inv = __uint_as_float((uint32_t)(127 - ec) << 23);
#pragma unroll
        for (int t = 0; t < KT; ++t)
#pragma unroll
            for (int w = 0; w < 4; ++w) {
                const float x0 = x[t][2 * w] * inv, x1 = x[t][2 * w + 1] * inv;
                const uint32_t b = pack2<KVDT>(x0, x1);
                qf[0][t][w] = b;
                qf[QT - 1][t][w] = pack2<KVDT>(x0 - kv_float<KVDT>((uint16_t)b), x1 - kv_float<KVDT>((uint16_t)(b >> 16)));
            }
    }
    const float sc = a.scale2 * qscale;            // scores to the exponent of 2

    // ---- LDS addresses within a buffer
    uint32_t ka[KT], va[MB];
#pragma unroll
    for (int t = 0; t < KT; ++t) ka[t] = lds_addr(ring) + ql * RB + 16 * ((2 * t + h) ^ swz_k<D>(ql));
    {
        const int j = lane & 15, key = 4 * h + (j >> 2), dg = (lane >> 4) & 1;   // keys 8 apart have the same place
#pragma unroll
        for (int mb = 0; mb < MB; ++mb)
            va[mb] = lds_addr(ring) + SB + key * RB + 16 * ((4 * mb + 2 * dg + ((j & 3) >> 1)) ^ swz_v<D>(key)) + 8 * (j & 1);
    }

    float base = -INFINITY, lsum = 0.f;            // the largest score so far (before scaling), the sum of the probabilities
    f32x16_t o[MB];
#pragma unroll
    for (int mb = 0; mb < MB; ++mb)
#pragma unroll
        for (int r = 0; r < 16; ++r) o[mb][r] = 0.f;

    for (int i = 0; i < turns; ++i) {
        const int st = s0 + kg + KG * i, buf = NB > 1 ? i % NB : 0;
        if constexpr (NB > 1) {
            if (i + NB - 2 < turns) wait_loads<(NB - 2) * NL>();   // this wave's loads of step i are there
            else wait_loads<0>();
            bare_barrier();                        // every wave's are, and the buffer of step i - 1 has been read
            if (i + NB - 1 < turns) issue(s0 + kg + KG * (i + NB - 1), (i + NB - 1) % NB);
        } else {
            wait_loads<0>();
        }
        // what this lane's query vector sees of the step, one bit a key
        const bool whole = full && AK * st >= it.kb && AK * st + AK <= it.ke;
        uint32_t see = ~0u, in = ~0u;
        bool work = true;
        if (!whole) {
            const int lo = max(it.kb - AK * st, 0), hi = min(it.ke - AK * st, AK);
            in = hi <= lo ? 0u : (~0u >> (AK - (hi - lo))) << lo;
            const int lim = ri.limit - AK * st;
            see = in & (lim <= 0 ? 0u : lim >= AK ? ~0u : ~0u >> (AK - lim));
            if (ri.mask >= 0 && see) see &= a.masks[(size_t)ri.mask + st];
            work = __any(see != 0u);
        }
        const uint32_t off = buf * 2 * SB;
        f32x16_t s;
        u32x4 vf[MB][2];
        if (work) {
            u32x4 kf[KT];
            uint32_t ad[KT];
#pragma unroll
            for (int t = 0; t < KT; ++t) ad[t] = ka[t] + off;
            if constexpr (KT == 8) lds_read8(kf, ad);
            else lds_read4(kf, ad[0], ad[1], ad[2], ad[3]);
#pragma unroll
            for (int r = 0; r < 16; ++r) s[r] = 0.f;
#pragma unroll
            for (int t = 0; t < KT; ++t) {
                s = mma32<KVDT>(kf[t], qf[0][t], s);
                if constexpr (QT == 2) s = mma32<KVDT>(kf[t], qf[1][t], s);
            }
#pragma unroll
            for (int mb = 0; mb < MB; ++mb) {
                u32x2 p[4];
                lds_read_v<RB>(p, va[mb] + off);
#pragma unroll
                for (int t = 0; t < 2; ++t) vf[mb][t] = u32x4{p[2 * t][0], p[2 * t][1], p[2 * t + 1][0], p[2 * t + 1][1]};
            }
        }
        if constexpr (NB == 1) {
            if (i + 1 < turns) issue(s0 + kg + KG * (i + 1), 0);   // the buffer is read
        }
        if (!work) continue;

        if (!whole) {
            const uint32_t b = see >> (4 * h);
#pragma unroll
            for (int r = 0; r < 16; ++r) s[r] = (b >> (8 * (r / 4) + r % 4)) & 1u ? s[r] : -INFINITY;
        }
        float mx = s[0];
#pragma unroll
        for (int r = 1; r < 16; ++r) mx = fmaxf(mx, s[r]);
        if (__any(mx > base)) {
            float lo, hi;
            halves(mx, lo, hi);
            const float top = fmaxf(base, fmaxf(lo, hi));
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
        if (!whole) {
            // Rows outside the run enter as zeros: what they hold is nobody's.  Of the others, a value that is no number must
            // reach the query vectors that see it and no other (0 times it is no number either): it is taken out of the
            // products and added where it is seen.
            uint32_t any = 0u;
#pragma unroll
            for (int t = 0; t < 2; ++t)
#pragma unroll
                for (int w = 0; w < 4; ++w) {
                    const uint32_t bits = in >> (16 * t + 8 * (w >> 1) + 4 * h + 2 * (w & 1));
                    const uint32_t m = (bits & 1u ? 0xFFFFu : 0u) | (bits & 2u ? 0xFFFF0000u : 0u);
#pragma unroll
                    for (int mb = 0; mb < MB; ++mb) {
                        vf[mb][t][w] &= m;
                        any |= not_numbers<KVDT>(vf[mb][t][w]);
                    }
                }
            if (__any(any != 0u)) {
#pragma unroll
                for (int mb = 0; mb < MB; ++mb)
#pragma unroll
                    for (int t = 0; t < 2; ++t)
#pragma unroll
                        for (int w = 0; w < 4; ++w) vf[mb][t][w] &= ~((not_numbers<KVDT>(vf[mb][t][w]) >> 15) * 0xFFFFu);
#pragma unroll 1
                for (int key = 0; key < AK; ++key) {
                    if (!((in >> key) & 1u)) continue;
                    float p = 0.f;
#pragma unroll
                    for (int r = 0; r < 16; ++r) p = 4 * (key / 8) + key % 4 == r ? pv[r] : p;
                    float lo, hi;
                    halves(p, lo, hi);
                    p = key & 4 ? hi : lo;
                    const int j = AK * st + key;
                    const int page = uniform_load(a.tables, (size_t)it.table + (j >> a.shift));
                    const uint16_t* vr = a.v + ((((size_t)page * a.Hkv + g) << a.shift) + (j & pmask)) * D + 4 * h;
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
    }

    // ---- results: 4 neighbouring dims 32 mb + 8 r4 + 4 h .. of the lane's query vector at a time
    {
        float lo, hi;
        halves(lsum, lo, hi);
        lsum = lo + hi;
    }
    base = base == -INFINITY ? base : base * sc;
    const size_t prow_ = ((size_t)(ri.part + it.slot) * Hq + head);
    auto put = [&](int d, const f32x4_t& v, float inv) {
        if (!mine) return;
        if (ri.nparts > 1) {
            *(f32x4_t*)(a.part_o + prow_ * D + d) = v;
            return;
        }
        const size_t at = (size_t)row * a.ldo + (size_t)head * D + d;
        if (a.out_dt == DT_F32) {
            *(f32x4_any*)((float*)a.out + at) = v * inv;
        } else {
            u32x2 b;
#pragma unroll
            for (int e = 0; e < 2; ++e)
                b[e] = (uint32_t)to_half_bits(v[2 * e] * inv, a.out_dt) | ((uint32_t)to_half_bits(v[2 * e + 1] * inv, a.out_dt) << 16);
            *(u32x2_any*)((uint16_t*)a.out + at) = b;
        }
    };
    auto quad = [&](const f32x16_t& x, int r4) { return f32x4_t{x[4 * r4], x[4 * r4 + 1], x[4 * r4 + 2], x[4 * r4 + 3]}; };
    if constexpr (KG == 1) {
        if (mine && ri.nparts > 1 && h == 0) a.part_ml[prow_] = float2{base, lsum};
        const float inv = lsum == 0.f ? 0.f : 1.0f / lsum;
#pragma unroll
        for (int mb = 0; mb < MB; ++mb)
#pragma unroll
            for (int r4 = 0; r4 < 4; ++r4) put(32 * mb + 8 * r4 + 4 * h, quad(o[mb], r4), inv);
    } else {
        __syncthreads();                           // every wave has read its last step
        f32x4_t* so = (f32x4_t*)lds;               // [wave][MB][4][64]
        if (h == 0) sml[wave * 32 + ql] = float2{base, lsum};
#pragma unroll
        for (int mb = 0; mb < MB; ++mb)
#pragma unroll
            for (int r4 = 0; r4 < 4; ++r4) so[((wave * MB + mb) * 4 + r4) * 64 + lane] = quad(o[mb], r4);
        __syncthreads();
        float top = -INFINITY, sum = 0.f, f[KG];
#pragma unroll
        for (int k = 0; k < KG; ++k) top = fmaxf(top, sml[(k * NQT + qt) * 32 + ql].x);
#pragma unroll
        for (int k = 0; k < KG; ++k) {
            const float2 ml = sml[(k * NQT + qt) * 32 + ql];
            f[k] = ml.x == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(ml.x - top);
            sum += ml.y * f[k];
        }
        if (mine && ri.nparts > 1 && h == 0 && kg == 0) a.part_ml[prow_] = float2{top, sum};
        const float inv = sum == 0.f ? 0.f : 1.0f / sum;
        for (int q = kg; q < MB * 4; q += KG) {    // the tile's waves share its dims
            f32x4_t v = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int k = 0; k < KG; ++k) {
                const f32x4_t x = so[((k * NQT + qt) * MB * 4 + q) * 64 + lane];
                v += x * f[k];
            }
            put(32 * (q / 4) + 8 * (q % 4) + 4 * h, v, inv);
        }
    }
}

template <int D, int KVDT, int QT, int PT>
__global__ __launch_bounds__(256, 2) void paged_attend_kernel(PagedAttend a) {
    __shared__ __attribute__((aligned(1024))) uint8_t lds[4 * 2 * AK * 2 * D];
    __shared__ float2 sml[128];
    const int b = __builtin_amdgcn_readfirstlane(blockIdx.x / a.Hkv), g = __builtin_amdgcn_readfirstlane(blockIdx.x % a.Hkv);
    const PagedItem it = uniform_load(a.items, b);
    const int nqt = it.form & 7;
    if (nqt == 1) attend_item<D, KVDT, QT, 2, 1>(a, it, g, lds, sml);
    else if (nqt == 2) attend_item<D, KVDT, QT, 2, 2>(a, it, g, lds, sml);
    else attend_item<D, KVDT, QT, PT, 4>(a, it, g, lds, sml);
}

// Rows with several partial results: m = max m_r, o = sum o_r 2^(m_r - m) / sum l_r 2^(m_r - m), added in the order of the
// runs.  One wave per row and head.
template <int D>
__global__ __launch_bounds__(256) void paged_merge_kernel(PagedAttend a) {
    constexpr int E = D / 64;
    const int lane = threadIdx.x & 63, Hq = a.Hkv * a.gs;
    const int id = __builtin_amdgcn_readfirstlane(4 * blockIdx.x + (threadIdx.x >> 6));
    if (id >= a.M * Hq) return;
    const int row = id / Hq, head = id % Hq;
    const PagedRow ri = uniform_load(a.rows, row);
    const int n = ri.nparts;
    if (n < 2) return;
    float top = -INFINITY;
    for (int p0 = 0; p0 < n; p0 += 64) {
        float m = p0 + lane < n ? a.part_ml[(size_t)(ri.part + p0 + lane) * Hq + head].x : -INFINITY;
#pragma unroll
        for (int x = 1; x < 64; x <<= 1) m = fmaxf(m, __shfl_xor(m, x));
        top = fmaxf(top, m);
    }
    float acc[E] = {}, sum = 0.f;
    for (int p0 = 0; p0 < n; p0 += 64) {
        const bool have = p0 + lane < n;
        const float2 ml = have ? a.part_ml[(size_t)(ri.part + p0 + lane) * Hq + head] : float2{-INFINITY, 0.f};
        const float w = ml.x == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(ml.x - top);
        const float l = w * ml.y;
        const int cnt = min(64, n - p0);
        for (int p = 0; p < cnt; p += 4) {
            float x[4][E];
#pragma unroll
            for (int u = 0; u < 4; ++u)
                __builtin_memcpy(x[u], a.part_o + ((size_t)(ri.part + p0 + min(p + u, cnt - 1)) * Hq + head) * D + E * lane, 4 * E);
#pragma unroll
            for (int u = 0; u < 4; ++u) {
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
    const size_t grid = (size_t)a.n_items * a.Hkv, waves = (size_t)a.M * a.Hkv * a.gs;
    if (a.n_items < 1 || grid >= (1u << 24) || waves >= (1u << 24)) return hipErrorInvalidValue;
    const bool f32 = a.q_dt == DT_F32;
    if (!f32 && a.q_dt != kv_dt) return hipErrorInvalidValue;
    const hipEvent_t d0 = a.merge ? nullptr : done;
    hipError_t e = hipErrorInvalidValue;
#define PAGED_ATTEND(D_, KV_)                                                                                     \
    e = f32 ? launch_done(paged_attend_kernel<D_, KV_, 2, 2>, dim3((unsigned)grid), dim3(256), 0, st, d0, a)      \
            : launch_done(paged_attend_kernel<D_, KV_, 1, 1>, dim3((unsigned)grid), dim3(256), 0, st, d0, a)
    if (D == 128 && kv_dt == DT_BF16) PAGED_ATTEND(128, DT_BF16);
    else if (D == 128) PAGED_ATTEND(128, DT_F16);
    else if (D == 64 && kv_dt == DT_BF16) PAGED_ATTEND(64, DT_BF16);
    else if (D == 64) PAGED_ATTEND(64, DT_F16);
#undef PAGED_ATTEND
    if (e != hipSuccess || !a.merge) return e;
    const dim3 mg((unsigned)((waves + 3) / 4));
    return D == 128 ? launch_done(paged_merge_kernel<128>, mg, dim3(256), 0, st, done, a)
                    : launch_done(paged_merge_kernel<64>, mg, dim3(256), 0, st, done, a);
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
