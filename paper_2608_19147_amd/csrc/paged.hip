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


// A maximum that rises by less than this (in powers of two) does not move the base that is subtracted: probabilities up to
// 2^LAG cost no bits, in 16-bit floats either, and the outputs are seldom rescaled (a wave does when one of its query
// vectors has to, which for 32 of them was nearly every step: 4 x 1024 rows behind 2048 224 -> 211 us).
constexpr float LAG = 8.f;

template <int D>
__device__ __forceinline__ int swz_k(int row) { return D == 128 ? row & 15 : (row >> 1) & 7; }
template <int D>
__device__ __forceinline__ int swz_v(int row) { return D == 128 ? 2 * (row & 7) : 2 * ((row >> 1) & 3); }

// The value, as one that is only known here: what is computed from it is not kept in registers through a loop.
__device__ __forceinline__ uint32_t here(uint32_t v) {
    asm volatile("" : "+v"(v));
    return v;
}

// Values that were loaded are there from here on: first used inside a loop, they would be waited for in every turn of it,
// and the rows under way with them (64 rows behind 4096 shared ones 38 -> 32.5 us).
template <int N>
__device__ __forceinline__ void settle(u32x4 (&v)[N]) {
#pragma unroll
    for (int i = 0; i < N; ++i) asm volatile("" : "+v"(v[i]));
}

// The place in the wave, from no register, so that none is kept for an item's second pass.
__device__ __forceinline__ int lane_id() { return __builtin_amdgcn_mbcnt_hi(~0u, __builtin_amdgcn_mbcnt_lo(~0u, 0u)); }

// This lane's part of the direct loads of 16 rows of a page, a kilobyte (1024 / (2 D) rows) an instruction: byte offsets
// into the rows, for K and V.
template <int D>
__device__ __forceinline__ uint32_t lane_k(int l) { const int r = l / (D / 8); return r * 2 * D + 16 * (l % (D / 8) ^ swz_k<D>(r)); }
template <int D>
__device__ __forceinline__ uint32_t lane_v(int l) { const int r = l / (D / 8); return r * 2 * D + 16 * (l % (D / 8) ^ swz_v<D>(r)); }
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
__device__ __forceinline__ void load_word(const uint32_t* src, uint32_t* lds) {   // one a lane
    __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)src, (__attribute__((address_space(3))) void*)lds, 4, 0, 0);
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
__device__ __forceinline__ uint32_t read_word(uint32_t at) {
    uint32_t v;
    asm volatile("ds_read_b32 %0, %1\n\ts_waitcnt lgkmcnt(0)" : "=v"(v) : "v"(at) : "memory");
    return v;
}
// All of a step of 32 keys: K's fragments and V's, 32 dims of V at v ^ (64 t), its reads 8 keys apart (RB bytes a row).
template <int D>
__device__ __forceinline__ void read_step32(uint32_t k, uint32_t v, u32x4* f, u32x2* w) {
    constexpr int RB = 2 * D;
    if constexpr (D == 128)
        asm volatile(
            "ds_read_b128 %0, %24\n\t"
            "ds_read_b128 %1, %25\n\t"
            "ds_read_b128 %2, %26\n\t"
            "ds_read_b128 %3, %27\n\t"
            "ds_read_b128 %4, %28\n\t"
            "ds_read_b128 %5, %29\n\t"
            "ds_read_b128 %6, %30\n\t"
            "ds_read_b128 %7, %31\n\t"
            "ds_read_b64_tr_b16 %8, %32\n\t"
            "ds_read_b64_tr_b16 %9, %32 offset:%36\n\t"
            "ds_read_b64_tr_b16 %10, %32 offset:%37\n\t"
            "ds_read_b64_tr_b16 %11, %32 offset:%38\n\t"
            "ds_read_b64_tr_b16 %12, %33\n\t"
            "ds_read_b64_tr_b16 %13, %33 offset:%36\n\t"
            "ds_read_b64_tr_b16 %14, %33 offset:%37\n\t"
            "ds_read_b64_tr_b16 %15, %33 offset:%38\n\t"
            "ds_read_b64_tr_b16 %16, %34\n\t"
            "ds_read_b64_tr_b16 %17, %34 offset:%36\n\t"
            "ds_read_b64_tr_b16 %18, %34 offset:%37\n\t"
            "ds_read_b64_tr_b16 %19, %34 offset:%38\n\t"
            "ds_read_b64_tr_b16 %20, %35\n\t"
            "ds_read_b64_tr_b16 %21, %35 offset:%36\n\t"
            "ds_read_b64_tr_b16 %22, %35 offset:%37\n\t"
            "ds_read_b64_tr_b16 %23, %35 offset:%38\n\t"
            "s_waitcnt lgkmcnt(0)"
            : "=&v"(f[0]), "=&v"(f[1]), "=&v"(f[2]), "=&v"(f[3]), "=&v"(f[4]), "=&v"(f[5]), "=&v"(f[6]), "=&v"(f[7]), "=&v"(w[0]), "=&v"(w[1]), "=&v"(w[2]), "=&v"(w[3]), "=&v"(w[4]), "=&v"(w[5]), "=&v"(w[6]), "=&v"(w[7]), "=&v"(w[8]), "=&v"(w[9]), "=&v"(w[10]), "=&v"(w[11]), "=&v"(w[12]), "=&v"(w[13]), "=&v"(w[14]), "=&v"(w[15])
            : "v"(k), "v"(k ^ 32u), "v"(k ^ 64u), "v"(k ^ 96u), "v"(k ^ 128u), "v"(k ^ 160u), "v"(k ^ 192u), "v"(k ^ 224u), "v"(v), "v"(v ^ 64u), "v"(v ^ 128u), "v"(v ^ 192u), "n"(8 * RB), "n"(16 * RB), "n"(24 * RB)
            : "memory");
    else
        asm volatile(
            "ds_read_b128 %0, %12\n\t"
            "ds_read_b128 %1, %13\n\t"
            "ds_read_b128 %2, %14\n\t"
            "ds_read_b128 %3, %15\n\t"
            "ds_read_b64_tr_b16 %4, %16\n\t"
            "ds_read_b64_tr_b16 %5, %16 offset:%18\n\t"
            "ds_read_b64_tr_b16 %6, %16 offset:%19\n\t"
            "ds_read_b64_tr_b16 %7, %16 offset:%20\n\t"
            "ds_read_b64_tr_b16 %8, %17\n\t"
            "ds_read_b64_tr_b16 %9, %17 offset:%18\n\t"
            "ds_read_b64_tr_b16 %10, %17 offset:%19\n\t"
            "ds_read_b64_tr_b16 %11, %17 offset:%20\n\t"
            "s_waitcnt lgkmcnt(0)"
            : "=&v"(f[0]), "=&v"(f[1]), "=&v"(f[2]), "=&v"(f[3]), "=&v"(w[0]), "=&v"(w[1]), "=&v"(w[2]), "=&v"(w[3]), "=&v"(w[4]), "=&v"(w[5]), "=&v"(w[6]), "=&v"(w[7])
            : "v"(k), "v"(k ^ 32u), "v"(k ^ 64u), "v"(k ^ 96u), "v"(v), "v"(v ^ 64u), "n"(8 * RB), "n"(16 * RB), "n"(24 * RB)
            : "memory");
}

// The larger magnitudes of two pairs of 16-bit floats, as integers; whether one of a pair is no number.
__device__ __forceinline__ uint32_t larger(uint32_t m, uint32_t x) {
    typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));
    return __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(u16x2, m), __builtin_bit_cast(u16x2, x & 0x7fff7fffu)));
}
template <int KVDT>
__device__ __forceinline__ bool no_number(uint32_t m) {
    constexpr uint32_t INF = KVDT == DT_BF16 ? 0x7f80u : 0x7c00u;
    return (m & 0xffffu) >= INF || (m >> 16) >= INF;
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

// Whether one of these results is infinite or no number.
template <int MB, class V>
__device__ __forceinline__ bool no_numbers(const V (&o)[MB]) {
    float t = 0.f;                                 // 0 times a number is 0
#pragma unroll
    for (int mb = 0; mb < MB; ++mb)
#pragma unroll
        for (unsigned j = 0; j < sizeof(V) / 4; ++j) t = __builtin_fmaf(o[mb][j], 0.f, t);
    return t != 0.f;
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

// Whether one of the four waves has said so in its words, `apart` words from each other.
__device__ __forceinline__ bool any_wave(const uint32_t* words, int apart) {
    return (words[0] | words[apart]) | (words[2 * apart] | words[3 * apart]);
}

// s where bit b of the bits is set, else -infinity.
__device__ __forceinline__ float seen(float s, uint32_t bits, int b) {
    const uint32_t m = (uint32_t)__builtin_amdgcn_sbfe((int)bits, b, 1);
    return __uint_as_float((__float_as_uint(s) & m) | (~m & 0xff800000u));
}

// The bits of a step of AK keys from key k0 on that lie in the item's run, and of those the ones below `limit`.
template <int AK>
__device__ __forceinline__ uint32_t run_bits(int kb, int ke, int k0) {
    const int lo = max(kb - k0, 0), hi = min(ke - k0, AK);
    return hi <= lo ? 0u : (~0u >> (32 - (hi - lo))) << lo;
}
__device__ __forceinline__ uint32_t bits_below(int n) { return n <= 0 ? 0u : n >= 32 ? ~0u : ~0u >> (32 - n); }

// ---- tiles of up to 16 query vectors
//
// Decoding rows.  The four waves take alternate steps of 16 keys (one page's) and are merged through LDS.  Bound by memory
// (four caches of 81920 to 131072 rows of 8 x 128: 308 us, 5.67 TB/s; a large read 6.2): what counts is bytes in flight.
// A wave holds NB steps in LDS of its own; it reads all of a step into registers, then asks for the step NB further on in
// its place, so that no barrier stands between.  A probability enters as its rounded
// part and the residual (2^-17 in bf16), in one product: the second operand's 32 k slots hold 16 keys twice, those of V^T
// repeat them.
//
// Values of V that are no numbers are looked for in steps that not every row sees whole.  In the others an infinite one would
// be NaN by the probability's two terms (p inf + r inf, r <= 0), or by a probability that is zero in 16 bits.  An item with
// such a result (true is returned, nothing is written) is computed again with every step looked at (EACH), unless the sum of
// the probabilities is none either (a query or key with NaN: the result stays NaN): what holds numbers pays a look at its
// results, not at its values (one row 8.8 -> 9.0 us, four trees 15.3 -> 15.5, other batches within 1%).
template <int D, int KVDT, int QT, int NB, bool EACH = false>
__device__ __forceinline__ bool few_item(const PagedAttend& a, const PagedItem& it, int g, int wave, uint8_t* lds, float2* sml, uint32_t* words) {
    constexpr int AK = 16, RB = 2 * D, SB = AK * RB, KT = D / 32, MB = D / 16, KG = 4;
    constexpr int NL = 2 * SB / 1024;              // loads of a step
    const int lane = EACH ? (int)here(lane_id()) : lane_id(), ql = lane & 15, lg = lane >> 4;
    const int Hq = a.Hkv * a.gs, pmask = (1 << a.shift) - 1;
    const int s0 = it.kb / AK, s1 = (it.ke + AK - 1) / AK, turns = (s1 - s0 + KG - 1) / KG;
    uint8_t* ring = lds + wave * NB * 2 * SB;
    words += wave * NB * 64;
    const bool open = it.open & 1, masked = it.open & 2;

    int limit, mask;                               // of the lane's row
    {
        const PagedRow* r = a.list + it.rows + min(it.q0 + ql, it.q0 + it.nq - 1) / a.gs;
        limit = r->limit;
        mask = r->mask;
    }
    const size_t head_at = ((size_t)g << a.shift) * RB, page_bytes = ((size_t)a.Hkv << a.shift) * RB;
    const uint32_t lk = lane_k<D>(lane), lv = lane_v<D>(lane);
    auto page_of = [&](int i) { return uniform_load(a.tables, (size_t)it.table + (min(AK * (s0 + wave + KG * i), it.ke - 1) >> a.shift)); };
    int page = page_of(0);                         // of the step asked for next, known a step ahead
    auto issue = [&](int i) {                      // this wave's step i; every row of a page may be read
        const int key = AK * (s0 + wave + KG * i);
        const size_t at = (size_t)page * page_bytes + head_at + (size_t)(key & pmask) * RB;
        uint8_t* buf = ring + i % NB * 2 * SB;
        load_rows16<D, false>((const uint8_t*)a.k + at, lk, buf);
        load_rows16<D, true>((const uint8_t*)a.v + at, lv, buf + SB);
        if (masked) load_word(a.masks + (size_t)max(mask, 0) + min(key, it.ke - 1) / 32, words + i % NB * 64);   // (to registers it would hold up the rows)
        page = page_of(i + 1);
    };
#pragma unroll
    for (int i = 0; i < NB; ++i)
        if (i < turns) issue(i);

    u32x4 qf[QT][KT];
    float sc = a.scale2;
    {
        const int cq = min(it.q0 + ql, it.q0 + it.nq - 1);
        sc = fmaxf(sc * load_query<KVDT, QT, KT, 4>(a, (size_t)a.list[it.rows + cq / a.gs].row * a.ldq + (size_t)(g * a.gs + cq % a.gs) * D + 8 * lg, 32, qf), 0x1p-149f);   // (above zero: no score is the base's times zero)
    }
    limit = (int)here((uint32_t)limit);
    mask = (int)here((uint32_t)mask);
#pragma unroll
    for (int t = 0; t < QT; ++t) settle(qf[t]);
    const uint32_t ka = lds_addr(ring) + ql * RB + 16 * (lg ^ swz_k<D>(ql));
    const int vkey = 4 * lg + (ql >> 2);
    const uint32_t va = lds_addr(ring) + SB + vkey * RB + 16 * (swz_v<D>(vkey) + ((ql & 3) >> 1)) + 8 * (ql & 1);

    float base = -INFINITY, lsum = 0.f;            // the largest score so far (before scaling), the sum of the probabilities
    f32x4_t o[MB];
#pragma unroll
    for (int mb = 0; mb < MB; ++mb) o[mb] = f32x4_t{0.f, 0.f, 0.f, 0.f};

    for (int i = 0; i < turns; ++i) {
        const int k0 = AK * (s0 + wave + KG * i);
        if (NB == 1 || i + NB - 1 >= turns) wait_loads<0>();   // step i is there
        else if (masked) wait_loads<(NB - 1) * (NL + 1)>();
        else wait_loads<(NB - 1) * NL>();
        const bool whole = !EACH && open && k0 >= it.kb && k0 + AK <= it.ke;
        uint32_t in = 0xFFFFu, see = 0xFFFFu;      // keys of the step in the run; those that this lane's query vector sees
        bool work = true;
        if (!whole) {
            in = run_bits<AK>(it.kb, it.ke, k0);
            see = in & bits_below(limit - k0);
            if (masked) {
                const uint32_t w = read_word(lds_addr(words) + i % NB * 256 + 4 * lane);
                see &= mask >= 0 ? w >> (k0 & 16) : ~0u;
            }
            work = __any(see != 0u);
        }
        f32x4_t s = {0.f, 0.f, 0.f, 0.f};
        u32x2 vf[MB];
        const uint32_t off = i % NB * (2 * SB);
        if (work) {
            u32x4 kf[KT];
            read_k16<D>(here(ka + off), kf);
#pragma unroll
            for (int t = 0; t < KT; ++t) {
                s = mma16<KVDT>(kf[t], qf[0][t], s);
                if constexpr (QT == 2) s = mma16<KVDT>(kf[t], qf[1][t], s);
            }
            const uint32_t v = here(va + off);
            read_v16(v, vf);
            if constexpr (MB == 8) read_v16(v ^ 128u, vf + 4);
        }
        if (i + NB < turns) issue(i + NB);         // the step's place is free
        if (!work) continue;
        if (!whole) {
#pragma unroll
            for (int j = 0; j < 4; ++j) s[j] = seen(s[j], see >> (4 * lg), j);
        }
        const float mx = fmaxf(fmaxf(s[0], s[1]), fmaxf(s[2], s[3]));
        if (__any((mx - base) * sc > LAG)) {
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
#pragma unroll
        for (int j = 0; j < 4; ++j) s[j] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[j], sc, nb));   // the probabilities
        lsum += (s[0] + s[1]) + (s[2] + s[3]);
        bool bad = false;
        if (!whole) {
            // Rows outside the run enter as zeros: what they hold is nobody's.  Of the others, a value that is no number must
            // reach the query vectors that see it and no other (0 times it is no number either): it is taken out of the
            // products and added where it is seen.
            if (in != 0xFFFFu) {
#pragma unroll
                for (int w = 0; w < 2; ++w) {
                    const uint32_t bits = in >> (4 * lg + 2 * w), m = (bits & 1u ? 0xFFFFu : 0u) | (bits & 2u ? 0xFFFF0000u : 0u);
#pragma unroll
                    for (int mb = 0; mb < MB; ++mb) vf[mb][w] &= m;
                }
            }
            uint32_t top = 0u;
#pragma unroll
            for (int mb = 0; mb < MB; ++mb) top = larger(larger(top, vf[mb][0]), vf[mb][1]);
            bad = __any(no_number<KVDT>(top));
            if (bad) {
#pragma unroll
                for (int mb = 0; mb < MB; ++mb)
#pragma unroll
                    for (int w = 0; w < 2; ++w) vf[mb][w] &= ~((not_numbers<KVDT>(vf[mb][w]) >> 15) * 0xFFFFu);
            }
        }
        u32x4 pb;
#pragma unroll
        for (int w = 0; w < 2; ++w) {
            pb[w] = pack2<KVDT>(s[2 * w], s[2 * w + 1]);
            pb[2 + w] = pack2<KVDT>(s[2 * w] - kv_float<KVDT>((uint16_t)pb[w]), s[2 * w + 1] - kv_float<KVDT>((uint16_t)(pb[w] >> 16)));
        }
#pragma unroll
        for (int mb = 0; mb < MB; ++mb) o[mb] = mma16<KVDT>(u32x4{vf[mb][0], vf[mb][1], vf[mb][0], vf[mb][1]}, pb, o[mb]);
        if (bad) {
#pragma unroll 1
            for (int key = 0; key < AK; ++key) {
                if (!((in >> key) & 1u)) continue;
                float p = 0.f;
#pragma unroll
                for (int j = 0; j < 4; ++j) p = (key & 3) == j ? s[j] : p;
                p = __shfl(p, 16 * (key >> 2) + ql);
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
    __syncthreads();                               // every wave has read its last step
    f32x4_t* so = (f32x4_t*)lds;                   // [wave][MB][64]
    if (lg == 0) sml[wave * 16 + ql] = float2{base, lsum};
    if constexpr (!EACH) {
        const bool bad = __any(lsum - lsum == 0.f && no_numbers(o));
        if (lane == 0) words[0] = bad;             // (the wave has read its words)
    }
#pragma unroll
    for (int mb = 0; mb < MB; ++mb) so[(wave * MB + mb) * 64 + lane] = o[mb];
    __syncthreads();
    if constexpr (!EACH)
        if (any_wave(words - wave * NB * 64, NB * 64)) return true;
    int cq = it.q0 + ql;
    asm volatile("" : "+v"(cq));                   // its row is read again: it need not stay in registers through the loop
    if (cq >= it.q0 + it.nq) return false;
    const PagedRow ri = a.list[it.rows + cq / a.gs];
    if (it.slot >= ri.nparts) return false;        // (a row that ends before this run has no part of it)
    const int head = g * a.gs + cq % a.gs;
    const size_t part = ((size_t)(ri.part + it.slot) * Hq + head);
    float top = -INFINITY, sum = 0.f, f[KG];
#pragma unroll
    for (int k = 0; k < KG; ++k) top = fmaxf(top, sml[k * 16 + ql].x);
#pragma unroll
    for (int k = 0; k < KG; ++k) {
        const float2 ml = sml[k * 16 + ql];
        f[k] = ml.x == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(ml.x - top);
        sum += ml.y * f[k];
    }
    if (ri.nparts > 1 && lg == 0 && wave == 0) a.part_ml[part] = float2{top, sum};
    const float inv = sum == 0.f ? 0.f : 1.0f / sum;
#pragma unroll
    for (int u = 0; u < MB / KG; ++u) {            // the waves share the dims
        const int mb = wave + KG * u;
        f32x4_t v = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int k = 0; k < KG; ++k) v += so[(k * MB + mb) * 64 + lane] * f[k];
        put_result<D>(a, ri, part, head, 16 * mb + 4 * lg, v, inv);
    }
    return false;
}

// Every query vector of an item, 16 at a time, each step looked at.  LDS may still be read by the item's first pass.
template <int D, int KVDT, int QT, int NB>
__device__ __forceinline__ void each_step(const PagedAttend& a, PagedItem it, int g, int wave, uint8_t* lds, float2* sml, uint32_t* words) {
    const int end = it.q0 + it.nq;
#pragma unroll 1
    for (; it.q0 < end; it.q0 += PAGED_FEW) {
        __syncthreads();
        it.nq = min(end - it.q0, PAGED_FEW);
        few_item<D, KVDT, QT, NB, true>(a, it, g, wave, lds, sml, words);
    }
}

// Batches of nothing else: at most 128 registers a wave and 33 KB of LDS, so that four workgroups share a CU (16 x 8 KB
// under way; four caches of 81920 to 131072 rows: two workgroups of 16 KB a wave 359 us, four of 8 KB 315).
template <int D, int KVDT, int QT>
__global__ __launch_bounds__(256, 4) void paged_few_kernel(PagedAttend a) {
    __shared__ __attribute__((aligned(1024))) uint8_t lds[32768];
    __shared__ float2 sml[64];
    __shared__ uint32_t words[4 * 128 / D * 64];
    const int b = __builtin_amdgcn_readfirstlane(blockIdx.x / a.Hkv), g = __builtin_amdgcn_readfirstlane(blockIdx.x % a.Hkv);
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const PagedItem it = uniform_load(a.items, b);
    if (few_item<D, KVDT, QT, 128 / D>(a, it, g, wave, lds, sml, words)) each_step<D, KVDT, QT, 128 / D>(a, it, g, wave, lds, sml, words);
}

// ---- tiles of up to 128 query vectors
//
// Verifies, what many rows share, prompts.  On 32 x 32 x 16 products: NQT tiles of 32 query vectors by KG = 4 / NQT key
// groups, which take alternate steps of 32 keys.  A group's waves share a ring of NQT steps; alone (NQT = 1) a wave reads
// its step into registers before it asks for the next.  A step of a wave takes 512 cycles of products, some 640 of vector
// instructions (256 of them exponentials) and a share of LDS, which its two waves a SIMD hardly overlap: 4 x 1024 rows of 32
// heads of 128 behind 2048 take 197 to 209 us, 825 to 875 TFLOP/s, where a product of 8192 x 8192 x 8192 reaches 1077.  (The next step's
// scores under way while this one's become probabilities: 12% slower; steps of 64 keys: 4%; wave priorities: 1% faster to 9% slower.)
// PT: terms of a probability.  One (rounded to the cache's type, while the sum keeps it whole) for prompts alone, whose products
// bound them (4 x 1024 rows 208 us, two terms 267; 4 x 128 rows 50 and 58) and whose tiles hold nobody else's rows: a row's bits
// must not follow from what is batched with it.  Two cost the others 5 to 13% (64 rows 32.8 -> 34.7 us, trees 15.5 -> 16.7,
// verifies 32.4 -> 35.2, 12 x 10 rows 42.7 -> 48.8).
template <int D, int KVDT, int QT, int PT, int NQT>
__device__ __forceinline__ bool many_item(const PagedAttend& a, const PagedItem& it, int g, int wave, uint8_t* lds, float2* sml, uint32_t* words) {
    constexpr int AK = 32, RB = 2 * D, SB = AK * RB, KT = D / 16, MB = D / 32, KG = 4 / NQT, NB = NQT;
    constexpr int NL = 2 * SB / 1024 / NQT;        // a wave's loads of a step
    const int lane = lane_id(), qt = wave % NQT, kg = wave / NQT, ql = lane & 31, h = lane >> 5;
    const int Hq = a.Hkv * a.gs, pmask = (1 << a.shift) - 1;
    const int s0 = it.kb / AK, s1 = (it.ke + AK - 1) / AK, turns = (s1 - s0 + KG - 1) / KG;
    uint8_t* ring = lds + kg * NB * 2 * SB;
    words += wave * NB * 64;
    const bool open = it.open & 1, masked = it.open & 2;

    const int c0 = it.q0 + 32 * qt + ql;
    int limit, mask;
    {
        const PagedRow* r = a.list + it.rows + min(c0, it.q0 + it.nq - 1) / a.gs;
        limit = r->limit;
        mask = r->mask;
    }

    const size_t head_at = ((size_t)g << a.shift) * RB, page_bytes = ((size_t)a.Hkv << a.shift) * RB;
    const uint32_t lk = lane_k<D>(lane), lv = lane_v<D>(lane);
    // a wave's 16-row parts of a step's K and V: all four, two of one, or one; their pages are known a step ahead
    constexpr int NP = 4 / NQT, PG = NQT == 4 ? 1 : 2;
    int page[PG];
    auto pages_of = [&](int i) {
#pragma unroll
        for (int u = 0; u < PG; ++u)
            page[u] = uniform_load(a.tables, (size_t)it.table + (min(AK * (s0 + kg + KG * i) + 16 * (NQT == 4 ? qt & 1 : u), it.ke - 1) >> a.shift));
    };
    pages_of(0);
    auto issue = [&](int i) {
        uint8_t* buf = ring + (NB > 1 ? i % NB : 0) * 2 * SB;
#pragma unroll
        for (int u = 0; u < NP; ++u) {
            const int p = qt * NP + u, half = p & 1, key = AK * (s0 + kg + KG * i) + 16 * half;
            const size_t at = (size_t)page[PG == 2 ? u & 1 : 0] * page_bytes + head_at + (size_t)(key & pmask) * RB;
            if (p < 2) load_rows16<D, false>((const uint8_t*)a.k + at, lk, buf + half * 16 * RB);
            else load_rows16<D, true>((const uint8_t*)a.v + at, lv, buf + SB + half * 16 * RB);
        }
        if (masked) load_word(a.masks + (size_t)max(mask, 0) + min(AK * (s0 + kg + KG * i), it.ke - 1) / 32, words + (NB > 1 ? i % NB : 0) * 64);
        pages_of(i + 1);
    };
#pragma unroll
    for (int i = 0; i < (NB > 1 ? NB - 1 : 1); ++i)
        if (i < turns) issue(i);

    u32x4 qf[QT][KT];
    float sc = a.scale2;
    {
        const int cq = min(c0, it.q0 + it.nq - 1);
        sc = fmaxf(sc * load_query<KVDT, QT, KT, 2>(a, (size_t)a.list[it.rows + cq / a.gs].row * a.ldq + (size_t)(g * a.gs + cq % a.gs) * D + 8 * h, 16, qf), 0x1p-149f);   // (above zero: no score is the base's times zero)
    }

    limit = (int)here((uint32_t)limit);
    mask = (int)here((uint32_t)mask);
#pragma unroll
    for (int t = 0; t < QT; ++t) settle(qf[t]);
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
        const int k0 = AK * (s0 + kg + KG * i);
        if (NB == 1 || i + NB - 2 >= turns) wait_loads<0>();   // this wave's loads of step i are there
        else if (masked) wait_loads<(NB > 1 ? NB - 2 : 0) * (NL + 1)>();
        else wait_loads<(NB > 1 ? NB - 2 : 0) * NL>();
        if constexpr (NB > 1) {
            bare_barrier();                        // every wave's are, and the buffer of step i - 1 has been read
            if (i + NB - 1 < turns) issue(i + NB - 1);
        }
        uint32_t in = ~0u, see = ~0u;              // keys of the step in the run; those that this lane's query vector sees
        bool whole = open && k0 >= it.kb && k0 + AK <= it.ke, work = true;
        if (!whole) {
            in = run_bits<AK>(it.kb, it.ke, k0);
            see = in & bits_below(limit - k0);
            if (masked) {
                const uint32_t w = read_word(lds_addr(words) + (NB > 1 ? i % NB * 256 : 0) + 4 * lane);
                see &= mask >= 0 ? w : ~0u;
            }
            work = __any(see != 0u);
            whole = !__any(see != ~0u);            // a prompt's rows see whole steps well before their own keys
        }
        const uint32_t off = NB > 1 ? i % NB * (2 * SB) : 0;
        f32x16_t s;
        u32x4 vf[MB][2];
        if (work) {
            u32x4 kf[KT];
            u32x2 p[4 * MB];
            read_step32<D>(here(ka + off), here(va + off), kf, p);
#pragma unroll
            for (int e = 0; e < 2 * MB; ++e) vf[e / 2][e % 2] = u32x4{p[2 * e][0], p[2 * e][1], p[2 * e + 1][0], p[2 * e + 1][1]};
#pragma unroll
            for (int r = 0; r < 16; ++r) s[r] = 0.f;
#pragma unroll
            for (int u = 0; u < KT; ++u) {
                s = mma32<KVDT>(kf[u], qf[0][u], s);
                if constexpr (QT == 2) s = mma32<KVDT>(kf[u], qf[1][u], s);
            }
        }
        if constexpr (NB == 1) {
            if (i + 1 < turns) issue(i + 1);       // the buffer is read
        }
        if (!work) continue;
        if (!whole) {
            const uint32_t x = see >> (4 * h);
#pragma unroll
            for (int r = 0; r < 16; ++r) s[r] = seen(s[r], x, 8 * (r / 4) + r % 4);
        }
        float mx = s[0];
#pragma unroll
        for (int r = 1; r < 16; ++r) mx = fmaxf(mx, s[r]);
        if (__any((mx - base) * sc > LAG)) {
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
        bool bad = false;
        if (!whole) {                              // as in few_item
            if (in != ~0u) {
#pragma unroll
                for (int t = 0; t < 2; ++t)
#pragma unroll
                    for (int w = 0; w < 4; ++w) {
                        const uint32_t bits = in >> (16 * t + 8 * (w >> 1) + 4 * h + 2 * (w & 1));
                        const uint32_t m = (bits & 1u ? 0xFFFFu : 0u) | (bits & 2u ? 0xFFFF0000u : 0u);
#pragma unroll
                        for (int mb = 0; mb < MB; ++mb) vf[mb][t][w] &= m;
                    }
            }
            uint32_t top = 0u;
#pragma unroll
            for (int mb = 0; mb < MB; ++mb)
#pragma unroll
                for (int w = 0; w < 8; ++w) top = larger(top, vf[mb][w / 4][w % 4]);
            bad = __any(no_number<KVDT>(top));
            if (bad) {
#pragma unroll
                for (int mb = 0; mb < MB; ++mb)
#pragma unroll
                    for (int w = 0; w < 8; ++w) vf[mb][w / 4][w % 4] &= ~((not_numbers<KVDT>(vf[mb][w / 4][w % 4]) >> 15) * 0xFFFFu);
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
        if (bad) {
#pragma unroll 1
            for (int key = 0; key < AK; ++key) {
                if (!((in >> key) & 1u)) continue;
                float p = 0.f;
#pragma unroll
                for (int r = 0; r < 16; ++r) p = 4 * (key / 8) + key % 4 == r ? pv[r] : p;
                p = __shfl(p, 32 * ((key >> 2) & 1) + ql);
                const int pg = uniform_load(a.tables, (size_t)it.table + ((k0 + key) >> a.shift));
                const uint16_t* vr = a.v + ((((size_t)pg * a.Hkv + g) << a.shift) + ((k0 + key) & pmask)) * D + here(4 * h);
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
    auto quad = [&](int q) { return f32x4_t{o[q / 4][q % 4 * 4], o[q / 4][q % 4 * 4 + 1], o[q / 4][q % 4 * 4 + 2], o[q / 4][q % 4 * 4 + 3]}; };
    f32x4_t* so = (f32x4_t*)lds;                   // [wave][MB][4][64]
    const bool bad = __any(lsum - lsum == 0.f && no_numbers(o));   // as in few_item
    if (lane == 0) words[0] = bad;
    if constexpr (KG > 1) {
        __syncthreads();                           // every wave has read its last step
        if (h == 0) sml[wave * 32 + ql] = float2{base, lsum};
#pragma unroll
        for (int q = 0; q < 4 * MB; ++q) so[(wave * MB * 4 + q) * 64 + lane] = quad(q);
    }
    __syncthreads();
    if (any_wave(words - wave * NB * 64, NB * 64)) return true;
    int cq = c0;
    asm volatile("" : "+v"(cq));
    if (cq >= it.q0 + it.nq) return false;
    const PagedRow ri = a.list[it.rows + cq / a.gs];
    if (it.slot >= ri.nparts) return false;
    const int head = g * a.gs + cq % a.gs;
    const size_t part = ((size_t)(ri.part + it.slot) * Hq + head);
    if constexpr (KG == 1) {
        if (ri.nparts > 1 && h == 0) a.part_ml[part] = float2{base, lsum};
        const float inv = lsum == 0.f ? 0.f : 1.0f / lsum;
#pragma unroll
        for (int q = 0; q < 4 * MB; ++q) put_result<D>(a, ri, part, head, 8 * q + 4 * h, quad(q), inv);
    } else {
        float top = -INFINITY, sum = 0.f, f[KG];
#pragma unroll
        for (int k = 0; k < KG; ++k) top = fmaxf(top, sml[(k * NQT + qt) * 32 + ql].x);
#pragma unroll
        for (int k = 0; k < KG; ++k) {
            const float2 ml = sml[(k * NQT + qt) * 32 + ql];
            f[k] = ml.x == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(ml.x - top);
            sum += ml.y * f[k];
        }
        if (ri.nparts > 1 && h == 0 && kg == 0) a.part_ml[part] = float2{top, sum};
        const float inv = sum == 0.f ? 0.f : 1.0f / sum;
        for (int q = kg; q < MB * 4; q += KG) {    // the tile's waves share its dims
            f32x4_t v = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int k = 0; k < KG; ++k) v += so[((k * NQT + qt) * MB * 4 + q) * 64 + lane] * f[k];
            put_result<D>(a, ri, part, head, 8 * q + 4 * h, v, inv);
        }
    }
    return false;
}

template <int D, int KVDT, int QT>
__global__ __launch_bounds__(256, 2) void paged_many_kernel(PagedAttend a) {
    __shared__ __attribute__((aligned(1024))) uint8_t lds[4 * 2 * 32 * 2 * D];
    __shared__ float2 sml[128];
    __shared__ uint32_t words[4 * 4 * 64];
    const int b = __builtin_amdgcn_readfirstlane(blockIdx.x / a.Hkv), g = __builtin_amdgcn_readfirstlane(blockIdx.x % a.Hkv);
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const PagedItem it = uniform_load(a.items, b);
    const bool two = QT == 2 || (it.open & 4);
    const bool again = it.nq <= 16   ? few_item<D, KVDT, QT, 2>(a, it, g, wave, lds, sml, words)
                       : it.nq <= 32 ? two ? many_item<D, KVDT, QT, 2, 1>(a, it, g, wave, lds, sml, words)
                                           : many_item<D, KVDT, QT, QT, 1>(a, it, g, wave, lds, sml, words)
                       : it.nq <= 64 ? two ? many_item<D, KVDT, QT, 2, 2>(a, it, g, wave, lds, sml, words)
                                           : many_item<D, KVDT, QT, QT, 2>(a, it, g, wave, lds, sml, words)
                       : two         ? many_item<D, KVDT, QT, 2, 4>(a, it, g, wave, lds, sml, words)
                                     : many_item<D, KVDT, QT, QT, 4>(a, it, g, wave, lds, sml, words);
    if (again) each_step<D, KVDT, QT, 2>(a, it, g, wave, lds, sml, words);
}

// Rows with several partial results: m = max m_r, o = sum o_r 2^(m_r - m) / sum l_r 2^(m_r - m), added in the order of the
// runs.  One wave per row and head; the first eight results are under way before their weights are known.  Bound by latency:
// 4 us for one row, 6 for 3840 rows and heads of 7 results.
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
// bits); k and v go to their rows of the pages.  Bound by memory (4096 rows of 64 + 16 heads of 128, fp32 to bf16: 52 us,
// 4.8 TB/s; a large copy 4.9).  A thread takes four neighbouring pairs, so 16 (or 8) threads a head; the angles of a row are
// read once per thread and reused for the heads that it walks.
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
// up to 64 rows of it, four loads a thread in flight (16 layers of 8 x 128: 40 rows to each of 64 pages 37 us, 4.8 TB/s; 3400
// rows closed up 81 us, 5.5 TB/s).

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

__global__ __launch_bounds__(256) void paged_send_kernel(const u32x4* host, u32x4* dev, int n) {
    const int i = blockIdx.x * 256 + threadIdx.x;
    if (i < n) dev[i] = host[i];
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
    const size_t items = (size_t)a.n_items * a.Hkv, waves = (size_t)a.M * a.Hkv * a.gs;
    if (a.n_items < 1 || items >= (1u << 24) || waves >= (1u << 24)) return hipErrorInvalidValue;
    const bool f32 = a.q_dt == DT_F32, bf = kv_dt == DT_BF16;
    if ((!f32 && a.q_dt != kv_dt) || (D != 64 && D != 128)) return hipErrorInvalidValue;
    const dim3 block(256), grid((unsigned)items), mg((unsigned)((waves + 3) / 4));
    const hipEvent_t d = a.merge ? nullptr : done;
#define PAGED_KERNEL(D_, KV_)                                                                                                  \
    (a.many ? f32 ? launch_done(paged_many_kernel<D_, KV_, 2>, grid, block, 0, st, d, a)                                       \
                  : launch_done(paged_many_kernel<D_, KV_, 1>, grid, block, 0, st, d, a)                                       \
            : f32 ? launch_done(paged_few_kernel<D_, KV_, 2>, grid, block, 0, st, d, a)                                        \
                  : launch_done(paged_few_kernel<D_, KV_, 1>, grid, block, 0, st, d, a))
    const hipError_t e = D == 128 ? (bf ? PAGED_KERNEL(128, DT_BF16) : PAGED_KERNEL(128, DT_F16))
                                  : (bf ? PAGED_KERNEL(64, DT_BF16) : PAGED_KERNEL(64, DT_F16));
#undef PAGED_KERNEL
    if (e != hipSuccess || !a.merge) return e;
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

hipError_t launch_paged_send(const void* host, void* dev, size_t bytes, hipStream_t st, hipEvent_t done) {
    const int n = (int)((bytes + 15) / 16);
    if (n < 1 || bytes > (1u << 24)) return hipErrorInvalidValue;
    return launch_done(paged_send_kernel, dim3((n + 255) / 256), dim3(256), 0, st, done, (const u32x4*)host, (u32x4*)dev, n);
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
