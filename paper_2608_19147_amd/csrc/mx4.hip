// MXFP4 (blocks of 32 values along a row: E2M1 codes and one power-of-two E8M0
// scale) on the gfx950 matrix cores.
//
// Rounding a block x[0..31]: byte = floor(log2 max|x|) - 2 + 127, at least 0;
// code = x / 2^(byte - 127) to the nearest E2M1 value, ties to the even code, at
// most 6 in magnitude.  A block of zeros has byte 0; a block with a NaN or an
// infinity has byte 255 (every value of it reads as NaN) and zero codes.
//
// Products: out[m][n] = sum_k x[m][k] W[n][k], W in MXFP4.  The scaled matrix
// instruction takes E2M1 codes with their scale bytes as they are, so weights
// are never unpacked.  Activations of 16 bits go in as sums of E4M3 terms, each
// with its own block scales: t1 = E4M3(x), t2 = E4M3(x - t1), ...  Measured on
// the instruction: the 8 products of neighbouring elements are added in units of
// 2^-13 of the largest one's power of two, what is below is cut off; groups of 8
// and the accumulator are added as fp32.  A term is therefore scaled to a largest
// magnitude in [1, 2): E4M3's smallest step is 2^-9, so that every product is a
// multiple of 2^-10 and below 12, and nothing is cut.  (Scaled to E4M3's full
// range instead, results of 32 bits were 1e-5 off.)  What a term leaves of x is
// at most 2^-4 of x and of a block at most 2^-4 of its largest magnitude (half
// the last of 4 bits), or 2^-10 where E4M3's smallest step decides: three terms
// come within 2^-18 of a block's largest magnitude, and the larger elements are
// exact.  (Two terms, 2^-14, kept some 6 of the 8 bits of a bf16 element 2^-8
// below its block's largest: 16-bit results were 3e-4 apart from those of products
// in fp32, single ones by a step; three terms take 85 us at 517 x 4096 x 14336 and
// 7.0 for one row of 4096 x 4096, two took 66 and 6.7.)
// Activations of 4 bits are one E2M1 term.
#include "device.h"

namespace stg {

typedef int v8i __attribute__((ext_vector_type(8)));
typedef float v16f __attribute__((ext_vector_type(16)));

// ------------------------------------------------------------------ E2M1, E4M3

// Codes of eight values times `inv` (then below 8 in magnitude): nearest, ties
// to even, at most 6; the first value in the low bits.  The conversion does all
// of that; its scale operand is left at 1 and the power of two multiplied in
// before, exactly, also where it is subnormal.
__device__ __forceinline__ uint32_t e2m1x8(const float (&v)[8], float inv) {
    uint32_t w = 0;
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, v[0] * inv, v[1] * inv, 1.0f, 0);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, v[2] * inv, v[3] * inv, 1.0f, 1);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, v[4] * inv, v[5] * inv, 1.0f, 2);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, v[6] * inv, v[7] * inv, 1.0f, 3);
    return w;
}

__device__ __forceinline__ float e2m1_value(uint32_t c) {
    const uint32_t m = c & 7u;
    const float a = m < 2u ? 0.5f * (float)m : __uint_as_float((126u + (m >> 1)) << 23 | (m & 1u) << 22);
    return (c & 8u) ? -a : a;
}

// 2^(byte - 127); byte 255 is NaN.
__device__ __forceinline__ float e8m0(uint32_t byte) {
    return __uint_as_float(byte == 255u ? 0x7fc00000u : byte == 0u ? 0x00400000u : byte << 23);
}
// 2^(127 - byte), byte <= 252.
__device__ __forceinline__ float e8m0_inv(uint32_t byte) { return __uint_as_float((254u - byte) << 23); }

// Scale byte of a block whose largest magnitude has the fp32 bits `top`, with
// the block's largest scaled magnitude in [2^e, 2^(e+1)).
__device__ __forceinline__ uint32_t block_byte(uint32_t top, int e) {
    if (top >= 0x7f800000u) return 255u;
    const int b = (int)(top >> 23) - e;
    return (uint32_t)(b < 0 ? 0 : b);
}

__device__ __forceinline__ uint32_t absbits(float v) { return __float_as_uint(v) & 0x7fffffffu; }

// ------------------------------------------------------------------ quantize

// Eight values of a row a thread, four neighbouring threads a block: their
// largest magnitude is shared by lane exchanges, each writes 4 bytes of codes.
// Bound by memory: 2 bytes a value read (16 bits), 17/32 written (2048 x 14336:
// 13.8 us, 5.4 TB/s where a large copy reaches 5.1; one row of 4096: 2.0 us, the
// least a launch takes).
template <int DT>
__global__ __launch_bounds__(256) void mx4_quantize_kernel(const void* __restrict__ x, size_t ld, int m, int k, int chunks,
                                                           uint8_t* __restrict__ codes, uint8_t* __restrict__ scales) {
    // chunks: of 8 values in a row, a multiple of 4
    const size_t idx = blockIdx.x * (size_t)256 + threadIdx.x;
    if (idx >= (size_t)m * chunks) return;                         // whole blocks of 32 leave together
    const bool small = (size_t)m * chunks < ((size_t)1 << 32);
    const size_t r = small ? (size_t)((uint32_t)idx / (uint32_t)chunks) : idx / chunks;
    const int c = (int)(idx - r * chunks), i0 = 8 * c;
    float v[8];
    if (i0 + 8 <= k) {
        if constexpr (DT == DT_F32) {
            const u32x4_any* p = (const u32x4_any*)((const float*)x + r * ld + i0);
            const u32x4 a = p[0], b = p[1];
#pragma unroll
            for (int j = 0; j < 4; ++j) { v[j] = __uint_as_float(a[j]); v[4 + j] = __uint_as_float(b[j]); }
        } else {
            const u32x4 a = *(const u32x4_any*)((const uint16_t*)x + r * ld + i0);
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] = half_bits_to_f32((uint16_t)(a[j >> 1] >> (16 * (j & 1))), DT);
        }
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = i0 + j < k ? load_val(x, DT, r * ld + i0 + j) : 0.0f;
    }
    uint32_t top = 0;
#pragma unroll
    for (int j = 0; j < 8; ++j) top = max(top, absbits(v[j]));
    top = max(top, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)top, 0xB1, 0xF, 0xF, false));   // lane ^ 1
    top = max(top, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)top, 0x4E, 0xF, 0xF, false));   // lane ^ 2
    if (i0 >= k) return;
    const uint32_t byte = block_byte(top, 2);
    const uint32_t w = byte == 255u ? 0u : e2m1x8(v, e8m0_inv(byte));
    uint8_t* o = codes + r * ((size_t)(k + 1) / 2) + i0 / 2;
    if (i0 + 8 <= k) {
        *(u32_any*)o = w;
    } else {
#pragma unroll
        for (int j = 0; j < 4; ++j)
            if (i0 + 2 * j < k) o[j] = (uint8_t)(w >> (8 * j));
    }
    if ((c & 3) == 0) scales[r * (size_t)(chunks / 4) + c / 4] = (uint8_t)byte;
}

hipError_t launch_mx4_quantize(const void* x, int dt, int64_t ld, int m, int k, uint8_t* codes, uint8_t* scales, hipStream_t st) {
    const int chunks = (k + 31) / 32 * 4;
    const size_t n = (size_t)m * chunks;
    const dim3 g((unsigned)((n + 255) / 256)), b(256);
#define MX4_Q(DT) mx4_quantize_kernel<DT><<<g, b, 0, st>>>(x, (size_t)ld, m, k, chunks, codes, scales)
    if (dt == DT_F32) MX4_Q(DT_F32);
    else if (dt == DT_F16) MX4_Q(DT_F16);
    else MX4_Q(DT_BF16);
#undef MX4_Q
    return hipGetLastError();
}

// Eight values a thread.  Reads 17/32 bytes a value and writes 2 (16 bits; 2048 x 14336:
// 20 us, 3.7 TB/s).  Bound by the issue of vector instructions, 29 a value: 12,800 a SIMD
// in 42,800 busy cycles; a fill writes as much in 10 us.  PAST_L2: the values are stored
// past the L2s, which they would fill (2048 x 14336 rounded and back: 36.6 us through
// them, 32.6 past them).
template <int DT, bool PAST_L2>
__global__ __launch_bounds__(256) void mx4_dequantize_kernel(const uint8_t* __restrict__ codes, const uint8_t* __restrict__ scales,
                                                             int m, int k, int chunks, void* __restrict__ out, size_t ld) {
    const size_t idx = blockIdx.x * (size_t)256 + threadIdx.x;
    if (idx >= (size_t)m * chunks) return;
    const bool small = (size_t)m * chunks < ((size_t)1 << 32);
    const size_t r = small ? (size_t)((uint32_t)idx / (uint32_t)chunks) : idx / chunks;
    const int c = (int)(idx - r * chunks), i0 = 8 * c;
    const uint8_t* p = codes + r * ((size_t)(k + 1) / 2) + i0 / 2;
    uint32_t w = 0;
    const bool whole = i0 + 8 <= k;
    if (whole) {
        w = *(const u32_any*)p;
    } else {
#pragma unroll
        for (int j = 0; j < 4; ++j)
            if (i0 + 2 * j < k) w |= (uint32_t)p[j] << (8 * j);
    }
    const float s = e8m0(scales[r * (size_t)((k + 31) / 32) + c / 4]);
    float v[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = e2m1_value(w >> (4 * j)) * s;
    const size_t at = r * ld + i0;
    if constexpr (DT == DT_F32) {
        if (whole) {
            u32x4_any* o = (u32x4_any*)((float*)out + at);
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                const u32x4 q = {__float_as_uint(v[4 * j]), __float_as_uint(v[4 * j + 1]), __float_as_uint(v[4 * j + 2]), __float_as_uint(v[4 * j + 3])};
                if constexpr (PAST_L2) __builtin_nontemporal_store(q, o + j);
                else o[j] = q;
            }
        } else {
#pragma unroll
            for (int j = 0; j < 8; ++j)
                if (i0 + j < k) ((float*)out)[at + j] = v[j];
        }
    } else {
        if (whole) {
            u32x4 o;
#pragma unroll
            for (int j = 0; j < 4; ++j) o[j] = (uint32_t)to_half_bits(v[2 * j], DT) | (uint32_t)to_half_bits(v[2 * j + 1], DT) << 16;
            u32x4_any* q = (u32x4_any*)((uint16_t*)out + at);
            if constexpr (PAST_L2) __builtin_nontemporal_store(o, q);
            else *q = o;
        } else {
#pragma unroll
            for (int j = 0; j < 8; ++j)
                if (i0 + j < k) ((uint16_t*)out)[at + j] = to_half_bits(v[j], DT);
        }
    }
}

hipError_t launch_mx4_dequantize(const uint8_t* codes, const uint8_t* scales, int m, int k, void* out, int dt, int64_t ld,
                                 hipStream_t st) {
    const int chunks = (k + 7) / 8;
    const size_t n = (size_t)m * chunks;
    const dim3 g((unsigned)((n + 255) / 256)), b(256);
    const bool past = (size_t)m * k * (dt == DT_F32 ? 4 : 2) > ((size_t)32 << 20);     // 8 L2s of 4 MB
#define MX4_D(DT, PAST) mx4_dequantize_kernel<DT, PAST><<<g, b, 0, st>>>(codes, scales, m, k, chunks, out, (size_t)ld)
    if (dt == DT_F32) past ? MX4_D(DT_F32, true) : MX4_D(DT_F32, false);
    else if (dt == DT_F16) past ? MX4_D(DT_F16, true) : MX4_D(DT_F16, false);
    else past ? MX4_D(DT_BF16, true) : MX4_D(DT_BF16, false);
#undef MX4_D
    return hipGetLastError();
}

// ------------------------------------------------------------------ weights

// One thread per 16-byte piece (32 codes: one row and block) of the packed form.
// Runs once a matrix, so it reads the codes byte by byte.
__global__ __launch_bounds__(256) void mx4_pack_kernel(const uint8_t* __restrict__ codes, const uint8_t* __restrict__ scales,
                                                       Mx4Mat w) {
    const size_t idx = blockIdx.x * (size_t)256 + threadIdx.x;     // [group][step][j][lane]
    if (idx >= (size_t)w.groups * w.steps * 128) return;
    const int lane = (int)(idx & 63), j = (int)(idx >> 6) & 1;
    const size_t gs = idx >> 7;
    const int s = (int)(gs % w.steps), g = (int)(gs / w.steps);
    const int row = 64 * g + 2 * (lane & 31) + j, b = 2 * s + (lane >> 5);
    const size_t rb = (size_t)(w.k + 1) / 2;
    uint8_t c[16];
    uint8_t byte = 127;
    const bool in = row < w.n && 32 * b < w.k;
    for (int i = 0; i < 16; ++i) {
        const int kk = 32 * b + 2 * i;
        uint8_t v = in && kk < w.k ? codes[row * rb + kk / 2] : 0;
        if (kk + 1 >= w.k) v &= 15;                                // an odd k leaves the high nibble unused
        c[i] = v;
    }
    if (in) byte = scales[(size_t)row * ((w.k + 31) / 32) + b];
    u32x4 o;
    for (int i = 0; i < 4; ++i) o[i] = c[4 * i] | c[4 * i + 1] << 8 | c[4 * i + 2] << 16 | (uint32_t)c[4 * i + 3] << 24;
    ((u32x4*)w.w)[idx] = o;
    ((uint8_t*)w.s)[((((size_t)g * (w.steps / 4) + s / 4) * 64 + lane) * 2 + j) * 4 + (s & 3)] = byte;
}

hipError_t launch_mx4_pack(const uint8_t* codes, const uint8_t* scales, const Mx4Mat& w, hipStream_t st) {
    const size_t n = (size_t)w.groups * w.steps * 128;
    mx4_pack_kernel<<<dim3((unsigned)((n + 255) / 256)), dim3(256), 0, st>>>(codes, scales, w);
    return hipGetLastError();
}

// ------------------------------------------------------------------ activations

// Values at .. at + 15 of x, zero from `left` on.
template <int DT>
__device__ __forceinline__ void load16(const void* x, size_t at, int left, float (&v)[16]) {
    if constexpr (DT == DT_F32) {
        const float* f = (const float*)x + at;
        if (left >= 16) {
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const u32x4 a = ((const u32x4_any*)f)[q];
#pragma unroll
                for (int j = 0; j < 4; ++j) v[4 * q + j] = __uint_as_float(a[j]);
            }
        } else {
#pragma unroll
            for (int j = 0; j < 16; ++j) v[j] = j < left ? f[j] : 0.0f;
        }
    } else {
        const uint16_t* f = (const uint16_t*)x + at;
        u32x4 a[2];
        if (left >= 16) {
            a[0] = ((const u32x4_any*)f)[0];
            a[1] = ((const u32x4_any*)f)[1];
        } else {
#pragma unroll
            for (int j = 0; j < 8; ++j)
                a[j >> 2][j & 3] = (2 * j < left ? (uint32_t)f[2 * j] : 0u) | (2 * j + 1 < left ? (uint32_t)f[2 * j + 1] << 16 : 0u);
        }
#pragma unroll
        for (int j = 0; j < 16; ++j) v[j] = half_bits_to_f32((uint16_t)(a[j >> 3][(j >> 1) & 3] >> (16 * (j & 1))), DT);
    }
}

// One E4M3 term of 16 values: 16 bytes; v keeps what is left.
__device__ __forceinline__ u32x4 take_term(float (&v)[16]) {
    u32x4 o;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        int w = __builtin_amdgcn_cvt_pk_fp8_f32(v[4 * i], v[4 * i + 1], 0, false);
        w = __builtin_amdgcn_cvt_pk_fp8_f32(v[4 * i + 2], v[4 * i + 3], w, true);
        o[i] = (uint32_t)w;
        v[4 * i] -= __builtin_amdgcn_cvt_f32_fp8(w, 0);
        v[4 * i + 1] -= __builtin_amdgcn_cvt_f32_fp8(w, 1);
        v[4 * i + 2] -= __builtin_amdgcn_cvt_f32_fp8(w, 2);
        v[4 * i + 3] -= __builtin_amdgcn_cvt_f32_fp8(w, 3);
    }
    return o;
}

// The first term's scale byte of a block: largest scaled magnitude in [1, 2).
__device__ __forceinline__ int term_byte(uint32_t top) { return min((int)block_byte(top, 0), 252); }
// The next one's, from what is left (scaled by the last one's), and the power of two between them.
__device__ __forceinline__ int next_byte(int byte, uint32_t rest, float* up) {
    int e = rest ? (int)(rest >> 23) - 127 : 0;
    e = max(e, max(-byte, -127));
    *up = __uint_as_float((uint32_t)(127 - e) << 23);
    return byte + e;
}
__device__ __forceinline__ uint32_t top16(const float (&v)[16]) {
    uint32_t top = 0;
#pragma unroll
    for (int i = 0; i < 16; ++i) top = max(top, absbits(v[i]));
    return top;
}

// 16 values of one row (half a block) a thread; the two threads of a block are
// neighbours and share its largest magnitude.  A workgroup takes 32 rows by two
// steps: it reads 256 bytes of a 16-bit row and writes whole fragments.  Rows from
// m and columns from k on are zero.  T terms of E4M3 (T = 0: one E2M1 term).  Bound
// by memory (517 x 14336 in three terms: 14.8 MB read, 24 written, 9.0 us), for few
// rows by its launch (20 x 4096 in three: 5.1 us).
template <int T, int DT>
__global__ __launch_bounds__(256) void mx4_prep_kernel(const void* __restrict__ x, size_t ld, int m, int k, int steps,
                                                       uint8_t* __restrict__ a, uint8_t* __restrict__ as) {
    constexpr int NT = T ? T : 1, U = T ? 2 : 1;
    const int p = threadIdx.x & 3;                                 // quarter of the step of 64
    const int s = 2 * blockIdx.x + (threadIdx.x >> 7), row = 32 * blockIdx.y + ((threadIdx.x >> 2) & 31);
    const int k0 = 64 * s + 16 * p;
    float v[16];
    load16<DT>(x, (size_t)row * ld + k0, row < m ? k - k0 : 0, v);
    uint32_t top = top16(v);
    top = max(top, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)top, 0xB1, 0xF, 0xF, false));   // lane ^ 1
    const size_t tile = row >> 5;
    const int r = row & 31, b = p >> 1;
    const size_t frag = (tile * steps + s) * (size_t)(NT * U) * 1024;
    const size_t sc = ((((tile >> 2) * (steps / 4) + s / 4) * NT * 64 + b * 32 + r) * 4 + (tile & 3)) * 4 + (s & 3);
    if constexpr (T == 0) {
        const uint32_t byte = block_byte(top, 2);
        const float inv = byte == 255u ? 0.0f : e8m0_inv(byte);
        float h[2][8];
#pragma unroll
        for (int i = 0; i < 16; ++i) h[i >> 3][i & 7] = byte == 255u ? 0.0f : v[i];
        const u32x2 o = {e2m1x8(h[0], inv), e2m1x8(h[1], inv)};
        *(u32x2*)(a + frag + (b * 32 + r) * 16 + (p & 1) * 8) = o;
        if (!(p & 1)) as[sc] = (uint8_t)byte;
    } else {
        const bool bad = top >= 0x7f800000u;
        int byte = bad ? 0 : term_byte(top);
        const float inv = bad ? 0.0f : e8m0_inv((uint32_t)byte);
#pragma unroll
        for (int i = 0; i < 16; ++i) v[i] = bad ? 0.0f : v[i] * inv;
#pragma unroll
        for (int t = 0; t < NT; ++t) {
            // element e of lane 32 g + r: k = 16 g + e for the first 16, 32 + 16 g + e - 16 for the others
            *(u32x4*)(a + frag + ((size_t)t * 2 + b) * 1024 + ((p & 1) * 32 + r) * 16) = take_term(v);
            if (!(p & 1)) as[sc + (size_t)t * 1024] = (uint8_t)(bad ? 255 : byte);
            if (t + 1 < NT) {
                uint32_t rest = top16(v);
                rest = max(rest, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)rest, 0xB1, 0xF, 0xF, false));
                float up;
                byte = next_byte(byte, rest, &up);
#pragma unroll
                for (int i = 0; i < 16; ++i) v[i] *= up;
            }
        }
    }
}

hipError_t launch_mx4_prep(const Mx4Act& a, const void* x, int dt, int64_t ld, int m, int k, hipStream_t st) {
    const dim3 g((unsigned)(a.steps / 2), (unsigned)a.tiles), b(256);
#define MX4_PREP(T, DT) mx4_prep_kernel<T, DT><<<g, b, 0, st>>>(x, (size_t)ld, m, k, a.steps, a.a, a.s)
    switch (a.terms * 4 + dt) {
        case DT_F32: MX4_PREP(0, DT_F32); break;
        case DT_F16: MX4_PREP(0, DT_F16); break;
        case DT_BF16: MX4_PREP(0, DT_BF16); break;
        case 12 + DT_F32: MX4_PREP(3, DT_F32); break;
        case 12 + DT_F16: MX4_PREP(3, DT_F16); break;
        case 12 + DT_BF16: MX4_PREP(3, DT_BF16); break;
        default: return hipErrorInvalidValue;
    }
#undef MX4_PREP
    return hipGetLastError();
}

// ------------------------------------------------------------------ product

// Outputs v of row `row`, columns col .. col + N - 1 (N 4 or 8), as far as the n columns go.
template <int DT, int N>
__device__ __forceinline__ void store_run(void* out, size_t ld, int n, int row, int col, const float (&v)[N]) {
    const size_t at = (size_t)row * ld + col;
    if constexpr (DT == DT_F32) {
        float* o = (float*)out + at;
        if (col + N <= n) {
#pragma unroll
            for (int j = 0; j < N; j += 4)
                *(u32x4_any*)(o + j) = u32x4{__float_as_uint(v[j]), __float_as_uint(v[j + 1]), __float_as_uint(v[j + 2]), __float_as_uint(v[j + 3])};
        } else {
#pragma unroll
            for (int j = 0; j < N; ++j)
                if (col + j < n) o[j] = v[j];
        }
    } else {
        typedef __bf16 bf2 __attribute__((ext_vector_type(2)));
        uint16_t* o = (uint16_t*)out + at;
        uint32_t h[N / 2];
#pragma unroll
        for (int j = 0; j < N / 2; ++j)
            h[j] = DT == DT_BF16 ? __builtin_bit_cast(uint32_t, bf2{(__bf16)v[2 * j], (__bf16)v[2 * j + 1]}) : pack_f16x2(v[2 * j], v[2 * j + 1]);
        if (col + N <= n) {
            if constexpr (N == 8) *(u32x4_any*)o = u32x4{h[0], h[1], h[2], h[3]};
            else *(u32x2_any*)o = u32x2{h[0], h[1]};
        } else {
#pragma unroll
            for (int j = 0; j < N; ++j)
                if (col + j < n) o[j] = (uint16_t)(h[j / 2] >> (16 * (j & 1)));
        }
    }
}

// The product of a fragment pair; the scale bytes are byte `step` (0..3) of their words.
template <int FMT>
__device__ __forceinline__ v16f mx4_mfma(v8i a, v8i b, v16f c, int step, uint32_t sa, uint32_t sb) {
    switch (step) {                                                // a constant where this is used
        case 0: return __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(a, b, c, FMT, 4, 0, (int)sa, 0, (int)sb);
        case 1: return __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(a, b, c, FMT, 4, 1, (int)sa, 1, (int)sb);
        case 2: return __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(a, b, c, FMT, 4, 2, (int)sa, 2, (int)sb);
        default: return __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(a, b, c, FMT, 4, 3, (int)sa, 3, (int)sb);
    }
}

// The outputs of a wave: MT row tiles from mt0, group g.  Lane l holds outputs
// 64 g + 2 (l mod 32) + j of rows 8 (r / 4) + 4 (l / 32) + r mod 4.  Sums of a split
// go straight to their rows, which are whole tiles, a group's even outputs ahead of
// its odd ones (as pairs they would have to be moved to neighbouring registers first).
// Results go through LDS of the wave's own, two tiles at a time, so that short loops
// store their rows, 16 or 32 bytes a lane: stores straight from the registers were
// 20 KB of instructions for 8 tiles, and fetching them took most of 12 us a workgroup.
constexpr int STORE_LD = 72;                                       // rows 4 apart lie in other banks
constexpr int store_lds(int mt) { return 4 * (mt < 2 ? 1 : 2) * 32 * STORE_LD * 4; }
// LDS accesses of a wave's lanes on either side keep their order (the unit takes a wave's in order).
__device__ __forceinline__ void wave_lds_order() {
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
}
template <bool WIDE>
__device__ __forceinline__ void store_rows(const float* buf, const Mx4Gemm& p, int row0, int rows, int col0) {
    const int lane = threadIdx.x & 63, c = 8 * (lane & 7);
    const bool whole = col0 + c + 8 <= p.w.n;
#pragma unroll 1
    for (int i0 = 0; i0 < rows; i0 += 32) {
        float4 a[4], b[4];
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            const float* f = buf + (i0 + 8 * q + (lane >> 3)) * STORE_LD + c / 2;
            a[q] = *(const float4*)f;
            b[q] = *(const float4*)(f + 32);
        }
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            const int i = i0 + 8 * q + (lane >> 3);
            const float v[8] = {a[q].x, b[q].x, a[q].y, b[q].y, a[q].z, b[q].z, a[q].w, b[q].w};
            if (i >= rows) break;
            if (whole) {
                if constexpr (WIDE) store_run<DT_F32, 8>(p.out, p.ld, p.w.n, row0 + i, col0 + c, v);
                else if (p.dt == DT_F16) store_run<DT_F16, 8>(p.out, p.ld, p.w.n, row0 + i, col0 + c, v);
                else store_run<DT_BF16, 8>(p.out, p.ld, p.w.n, row0 + i, col0 + c, v);
            }
        }
    }
    if (whole) return;
#pragma unroll 1
    for (int i = lane >> 3; i < rows; i += 8)
#pragma unroll 1
        for (int j = c; col0 + j < p.w.n; ++j) {
            const float f = buf[i * STORE_LD + (j & 1) * 32 + j / 2];
            const size_t at = (size_t)(row0 + i) * p.ld + col0 + j;
            if constexpr (WIDE) ((float*)p.out)[at] = f;
            else ((uint16_t*)p.out)[at] = to_half_bits(f, p.dt);
        }
}
template <int MT>
__device__ __forceinline__ void store_tiles(const Mx4Gemm& p, int mt0, int g, const v16f (&acc)[MT][2], uint8_t* lds) {
    constexpr int PASS = MT < 2 ? 1 : 2;
    const int lane = threadIdx.x & 63;
    const int tiles = min(MT, p.a.tiles - mt0);
    if (p.split > 1) {
        g = __builtin_amdgcn_readfirstlane(g);
        float* part = p.part + ((size_t)blockIdx.z * p.a.tiles + mt0) * 32 * p.part_ld + 64 * g;
        const uint32_t at = 4 * (lane >> 5) * p.part_ld + (lane & 31);
#pragma unroll
        for (int t = 0; t < MT; ++t) {
            if (t >= tiles) return;
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                float* o = part + (size_t)(32 * t + 8 * (r >> 2) + (r & 3)) * p.part_ld;
                o[at] = acc[t][0][r];
                o[at + 32] = acc[t][1][r];
            }
        }
        return;
    }
    float* buf = (float*)lds + PASS * 32 * STORE_LD * (threadIdx.x >> 6);
    float* own = buf + 4 * (lane >> 5) * STORE_LD + (lane & 31);
#pragma unroll
    for (int t0 = 0; t0 < MT; t0 += PASS) {
        if (t0 >= tiles) return;
#pragma unroll
        for (int t = t0; t < t0 + PASS; ++t)
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                float* o = own + ((t - t0) * 32 + 8 * (r >> 2) + (r & 3)) * STORE_LD;
                o[0] = acc[t][0][r];
                o[32] = acc[t][1][r];
            }
        wave_lds_order();
        const int row0 = (mt0 + t0) * 32, rows = min(32 * PASS, p.m - row0);
        if (p.dt == DT_F32) store_rows<true>(buf, p, row0, rows, 64 * g);
        else store_rows<false>(buf, p, row0, rows, 64 * g);
        wave_lds_order();
    }
}

// Scale words of MT row tiles (1, 2 or 4, from a multiple of MT on) and a group of W,
// four steps at once.
template <int NT, int MT>
struct ScaleLoad {
    const uint32_t* a;
    const u32x2* w;
    __device__ __forceinline__ ScaleLoad(const Mx4Gemm& p, int mt0, int g, int lane) {
        const int quads = p.w.steps / 4;
        a = (const uint32_t*)p.a.s + ((size_t)(mt0 / 4) * quads * NT * 64 + lane) * 4 + mt0 % 4;
        w = (const u32x2*)p.w.s + (size_t)g * quads * 64 + lane;
    }
    __device__ __forceinline__ void load(int quad, uint32_t (&as)[MT][NT], uint32_t (&ws)[2]) const {
        const u32x2 v = w[(size_t)quad * 64];
        ws[0] = v[0];
        ws[1] = v[1];
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            const uint32_t* s = a + ((size_t)quad * NT + n) * 256;
            if constexpr (MT == 1) as[0][n] = s[0];
            else if constexpr (MT == 2) {
                const u32x2 t = *(const u32x2*)s;
                as[0][n] = t[0];
                as[1][n] = t[1];
            } else {
                const u32x4 t = *(const u32x4*)s;
#pragma unroll
                for (int i = 0; i < 4; ++i) as[i][n] = t[i];
            }
        }
    }
};

// Neighbouring workgroups go to different XCDs: gives each XCD a run of tiles,
// row tiles first, so that its L2 holds the weights of few groups and every tile
// of them.
__device__ __forceinline__ int xcd_run(int bid, int nwg) {
    const int per = nwg >> 3, more = nwg & 7, x = bid & 7;
    return x * per + min(x, more) + (bid >> 3);
}

// One workgroup: 32 MT rows of x by 256 outputs, one 64-row group of W a wave,
// over steps_per = a multiple of 4 steps of K (blockIdx.z: the split).  The
// activations' fragments are shared by the four waves through LDS, double
// buffered; W's go from memory to the registers that the product reads, each
// used for MT tiles.  T terms of E4M3 (0: one of E2M1), KS steps a buffer.  With few
// rows bound by reading the weights (20 x 128256 x 4096: 53 us, 5.2 TB/s), with some
// hundred by what a CU reads, 14 KB a step of one tile with three terms, 0.35 us (256 x
// 4096 x 4096: 19 us; a second set of waves on the other half of K gained 3%).
//
// split > 1: fp32 sums to part [split][tiles of 32 rows][n], joined by mx4_reduce_kernel.
template <int T, int MT, int KS>
__global__ __launch_bounds__(256) void mx4_gemm_kernel(Mx4Gemm p) {
    constexpr int NT = T ? T : 1, U = T ? 2 : 1, FMT = T ? 0 : 4;
    constexpr int PIECES = MT * KS * NT * U;                       // kilobytes of a buffer
    constexpr int PW = PIECES / 4;                                 // loaded by a wave
    constexpr int FRAGS = MT * KS * NT, DEPTH = FRAGS < 4 ? FRAGS : T ? 2 : 4;
    static_assert(PIECES % 4 == 0 && 4 % KS == 0, "buffer");
    extern __shared__ __attribute__((aligned(16))) uint8_t smem[];
    u32x4* lds = (u32x4*)smem;                                     // [2][PIECES * 64]
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int bid = xcd_run(blockIdx.x, gridDim.x);
    const int mt0 = (bid % p.mtiles) * MT;
    int g = (bid / p.mtiles) * 4 + wave;
    const bool off = g >= p.w.groups;                              // a wave without outputs keeps step with the others
    if (off) g = p.w.groups - 1;
    const int steps = p.w.steps, s0 = blockIdx.z * p.steps_per, s1 = min(steps, s0 + p.steps_per);
    const u32x4* wp = (const u32x4*)p.w.w + (size_t)g * steps * 128 + lane;
    const ScaleLoad<NT, MT> sl(p, mt0, g, lane);
    // this wave's pieces of a buffer: piece q of tile q / (KS NT U); tiles past the last are the last one again
    const u32x4* ap[PW];
#pragma unroll
    for (int q = 0; q < PW; ++q) {
        const int i = wave * PW + q, tile = min(mt0 + i / (KS * NT * U), p.a.tiles - 1);
        ap[q] = (const u32x4*)p.a.a + ((size_t)tile * steps * (NT * U) + i % (KS * NT * U)) * 64 + lane;
    }
    v16f acc[MT][2] = {};
    u32x4 ar[PW], wr[2][KS][2];
    uint32_t wsc[2], asc[MT][NT], wsn[2], asn[MT][NT];
    auto load_a = [&](int s) {
#pragma unroll
        for (int q = 0; q < PW; ++q) ar[q] = ap[q][(size_t)s * (NT * U * 64)];
    };
    auto load_w = [&](int s, u32x4 (&r)[KS][2]) {
#pragma unroll
        for (int i = 0; i < KS; ++i)
#pragma unroll
            for (int j = 0; j < 2; ++j) r[i][j] = wp[(size_t)(s + i) * 128 + j * 64];
    };
    auto load_s = [&](int s) { sl.load(s / 4, asn, wsn); };
    load_s(s0);
    load_a(s0);
    load_w(s0, wr[0]);
#pragma unroll
    for (int q = 0; q < PW; ++q) lds[(wave * PW + q) * 64 + lane] = ar[q];
    for (int s = s0; s < s1; s += 4) {
#pragma unroll
        for (int j = 0; j < 2; ++j) wsc[j] = wsn[j];
#pragma unroll
        for (int t = 0; t < MT; ++t)
#pragma unroll
            for (int n = 0; n < NT; ++n) asc[t][n] = asn[t][n];
        const int s_next = s + 4 < s1 ? s + 4 : s;
#pragma unroll
        for (int h = 0; h < 4 / KS; ++h) {
            constexpr int PAR = (4 / KS) & 1;                      // buffers alternate; with one a round, by rounds
            const int cur = PAR ? ((s - s0) >> 2) & 1 : h & 1;
            __syncthreads();                                       // this buffer is written, the other one read
            const int sn = h + 1 < 4 / KS ? s + (h + 1) * KS : s_next;
            load_a(sn);
            load_w(sn, wr[1]);
            if (h == 4 / KS - 1) load_s(s_next);
            // fragments in the order of use, read DEPTH ahead of their products; the scheduling barriers keep the loads
            // above in front (the compiler had sunk them behind the products that cover them) and the reads ahead
            const u32x4* buf = lds + cur * PIECES * 64 + lane;
            u32x4 fr[DEPTH + 1][U];
            auto read = [&](int e) {
                const int i = e / (MT * NT), t = e / NT % MT, n = e % NT;
#pragma unroll
                for (int u = 0; u < U; ++u) fr[e % (DEPTH + 1)][u] = buf[(((t * KS + i) * NT + n) * U + u) * 64];
            };
#pragma unroll
            for (int e = 0; e < DEPTH; ++e) read(e);
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int e = 0; e < FRAGS; ++e) {
                const int i = e / (MT * NT), t = e / NT % MT, n = e % NT;
                if (e + DEPTH < FRAGS) read(e + DEPTH);
                const u32x4 lo = fr[e % (DEPTH + 1)][0], hi = U == 2 ? fr[e % (DEPTH + 1)][U - 1] : u32x4{0u, 0u, 0u, 0u};
                const v8i a = {(int)lo[0], (int)lo[1], (int)lo[2], (int)lo[3], (int)hi[0], (int)hi[1], (int)hi[2], (int)hi[3]};
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    const u32x4 f = wr[0][i][j];
                    const v8i b = {(int)f[0], (int)f[1], (int)f[2], (int)f[3], 0, 0, 0, 0};
                    acc[t][j] = mx4_mfma<FMT>(a, b, acc[t][j], h * KS + i, asc[t][n], wsc[j]);
                }
                __builtin_amdgcn_sched_barrier(0);
            }
#pragma unroll
            for (int q = 0; q < PW; ++q) lds[(cur ^ 1) * PIECES * 64 + (wave * PW + q) * 64 + lane] = ar[q];
#pragma unroll
            for (int i = 0; i < KS; ++i)
#pragma unroll
                for (int j = 0; j < 2; ++j) wr[0][i][j] = wr[1][i][j];
        }
    }
    __syncthreads();                                               // the buffers are read
    if (off) return;
    store_tiles<MT>(p, mt0, g, acc, smem);
}

// The same product for many rows, where the matrix cores are to be the bound: 2048 x
// 28672 x 8192 with 4-bit rows runs at 3.7 to 4.0 PFLOP/s.  Random codes draw so much
// power that the clock falls to 1.5 GHz from 2.1 with equal ones (same cycles); the
// instruction alone, out of registers, does 6.5 on them.  A product is at work in 57% of
// a CU's cycles: the others are starts, stores and the end of 3.5 rounds of workgroups.
// With three terms (517 x 4096 x 14336: 76 us) it is at work in 87%.
// A step of 64 k is 2 MT NT products of 32 or 64 cycles a wave, and with 16-bit rows
// one wave a SIMD, which issues in order: whatever the wave waits for or cannot issue
// leaves the matrix core idle.  So
//  - loads run D steps ahead in registers, W's fragments to their use, the
//    activations' (a wave loads a quarter of a step's) into one of two LDS
//    buffers;
//  - memory instructions stand one by one between the products (four waves that
//    each issue six at a time had the products wait for 35% of the cycles);
//  - fragments are read AHEAD of their products, across the step's end: the
//    barrier that frees one buffer and opens the other stands where the first
//    fragment of the next step is read, under the products in between.
// Everything is unrolled over D = 4 steps (steps_per is a multiple), so that the rings
// are registers.  With 4-bit rows they leave room for two workgroups a CU, one of which
// works while the other one starts or stores (tiles of 8 x 32 rows, one a CU, and of
// 4 x 32, two a CU: 2048 x 28672 x 8192 253 and 261 us, 2048 x 14336 x 4096 78 and 75,
// 2048 x 4096 x 14336 96 and 77).
template <int T, int MT>
__global__ __launch_bounds__(256, T ? 1 : 2) void mx4_pipe_kernel(Mx4Gemm p) {
    constexpr int NT = T ? T : 1, U = T ? 2 : 1, FMT = T ? 0 : 4;
    constexpr int PIECES = MT * NT * U, PW = PIECES / 4;           // kilobytes of a step's fragments; loaded by a wave
    constexpr int FRAGS = MT * NT;                                 // of a step
    constexpr int AHEAD = 3, RING = AHEAD + 1;                     // fragments read before their products
    constexpr int D = 4, OPEN = FRAGS - AHEAD;                     // OPEN: the fragment before whose products the barrier stands
    static_assert(PIECES % 4 == 0 && FRAGS % RING == 0 && PW <= OPEN && PW + 2 <= FRAGS, "rings");
    constexpr int BUF = PIECES * 1024;
    __shared__ __attribute__((aligned(16))) uint8_t smem[2 * BUF > store_lds(MT) ? 2 * BUF : store_lds(MT)];
    u32x4* const lds[2] = {(u32x4*)smem, (u32x4*)(smem + BUF)};
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int bid = xcd_run(blockIdx.x, gridDim.x);
    const int mt0 = (bid % p.mtiles) * MT;
    int g = (bid / p.mtiles) * 4 + wave;
    const bool off = g >= p.w.groups;                              // a wave without outputs keeps step with the others
    if (off) g = p.w.groups - 1;
    const int steps = p.w.steps, s0 = blockIdx.z * p.steps_per, s1 = min(steps, s0 + p.steps_per), last = s1 - 1;
    const u32x4* wp = (const u32x4*)p.w.w + (size_t)g * steps * 128 + lane;
    const ScaleLoad<NT, MT> sl(p, mt0, g, lane);
    const u32x4* ap[PW];                                           // tiles past the last are the last one again
#pragma unroll
    for (int q = 0; q < PW; ++q) {
        const int i = wave * PW + q, tile = min(mt0 + i / (NT * U), p.a.tiles - 1);
        ap[q] = (const u32x4*)p.a.a + ((size_t)tile * steps * (NT * U) + i % (NT * U)) * 64 + lane;
    }
    v16f acc[MT][2] = {};
    u32x4 ar[D][PW], wr[D][2], fr[RING][U];
    uint32_t ws[2], as[MT][NT], wsn[2], asn[MT][NT];             // scales of these four steps and of the next
    auto load_a = [&](int slot, int q, int s) { ar[slot][q] = ap[q][(size_t)min(s, last) * (NT * U * 64)]; };
    auto load_w = [&](int slot, int j, int s) { wr[slot][j] = wp[(size_t)min(s, last) * 128 + j * 64]; };
    auto write_a = [&](int slot, int q, int buf) { lds[buf][(wave * PW + q) * 64 + lane] = ar[slot][q]; };
    auto read = [&](int ring, int buf, int f) {                    // fragment f (tile, term) of a step
#pragma unroll
        for (int u = 0; u < U; ++u) fr[ring][u] = lds[buf][(f * U + u) * 64 + lane];
    };
    // steps s0 .. s0 + D - 1 of both operands; step s0 to LDS, and its first fragments to registers
    sl.load(s0 / 4, as, ws);
#pragma unroll
    for (int d = 0; d < D; ++d) {
#pragma unroll
        for (int q = 0; q < PW; ++q) load_a(d, q, s0 + d);
#pragma unroll
        for (int j = 0; j < 2; ++j) load_w(d, j, s0 + d);
    }
#pragma unroll
    for (int q = 0; q < PW; ++q) {
        write_a(0, q, 0);
        load_a(0, q, s0 + D);
    }
    __syncthreads();
#pragma unroll
    for (int f = 0; f < AHEAD; ++f) read(f, 0, f);
    for (int s = s0; s < s1; s += D) {
#pragma unroll
        for (int d = 0; d < D; ++d) {
            // step s + d stands in buffer d mod 2; step s + d + 1 goes into the other one, which the last barrier freed
#pragma unroll
            for (int f = 0; f < FRAGS; ++f) {
                if (f == OPEN) __syncthreads();                    // step s + d + 1 is written, and step s + d read
                if (f < OPEN) read((f + AHEAD) % RING, d & 1, f + AHEAD);
                else read((f + AHEAD) % RING, (d + 1) & 1, f - OPEN);
                if (f < PW) {
                    write_a((d + 1) % D, f, (d + 1) & 1);
                    load_a((d + 1) % D, f, s + d + 1 + D);
                } else if (f < PW + 2) {
                    load_w((d + D - 1) % D, f - PW, s + d - 1 + D);     // the step before is done with its own
                } else if (f == PW + 2 && d == 0) {
                    sl.load(min(s + 4, last) / 4, asn, wsn);
                }
                const u32x4 lo = fr[f % RING][0], hi = U == 2 ? fr[f % RING][U - 1] : u32x4{0u, 0u, 0u, 0u};
                const v8i a = {(int)lo[0], (int)lo[1], (int)lo[2], (int)lo[3], (int)hi[0], (int)hi[1], (int)hi[2], (int)hi[3]};
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    const u32x4 w = wr[d][j];
                    const v8i b = {(int)w[0], (int)w[1], (int)w[2], (int)w[3], 0, 0, 0, 0};
                    acc[f / NT][j] = mx4_mfma<FMT>(a, b, acc[f / NT][j], d, as[f / NT][f % NT], ws[j]);
                }
                __builtin_amdgcn_sched_barrier(0);
            }
        }
#pragma unroll
        for (int j = 0; j < 2; ++j) ws[j] = wsn[j];
#pragma unroll
        for (int t = 0; t < MT; ++t)
#pragma unroll
            for (int n = 0; n < NT; ++n) as[t][n] = asn[t][n];
    }
    __syncthreads();                                               // the buffers are read
    if (off) return;
    store_tiles<MT>(p, mt0, g, acc, smem);
}

// Few rows of x, in one launch and without a workspace: 16 of them by 16 outputs a
// workgroup (every second row of a group, so that their fragments are the packed
// ones), K over its eight waves, 128 k at a time on the 16 x 16 x 128 product.
// The workgroup turns x into terms in LDS, a segment of K at a time, while its
// first weights are on their way; the waves' sums meet in LDS, in their order.
// Bound by the latency of one read after a launch and by fetching the code, so
// there is one copy of the conversion; where many outputs or long rows make the
// terms that every workgroup makes for itself the larger part, the rows are
// prepared once instead (mx4_rows_direct below).  One row of 4096 x 4096: 5.4 us, of
// which the weights' 8.9 MB could be read in 1.8.
constexpr int ROW_WAVES = 8, ROW_LDS = 48 * 1024, ROW_SEG = 128 * ROW_WAVES;
template <int T, int DT>
__global__ __launch_bounds__(64 * ROW_WAVES) void mx4_rows_kernel(Mx4Gemm p, const void* __restrict__ x, size_t ldx, int seg) {
    constexpr int NT = T ? T : 1, U = T ? 2 : 1, FMT = T ? 0 : 4;
    // chunks whose weights are on their way at once: with three terms 4 took 165 registers, one workgroup a CU where 2 take
    // 107, two (one row of 28672 x 8192: 42 and 30 us)
    constexpr int ROW_BATCH = T ? 2 : 4;
    typedef float v4f __attribute__((ext_vector_type(4)));
    // fragments [chunk][term][half][block or quarter kb][row]; scales [chunk][term][row] words of 4 blocks; sums
    __shared__ __attribute__((aligned(16))) uint8_t frags[ROW_LDS];
    __shared__ uint32_t scales[T ? ROW_LDS / 128 : ROW_LDS / 64];  // a word for the 128 or 64 bytes of a chunk's row
    __shared__ float part[ROW_WAVES][256];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, r16 = lane & 15, kb = lane >> 4;
    const int g = blockIdx.x >> 2, j = blockIdx.x & 1, h = (blockIdx.x >> 1) & 1;
    const int row0 = 16 * blockIdx.y, m = min(16, p.m - row0);
    const int steps = p.w.steps, chunks = steps / 2;
    // lane: row 16 h + r16 of the tile j, block kb of the chunk
    const int at = (kb & 1) * 32 + 16 * h + r16;
    const u32x4* wp = (const u32x4*)p.w.w + ((size_t)g * steps * 2 + j) * 64 + at;
    const uint32_t* sp = p.w.s + ((size_t)g * (steps / 4) * 64 + at) * 2 + j;
    v4f acc = {};
#pragma unroll 1
    for (int k0 = 0; k0 < 64 * steps; k0 += seg) {                 // seg: a multiple of 128
        const int n = min(seg / 128, chunks - k0 / 128);           // chunks of the segment; a run of them is the wave's
        const int per = (n + ROW_WAVES - 1) / ROW_WAVES, c0 = min(n, wave * per), c1 = min(n, c0 + per);
        u32x4 w[ROW_BATCH];
        uint32_t ws[ROW_BATCH];
        auto load = [&](int c) {
#pragma unroll
            for (int i = 0; i < ROW_BATCH; ++i) {
                const int s = k0 / 64 + 2 * min(c + i, n - 1) + (kb >> 1);
                w[i] = wp[(size_t)s * 128];
                ws[i] = sp[(size_t)(s / 4) * 128] >> (8 * (s & 3));
            }
        };
        load(c0);
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll 1
        for (int i = tid; i < m * 8 * n; i += 64 * ROW_WAVES) {    // 16 values; neighbours share a block
            const int q = i & 7, rc = i >> 3, row = rc / n, c = rc - row * n, k = k0 + 128 * c + 16 * q;
            float v[16];
            load16<DT>(x, (size_t)(row0 + row) * ldx + k, p.w.k - k, v);
            uint32_t top = top16(v);
            top = max(top, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)top, 0xB1, 0xF, 0xF, false));   // lane ^ 1
            const bool bad = top >= 0x7f800000u;
            if constexpr (T == 0) {
                const uint32_t byte = block_byte(top, 2);
                const float inv = bad ? 0.0f : e8m0_inv(byte);
                float e[2][8];
#pragma unroll
                for (int z = 0; z < 16; ++z) e[z >> 3][z & 7] = bad ? 0.0f : v[z];
                *(u32x2*)(frags + ((size_t)(c * 4 + (q >> 1)) * m + row) * 16 + (q & 1) * 8) = u32x2{e2m1x8(e[0], inv), e2m1x8(e[1], inv)};
                ((uint8_t*)scales)[(c * m + row) * 4 + (q >> 1)] = (uint8_t)byte;
            } else {
                // element e of lane 16 kb + r: k = 16 kb + e for the first 16, 64 + 16 kb + e - 16 for the others
                int byte = bad ? 0 : term_byte(top);
                const float inv = bad ? 0.0f : e8m0_inv((uint32_t)byte);
#pragma unroll
                for (int z = 0; z < 16; ++z) v[z] = bad ? 0.0f : v[z] * inv;
#pragma unroll
                for (int t = 0; t < NT; ++t) {
                    *(u32x4*)(frags + ((size_t)((c * NT + t) * 8 + q) * m + row) * 16) = take_term(v);
                    ((uint8_t*)scales)[((c * NT + t) * m + row) * 4 + (q >> 1)] = (uint8_t)(bad ? 255 : byte);
                    if (t + 1 < NT) {
                        uint32_t rest = top16(v);
                        rest = max(rest, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)rest, 0xB1, 0xF, 0xF, false));
                        float up;
                        byte = next_byte(byte, rest, &up);
#pragma unroll
                        for (int z = 0; z < 16; ++z) v[z] *= up;
                    }
                }
            }
        }
        __syncthreads();
#pragma unroll 1
        for (int c = c0; c < c1; c += ROW_BATCH) {
            if (c != c0) load(c);
#pragma unroll
            for (int i = 0; i < ROW_BATCH; ++i) {
                if (c + i >= c1) break;
                const v8i b = {(int)w[i][0], (int)w[i][1], (int)w[i][2], (int)w[i][3], 0, 0, 0, 0};
#pragma unroll
                for (int t = 0; t < NT; ++t) {
                    u32x4 f[2] = {u32x4{0u, 0u, 0u, 0u}, u32x4{0u, 0u, 0u, 0u}};
                    uint32_t sa = 0x7f7f7f7fu;
                    if (r16 < m) {
#pragma unroll
                        for (int u = 0; u < U; ++u) f[u] = *(const u32x4*)(frags + ((size_t)(((c + i) * NT + t) * 4 * U + 4 * u + kb) * m + r16) * 16);
                        sa = scales[((c + i) * NT + t) * m + r16] >> (8 * kb);
                    }
                    const v8i a = {(int)f[0][0], (int)f[0][1], (int)f[0][2], (int)f[0][3], (int)f[1][0], (int)f[1][1], (int)f[1][2], (int)f[1][3]};
                    acc = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(a, b, acc, FMT, 4, 0, (int)sa, 0, (int)ws[i]);
                }
            }
        }
        __syncthreads();
    }
    // lane l holds output l mod 16 of rows 4 (l / 16) + r
#pragma unroll
    for (int r = 0; r < 4; ++r) part[wave][(4 * kb + r) * 16 + r16] = acc[r];
    __syncthreads();
    if (tid >= 256) return;
    float sum = 0.0f;
#pragma unroll
    for (int w = 0; w < ROW_WAVES; ++w) sum += part[w][tid];
    const int row = tid >> 4, col = 64 * g + 2 * (16 * h + (tid & 15)) + j;
    if (row < m && col < p.w.n) {
        const size_t o = (size_t)(row0 + row) * p.ld + col;
        if (p.dt == DT_F32) ((float*)p.out)[o] = sum;
        else ((uint16_t*)p.out)[o] = to_half_bits(sum, p.dt);
    }
}

hipError_t launch_mx4_rows(const Mx4Gemm& p, const void* x, int dt, int64_t ldx, hipStream_t st) {
    const dim3 g((unsigned)(4 * p.w.groups), (unsigned)((p.m + 15) / 16)), b(64 * ROW_WAVES);
    // the longest segment of K that LDS holds, the same number of chunks for each wave
    const int per_k = (p.m < 16 ? p.m : 16) * (p.a.terms ? 2 * p.a.terms : 1);       // half bytes
    int seg = ROW_LDS * 2 / per_k / ROW_SEG * ROW_SEG;
    if (seg > 64 * p.w.steps) seg = 64 * p.w.steps;
#define MX4_ROWS(T, DT) mx4_rows_kernel<T, DT><<<g, b, 0, st>>>(p, x, (size_t)ldx, seg)
    switch (p.a.terms * 4 + dt) {
        case DT_F32: MX4_ROWS(0, DT_F32); break;
        case DT_F16: MX4_ROWS(0, DT_F16); break;
        case DT_BF16: MX4_ROWS(0, DT_BF16); break;
        case 12 + DT_F16: MX4_ROWS(3, DT_F16); break;
        case 12 + DT_BF16: MX4_ROWS(3, DT_BF16); break;
        default: return hipErrorInvalidValue;
    }
#undef MX4_ROWS
    return hipGetLastError();
}

// out = the sum of the splits, in their order: four outputs a thread, and eight
// splits' on their way at a time (other XCDs wrote them: a read takes over a us).
// Bound by memory (517 x 4096 in three splits: 27 MB read, 7.5 us).
__global__ __launch_bounds__(256) void mx4_reduce_kernel(Mx4Gemm p) {
    const int quads = (p.w.n + 3) / 4;
    const size_t idx = blockIdx.x * (size_t)256 + threadIdx.x;
    if (idx >= (size_t)p.m * quads) return;
    const int row = (int)(idx / quads), col = 4 * (int)(idx % quads);
    // two of a group's even outputs and two of its odd ones
    const float2* part = (const float2*)(p.part + (size_t)row * p.part_ld + (col & ~63) + (col & 63) / 2);
    const size_t step = (size_t)p.a.tiles * 16 * p.part_ld;        // a split's rows are whole tiles
    float v[4] = {};
    for (int z0 = 0; z0 < p.split; z0 += 8) {
        float2 a[8], b[8];
#pragma unroll
        for (int z = 0; z < 8; ++z) {
            const float2* at = part + (size_t)min(z0 + z, p.split - 1) * step;
            a[z] = at[0];
            b[z] = at[16];
        }
#pragma unroll
        for (int z = 0; z < 8; ++z) {
            if (z0 + z >= p.split) break;
            v[0] += a[z].x; v[1] += b[z].x; v[2] += a[z].y; v[3] += b[z].y;
        }
    }
    if (p.dt == DT_F32) store_run<DT_F32, 4>(p.out, p.ld, p.w.n, row, col, v);
    else if (p.dt == DT_F16) store_run<DT_F16, 4>(p.out, p.ld, p.w.n, row, col, v);
    else store_run<DT_BF16, 4>(p.out, p.ld, p.w.n, row, col, v);
}

static hipError_t run_reduce(const Mx4Gemm& p, hipStream_t st, hipEvent_t done) {
    const size_t n = (size_t)p.m * ((p.w.n + 3) / 4);
    return launch_done(mx4_reduce_kernel, dim3((unsigned)((n + 255) / 256)), dim3(256), 0, st, done, p);
}

template <int T, int MT, int KS>
hipError_t run_gemm(Mx4Gemm p, hipStream_t st, hipEvent_t done) {
    p.mtiles = (p.a.tiles + MT - 1) / MT;
    const int ntiles = (p.w.groups + 3) / 4;
    constexpr int BUFS = 2 * MT * KS * (T ? 2 * T : 1) * 1024, LDS = BUFS > store_lds(MT) ? BUFS : store_lds(MT);
    hipError_t e = hipSuccess;
    if (LDS > 65536) e = hipFuncSetAttribute((const void*)mx4_gemm_kernel<T, MT, KS>, hipFuncAttributeMaxDynamicSharedMemorySize, LDS);
    if (e != hipSuccess) return e;
    e = launch_done(mx4_gemm_kernel<T, MT, KS>, dim3((unsigned)(p.mtiles * ntiles), 1, (unsigned)p.split), dim3(256), LDS, st,
                    p.split > 1 ? nullptr : done, p);
    return e == hipSuccess && p.split > 1 ? run_reduce(p, st, done) : e;
}

template <int T, int MT>
hipError_t run_pipe(Mx4Gemm p, hipStream_t st, hipEvent_t done) {
    p.mtiles = (p.a.tiles + MT - 1) / MT;
    const int ntiles = (p.w.groups + 3) / 4;
    const hipError_t e = launch_done(mx4_pipe_kernel<T, MT>, dim3((unsigned)(p.mtiles * ntiles), 1, (unsigned)p.split), dim3(256), 0,
                                     st, p.split > 1 ? nullptr : done, p);
    return e == hipSuccess && p.split > 1 ? run_reduce(p, st, done) : e;
}

// Row tiles of 32 a workgroup (MT) and splits of K: the pair of least time by what
// the parts cost, measured from 16 x 4096 x 4096 to 2048 x 28672 x 8192 (the picks are
// within 1% of the best pair on average, 7% at worst).  A workgroup's step of 64 k
// costs STEP (us), and a CU's workgroups take turns: larger tiles read less per
// product, so they win once every CU has work (2048 x 4096 x 4096: 102, 84 and 77 us
// with MT 1, 2 and 4).  START is what a tile's code and stores add, which is why small
// products take small tiles (300 x 300 x 300 with 4-bit rows: 12, 15 and 20 us with MT
// 1, 2 and 4); where MT 4 has one workgroup a CU, each round pays it.  Splits cost a
// launch and their sums' way to memory and back (33 x 256 x 14336: 84 us unsplit, 21 in
// 12 splits; 700 x 2048 x 700: 15 and 22 in two).  The split alone says in which order
// a row's sums are added.
float mx4_plan(Mx4Gemm& p, int n_cus, int only_split) {
    constexpr int MTS[3] = {1, 2, 4};
    constexpr float START[3] = {0.0f, 1.8f, 6.5f};
    constexpr float STEP[2][3] = {{0.15f, 0.185f, 0.25f}, {0.35f, 0.55f, 0.75f}};      // one E2M1 term, three E4M3 terms
    constexpr float BASE = 11.0f, JOIN = 4.0f, RATE = 7e6f;        // launches; the sums' launch; bytes a us
    constexpr int MAX_SPLIT = 24;
    const int units = p.w.steps / 4;
    const float* step = STEP[p.a.terms ? 1 : 0];
    const float sums = (float)p.a.tiles * 32.0f * (float)p.w.groups * 64.0f * 8.0f / RATE;
    float least = 3.4e38f;
    for (int i = 0; i < 3; ++i) {
        const float wgs = (float)((p.a.tiles + MTS[i] - 1) / MTS[i]) * (float)((p.w.groups + 3) / 4);
        for (int s = 1; s <= MAX_SPLIT && s <= units; ++s) {
            const int per = (units + s - 1) / s, split = (units + per - 1) / per;
            if (split != s || (only_split && s != only_split)) continue;
            float rounds = fmaxf(1.0f, wgs * (float)s / (float)n_cus);
            if (MTS[i] < 4 || p.a.terms) rounds = ceilf(rounds);       // else two workgroups a CU fill each other's gaps
            const float us = BASE + rounds * (float)(per * 4) * step[i] + (MTS[i] == 4 && p.a.terms ? rounds : 1.0f) * START[i] +
                             (s > 1 ? JOIN + (float)s * sums : 0.0f);
            if (us < least) {
                least = us;
                p.mt = MTS[i];
                p.split = s;
                p.steps_per = per * 4;
            }
        }
    }
    return least;
}

// Whether up to 64 rows go through mx4_rows_kernel: its workgroups share CUs, each
// makes the terms of 16 rows for itself (TERMS, us for 1000 values) after START, and
// reads weights.  8 x 4096 x 4096 in three terms: 9.9 us so, 18.9 through the plan's three
// launches; 16 x 14336 x 4096: 49 and 20; one row of 14336 x 14336: 29 and 34, two: 35
// and 34.  The picks of 196 sizes from 64 x 256 to 28672 x 14336 and 1 to 64 rows are the
// faster way or within 10% of it but for three (13 to 19% where K is long).
bool mx4_rows_direct(const Mx4Gemm& rows, int n_cus) {
    constexpr float BASE = 6.0f, SHARE = 0.65f, RATE = 16e6f;
    constexpr float START[2] = {0.8f, 1.0f}, TERMS[2] = {0.06f, 0.21f};
    Mx4Gemm p = rows;
    if (p.m > MX4_ROWS_MAX) return false;
    const int t = p.a.terms ? 1 : 0;
    const float wgs = 4.0f * (float)p.w.groups * (float)((p.m + 15) / 16);
    const float own = START[t] + TERMS[t] * (float)(p.m < 16 ? p.m : 16) * (float)p.w.k * 1e-3f;
    const float us = BASE + fmaxf(1.0f, SHARE * wgs / (float)n_cus) * own + (float)p.w.n * (float)p.w.k * 0.53f / RATE;
    p.a.tiles = (p.m + 31) / 32;
    return us < mx4_plan(p, n_cus);
}

hipError_t launch_mx4_gemm(const Mx4Gemm& p, hipStream_t st, hipEvent_t done) {
    switch (p.a.terms * 10 + p.mt) {
        case 1: return run_gemm<0, 1, 4>(p, st, done);
        case 2: return run_gemm<0, 2, 4>(p, st, done);
        case 4: return run_pipe<0, 4>(p, st, done);
        case 31: return run_gemm<3, 1, 4>(p, st, done);
        case 32: return run_gemm<3, 2, 2>(p, st, done);
        case 34: return run_pipe<3, 4>(p, st, done);
        default: return hipErrorInvalidValue;
    }
}

// out[m][H] = RMSNorm(row) * gamma in fp32: the input of an MXFP4 head, whose E4M3
// terms then take it at whatever power of two gamma gives it (fp16 rows ended at
// 65504) and leave 2^-12 of a block's larger elements.
__global__ __launch_bounds__(256) void rms_rows_kernel(const void* __restrict__ x, int dt, const uint16_t* __restrict__ gamma, int H,
                                                       float eps, float* __restrict__ out) {
    __shared__ float buf[256];
    const size_t row = (size_t)blockIdx.x * H;
    float s = 0.0f;
    for (int i = threadIdx.x; i < H; i += 256) {
        const float v = load_val(x, dt, row + i);
        s += v * v;
    }
    const float rs = rsqrtf(block_sum256(s, buf) / (float)H + eps);
    for (int i = threadIdx.x; i < H; i += 256) out[row + i] = load_val(x, dt, row + i) * rs * load_val(gamma, dt, i);
}

hipError_t launch_rms_rows(const void* x, int dt, const uint16_t* gamma, int m, int H, float eps, float* out, hipStream_t st) {
    rms_rows_kernel<<<dim3((unsigned)m), dim3(256), 0, st>>>(x, dt, gamma, H, eps, out);
    return hipGetLastError();
}

}  // namespace stg
