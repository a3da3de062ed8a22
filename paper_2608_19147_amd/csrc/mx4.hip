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
// the last of 4 bits), or 2^-10 where E4M3's smallest step decides: two terms
// come within 2^-14 of a block's largest magnitude, three within 2^-18, and the
// larger elements of bf16 (8 significant bits) and f16 (11) are exact in two and
// three terms.  Two terms are taken for bf16 rows with 16-bit results, three
// otherwise.  Activations of 4 bits are one E2M1 term.
#include "device.h"

namespace stg {

typedef int v8i __attribute__((ext_vector_type(8)));
typedef float v16f __attribute__((ext_vector_type(16)));

// ------------------------------------------------------------------ E2M1, E4M3

// Code of a value scaled to [0, 8) in magnitude: nearest, ties to even, at most 6.
__device__ __forceinline__ uint32_t e2m1(float v) {
    const float a = fabsf(v);
    const float inv = a < 2.0f ? 2.0f : a < 4.0f ? 1.0f : 0.5f;    // steps of 0.5, 1 and 2
    const float r = rintf(a * inv);                                // 0..4, 2..4, 2..4 steps
    const uint32_t c = (uint32_t)r + (a < 2.0f ? 0u : a < 4.0f ? 2u : 4u);
    return (c > 7u ? 7u : c) | ((__float_as_uint(v) >> 28) & 8u);
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

__global__ __launch_bounds__(256) void mx4_quantize_kernel(const void* __restrict__ x, int dt, size_t ld, int m, int k,
                                                           uint8_t* __restrict__ codes, uint8_t* __restrict__ scales) {
    const int nb = (k + 31) / 32;
    const size_t idx = blockIdx.x * (size_t)256 + threadIdx.x;     // one block of 32 a thread
    if (idx >= (size_t)m * nb) return;
    const int r = (int)(idx / nb), b = (int)(idx % nb);
    const int n = min(32, k - 32 * b);
    uint32_t top = 0;
    float v[32];
    for (int i = 0; i < 32; ++i) {
        v[i] = i < n ? load_val(x, dt, r * ld + 32 * (size_t)b + i) : 0.0f;
        top = max(top, absbits(v[i]));
    }
    const uint32_t byte = block_byte(top, 2);
    const float inv = byte == 255u ? 0.0f : e8m0_inv(byte);
    uint8_t* c = codes + (size_t)r * ((k + 1) / 2) + 16 * (size_t)b;
    for (int i = 0; i < n; i += 2) {
        const uint32_t lo = byte == 255u ? 0u : e2m1(v[i] * inv), hi = byte == 255u ? 0u : e2m1(v[i + 1] * inv);
        c[i / 2] = (uint8_t)(lo | (hi << 4));
    }
    scales[(size_t)r * nb + b] = (uint8_t)byte;
}

hipError_t launch_mx4_quantize(const void* x, int dt, int64_t ld, int m, int k, uint8_t* codes, uint8_t* scales, hipStream_t st) {
    const size_t n = (size_t)m * ((k + 31) / 32);
    mx4_quantize_kernel<<<dim3((unsigned)((n + 255) / 256)), dim3(256), 0, st>>>(x, dt, (size_t)ld, m, k, codes, scales);
    return hipGetLastError();
}

__global__ __launch_bounds__(256) void mx4_dequantize_kernel(const uint8_t* __restrict__ codes, const uint8_t* __restrict__ scales,
                                                             int m, int k, void* __restrict__ out, int dt, size_t ld) {
    const size_t idx = blockIdx.x * (size_t)256 + threadIdx.x;
    if (idx >= (size_t)m * k) return;
    const size_t r = idx / k, c = idx % k;
    const uint32_t code = (codes[r * ((k + 1) / 2) + c / 2] >> (4 * (c & 1))) & 15u;
    const float v = e2m1_value(code) * e8m0(scales[r * ((k + 31) / 32) + c / 32]);
    if (dt == DT_F32) ((float*)out)[r * ld + c] = v;
    else ((uint16_t*)out)[r * ld + c] = to_half_bits(v, dt);
}

hipError_t launch_mx4_dequantize(const uint8_t* codes, const uint8_t* scales, int m, int k, void* out, int dt, int64_t ld,
                                 hipStream_t st) {
    const size_t n = (size_t)m * k;
    mx4_dequantize_kernel<<<dim3((unsigned)((n + 255) / 256)), dim3(256), 0, st>>>(codes, scales, m, k, out, dt, (size_t)ld);
    return hipGetLastError();
}

// ------------------------------------------------------------------ weights

// One thread per 16-byte piece (32 codes: one row and block) of the packed form.
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
    ((uint8_t*)w.s)[((((size_t)g * (w.steps / 4) + s / 4) * 2 + j) * 64 + lane) * 4 + (s & 3)] = byte;
}

hipError_t launch_mx4_pack(const uint8_t* codes, const uint8_t* scales, const Mx4Mat& w, hipStream_t st) {
    const size_t n = (size_t)w.groups * w.steps * 128;
    mx4_pack_kernel<<<dim3((unsigned)((n + 255) / 256)), dim3(256), 0, st>>>(codes, scales, w);
    return hipGetLastError();
}

// ------------------------------------------------------------------ activations

// 16 values of one row (half a block) a thread; the two threads of a block are
// neighbours and share its largest magnitude.  Rows from m and columns from k
// on are zero.  T terms of E4M3 (T = 0: one E2M1 term).
template <int T>
__global__ __launch_bounds__(256) void mx4_prep_kernel(const void* __restrict__ x, int dt, size_t ld, int m, int k, int steps,
                                                       int tiles, uint8_t* __restrict__ a, uint8_t* __restrict__ as) {
    constexpr int NT = T ? T : 1, U = T ? 2 : 1;
    const size_t idx = blockIdx.x * (size_t)256 + threadIdx.x;
    if (idx >= (size_t)tiles * 32 * steps * 4) return;             // whole waves: a block's two threads stay together
    const int p = (int)(idx & 3);                                  // quarter of the step of 64
    const size_t rs = idx >> 2;
    const int s = (int)(rs % steps), row = (int)(rs / steps);
    const int k0 = 64 * s + 16 * p;
    float v[16];
    uint32_t top = 0;
#pragma unroll
    for (int i = 0; i < 16; ++i) {
        v[i] = row < m && k0 + i < k ? load_val(x, dt, row * ld + k0 + i) : 0.0f;
        top = max(top, absbits(v[i]));
    }
    top = max(top, (uint32_t)__shfl_xor((int)top, 1));
    const size_t tile = row >> 5;
    const int r = row & 31, b = p >> 1;
    const size_t frag = (tile * steps + s) * (size_t)(NT * U) * 1024;
    const size_t sc = ((tile * (steps / 4) + s / 4) * NT * 64 + b * 32 + r) * 4 + (s & 3);
    if constexpr (T == 0) {
        const uint32_t byte = block_byte(top, 2);
        const float inv = byte == 255u ? 0.0f : e8m0_inv(byte);
        u32x2 o = {0u, 0u};
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            const uint32_t c = byte == 255u ? 0u : e2m1(v[i] * inv);
            o[i >> 3] |= c << (4 * (i & 7));
        }
        *(u32x2*)(a + frag + (b * 32 + r) * 16 + (p & 1) * 8) = o;
        if (!(p & 1)) as[sc] = (uint8_t)byte;
    } else {
        int byte = (int)block_byte(top, 0);                        // largest scaled magnitude in [1, 2)
        const bool bad = top >= 0x7f800000u;
        byte = min(byte, 252);
        const float inv = bad ? 0.0f : e8m0_inv((uint32_t)byte);
#pragma unroll
        for (int i = 0; i < 16; ++i) v[i] = bad ? 0.0f : v[i] * inv;
#pragma unroll
        for (int t = 0; t < NT; ++t) {
            u32x4 o;
            uint32_t rest = 0;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                int w = __builtin_amdgcn_cvt_pk_fp8_f32(v[4 * i], v[4 * i + 1], 0, false);
                w = __builtin_amdgcn_cvt_pk_fp8_f32(v[4 * i + 2], v[4 * i + 3], w, true);
                o[i] = (uint32_t)w;
                v[4 * i] -= __builtin_amdgcn_cvt_f32_fp8(w, 0);
                v[4 * i + 1] -= __builtin_amdgcn_cvt_f32_fp8(w, 1);
                v[4 * i + 2] -= __builtin_amdgcn_cvt_f32_fp8(w, 2);
                v[4 * i + 3] -= __builtin_amdgcn_cvt_f32_fp8(w, 3);
#pragma unroll
                for (int q = 0; q < 4; ++q) rest = max(rest, absbits(v[4 * i + q]));
            }
            // element e of lane 32 g + r: k = 16 g + e for the first 16, 32 + 16 g + e - 16 for the others
            *(u32x4*)(a + frag + ((size_t)t * 2 + b) * 1024 + ((p & 1) * 32 + r) * 16) = o;
            if (!(p & 1)) as[sc + (size_t)t * 256] = (uint8_t)(bad ? 255 : byte);
            if (t + 1 < NT) {
                rest = max(rest, (uint32_t)__shfl_xor((int)rest, 1));
                int e = rest ? (int)(rest >> 23) - 127 : 0;        // the rest's largest magnitude to [1, 2)
                e = max(e, max(-byte, -127));
                byte += e;
                const float up = __uint_as_float((uint32_t)(127 - e) << 23);
#pragma unroll
                for (int i = 0; i < 16; ++i) v[i] *= up;
            }
        }
    }
}

hipError_t launch_mx4_prep(const Mx4Act& a, const void* x, int dt, int64_t ld, int m, int k, hipStream_t st) {
    const size_t n = (size_t)a.tiles * 32 * a.steps * 4;
    const dim3 g((unsigned)((n + 255) / 256)), b(256);
    switch (a.terms) {
        case 0: mx4_prep_kernel<0><<<g, b, 0, st>>>(x, dt, (size_t)ld, m, k, a.steps, a.tiles, a.a, a.s); break;
        case 2: mx4_prep_kernel<2><<<g, b, 0, st>>>(x, dt, (size_t)ld, m, k, a.steps, a.tiles, a.a, a.s); break;
        case 3: mx4_prep_kernel<3><<<g, b, 0, st>>>(x, dt, (size_t)ld, m, k, a.steps, a.tiles, a.a, a.s); break;
        default: return hipErrorInvalidValue;
    }
    return hipGetLastError();
}

// ------------------------------------------------------------------ product

__device__ __forceinline__ void store_out(void* out, int dt, size_t i, float v) {
    if (dt == DT_F32) ((float*)out)[i] = v;
    else ((uint16_t*)out)[i] = to_half_bits(v, dt);
}

// One 32 x 32 tile a wave.
template <int T>
__global__ __launch_bounds__(64) void mx4_gemm_kernel(Mx4Mat w, const uint8_t* __restrict__ a, const uint8_t* __restrict__ as,
                                                      int m, void* __restrict__ out, int dt, size_t ld) {
    constexpr int NT = T ? T : 1, U = T ? 2 : 1, FMT = T ? 0 : 4;
    const int lane = threadIdx.x, g = blockIdx.x >> 1, j = blockIdx.x & 1;
    const size_t tile = blockIdx.y;
    v16f acc = {};
    for (int s = 0; s < w.steps; ++s) {
        const u32x4 wf = ((const u32x4*)w.w)[(((size_t)g * w.steps + s) * 2 + j) * 64 + lane];
        const uint32_t ws = w.s[(((size_t)g * (w.steps / 4) + s / 4) * 2 + j) * 64 + lane] >> (8 * (s & 3));
        const v8i b = {(int)wf[0], (int)wf[1], (int)wf[2], (int)wf[3], 0, 0, 0, 0};
#pragma unroll
        for (int t = 0; t < NT; ++t) {
            const u32x4* f = (const u32x4*)(a + ((tile * w.steps + s) * NT + t) * (size_t)(U * 1024));
            const uint32_t sa = ((const uint32_t*)as)[((tile * (w.steps / 4) + s / 4) * NT + t) * 64 + lane] >> (8 * (s & 3));
            const u32x4 lo = f[lane], hi = U == 2 ? f[64 + lane] : u32x4{0u, 0u, 0u, 0u};
            const v8i av = {(int)lo[0], (int)lo[1], (int)lo[2], (int)lo[3], (int)hi[0], (int)hi[1], (int)hi[2], (int)hi[3]};
            acc = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(av, b, acc, FMT, 4, 0, (int)sa, 0, (int)ws);
        }
    }
    const int col = 64 * g + 2 * (lane & 31) + j;
#pragma unroll
    for (int r = 0; r < 16; ++r) {
        const int row = (int)tile * 32 + 8 * (r >> 2) + 4 * (lane >> 5) + (r & 3);
        if (row < m && col < w.n) store_out(out, dt, row * ld + col, acc[r]);
    }
}

hipError_t launch_mx4_gemm(const Mx4Mat& w, const Mx4Act& a, int m, void* out, int dt, int64_t ld, hipStream_t st) {
    const dim3 g((unsigned)(2 * w.groups), (unsigned)((m + 31) / 32)), b(64);
    switch (a.terms) {
        case 0: mx4_gemm_kernel<0><<<g, b, 0, st>>>(w, a.a, a.s, m, out, dt, (size_t)ld); break;
        case 2: mx4_gemm_kernel<2><<<g, b, 0, st>>>(w, a.a, a.s, m, out, dt, (size_t)ld); break;
        case 3: mx4_gemm_kernel<3><<<g, b, 0, st>>>(w, a.a, a.s, m, out, dt, (size_t)ld); break;
        default: return hipErrorInvalidValue;
    }
    return hipGetLastError();
}

// out[m][H] = fp16(RMSNorm(row) * gamma): the input of an MXFP4 head.
__global__ __launch_bounds__(256) void rms_rows_kernel(const void* __restrict__ x, int dt, const uint16_t* __restrict__ gamma, int H,
                                                       float eps, uint16_t* __restrict__ out) {
    __shared__ float buf[256];
    const size_t row = (size_t)blockIdx.x * H;
    float s = 0.0f;
    for (int i = threadIdx.x; i < H; i += 256) {
        const float v = load_val(x, dt, row + i);
        s += v * v;
    }
    const float rs = rsqrtf(block_sum256(s, buf) / (float)H + eps);
    for (int i = threadIdx.x; i < H; i += 256) out[row + i] = f32_to_f16(load_val(x, dt, row + i) * rs * load_val(gamma, dt, i));
}

hipError_t launch_rms_rows(const void* x, int dt, const uint16_t* gamma, int m, int H, float eps, uint16_t* out, hipStream_t st) {
    rms_rows_kernel<<<dim3((unsigned)m), dim3(256), 0, st>>>(x, dt, gamma, H, eps, out);
    return hipGetLastError();
}

}  // namespace stg
