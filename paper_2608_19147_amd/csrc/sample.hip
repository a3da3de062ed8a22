// Sampling from logits rows, and the walk of a drafted tree.
//
// The tokens of a row are ranked highest logit first, lowest index first among
// equal logits.  Temperature, top-k, top-p and min-p each keep a run of that
// ranking from its start, so what is kept is its first C tokens, and the token
// drawn is the first whose running weight passes u times the kept weight.  Every
// step is then a search for a place in the ranking by count, by weight or by
// value, and none needs the row sorted: a histogram over bins of the scaled
// logit says which bins hold the places, and only those bins' tokens are ranked.
//
// Bins: x = logit * 32 / T, q = floor(x), bin = q_max - q, weight exp((x - x_max)
// / 32), up to a common factor exp(d) E[bin] with d = (x - q) / 32 - 1 / 64 and
// E[b] = exp(-b / 32).  The grid does not move with the row's largest logit, so
// slices of a row are counted apart and joined by shifting whole bins.  exp(d)
// is summed as an integer in units of 2^-36 (any order of addition gives the same
// sum; below 2^57 for 2^20 tokens), the bins' sums are joined in 64-bit floating
// point.  Bins from 1024 on (weights below e^-31.9 of the largest, together less
// than 2^20 e^-31.9 = 1.5e-8 of the kept weight) are left out: neither u nor
// top_p, 24-bit numbers below 1, comes nearer to 1 than 6e-8, so no draw and no
// cut falls there.
//
// What bounds it is not the reading (64 bf16 rows of 128256: 16 MB, 3.3 us).  For one
// row to some it is the chain of small steps: count, plan, gather, draw, each a launch
// or a workgroup's code run once, from memory.  With 64 rows the counting itself is
// bound by the issue of vector instructions, most of them on 64-bit numbers: 47 a token,
// 5,900 a SIMD, which at 4 cycles each are 23,600 of a CU's 28,300 busy cycles.  Rows
// whose logits are nearly equal have more tokens in the bins that matter than are
// gathered, and are read again, place by place, by one workgroup: a row of 128256 equal
// ones takes 0.2 to 0.6 ms.
#include "device.h"

namespace stg {

constexpr int SB_BINS = 1024;        // bins of 1/32 of a unit of logit / T
constexpr int SB_CAP = 8192;         // tokens of the bins that matter that are gathered: 128256 spread over 2 units of
                                     // logit / T are up to 1600 a bin, and two or three bins matter
constexpr int SB_CAP_SMALL = 4096;   // and of a row held in LDS
constexpr int SB_RANK = 256;         // tokens that are ranked by counting larger ones
constexpr int SB_RANGES = 4;         // runs of bins that are gathered
constexpr int SB_THREADS = 512;      // of a workgroup
constexpr int SB_PER = SB_BINS / SB_THREADS;       // bins a thread, neighbours
constexpr int SL_LEN = SAMPLE_SLICE; // tokens of a slice: a bin's count fits the 14 bits below its sum
static_assert(SL_LEN == 16 * SB_THREADS && SL_LEN < (1 << 14), "slice");

// Order of finite logits as unsigned integers; NaN and -inf are not ranked (0), +inf ranks as the largest finite value, -0 as 0.
__device__ __forceinline__ uint32_t rank_key(float l) {
    if (!(l >= -3.402823466e38f)) return 0u;
    const uint32_t u = __float_as_uint(fminf(l, 3.402823466e38f) + 0.0f);
    return (u & 0x80000000u) ? ~u : (u | 0x80000000u);
}
__device__ __forceinline__ float key_logit(uint32_t k) { return __uint_as_float((k & 0x80000000u) ? (k & 0x7fffffffu) : ~k); }

// exp((f - 1/2) / 32) in units of 2^-36, f in [0, 1]: Taylor around f = 1/2 to the 5th power, the rest below 2.1e-14,
// 0.0015 of a unit, with the coefficients 2^36 / (32^n n!).  Added to 2^52, the units are the low bits of the sum.
__device__ __forceinline__ unsigned long long exp_units(double f) {
    const double c = f - 0.5;
    double p = 2048.0 / 120.0;
    p = fma(p, c, 65536.0 / 24.0);
    p = fma(p, c, 2097152.0 / 6.0);
    p = fma(p, c, 33554432.0);
    p = fma(p, c, 2147483648.0);
    p = fma(p, c, 4503599627370496.0 + 68719476736.0);
    return (unsigned long long)__double_as_longlong(p) & 0xfffffffffffffull;
}

// exp(-b / 32) and its inverse for b = 32 q + r, as products of exp(-q) and exp(-r / 32): correctly rounded values, so that
// a product is within 2 units in the last place.
__constant__ const double EXP_Q[32] = {
    0x1.0000000000000p+0, 0x1.78b56362cef38p-2, 0x1.152aaa3bf81ccp-3, 0x1.97db0ccceb0afp-5,
    0x1.2c155b8213cf4p-6, 0x1.b993fe00d5376p-8, 0x1.44e51f113d4d6p-9, 0x1.de16b9c24a98fp-11,
    0x1.5fc21041027adp-12, 0x1.02cf22526545ap-13, 0x1.7cd79b5647c9bp-15, 0x1.18354238f6764p-16,
    0x1.9c54c3b43bc8bp-18, 0x1.2f6053b981d98p-19, 0x1.be6c6fdb01612p-21, 0x1.4875ca227ec38p-22,
    0x1.e355bbaee85cbp-24, 0x1.639e3175a689dp-25, 0x1.05a628c699fa1p-26, 0x1.81056ff2c5772p-28,
    0x1.1b48655f37267p-29, 0x1.a0db0d0ddb3ecp-31, 0x1.32b48bf117da2p-32, 0x1.c3527e433fab1p-34,
    0x1.4c1078fe9228ap-35, 0x1.e8a37a45fc32ep-37, 0x1.67852a7007e42p-38, 0x1.0885298767e9ap-39,
    0x1.853f01d6d53bap-41, 0x1.1e642baeb84a0p-42, 0x1.a56e0c2ac7f75p-44, 0x1.36121e24d3bbap-45,
};
__constant__ const double EXP_R[32] = {
    0x1.0000000000000p+0, 0x1.f03f56a88b5d8p-1, 0x1.e0fabfbc702a4p-1, 0x1.d22e6a0197c03p-1,
    0x1.c3d6a24ed8222p-1, 0x1.b5efd29f24c26p-1, 0x1.a876812c0877cp-1, 0x1.9b674f8f2f3d8p-1,
    0x1.8ebef9eac820bp-1, 0x1.827a561889716p-1, 0x1.769652df22f7ep-1, 0x1.6b0ff72deb89dp-1,
    0x1.5fe4615e98e8fp-1, 0x1.5510c67cd2591p-1, 0x1.4a9271936fd09p-1, 0x1.4066c2ff39127p-1,
    0x1.368b2fc6f960ap-1, 0x1.2cfd40f8bdcaep-1, 0x1.23ba930c1568bp-1, 0x1.1ac0d5492c0dcp-1,
    0x1.120dc934993e8p-1, 0x1.099f41ffbe580p-1, 0x1.017323fd90020p-1, 0x1.f30ec8375038bp-2,
    0x1.e3b40ebefcd7ep-2, 0x1.d4d244cf4ea9ep-2, 0x1.c665b1e1f1e0dp-2, 0x1.b86ababeef8dfp-2,
    0x1.aadde095dad4bp-2, 0x1.9dbbc01e18268p-2, 0x1.910110be06976p-2, 0x1.84aaa3b8d514ep-2,
};
__constant__ const double INV_Q[32] = {
    0x1.0000000000000p+0, 0x1.5bf0a8b145769p+1, 0x1.d8e64b8d4ddaep+2, 0x1.415e5bf6fb106p+4,
    0x1.b4c902e273a58p+5, 0x1.28d389970338fp+7, 0x1.936dc5690c08fp+8, 0x1.122885aaeddaap+10,
    0x1.749ea7d470c6ep+11, 0x1.fa7157c470f82p+12, 0x1.5829dcf950560p+14, 0x1.d3c4488ee4f7fp+15,
    0x1.3de1654d37c9ap+17, 0x1.b00b5916ac955p+18, 0x1.259ac48bf05d7p+20, 0x1.8f0ccafad2a87p+21,
    0x1.0f2ebd0a80020p+23, 0x1.709348c0ea4f9p+24, 0x1.f4f22091940bdp+25, 0x1.546d8f9ed26e1p+27,
    0x1.ceb088b68e804p+28, 0x1.3a6e1fd9eecfdp+30, 0x1.ab5adb9c43600p+31, 0x1.226af33b1fdc1p+33,
    0x1.8ab7fb5475fb7p+34, 0x1.0c3d3920962c9p+36, 0x1.6c932696a6b5dp+37, 0x1.ef822f7f6731dp+38,
    0x1.50bba3796379ap+40, 0x1.c9aae4631c056p+41, 0x1.370470aec28edp+43, 0x1.a6b765d8cdf6dp+44,
};
__constant__ const double INV_R[32] = {
    0x1.0000000000000p+0, 0x1.08205601127edp+0, 0x1.1082b577d34edp+0, 0x1.192937074e0cdp+0,
    0x1.2216045b6f5cdp+0, 0x1.2b4b58b372c79p+0, 0x1.34cb8170b5835p+0, 0x1.3e98deaa11dccp+0,
    0x1.48b5e3c3e8186p+0, 0x1.5325180cfacf7p+0, 0x1.5de9176045ff5p+0, 0x1.690492cbf9433p+0,
    0x1.747a513dbef6ap+0, 0x1.804d30347b546p+0, 0x1.8c802477b0010p+0, 0x1.99163ad4b1dccp+0,
    0x1.a61298e1e069cp+0, 0x1.b3787dc80f95fp+0, 0x1.c14b431256446p+0, 0x1.cf8e5d84758a9p+0,
    0x1.de455df80e3c0p+0, 0x1.ed73f240dc142p+0, 0x1.fd1de6182f8c9p+0, 0x1.06a39207f0a09p+1,
    0x1.0ef9db467dcf8p+1, 0x1.1793e4652cc50p+1, 0x1.2073d3f1bd518p+1, 0x1.299be1f3e7f1cp+1,
    0x1.330e587b62b28p+1, 0x1.3ccd9432682b4p+1, 0x1.46dc04f4e5338p+1, 0x1.513c2e6c731d7p+1,
};
__device__ __forceinline__ double bin_weight(int b) { return EXP_Q[b >> 5] * EXP_R[b & 31]; }
__device__ __forceinline__ double bin_inverse(int b) { return INV_Q[b >> 5] * INV_R[b & 31]; }

struct RowBins {                      // the scaled logit of a row's tokens
    double per_t;                     // 32 / T
    double qmax;                      // floor(x) of the largest
    // Rounded by itself, wherever it is used: joined to the subtraction of its floor in one instruction, the product's
    // rounding would be in the fraction (more than 1 from x = 2^54 on), in one place and not in another.
    __device__ __forceinline__ double x(float logit) const {
#pragma clang fp contract(off)
        return (double)logit * per_t;
    }
    __device__ __forceinline__ double x(uint32_t key) const { return x(key_logit(key)); }
    __device__ __forceinline__ double bin(double xv) const { return qmax - floor(xv); }
    __device__ __forceinline__ unsigned long long units(double xv) const { return exp_units(xv - floor(xv)); }
};

struct RowArgs {
    const void* logits; int dt; size_t base; int V;
};

// Logits of tokens i .. i + 7 (i a multiple of 8) as they are; -inf past the row's end.
__device__ __forceinline__ void load_logits(const RowArgs& r, int i, float (&v)[8]) {
    if (i + 8 <= r.V) {
        if (r.dt == DT_F32) {
            const u32x4_any* p = (const u32x4_any*)((const float*)r.logits + r.base + i);
            const u32x4 a = p[0], b = p[1];
#pragma unroll
            for (int j = 0; j < 4; ++j) { v[j] = __uint_as_float(a[j]); v[4 + j] = __uint_as_float(b[j]); }
        } else {
            const u32x4 a = *(const u32x4_any*)((const uint16_t*)r.logits + r.base + i);
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] = half_bits_to_f32((uint16_t)(a[j >> 1] >> (16 * (j & 1))), r.dt);
        }
    } else {
        size_t off[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) off[j] = r.base + min(i + j, r.V - 1);
        load_vals<8>(r.logits, r.dt, off, v);
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = i + j < r.V ? v[j] : -INFINITY;
    }
}
// Their keys.
__device__ __forceinline__ void load_keys(const RowArgs& r, int i, uint32_t (&k)[8]) {
    float v[8];
    load_logits(r, i, v);
#pragma unroll
    for (int j = 0; j < 8; ++j) k[j] = rank_key(v[j]);
}
// A logit as its key orders it: -inf if it is not ranked.
__device__ __forceinline__ float ranked_logit(float l) { return fminf(l >= -3.402823466e38f ? l : -INFINITY, 3.402823466e38f); }

// One slice of a row: its largest token; its bins, counted from that one's
// (sum << 14 | count), stand apart.
struct SliceHead { double q; uint32_t top; uint32_t used; };   // used: bins up to the last that holds any

template <int NW>
__device__ __forceinline__ uint32_t block_max(uint32_t v, uint32_t* buf) {
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) v = max(v, (uint32_t)__shfl_xor((int)v, o));
    __syncthreads();
    if ((threadIdx.x & 63) == 0) buf[threadIdx.x >> 6] = v;
    __syncthreads();
    uint32_t t = 0;
#pragma unroll
    for (int w = 0; w < NW; ++w) t = max(t, buf[w]);
    return t;
}

// The keys of n tokens into LDS, from token `first` on in their order, and 0 up to
// the next multiple of SB_THREADS; the largest one.  (Loops over a thread's tokens stay loops: a workgroup
// runs this code once, and fetching instructions costs it about 0.9 us a kilobyte.)
__device__ __forceinline__ uint32_t load_tokens(const RowArgs& r, int first, int n, uint32_t* keys, uint32_t* buf) {
    uint32_t top = 0;
#pragma unroll 1
    for (int i = threadIdx.x * 8; i < (n + SB_THREADS - 1) / SB_THREADS * SB_THREADS; i += SB_THREADS * 8) {
        uint32_t k[8];
        load_keys(r, first + i, k);
        *(u32x4*)(keys + i) = u32x4{k[0], k[1], k[2], k[3]};
        *(u32x4*)(keys + i + 4) = u32x4{k[4], k[5], k[6], k[7]};
#pragma unroll
        for (int j = 0; j < 8; ++j) top = max(top, k[j]);
    }
    return block_max<SB_THREADS / 64>(top, buf);               // and a barrier: the keys are written
}

// Counts N tokens (keys, or ranked logits): their bins and units first, side by side, then the additions.  (Key 0 reads as
// NaN, which as -inf no bin takes.)
template <int N, class K>
__device__ __forceinline__ void count_keys(const K* k, const RowBins& rb, unsigned long long* hist) {
    unsigned long long v[N];
    int b[N];
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const double x = rb.x(k[i]), f = rb.bin(x);
        b[i] = f < (double)SB_BINS ? (int)f : -1;
        v[i] = rb.units(x) << 14 | 1ull;
    }
#pragma unroll
    for (int i = 0; i < N; ++i)
        if (b[i] >= 0) atomicAdd(&hist[b[i]], v[i]);
}

// hist[] of the slice's n tokens, counted from rb.qmax.
__device__ __forceinline__ void count_slice(const uint32_t* keys, int n, const RowBins& rb, unsigned long long* hist) {
#pragma unroll 1
    for (int i = threadIdx.x; i < SB_BINS; i += SB_THREADS) hist[i] = 0ull;
    __syncthreads();
#pragma unroll 1
    for (int i = threadIdx.x; i < n; i += 4 * SB_THREADS) {
        uint32_t k[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) k[j] = i + j * SB_THREADS < n ? keys[i + j * SB_THREADS] : 0u;
        count_keys<4>(k, rb, hist);
    }
    __syncthreads();
}

// What the counts of a row say before any token is ranked.
struct RowPlan {
    double qmax, all, thr;            // floor(x) of the largest; the row's weight; min_p's least units in bin 0
    unsigned long long units0;        // units of bin 0
    uint32_t top;                     // key of the largest, 0: nothing to draw from
    unsigned nall, n;                 // tokens; those of the runs of bins in which the places can be
    int kbin, vbin;                   // bins of top_k's cut and of min_p's (SB_BINS: none)
    int lo[SB_RANGES], hi[SB_RANGES]; // the runs (lo = SB_BINS: none)
    uint32_t klo[SB_RANGES], span[SB_RANGES];  // their least keys, and how many keys there are from it
    unsigned touched[SAMPLE_MAX_SLICES / 32];  // slices that hold some of those, one bit each
};

// Workspace of one row of a sampled batch: SAMPLE_ROW_BYTES, then the slices' heads and bins.
struct RowSpace {
    unsigned long long list[SB_CAP];  // gathered tokens, key << 32 | ~index
    double cum[SB_BINS];              // weight of the bins up to and with this one
    unsigned cumc[SB_BINS];           // their tokens
    RowPlan plan;
    unsigned arrived;                 // slices that are counted: zero between calls
    unsigned fill;                    // tokens in the list
};
static_assert(sizeof(RowSpace) <= SAMPLE_ROW_BYTES, "row workspace");

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
    unsigned long long hist[SB_BINS];          // units << 14 | count
    double cum[SB_BINS];                       // weight of the bins up to and with this one
    unsigned cumc[SB_BINS];                    // their tokens
    union {
        unsigned pieces[SB_BINS];              // tokens of the buckets of a part too large for the list
        struct {
            unsigned long long ranked[SB_RANK];    // tokens in order
            unsigned long long pre[SB_RANK];       // units of ranked[] up to and with each
        };
    };
    unsigned rank[SB_RANK];
    int shift[SAMPLE_MAX_SLICES];              // bins from the row's largest to the slice's (SB_BINS: nothing there)
    int used[SAMPLE_MAX_SLICES];               // and how many bins the slice has
    unsigned touched[SAMPLE_MAX_SLICES / 32];
    unsigned long long wave_u[SB_THREADS / 64];
    unsigned wave_c[SB_THREADS / 64];
    double wave_d[SB_THREADS / 64];
    uint32_t klo, khi;
    unsigned fill;
    unsigned c0;
    int found, flag;
    unsigned long long u0;
    Place place;
};

// Inclusive sum over the wave's lanes by lane permutes within the vector unit
// (__shfl goes through LDS, several times the latency).
template <int CTRL, int ROWS>
__device__ __forceinline__ unsigned dpp_u(unsigned v) { return (unsigned)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, ROWS, 0xF, false); }
template <int CTRL, int ROWS>
__device__ __forceinline__ unsigned long long dpp_u(unsigned long long v) {
    return (unsigned long long)dpp_u<CTRL, ROWS>((unsigned)(v >> 32)) << 32 | dpp_u<CTRL, ROWS>((unsigned)v);
}
template <int CTRL, int ROWS>
__device__ __forceinline__ double dpp_u(double v) {
    return __longlong_as_double((long long)dpp_u<CTRL, ROWS>((unsigned long long)__double_as_longlong(v)));
}
template <class S>
__device__ __forceinline__ S scan_wave(S v) {
    v += dpp_u<0x111, 0xF>(v);                  // row_shr 1, 2, 4, 8: within 16 lanes
    v += dpp_u<0x112, 0xF>(v);
    v += dpp_u<0x114, 0xF>(v);
    v += dpp_u<0x118, 0xF>(v);
    v += dpp_u<0x142, 0xA>(v);                  // the last lane of rows 0 and 2 to rows 1 and 3
    v += dpp_u<0x143, 0xC>(v);                  // and that of row 1 to rows 2 and 3
    return v;
}

// Inclusive sums of two values over the workgroup's threads, in thread order, and the totals.
template <class A, class B>
__device__ __forceinline__ void scan_block(A& a, B& b, A* wa, B* wb, A* ta, B* tb) {
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
    a = scan_wave(a);
    b = scan_wave(b);
    __syncthreads();                            // earlier readers of the waves' sums are done
    if (lane == 63) { wa[w] = a; wb[w] = b; }
    __syncthreads();
    const A pa = lane < SB_THREADS / 64 ? wa[lane] : A(0);
    const B pb = lane < SB_THREADS / 64 ? wb[lane] : B(0);
    A sa = scan_wave(pa);
    B sb = scan_wave(pb);
    *ta = __shfl(sa, SB_THREADS / 64 - 1);
    *tb = __shfl(sb, SB_THREADS / 64 - 1);
    sa = __shfl(sa, w ? w - 1 : 0);
    sb = __shfl(sb, w ? w - 1 : 0);
    if (w) { a += sa; b += sb; }
}

// The first i < n <= 4096 for which pred holds (it holds for all later ones), or
// n: 64 places at once, then the places between two of them.  Every wave finds
// it for itself, without a barrier.
template <class F>
__device__ __forceinline__ int wave_search(int n, F pred) {
    const int lane = threadIdx.x & 63, step = (n + 63) >> 6;
    const int i = lane * step + step - 1;
    const unsigned long long a = __ballot(pred(i < n ? i : n - 1));
    if (!a) return n;
    const int j = (__ffsll(a) - 1) * step + lane;
    const unsigned long long b = __ballot(lane < step && j < n && pred(j < n ? j : n - 1));
    return j - lane + __ffsll(b) - 1;
}

// hist[] of n tokens was filled: the first bucket with which the part reaches t
// (else the last one that holds any), and what is ahead of it.  c0, u0 and n
// become those of the bucket.
__device__ __forceinline__ int find_bucket(Want want, unsigned long long t, int& c0, unsigned long long& u0, int& n, SampleShared& sh) {
    const int tid = threadIdx.x;
    unsigned own[SB_PER], c = 0, tc;
    unsigned long long ownu[SB_PER], u = 0, tu;
#pragma unroll
    for (int j = 0; j < SB_PER; ++j) {
        const unsigned long long h = sh.hist[SB_PER * tid + j];
        own[j] = (unsigned)h & 16383u;
        ownu[j] = h >> 14;
        c += own[j];
        u += ownu[j];
    }
    if (tid == 0) sh.found = SB_BINS;
    unsigned upc = c;
    unsigned long long upu = u;
    scan_block(upc, upu, sh.wave_c, sh.wave_u, &tc, &tu);
    upc -= c;
    upu -= u;
    int mine = SB_BINS;
    unsigned ac = upc;
    unsigned long long au = upu;
#pragma unroll
    for (int j = 0; j < SB_PER; ++j) {
        const unsigned c1 = upc + own[j];
        const unsigned long long u1 = upu + ownu[j];
        const bool here = own[j] != 0u && ((want == BY_COUNT ? (unsigned long long)(c0 + (int)c1) >= t : u0 + u1 >= t) || c1 == tc);
        if (here && mine == SB_BINS) { mine = SB_PER * tid + j; ac = upc; au = upu; }
        upc = c1;
        upu = u1;
    }
    if (mine < SB_BINS) atomicMin(&sh.found, mine);
    __syncthreads();
    const int s = sh.found;
    if (mine == s) { sh.c0 = (unsigned)c0 + ac; sh.u0 = u0 + au; sh.fill = (unsigned)sh.hist[s] & 16383u; }
    __syncthreads();
    c0 = (int)sh.c0;
    u0 = sh.u0;
    n = (int)sh.fill;
    return s;
}

// ranked[0..n) sorted downwards (n <= SB_RANK) and summed: each token's rank is
// the number of larger ones, counted by four threads a token.
__device__ __forceinline__ void rank_tokens(int n, const RowBins& rb, SampleShared& sh) {
    const int tid = threadIdx.x, e = tid & (SB_RANK - 1), q = tid / SB_RANK;
    constexpr int PARTS = SB_THREADS / SB_RANK;
    if (tid < SB_RANK) sh.rank[tid] = 0u;
    __syncthreads();
    const unsigned long long v = e < n ? sh.ranked[e] : 0ull;
    unsigned larger = 0;
    if (e < n)
        for (int i = q; i < n; i += PARTS) larger += sh.ranked[i] > v;
    if (larger) atomicAdd(&sh.rank[e], larger);
    __syncthreads();
    const unsigned at = sh.rank[e];
    __syncthreads();
    if (q == 0 && e < n) sh.ranked[at] = v;
    __syncthreads();
    unsigned long long u = tid < n ? rb.units(rb.x((uint32_t)(sh.ranked[tid] >> 32))) : 0ull, tu;
    unsigned zero = 0, tz;
    scan_block(u, zero, sh.wave_u, sh.wave_c, &tu, &tz);
    if (tid < SB_RANK) sh.pre[tid] = u;
    __syncthreads();
}

// The place among ranked tokens at .. at + n - 1, with c0 tokens of u0 units of their part ahead.
__device__ __forceinline__ Place place_in_ranked(int at, int n, int c0, unsigned long long u0, Want want, unsigned long long t,
                                                 const RowBins& rb, const SampleShared& sh) {
    const unsigned long long base = at ? sh.pre[at - 1] : 0ull;
    int lo;                                     // the fewest that do (BY_VALUE: the first that does not)
    if (want == BY_COUNT) {
        const unsigned long long c = t - (unsigned)c0;
        lo = c < (unsigned)n ? (int)c : n;
    } else if (want == BY_MASS) {
        lo = min(n, wave_search(n, [&](int i) { return u0 + (sh.pre[at + i] - base) >= t; }) + 1);
    } else {
        lo = wave_search(n, [&](int i) { return rb.units(rb.x((uint32_t)(sh.ranked[at + i] >> 32))) < t; });
    }
    if (lo == 0) return Place{c0, u0, 0u, -1};
    const unsigned long long v = sh.ranked[at + lo - 1];
    return Place{c0 + lo, u0 + (sh.pre[at + lo - 1] - base), (uint32_t)(v >> 32), (int)~(uint32_t)v};
}

// The place in `part` that `want` asks for: its first `t` tokens (BY_COUNT), the
// fewest whose units together reach `t`, all of them if none do (BY_MASS), or
// those of at least `t` units each (BY_VALUE, which names no token).  listed > 0:
// the part's tokens stand among the list's first `listed`.  Otherwise, above
// cap of them, passes over the row narrow the part to a bucket of its keys' range (or
// find a token of equal ones by index), then gather it.  The part's tokens are
// narrowed the same way, in LDS (sel), until SB_RANK are left, which are ranked.
// Whole workgroup; every thread gets the result.  (One loop over the row serves
// every kind of pass, and the caller calls this in one place: a row is one
// workgroup's work once, so instructions come from memory, not from the cache.)
__device__ __forceinline__ Place find_place(const RowArgs& r, const RowBins& rb, Part part, unsigned long long* list, int cap, int listed, Want want,
                                            unsigned long long t, unsigned long long* sel, SampleShared& sh) {
    enum Pass : int { RANGE, PIECES, COUNT, PICK, VALUE, GATHER };
    const int tid = threadIdx.x;
    int c0 = 0;                                 // tokens and units of the part ahead of the piece looked at
    unsigned long long u0 = 0;
    if (listed <= 0) {
        const int run = ((r.V + SB_THREADS - 1) / SB_THREADS + 7) / 8 * 8;   // COUNT, PICK: neighbours of one thread
        int shift = 0, kth = 0;
        unsigned upto = 0, mine = 0;
        Pass pass = part.n <= cap ? GATHER : want == BY_VALUE ? VALUE : RANGE;
        for (;;) {
            __syncthreads();
            if (tid == 0) { sh.klo = 0xffffffffu; sh.khi = 0u; sh.fill = 0u; sh.place = Place{0, 0ull, 0u, -1}; }
            if (pass == RANGE)
                for (int i = tid; i < SB_BINS; i += SB_THREADS) { sh.pieces[i] = 0u; sh.hist[i] = 0ull; }
            __syncthreads();
            uint32_t lo = 0xffffffffu, hi = 0u;
            unsigned long long sum = 0;
            const unsigned ahead = upto - mine;
            unsigned n = 0;
            const bool runs = pass == COUNT || pass == PICK;
            const int first = runs ? min(r.V, tid * run) : tid * 8, end = runs ? min(r.V, first + run) : r.V, by = runs ? 8 : SB_THREADS * 8;
            for (int i = first; i < end; i += by) {
                uint32_t k[8];
                load_keys(r, i, k);
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    if (k[j] == 0u || k[j] < part.lo || k[j] > part.hi) continue;
                    const double x = rb.x(k[j]);
                    if (rb.bin(x) != (double)part.bin) continue;
                    if (pass == RANGE) {
                        lo = min(lo, k[j]);
                        hi = max(hi, k[j]);
                    } else if (pass == PIECES) {
                        const uint32_t s = (part.hi - k[j]) >> shift;
                        atomicAdd(&sh.pieces[s], 1u);
                        atomicAdd(&sh.hist[s], rb.units(x));
                    } else if (pass == VALUE) {
                        const unsigned long long e = rb.units(x);
                        if (e >= t) { ++n; sum += e; }
                    } else if (runs) {
                        ++n;
                        if (pass == PICK && ahead + n == (unsigned)kth) sh.place.index = i + j;
                    } else {
                        const unsigned f = atomicAdd(&sh.fill, 1u);
                        if (f < (unsigned)cap) store_coherent(&list[f], ((unsigned long long)k[j] << 32) | (uint32_t)~(i + j));
                    }
                }
            }
            if (pass == RANGE && hi) { atomicMin(&sh.klo, lo); atomicMax(&sh.khi, hi); }
            if (pass == GATHER) asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");   // the list is read by other waves
            __syncthreads();
            if (pass == GATHER) break;
            if (pass == RANGE) {
                part.lo = sh.klo;
                part.hi = sh.khi;
                shift = 0;
                while (((part.hi - part.lo) >> shift) >= (uint32_t)SB_BINS) ++shift;
                pass = part.lo == part.hi ? COUNT : PIECES;
            } else if (pass == PIECES) {
                if (tid == 0) {                 // the first piece that holds the place, else the last one
                    int last = 0, cc = c0, lc = c0;
                    unsigned long long uu = u0, lu = u0;
                    for (int s = 0; s < SB_BINS; ++s) {
                        if (!sh.pieces[s]) continue;
                        last = s; lc = cc; lu = uu;
                        cc += (int)sh.pieces[s];
                        uu += sh.hist[s];
                        if (want == BY_COUNT ? (unsigned long long)cc >= t : uu >= t) break;
                    }
                    sh.found = last;
                    sh.c0 = (unsigned)lc;
                    sh.u0 = lu;
                }
                __syncthreads();
                const int s = sh.found;
                const uint32_t nhi = part.hi - ((uint32_t)s << shift), span = (1u << shift) - 1u;
                part.lo = max(part.lo, nhi >= span ? nhi - span : 0u);
                part.hi = nhi;
                part.n = (int)sh.pieces[s];
                c0 = (int)sh.c0;
                u0 = sh.u0;
                pass = part.n > cap ? RANGE : GATHER;
            } else if (pass == VALUE) {
                unsigned tc;
                unsigned long long tu;
                scan_block(n, sum, sh.wave_c, sh.wave_u, &tc, &tu);
                return Place{(int)tc, tu, 0u, -1};
            } else if (pass == COUNT) {         // all equal: the kth-th by index
                const unsigned long long e = rb.units(rb.x(part.lo));
                unsigned long long q, none = 0, tn;
                if (want == BY_COUNT) q = t - (unsigned)c0;
                else q = t > u0 ? (t - u0 + e - 1) / e : 1u;
                kth = q < (unsigned)part.n ? (int)q : part.n;
                unsigned tot;
                upto = mine = n;
                scan_block(upto, none, sh.wave_c, sh.wave_u, &tot, &tn);
                pass = PICK;
            } else {
                return Place{c0 + kth, u0 + (unsigned long long)kth * rb.units(rb.x(part.lo)), part.lo, sh.place.index};
            }
        }
        listed = part.n;
    }
    // the part's tokens among the list's into LDS; by value, they are counted and summed at once
    __syncthreads();
    if (tid == 0) sh.fill = 0u;
    __syncthreads();
    unsigned cnt = 0, tc;
    unsigned long long sum = 0, tu;
#pragma unroll 1
    for (int i = tid; i < listed; i += SB_THREADS) {
        const unsigned long long v = load_coherent(&list[i]);
        const uint32_t k = (uint32_t)(v >> 32);
        if (k < part.lo || k > part.hi) continue;
        const double x = rb.x(k);
        if (rb.bin(x) != (double)part.bin) continue;
        if (want == BY_VALUE) {
            const unsigned long long e = rb.units(x);
            if (e >= t) { ++cnt; sum += e; }
        } else {
            sel[atomicAdd(&sh.fill, 1u)] = v;
        }
    }
    if (want == BY_VALUE) {
        scan_block(cnt, sum, sh.wave_c, sh.wave_u, &tc, &tu);
        return Place{(int)tc, tu, 0u, -1};
    }
    int n = part.n;
#pragma unroll 1
    while (n > SB_RANK) {
        // buckets of the keys' range, highest first; where all keys are equal, of the range of their indices, which differ.
        // Either range is that of the tokens left, so its two ends fall into different buckets and every pass ends with
        // fewer tokens.
        __syncthreads();
        uint32_t lo = 0xffffffffu, hi = 0u;
#pragma unroll 1
        for (int i = tid; i < n; i += SB_THREADS) {
            const uint32_t k = (uint32_t)(sel[i] >> 32);
            lo = min(lo, k);
            hi = max(hi, k);
        }
#pragma unroll 1
        for (int i = tid; i < SB_BINS; i += SB_THREADS) sh.hist[i] = 0ull;
        hi = block_max<SB_THREADS / 64>(hi, sh.wave_c);
        lo = ~block_max<SB_THREADS / 64>(~lo, sh.wave_c);
        const bool equal = lo == hi;
        if (equal) {
            lo = 0xffffffffu, hi = 0u;                               // of the list's lower words, ~index
#pragma unroll 1
            for (int i = tid; i < n; i += SB_THREADS) {
                const uint32_t k = (uint32_t)sel[i];
                lo = min(lo, k);
                hi = max(hi, k);
            }
            hi = block_max<SB_THREADS / 64>(hi, sh.wave_c);
            lo = ~block_max<SB_THREADS / 64>(~lo, sh.wave_c);
        }
        const int shift = max(0, 22 - (int)__clz((hi - lo) | 1u));   // (hi - lo) >> shift < 1024
        auto bucket = [&](unsigned long long v) { return (hi - (equal ? (uint32_t)v : (uint32_t)(v >> 32))) >> shift; };
#pragma unroll 1
        for (int i = tid; i < n; i += SB_THREADS) {
            const unsigned long long v = sel[i];
            atomicAdd(&sh.hist[bucket(v)], rb.units(rb.x((uint32_t)(v >> 32))) << 14 | 1ull);
        }
        __syncthreads();
        const int was = n;
        const uint32_t s = (uint32_t)find_bucket(want, t, c0, u0, n, sh);
        __syncthreads();
        if (tid == 0) sh.fill = 0u;
#pragma unroll 1
        for (int i0 = 0; i0 < was; i0 += SB_THREADS) {               // what stays moves down, behind what has been read
            const unsigned long long v = i0 + tid < was ? sel[i0 + tid] : 0ull;
            __syncthreads();
            if (v && bucket(v) == s) sel[atomicAdd(&sh.fill, 1u)] = v;
        }
    }
    __syncthreads();
#pragma unroll 1
    for (int i = tid; i < n; i += SB_THREADS) sh.ranked[i] = sel[i];
    __syncthreads();
    rank_tokens(n, rb, sh);
    const Place p = place_in_ranked(0, n, c0, u0, want, t, rb, sh);
    __syncthreads();
    return p;
}

// From a thread's SB_PER bins (tokens bc, units bu) to the row's running sums, in
// sh.cum and sh.cumc, and its plan: the runs of bins in which cuts and draw can fall.
__device__ __forceinline__ RowPlan make_plan(const SampleRow& p, float u, const RowBins& rb, uint32_t top, const unsigned (&bc)[SB_PER],
                                             const unsigned long long (&bu)[SB_PER], SampleShared& sh) {
    const int tid = threadIdx.x, lane = tid & 63;
    double all, upw = 0.0, wj[SB_PER];
    unsigned nall, upc = 0;
#pragma unroll
    for (int j = 0; j < SB_PER; ++j) {
        wj[j] = (double)bu[j] * bin_weight(SB_PER * tid + j);
        upw += wj[j];
        upc += bc[j];
    }
    const double w = upw;
    const unsigned c = upc;
    if (tid == 0) sh.u0 = bu[0];
    scan_block(upw, upc, sh.wave_d, sh.wave_c, &all, &nall);
    upc -= c;
    double run = upw - w;
#pragma unroll
    for (int j = 0; j < SB_PER; ++j) {
        // a thread's last bin takes the scan's own sum, so that the running weight never falls from one bin to the next
        run += wj[j];
        upc += bc[j];
        sh.cum[SB_PER * tid + j] = j == SB_PER - 1 ? upw : fmin(run, upw);
        sh.cumc[SB_PER * tid + j] = upc;
    }
    __syncthreads();
    auto before = [&](int b) { return b ? sh.cum[b - 1] : 0.0; };
    auto cbefore = [&](int b) { return b ? sh.cumc[b - 1] : 0u; };
    auto bin_reaching = [&](double t) { return wave_search(SB_BINS, [&](int i) { return sh.cum[i] >= t; }); };
    auto bin_of_count = [&](unsigned n) { return wave_search(SB_BINS, [&](int i) { return sh.cumc[i] >= n; }); };
    const bool by_k = p.top_k > 0 && (unsigned)p.top_k < nall, by_p = p.top_p < 1.0f;
    RowPlan pl;
    pl.qmax = rb.qmax;
    pl.all = all;
    pl.thr = (double)p.min_p * (double)rb.units(rb.x(top));    // exp(d) E[bin] >= min_p exp(d_max)
    pl.units0 = sh.u0;
    pl.top = top;
    pl.nall = nall;
    pl.kbin = bin_of_count(by_k ? (unsigned)p.top_k : nall);
    pl.vbin = SB_BINS;
    if (p.min_p > 0.0f) {
        // the first bin with tokens whose least weight fails min_p may hold some that pass, those behind it none
        const double least = (double)exp_units(0.0);
        const int f = wave_search(SB_BINS, [&](int i) { return bin_weight(i) * least < pl.thr; });
        if (f < SB_BINS) pl.vbin = bin_of_count(cbefore(f) + 1u);
    }
    // The places, whatever the tokens of the cut bins are: the kept weight lies between what is ahead of a cut's bin
    // and what is up to it.
    int lo[SB_RANGES] = {by_k ? pl.kbin : SB_BINS, SB_BINS, pl.vbin, SB_BINS}, hi[SB_RANGES] = {pl.kbin, 0, pl.vbin, 0};
    {
        double wlo = by_k ? before(pl.kbin) : all, whi = sh.cum[pl.kbin];
        int end = pl.kbin;                      // no later place is behind it
        if (by_p) {
            const double tlo = (double)p.top_p * wlo, thi = (double)p.top_p * whi;
            lo[1] = min(end, bin_reaching(tlo));
            hi[1] = min(end, bin_reaching(thi));
            wlo = fmax(tlo, before(lo[1]));
            whi = fmin(whi, sh.cum[hi[1]]);
            end = hi[1];
        }
        if (pl.vbin <= end) {
            wlo = fmin(wlo, before(pl.vbin));
            whi = fmin(whi, sh.cum[pl.vbin]);
            end = pl.vbin;
        }
        const double thi = (double)u * whi;
        lo[3] = min(end, bin_reaching((double)u * wlo));
        hi[3] = min(end, wave_search(SB_BINS, [&](int i) { return sh.cum[i] > thi; }));
    }
    // In order and apart: a run that starts in or right behind an earlier one is joined to it.  A run may lie within the
    // one ahead of it (top_p's from the first bin to top_k's cut, the draw's at its start, top_k's at its end), so each
    // takes the furthest end so far before they are joined.
#pragma unroll
    for (int i = 0; i < SB_RANGES; ++i)
#pragma unroll
        for (int j = 0; j < SB_RANGES - 1 - i; ++j)
            if (lo[j + 1] < lo[j]) {
                const int l = lo[j], h = hi[j];
                lo[j] = lo[j + 1]; hi[j] = hi[j + 1];
                lo[j + 1] = l; hi[j + 1] = h;
            }
#pragma unroll
    for (int i = 1; i < SB_RANGES; ++i)
        if (lo[i] < SB_BINS) hi[i] = max(hi[i], hi[i - 1]);
#pragma unroll
    for (int i = SB_RANGES - 1; i > 0; --i)
        if (lo[i] < SB_BINS && lo[i] <= hi[i - 1] + 1) {
            hi[i - 1] = hi[i];
            lo[i] = SB_BINS;
        }
    // The least key whose bin is b or less, for the ends of the runs: x rises with the key, so a logit next to q / per_t
    // is where floor(x) comes to q, to be found among 8 keys by 8 lanes; where the rounding of a large x leaves it
    // outside of them, by halving.  Lanes 0-7: the first run's low keys, 8-15: the end of its high ones, ...
    const int g = lane >> 4;
    const int b = (lane & 8) ? (g == 0 ? lo[0] : g == 1 ? lo[1] : g == 2 ? lo[2] : lo[3]) - 1
                             : (g == 0 ? hi[0] : g == 1 ? hi[1] : g == 2 ? hi[2] : hi[3]);
    const uint32_t near = max(rank_key((float)((rb.qmax - (double)b) / rb.per_t)), 0x00800004u) - 4u;
    const unsigned mask = (unsigned)(__ballot(rb.bin(rb.x(near + (lane & 7))) <= (double)b) >> (lane & 56)) & 255u;
    uint32_t key = near + (mask ? __ffs(mask) - 1 : 8);
    if (mask == 0u || mask == 255u) {
        uint32_t kl = 0x00800000u, kh = 0xff800000u;           // the finite numbers' keys
        while (kl < kh) {
            const uint32_t mid = kl + (kh - kl) / 2;
            if (rb.bin(rb.x(mid)) <= (double)b) kh = mid;
            else kl = mid + 1;
        }
        key = kl;
    }
    pl.n = 0;
#pragma unroll
    for (int i = 0; i < SB_RANGES; ++i) {
        pl.lo[i] = lo[i];
        pl.hi[i] = hi[i];
        pl.klo[i] = pl.span[i] = 0u;
        if (lo[i] >= SB_BINS) continue;
        pl.klo[i] = (uint32_t)__builtin_amdgcn_readlane((int)key, 16 * i);
        pl.span[i] = (lo[i] ? (uint32_t)__builtin_amdgcn_readlane((int)key, 16 * i + 8) : top + 1u) - pl.klo[i];
        pl.n += sh.cumc[hi[i]] - cbefore(lo[i]);
    }
    return pl;
}

// The slice's tokens (n of them) of the plan's runs go into the list; a wave asks
// once for their places.
template <class Put>
__device__ __forceinline__ void take_tokens(const RowPlan& pl, const uint32_t* keys, int slice, int n, int cap, unsigned* fill, Put put) {
    const int tid = threadIdx.x;
    unsigned m = 0;
#pragma unroll 2
    for (int i = 0; i < (n + SB_THREADS - 1) / SB_THREADS; ++i) {
        const uint32_t k = keys[i * SB_THREADS + tid];
        bool in = false;
#pragma unroll
        for (int q = 0; q < SB_RANGES; ++q) in |= k - pl.klo[q] < pl.span[q];
        m |= in ? 1u << i : 0u;
    }
    if (!__ballot(m != 0u)) return;
    const unsigned mine = (unsigned)__popc(m), upto = scan_wave(mine);
    unsigned at = 0;
    if ((tid & 63) == 63) at = atomicAdd(fill, upto);
    at = (unsigned)__builtin_amdgcn_readlane((int)at, 63) + upto - mine;
    while (m) {
        const int i = (__ffs(m) - 1) * SB_THREADS + tid;
        if (at < (unsigned)cap) put(at, ((unsigned long long)keys[i] << 32) | (uint32_t)~(slice * SL_LEN + i));
        ++at;
        m &= m - 1u;
    }
}

// The cuts and the draw of a row, by one workgroup: its running sums in sh.cum
// and sh.cumc, the tokens of the plan's runs in the list (unless they are more
// than cap: then the row is read again, place by place).
__device__ __forceinline__ void draw_row(const SampleArgs& a, int row, const RowArgs& r, const RowPlan& plan, float u,
                                         unsigned long long* list, int cap, unsigned long long* sel, SampleShared& sh) {
    const int tid = threadIdx.x;
    const SampleRow p = a.rows[row];
    const RowBins rb{p.per_t, plan.qmax};
    const double all = plan.all;
    const unsigned nall = plan.nall;
    const bool by_k = p.top_k > 0 && (unsigned)p.top_k < nall, by_p = p.top_p < 1.0f;
    auto before = [&](int b) { return b ? sh.cum[b - 1] : 0.0; };
    auto cbefore = [&](int b) { return b ? sh.cumc[b - 1] : 0u; };
    bool listed = plan.n <= (unsigned)cap, ranked = plan.n <= (unsigned)SB_RANK;
    if (ranked) {                               // few: ranked together, bin behind bin
        if (tid < (int)plan.n) sh.ranked[tid] = list[tid];
        __syncthreads();
        rank_tokens((int)plan.n, rb, sh);
    }
    // where bin b's tokens start among all of the runs', or -1
    auto start = [&](int b) {
        int at = -1;
        unsigned base = 0;
#pragma unroll
        for (int i = 0; i < SB_RANGES; ++i) {
            if (plan.lo[i] >= SB_BINS) continue;
            if (b >= plan.lo[i] && b <= plan.hi[i]) at = (int)(base + cbefore(b) - cbefore(plan.lo[i]));
            base += sh.cumc[plan.hi[i]] - cbefore(plan.lo[i]);
        }
        return at;
    };
    // kept: the first C tokens, of weight W; W0: the units of those in bin 0, where the largest is (E[0] = 1)
    int C = (int)nall;
    double W = all;
    unsigned long long W0 = plan.units0;
    // share * kept weight, in units of bin b and less what is ahead of it, rounded down or up.  Where all that is
    // kept is in bin 0 the product is exact: equal logits have no other way to agree with u or top_p times their number.
    auto target = [&](float share, int b, bool up) {
        if (C <= (int)sh.cumc[0]) {
            const unsigned long long f = (unsigned long long)((double)share * 18446744073709551616.0);
            return __umul64hi(W0, f) + (up && W0 * f != 0ull ? 1ull : 0ull);
        }
        const double t = fmax(0.0, ((double)share * W - before(b)) * bin_inverse(b));
        return (unsigned long long)(up ? ceil(t) : floor(t));
    };
    Place pl{0, 0ull, 0u, -1};
    int b = 0, end = plan.kbin;                 // end: the bin of the last token kept
#pragma unroll 1
    for (int step = 0; step < 5; ++step) {      // the three cuts, the draw, and the draw again where it came behind the last cut
        Want want = BY_MASS;
        unsigned long long t;
        if (step == 0) {
            if (!by_k) continue;
            b = plan.kbin;
            want = BY_COUNT;
            t = (unsigned)p.top_k - cbefore(b);
        } else if (step == 2) {
            if (plan.vbin >= SB_BINS || cbefore(plan.vbin) >= (unsigned)C) continue;
            b = plan.vbin;
            want = BY_VALUE;
            t = (unsigned long long)ceil(plan.thr * bin_inverse(b));
        } else if (step == 4) {
            if ((int)cbefore(b) + pl.count <= C) continue;
            want = BY_COUNT;
            t = (unsigned)C - cbefore(b);
        } else {
            if (step == 1 && !by_p) continue;
            // the bin in which the running weight reaches top_p of what is kept, or passes u of it
            const float share = step == 1 ? p.top_p : u;
            const double goal = (double)share * W;
            b = C <= (int)sh.cumc[0] ? 0 : min(end, wave_search(SB_BINS, [&](int i) { return step == 3 ? sh.cum[i] > goal : sh.cum[i] >= goal; }));
            // running weights are sums in different orders: an empty bin's may be a rounding step above that of the bins ahead,
            // with the goal in between, and the place is then where the next tokens start
            const unsigned c = cbefore(b);
            if (sh.cumc[b] == c) b = min(end, wave_search(SB_BINS, [&](int i) { return sh.cumc[i] > c; }));
            t = target(share, b, step == 1) + (step == 3 ? 1ull : 0ull);
        }
        const int at = start(b), cnt = (int)(sh.cumc[b] - cbefore(b));
        if (ranked && at >= 0) pl = place_in_ranked(at, cnt, 0, 0ull, want, t, rb, sh);
        else {
            pl = find_place(r, rb, Part{b, 0u, 0xffffffffu, cnt}, list, cap, listed && at >= 0 ? (int)plan.n : 0, want, t, sel, sh);
            listed = listed && at >= 0;         // find_place took the list's memory
            ranked = false;                     // and that of the ranked ones
        }
        const int c = (int)cbefore(b) + pl.count;
        if (step < 3 && c < C) {
            C = c;
            W = before(b) + (double)pl.units * bin_weight(b);
            if (b == 0) W0 = pl.units;
            end = pl.count ? b : wave_search(SB_BINS, [&](int i) { return sh.cumc[i] >= (unsigned)C; });
        }
    }
    if (tid == 0) {
        a.token[row] = pl.index;
        a.p[row] = (float)((double)rb.units(rb.x(pl.key)) * bin_weight(b) / W);
        if (a.top) a.top[row] = key_logit(plan.top);
    }
}

__device__ __forceinline__ void draw_nothing(const SampleArgs& a, int row) {
    if (threadIdx.x == 0) {
        a.token[row] = -1;
        a.p[row] = 0.0f;
        if (a.top) a.top[row] = -INFINITY;
    }
}

__device__ __forceinline__ float row_u(const SampleArgs& a, int row) { return a.u ? fminf(fmaxf(a.u[row], 0.0f), 0.99999994f) : 0.0f; }

// A row of up to SAMPLE_SMALL tokens by one workgroup, in LDS: one launch, and no
// workspace (1000 tokens 12 us; 16384 tokens, a row and 16 rows: 16 and 23 us, 23 and 31
// through the three kernels below; 24000 tokens: 21 and 27, 24 and 31).
struct SmallShared {
    SampleShared sh;
    alignas(16) unsigned long long list[SB_CAP_SMALL];
    alignas(16) uint32_t keys[SL_LEN];             // and those of the row's other slices behind them
};
static_assert(sizeof(SmallShared) + (SAMPLE_SMALL - SL_LEN) * 4 <= 160 * 1024 && SAMPLE_SMALL % SL_LEN == 0, "LDS");
__global__ __launch_bounds__(SB_THREADS) void sample_small_kernel(SampleArgs a) {
    extern __shared__ __attribute__((aligned(16))) uint8_t smem[];
    SmallShared& all = *(SmallShared*)smem;
    SampleShared& sh = all.sh;
    uint32_t* keys = all.keys;
    unsigned long long* list = all.list;
    const int row = blockIdx.x, tid = threadIdx.x, slices = (a.V + SL_LEN - 1) / SL_LEN;
    const RowArgs r{a.logits, a.dt, (size_t)row * a.ld, a.V};
    RowBins rb{a.rows[row].per_t, 0.0};
    const float u = row_u(a, row);
    if (tid == 0) sh.fill = 0u;
    const uint32_t top = load_tokens(r, 0, a.V, keys, sh.wave_c);
    if (!top) return draw_nothing(a, row);
    rb.qmax = floor(rb.x(top));
    unsigned bc[SB_PER] = {};
    unsigned long long bu[SB_PER] = {};
#pragma unroll 1
    for (int s = 0; s < slices; ++s) {             // a slice's counts at a time: they fit their bits
        count_slice(keys + s * SL_LEN, min(SL_LEN, a.V - s * SL_LEN), rb, sh.hist);
#pragma unroll
        for (int j = 0; j < SB_PER; ++j) {
            bc[j] += (unsigned)sh.hist[SB_PER * tid + j] & 16383u;
            bu[j] += sh.hist[SB_PER * tid + j] >> 14;
        }
        __syncthreads();
    }
    const RowPlan plan = make_plan(a.rows[row], u, rb, top, bc, bu, sh);
    if (plan.n <= (unsigned)SB_CAP_SMALL)
#pragma unroll 1
        for (int s = 0; s < slices; ++s)
            take_tokens(plan, keys + s * SL_LEN, s, min(SL_LEN, a.V - s * SL_LEN), SB_CAP_SMALL, &sh.fill, [&](unsigned at, unsigned long long v) { list[at] = v; });
    __syncthreads();
    draw_row(a, row, r, plan, u, list, SB_CAP_SMALL, (unsigned long long*)keys, sh);
}

// Counts one slice of a row; the row's last workgroup to end joins the counts and makes the plan.
// 20 rows of 128256: 17 us, of which a slice takes 5, the joining 3 and the plan 4; 64 rows: 26.
__global__ __launch_bounds__(SB_THREADS, 6) void sample_count_kernel(SampleArgs a) {
    __shared__ SampleShared sh;
    const int slice = blockIdx.x, row = blockIdx.y, ns = gridDim.x, tid = threadIdx.x;
    RowSpace* ws = (RowSpace*)(a.rows_ws + (size_t)row * SAMPLE_ROW_BYTES);
    SliceHead* heads = (SliceHead*)a.heads + (size_t)row * ns;
    unsigned long long* bins = a.bins + (size_t)row * ns * SB_BINS;
    RowBins rb{a.rows[row].per_t, 0.0};
    {
        const RowArgs r{a.logits, a.dt, (size_t)row * a.ld, a.V};
        // in registers: without them in LDS four workgroups share a CU; as keys they took 12 more instructions a token
        float l[2][8], most = -INFINITY;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            load_logits(r, slice * SL_LEN + h * (SL_LEN / 2) + tid * 8, l[h]);
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                l[h][j] = ranked_logit(l[h][j]);
                most = fmaxf(most, l[h][j]);
            }
        }
#pragma unroll 1
        for (int i = tid; i < SB_BINS; i += SB_THREADS) sh.hist[i] = 0ull;
        const uint32_t top = block_max<SB_THREADS / 64>(rank_key(most), sh.wave_c);
        rb.qmax = floor(rb.x(top));
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int j = 0; j < 8; j += 4) count_keys<4>(&l[h][j], rb, sh.hist);
        __syncthreads();
        if (tid == 0) sh.found = 0;
        __syncthreads();
#pragma unroll 1
        for (int i = tid; i < SB_BINS; i += SB_THREADS) {
            const unsigned long long some = __ballot(sh.hist[i] != 0ull);
            if (some && (tid & 63) == 0) atomicMax(&sh.found, i + 64 - __clzll(some));
        }
        __syncthreads();
        const int used = sh.found;
#pragma unroll 1
        for (int i = tid; i < used; i += SB_THREADS) store_coherent(&bins[(size_t)slice * SB_BINS + i], sh.hist[i]);
        if (tid == 0) {
            store_coherent((unsigned long long*)&heads[slice].q, (unsigned long long)__double_as_longlong(rb.qmax));
            store_coherent((unsigned long long*)&heads[slice].top, (unsigned long long)used << 32 | top);
        }
    }
    if (!last_arrival(&ws->arrived, (unsigned)ns, &sh.flag)) return;
    uint32_t top = 0;
    double q = 0.0;
    int used = 0;
    if (tid < ns) {
        q = __longlong_as_double((long long)load_coherent((unsigned long long*)&heads[tid].q));
        const unsigned long long v = load_coherent((unsigned long long*)&heads[tid].top);
        top = (uint32_t)v;
        used = (int)(v >> 32);
    }
    const uint32_t mytop = top;
    top = block_max<SB_THREADS / 64>(top, sh.wave_c);
    rb.qmax = floor(rb.x(top));
    if (tid < SAMPLE_MAX_SLICES) {
        const double d = rb.qmax - q;
        sh.shift[tid] = mytop != 0u && d < (double)SB_BINS ? (int)d : SB_BINS;
        sh.used[tid] = used;
    }
    if (tid < SAMPLE_MAX_SLICES / 32) sh.touched[tid] = 0u;
    __syncthreads();
    if (!top) {
        if (tid == 0) ws->plan.top = 0u;
        return;
    }
    unsigned bc[SB_PER] = {};
    unsigned long long bu[SB_PER] = {}, in_lo = 0, in_hi = 0;  // this thread's bins, and the slices that have tokens in them
#pragma unroll 1
    for (int s0 = 0; s0 < ns; s0 += 8) {
        unsigned long long v[8][SB_PER];
#pragma unroll
        for (int g = 0; g < 8; ++g) {
            const int s = min(s0 + g, ns - 1), d = sh.shift[s], end = s0 + g < ns ? sh.used[s] : 0;
#pragma unroll
            for (int j = 0; j < SB_PER; ++j) {
                const int i = SB_PER * tid + j - d;
                v[g][j] = i >= 0 && i < end ? load_coherent(&bins[(size_t)s * SB_BINS + i]) : 0ull;
            }
        }
#pragma unroll
        for (int g = 0; g < 8; ++g) {
            unsigned long long some = 0;
#pragma unroll
            for (int j = 0; j < SB_PER; ++j) {
                bc[j] += (unsigned)v[g][j] & 16383u;
                bu[j] += v[g][j] >> 14;
                some |= v[g][j];
            }
            const unsigned long long bit = some ? 1ull << ((s0 + g) & 63) : 0ull;
            if (s0 < 64) in_lo |= bit;
            else in_hi |= bit;
        }
    }
    RowPlan plan = make_plan(a.rows[row], row_u(a, row), rb, top, bc, bu, sh);
    bool mine = false;
#pragma unroll
    for (int i = 0; i < SB_RANGES; ++i)
        mine |= plan.lo[i] < SB_BINS && SB_PER * tid + SB_PER > plan.lo[i] && SB_PER * tid <= plan.hi[i];
    if (mine) {
#pragma unroll
        for (int w = 0; w < 2; ++w) {
            if ((unsigned)(in_lo >> (32 * w))) atomicOr(&sh.touched[w], (unsigned)(in_lo >> (32 * w)));
            if ((unsigned)(in_hi >> (32 * w))) atomicOr(&sh.touched[2 + w], (unsigned)(in_hi >> (32 * w)));
        }
    }
    for (int i = tid; i < SB_BINS; i += SB_THREADS) {
        ws->cum[i] = sh.cum[i];
        ws->cumc[i] = sh.cumc[i];
    }
    __syncthreads();
    if (tid == 0) {
#pragma unroll
        for (int w = 0; w < SAMPLE_MAX_SLICES / 32; ++w) plan.touched[w] = sh.touched[w];
        ws->plan = plan;
        ws->fill = 0u;
    }
}

// Gathers one slice's tokens of the plan's runs.  20 rows: 6 us; 64 rows, most of whose slices have some: 10.
__global__ __launch_bounds__(SB_THREADS) void sample_gather_kernel(SampleArgs a) {
    __shared__ __attribute__((aligned(16))) uint32_t keys[SL_LEN];
    __shared__ uint32_t buf[SB_THREADS / 64];
    const int slice = blockIdx.x, row = blockIdx.y;
    RowSpace* ws = (RowSpace*)(a.rows_ws + (size_t)row * SAMPLE_ROW_BYTES);
    const RowPlan& plan = ws->plan;
    if (!plan.top || plan.n > (unsigned)SB_CAP || !(plan.touched[slice >> 5] >> (slice & 31) & 1u)) return;
    const RowArgs r{a.logits, a.dt, (size_t)row * a.ld, a.V};
    const int n = min(SL_LEN, a.V - slice * SL_LEN);
    load_tokens(r, slice * SL_LEN, n, keys, buf);
    take_tokens(plan, keys, slice, n, SB_CAP, &ws->fill, [&](unsigned at, unsigned long long v) { ws->list[at] = v; });
}

// The cuts and the draw, one workgroup a row.  20 rows: 14 us, about 1 a step; 64 rows with up to some thousand
// gathered tokens each, narrowed in LDS: 27.
__global__ __launch_bounds__(SB_THREADS) void sample_draw_kernel(SampleArgs a) {
    __shared__ SampleShared sh;
    __shared__ unsigned long long sel[SB_CAP];
    const int row = blockIdx.x, tid = threadIdx.x;
    RowSpace* ws = (RowSpace*)(a.rows_ws + (size_t)row * SAMPLE_ROW_BYTES);
    const RowPlan plan = ws->plan;
    if (!plan.top) return draw_nothing(a, row);
    const RowArgs r{a.logits, a.dt, (size_t)row * a.ld, a.V};
#pragma unroll
    for (int j = 0; j < SB_PER; ++j) {
        sh.cum[j * SB_THREADS + tid] = ws->cum[j * SB_THREADS + tid];
        sh.cumc[j * SB_THREADS + tid] = ws->cumc[j * SB_THREADS + tid];
    }
    __syncthreads();
    draw_row(a, row, r, plan, row_u(a, row), ws->list, SB_CAP, sel, sh);
}

hipError_t launch_sample(const SampleArgs& a, int m, hipStream_t st, hipEvent_t done) {
    if (!a.slices) {
        // on every launch: the attribute belongs to the device that is current
        const int lds = (int)sizeof(SmallShared) + (a.V - 1) / SL_LEN * SL_LEN * 4;
        const hipError_t e = hipFuncSetAttribute((const void*)sample_small_kernel, hipFuncAttributeMaxDynamicSharedMemorySize, lds);
        if (e != hipSuccess) return e;
        return launch_done(sample_small_kernel, dim3((unsigned)m), dim3(SB_THREADS), lds, st, done, a);
    }
    const dim3 g((unsigned)a.slices, (unsigned)m);
    sample_count_kernel<<<g, dim3(SB_THREADS), 0, st>>>(a);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;                             // nothing behind it: the plan would be an earlier call's
    sample_gather_kernel<<<g, dim3(SB_THREADS), 0, st>>>(a);
    e = hipGetLastError();
    return e == hipSuccess ? launch_done(sample_draw_kernel, dim3((unsigned)m), dim3(SB_THREADS), 0, st, done, a) : e;
}

size_t sample_slice_bytes(int slices) { return (size_t)MAX_ROWS * slices * (sizeof(SliceHead) + 8 * SB_BINS); }

// The counters of every row's workspace, once.
__global__ void sample_clear_kernel(uint8_t* rows) {
    RowSpace* ws = (RowSpace*)(rows + (size_t)threadIdx.x * SAMPLE_ROW_BYTES);
    ws->arrived = 0u;
    ws->fill = 0u;
}

hipError_t launch_sample_clear(uint8_t* rows, hipStream_t st) {
    sample_clear_kernel<<<dim3(1), dim3(MAX_ROWS), 0, st>>>(rows);
    return hipGetLastError();
}

// ------------------------------------------------------------------ drafted tree

// One wave a slot, one lane a node.  A node is reached if its parent is and it
// is the parent's first child whose token is the one sampled there; node 0 is.
// Each step takes the lowest such child, so it goes to a later node and the walk
// ends after at most n steps.  One slot of 15 nodes 1.7 us, 256 of 64 nodes 2.9: the
// launch.
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
