// What the library's host code shares: errors, the stage and its KV states, the
// order of its calls on the device and the way metadata gets there.
#pragma once

#include "stage.h"
#include "common.h"

#include <algorithm>
#include <array>
#include <climits>
#include <cmath>
#include <cstdlib>
#include <cstring>
#include <memory>
#include <mutex>
#include <new>
#include <string>
#include <vector>

namespace stg {

inline thread_local std::string g_err;

inline int fail(int code, const std::string& msg) {
    g_err = msg;
    return code;
}

#define HIP_TRY(expr)                                                                          \
    do {                                                                                       \
        hipError_t e_ = (expr);                                                                \
        if (e_ != hipSuccess) return fail(STAGE_E_HIP, std::string(#expr) + ": " + hipGetErrorString(e_)); \
    } while (0)

constexpr int META_RING = 4;

struct DevMat {
    PackedMat pm;
    int ksplit = 1, cps = 1;
    int bp_split = 1, bp_kg = 1;   // prepared-operand product: splits of K, groups of 128 k per wave
};

struct LayerDev {
    DevMat qkv, o, gu, d;
    uint16_t* attn_norm = nullptr;
    uint16_t* ffn_norm = nullptr;
};

inline int dt_code(int stage_dt) { return stage_dt == STAGE_DTYPE_BF16 ? DT_BF16 : DT_F16; }
inline bool dtype_ok(int dt) { return dt == STAGE_DTYPE_F32 || dt == STAGE_DTYPE_F16 || dt == STAGE_DTYPE_BF16; }
inline int any_dt(int dt) { return dt == STAGE_DTYPE_F32 ? (int)DT_F32 : dt_code(dt); }

inline size_t align16(size_t x) { return (x + 15) & ~(size_t)15; }

}  // namespace stg

using namespace stg;

struct Stage {
    StageConfig cfg{};
    int device = 0;
    std::vector<LayerDev> layers;
    std::vector<void*> allocs;
    float2* rope = nullptr;
    float *x = nullptr, *qkv = nullptr, *attn = nullptr, *act = nullptr, *gpart = nullptr, *apart = nullptr, *ssq = nullptr;
    unsigned *gcnt = nullptr, *acnt = nullptr;
    int ntiles_h = 0;
    // prepared inputs of the matrix-core products (2..64 rows), double-buffered
    bool bp_ok = false;
    int kp = 0;                                        // row stride: max K rounded up to 128
    uint16_t* bp[2] = {nullptr, nullptr};              // [MAX_ROWS][kp] codes
    float* bc[2] = {nullptr, nullptr};                 // [MAX_ROWS][kp / 32] corrections
    float* cbf[2] = {nullptr, nullptr};                // [MAX_ROWS] scale each row was prepared with
    float* rsb = nullptr;                              // [MAX_ROWS] rs of the last normalization
    uint8_t* meta_dev = nullptr;
    size_t meta_cap = 0;
    uint8_t* meta_host[META_RING] = {};
    hipEvent_t meta_ev[META_RING] = {};
    bool meta_ev_used[META_RING] = {};
    int ring_i = 0;
    int64_t weight_bytes = 0;
    uint64_t fingerprint = 0;                          // of the config, rotary table and norm weights (KV blobs)
    // final-stage epilogue: final RMSNorm weight and INT4 LM head (stage_head_attach)
    bool head_ok = false;
    int vocab = 0;
    DevMat head;
    uint16_t* final_norm = nullptr;
    float4* top1_part = nullptr;                       // [MAX_ROWS][head tiles]
    Mx4Matrix* head4 = nullptr;                        // or an MXFP4 head (stage_head_attach_mx4), freed with the stage
    float* head_rows = nullptr;                        // its normalized input rows [MAX_ROWS][H]
    float *logits = nullptr, *head_p = nullptr;        // logits rows [MAX_ROWS][vocab] and [MAX_ROWS], on first need
    int32_t* head_tok = nullptr;
    // workspace of the MXFP4 products: activation fragments and their scales, grown on need
    // and the sums of split products
    uint8_t *mx_a = nullptr, *mx_s = nullptr, *mx_p = nullptr;
    size_t mx_a_cap = 0, mx_s_cap = 0, mx_p_cap = 0;
    // workspace of the sampling calls: the slices' counts, grown on need
    uint8_t *smp = nullptr, *smp_rows = nullptr;
    size_t smp_cap = 0;
    // first-stage role: token embedding table [embed_vocab][H] in act dtype (stage_embed_attach)
    uint16_t* embed = nullptr;
    int embed_vocab = 0;
    unsigned* embed_err = nullptr;                     // set by a gather that met an id outside the table
    // prefill workspace for pf_rows prompt rows: residual fp32 [rows][H], q|k|v fp32
    // [rows][NQKV], prepared inputs (64-row blocks; [1]: the down product's)
    float *pf_x = nullptr, *pf_qkv = nullptr, *pf_bc[2] = {nullptr, nullptr};
    uint16_t* pf_bp[2] = {nullptr, nullptr};
    float* pf_part = nullptr;                          // sums of the split residual products [splits][rows][H]
    size_t pf_rows = 0;
    // persistent-kernel weights (row layout) and barrier state
    bool ps_ok = false;
    int cpl_h = 0, cpl_q = 0, cpl_f = 0, kc_h = 0, kc_q = 0, kc_f = 0, ng_h = 0, ng_q = 0, ng_f = 0;
    std::vector<PsLayer> ps_host;
    PsLayer* ps_layers = nullptr;
    uint8_t* ps_wb[4] = {nullptr, nullptr, nullptr, nullptr};   // code slabs per matrix kind (all layers)
    size_t ps_wl[4] = {0, 0, 0, 0};                            // bytes per layer in each slab
    unsigned* err = nullptr;
    unsigned spin_limit = 1u << 20;                     // exchange wait passes (STAGE_PS_SPIN_LIMIT)
    int dbg_layer = -1, dbg_keys = 0, dbg_rows = 0;     // armed attention record (test support)
    float* dbg_q = nullptr;                             // [MAX_ROWS][Hq][D]
    float* dbg_logits = nullptr;                        // [MAX_ROWS][Hq][dbg_keys]
    int ps_nwg = 0;
    int n_cus = 0;                                      // compute units of the device
    int ps_rpw_qkv = 0, ps_rpw_h = 0, ps_rpw_gu = 0;    // rows per workgroup of the single-launch forward
    unsigned long long *ll_qkv = nullptr, *ll_o = nullptr, *ll_part = nullptr, *ll_act = nullptr;   // its flag-word
    unsigned* ll_x = nullptr;                                                                       // exchange buffers
    unsigned ll_epoch = 0;                              // flag numbers used so far
    bool ps_coop = false;                               // cooperative launch (STAGE_COOP=1), else a plain launch
    int attn_vector = 0;                                // attention on the vector units (STAGE_ATTN_VECTOR=1)
    bool attn_dma = true;                               // cache rows by direct loads where allowed (STAGE_ATTN_DMA=0: off)
    int gemm_min_rows = 1;                              // rows from which products use the matrix cores (STAGE_GEMM_MIN_ROWS)
    unsigned long long* trace = nullptr;   // phase stamps of the last persistent forward (STAGE_PS_TRACE=1)
    int prof_class = -1;
    std::vector<hipEvent_t> prof_ev;   // start/stop pairs
    size_t prof_used = 0;              // events recorded
    // Device work of every call on this stage (and on its KV states) runs in call
    // order: done_ev marks the end of the last call's work on last_stream, and a
    // call on another stream waits for it first (see order_on / mark_done).
    hipEvent_t done_ev = nullptr;
    hipStream_t last_stream = nullptr;
    bool done_used = false;

    std::array<void*, 7> pf_buffers() const { return {pf_x, pf_qkv, pf_bp[0], pf_bp[1], pf_bc[0], pf_bc[1], pf_part}; }

    ~Stage() {
        for (hipEvent_t e : prof_ev) (void)hipEventDestroy(e);
        if (pf_x) {
            (void)hipSetDevice(device);
            (void)hipDeviceSynchronize();
            for (void* p : pf_buffers()) (void)hipFree(p);
        }
        if (done_ev) (void)hipEventDestroy(done_ev);
        (void)hipSetDevice(device);
        (void)hipDeviceSynchronize();
        for (void* p : allocs) (void)hipFree(p);
        for (void* p : {(void*)mx_a, (void*)mx_s, (void*)mx_p, (void*)smp})
            if (p) (void)hipFree(p);
        if (meta_dev) (void)hipFree(meta_dev);
        for (int i = 0; i < META_RING; ++i) {
            if (meta_host[i]) (void)hipHostFree(meta_host[i]);
            if (meta_ev[i]) (void)hipEventDestroy(meta_ev[i]);
        }
    }

    template <class T>
    int alloc(T** p, size_t n_elems) {
        void* q = nullptr;
        if (n_elems == 0) n_elems = 1;
        if (hipMalloc(&q, n_elems * sizeof(T)) != hipSuccess) {
            (void)hipGetLastError();
            return fail(STAGE_E_OOM, "device allocation of " + std::to_string(n_elems * sizeof(T)) + " bytes failed");
        }
        allocs.push_back(q);
        *p = (T*)q;
        return STAGE_OK;
    }
};

struct Mx4Matrix {
    Stage* stage = nullptr;
    Mx4Mat m{};
};

struct KVState {
    Stage* stage = nullptr;
    int S = 0, cap = 0, P = 0;
    uint16_t* kc = nullptr;
    uint16_t* vc = nullptr;
    int16_t* table[2] = {nullptr, nullptr};
    int cur = 0;
};

namespace stg {

inline int ensure_meta(Stage* st, size_t bytes) {
    if (bytes <= st->meta_cap) return STAGE_OK;
    size_t cap = std::max<size_t>(bytes, 2 * st->meta_cap);
    cap = std::max<size_t>(cap, 1 << 16);
    HIP_TRY(hipDeviceSynchronize());   // old buffers may still be read by queued work
    if (st->meta_dev) HIP_TRY(hipFree(st->meta_dev));
    st->meta_dev = nullptr;
    for (int i = 0; i < META_RING; ++i) {
        if (st->meta_host[i]) HIP_TRY(hipHostFree(st->meta_host[i]));
        st->meta_host[i] = nullptr;
        st->meta_ev_used[i] = false;
    }
    if (hipMalloc(&st->meta_dev, cap) != hipSuccess) {
        (void)hipGetLastError();
        st->meta_cap = 0;
        return fail(STAGE_E_OOM, "metadata allocation failed");
    }
    for (int i = 0; i < META_RING; ++i) {
        if (hipHostMalloc(&st->meta_host[i], cap, hipHostMallocDefault) != hipSuccess) {
            (void)hipGetLastError();
            st->meta_cap = 0;
            return fail(STAGE_E_OOM, "pinned metadata allocation failed");
        }
    }
    st->meta_cap = cap;
    return STAGE_OK;
}

// Calls on one stage run on the device in the order they were made, whatever
// streams they are issued on: the workspace, the metadata buffer and the flag
// numbers of the single-launch forward are per stage.  A call on a stream other
// than the previous call's first makes its stream wait for that call's work.
inline hipError_t order_on(Stage* st, hipStream_t s) {
    if (st->done_used && s != st->last_stream) return hipStreamWaitEvent(s, st->done_ev, 0);
    return hipSuccess;
}
inline hipError_t mark_done(Stage* st, hipStream_t s) {
    const hipError_t e = hipEventRecord(st->done_ev, s);
    if (e == hipSuccess) {
        st->done_used = true;
        st->last_stream = s;
    }
    return e;
}

// A call's work on stream s, from order_on to launched(), after its last launch, which signals done_ev itself.  A call that
// ends before that, with an error, is marked behind whatever it has queued, which may still use the workspace.
struct WorkOn {
    Stage* st;
    hipStream_t s;
    bool open = true;
    WorkOn(Stage* st_, hipStream_t s_) : st(st_), s(s_) {}
    WorkOn(const WorkOn&) = delete;
    WorkOn& operator=(const WorkOn&) = delete;
    ~WorkOn() {
        if (open && mark_done(st, s) != hipSuccess) (void)hipGetLastError();   // the call reports its own error
    }
    void launched() {
        st->done_used = true;
        st->last_stream = s;
        open = false;
    }
};

// Copies `bytes` of host data into the next pinned metadata ring slot and from
// there to the device metadata buffer (stream-ordered); *dev is its device copy.
inline int meta_upload(Stage* st, const void* host, size_t bytes, hipStream_t s, const uint8_t** dev) {
    int rc = ensure_meta(st, std::max<size_t>(bytes, 16));
    if (rc) return rc;
    const int slot_i = st->ring_i;
    st->ring_i = (st->ring_i + 1) % META_RING;
    if (st->meta_ev_used[slot_i]) HIP_TRY(hipEventSynchronize(st->meta_ev[slot_i]));
    if (bytes) std::memcpy(st->meta_host[slot_i], host, bytes);
    HIP_TRY(hipMemcpyAsync(st->meta_dev, st->meta_host[slot_i], std::max<size_t>(bytes, 16), hipMemcpyHostToDevice, s));
    HIP_TRY(hipEventRecord(st->meta_ev[slot_i], s));
    st->meta_ev_used[slot_i] = true;
    *dev = st->meta_dev;
    return STAGE_OK;
}

// The current device of the calling thread, back when the call ends.
struct DeviceGuard {
    int prev = -1;
    hipError_t err;
    explicit DeviceGuard(int dev) {
        err = hipGetDevice(&prev);
        if (err == hipSuccess && prev != dev) err = hipSetDevice(dev);
        else prev = -1;
    }
    ~DeviceGuard() {
        if (prev >= 0) (void)hipSetDevice(prev);
    }
};

// No C++ exception leaves a C entry.
template <class F>
inline int guarded(F f) noexcept {
    try {
        return f();
    } catch (const std::bad_alloc&) {
        try { return fail(STAGE_E_OOM, "host allocation failed"); } catch (...) { return STAGE_E_OOM; }
    } catch (...) {
        try { return fail(STAGE_E_INVALID, "unexpected failure"); } catch (...) { return STAGE_E_INVALID; }
    }
}

// A call that uses the stage's workspace cannot be captured: a replay would not be ordered with the stage's other calls.
inline int captured(hipStream_t s, bool& yes) {
    hipStreamCaptureStatus c = hipStreamCaptureStatusNone;
    HIP_TRY(hipStreamIsCapturing(s, &c));
    yes = c != hipStreamCaptureStatusNone;
    return STAGE_OK;
}
inline int not_captured(hipStream_t s) {
    bool yes = false;
    const int rc = captured(s, yes);
    return rc ? rc : yes ? fail(STAGE_E_UNSUPPORTED, "this call cannot be captured into a graph") : STAGE_OK;
}

inline int grow(uint8_t** p, size_t* cap, size_t bytes) {
    if (*cap >= bytes) return STAGE_OK;
    HIP_TRY(hipDeviceSynchronize());                       // queued work may still read the old one
    if (*p) HIP_TRY(hipFree(*p));
    *p = nullptr;
    *cap = 0;
    if (hipMalloc(p, bytes) != hipSuccess) {
        (void)hipGetLastError();
        *p = nullptr;
        return fail(STAGE_E_OOM, "workspace allocation failed");
    }
    *cap = bytes;
    return STAGE_OK;
}

// One layer's attention of a forward: reads the stage's q|k|v rows; writes the o product's input, as prepared rows
// (bp, bc) or, where these are null, as rows of the stage's attn buffer.
struct LayerAttention {
    virtual hipError_t run(int layer, uint16_t* bp, float* bc) = 0;
};
// The layers of a forward of M rows, launch by launch.
int run_layers(Stage* st, int M, const void* hidden_in, void* hidden_out, hipStream_t s, LayerAttention& attention);

}  // namespace stg
