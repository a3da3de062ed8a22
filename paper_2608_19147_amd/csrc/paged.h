// The paged cache: what its host code (kv_pages.hip) and its kernels (paged.hip) share.
#pragma once

#include "common.h"

namespace stg {

// One pool: K and V [layers][pages][Hkv][page_rows][D].  Row r of page p is slot (p << shift) + r.
struct PagedPool {
    uint16_t *k, *v;
    int layers, n_pages, shift, Hkv, D, kv_dt;
    __host__ __device__ size_t layer_elems() const { return ((size_t)n_pages * Hkv << shift) * D; }
};

// A run of keys that some rows see, met by a tile of their query vectors: one workgroup per kv head.  Query vector c of
// the run's rows is head c % gs (of the kv head's) of row list[rows + c / gs]; the tile takes q0 <= c < q0 + nq.
struct PagedItem {
    int rows, q0, nq;
    int kb, ke;                                    // keys, by their place in the sequence
    int table;                                     // of a sequence that holds the run: tables[table + key / page_rows] is its page
    int slot;                                      // which of a row's partial results this is
    int open;                                      // 1: no row's limit or mask cuts the run, 2: some row has a mask; + 4: probabilities in two terms
};
struct PagedRow {
    int row;
    int limit;                                     // keys below it are seen
    int mask;                                      // word offset of its bits in masks, or -1
    int part, nparts;                              // its partial results: [part, part + nparts); one: it goes straight to out
    int spare[3];
};
constexpr int PAGED_FEW = 16, PAGED_MANY = 128;    // most query vectors of a tile, of the two kernels

struct PagedAttend {
    const void* q; int q_dt; size_t ldq;           // [M][Hq D], rotated
    void* out; int out_dt; size_t ldo;
    const uint16_t *k, *v;                         // the layer's
    int shift, Hkv, gs;
    const PagedItem* items; int n_items; bool many;   // many: some tile has more than PAGED_FEW query vectors
    const PagedRow* list; const PagedRow* rows; int M;   // of the runs; [M]
    const int* tables; const uint32_t* masks;
    float scale2;                                  // log2(e) times the softmax's scale
    float* part_o; float2* part_ml;                // [parts][Hq][D], [parts][Hq] (max, sum)
    bool merge;                                    // some row has more than one partial result
};
hipError_t launch_paged_attend(const PagedAttend& a, int D, int kv_dt, hipStream_t st, hipEvent_t done);

struct PagedWrite {
    const void *q, *k, *v; int dt; size_t ldq, ldk, ldv;
    void* q_out; int q_out_dt; size_t ldqo;
    uint16_t *kp, *vp;                             // the layer's pages
    const int* slots;                              // [M]
    const int* pos; int M;                         // [axes][M], or null: nothing is turned
    const uint8_t* axis;                           // [D / 2], or null: the first
    const float2* rope;                            // [positions][D / 2] (cos, sin)
    int shift, Hq, Hkv, kv_dt;
};
hipError_t launch_paged_write(const PagedWrite& a, int D, hipStream_t st, hipEvent_t done);

// Bytes (rounded up to 16) from pinned host memory to the device.
hipError_t launch_paged_send(const void* host, void* dev, size_t bytes, hipStream_t st, hipEvent_t done);
// Rows moves[i].x -> moves[i].y (slots) of every layer, K and V; no row is both read and written.
hipError_t launch_paged_copy(const PagedPool& p, const int2* moves, int n, hipStream_t st, hipEvent_t done);
// The same where rows may overlap: sources and destinations ascend, a source is never below its destination's place in
// the sequence, so each piece of a row is moved by one thread, in order.
hipError_t launch_paged_slide(const PagedPool& p, const int2* moves, int n, hipStream_t st, hipEvent_t done);
// Rows from dense ones [layers][S][Hkv][cap][D]: row start + i of `slot`, read through `table` [S][cap] (null: as they lie),
// to slots[i].
hipError_t launch_paged_fill(const PagedPool& p, const uint16_t* k, const uint16_t* v, const int16_t* table, int S, int slot, int cap,
                             int start, const int* slots, int n, hipStream_t st, hipEvent_t done);
// Rows slots[i] of one layer to k, v [Hkv][n][D].
hipError_t launch_paged_read(const PagedPool& p, int layer, const int* slots, int n, uint16_t* k, uint16_t* v, hipStream_t st, hipEvent_t done);

// fp32 rows [M][K] as a product's prepared input, unnormalized (kernels.hip).
hipError_t launch_bprep_plain(const float* in, int K, int M, uint16_t* bp, float* bc, int kp, hipStream_t st);

}  // namespace stg
