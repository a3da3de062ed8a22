// A stand-in for the HIP runtime on the host: device memory is host memory,
// kernels do nothing, and every launch, event and allocation is noted, so that
// what the library's host code does around a failing call can be tested without a
// GPU.  Preloaded ahead of libstage.so; the functions at the end are the test's.
#include <stdint.h>
#include <stdio.h>
#include <stdlib.h>
#include <string.h>

#include <new>
#include <string>

typedef int hipError_t;
typedef void* ptr;
struct dim3 { uint32_t x, y, z; };

namespace {
std::string notes;
int last = 0, fail_at = 0, launches = 0, capturing = 0;
long alloc_fail_at = 0, allocs = 0, malloc_fail_at = 0, mallocs = 0, live = 0, syncs = 0;
intptr_t handles = 100;
long long max_malloc = 0;
dim3 cfg_grid, cfg_block;
size_t cfg_shmem;
ptr cfg_stream;

void note(char kind, ptr stream, ptr event) {
    char b[64];
    snprintf(b, sizeof b, "%c %lld %lld\n", kind, (long long)(intptr_t)stream, (long long)(intptr_t)event);
    notes += b;
}
int launch(ptr stream, ptr done) {
    if (++launches == fail_at) return last = 719;                  // hipErrorLaunchFailure
    note('L', stream, 0);
    if (done) note('R', stream, done);
    return 0;
}
}  // namespace

// The library's operator new, failing on request.
void* operator new(size_t n) {
    if (alloc_fail_at && ++allocs == alloc_fail_at) throw std::bad_alloc();
    void* p = malloc(n ? n : 1);
    if (!p) throw std::bad_alloc();
    return p;
}
void operator delete(void* p) noexcept { free(p); }
void operator delete(void* p, size_t) noexcept { free(p); }

extern "C" {

int __hipPushCallConfiguration(dim3 g, dim3 b, size_t s, ptr st) { cfg_grid = g; cfg_block = b; cfg_shmem = s; cfg_stream = st; return 0; }
int __hipPopCallConfiguration(dim3* g, dim3* b, size_t* s, ptr* st) { *g = cfg_grid; *b = cfg_block; *s = cfg_shmem; *st = cfg_stream; return 0; }
ptr* __hipRegisterFatBinary(const void*) { static ptr p; return &p; }
void __hipRegisterFunction(ptr*, const void*, char*, const char*, unsigned, ptr, ptr, ptr, ptr, int*) {}
void __hipRegisterVar(ptr*, void*, char*, char*, int, size_t, int, int) {}
void __hipUnregisterFatBinary(ptr*) {}

int hipLaunchKernel(const void*, dim3, dim3, ptr*, size_t, ptr st) { return launch(st, 0); }
int hipExtLaunchKernel(const void*, dim3, dim3, ptr*, size_t, ptr st, ptr, ptr done, int) { return launch(st, done); }
int hipLaunchCooperativeKernel(const void*, dim3, dim3, ptr*, unsigned, ptr st) { return launch(st, 0); }

int hipMalloc(ptr* p, size_t n) {
    if (malloc_fail_at && ++mallocs == malloc_fail_at) return last = 2;   // hipErrorOutOfMemory
    if ((long long)n > max_malloc) max_malloc = (long long)n;
    *p = calloc(n ? n : 1, 1);
    ++live;
    return *p ? 0 : (last = 2);
}
int hipFree(ptr p) { live -= p ? 1 : 0; ++syncs; free(p); return 0; }
int hipHostMalloc(ptr* p, size_t n, unsigned) { *p = calloc(n ? n : 1, 1); return *p ? 0 : 2; }
int hipHostFree(ptr p) { ++syncs; free(p); return 0; }
int hipMemcpy(void* d, const void* s, size_t n, int) { memcpy(d, s, n); return 0; }
int hipMemcpyAsync(void* d, const void* s, size_t n, int, ptr) { memcpy(d, s, n); return 0; }
int hipMemset(void* d, int v, size_t n) { memset(d, v, n); return 0; }
int hipMemsetAsync(void* d, int v, size_t n, ptr) { memset(d, v, n); return 0; }
int hipGetSymbolAddress(ptr* p, const void*) { static char room[256]; *p = room; return 0; }

int hipEventCreate(ptr* e) { *e = (ptr)++handles; return 0; }
int hipEventCreateWithFlags(ptr* e, unsigned) { *e = (ptr)++handles; return 0; }
int hipEventDestroy(ptr) { return 0; }
int hipEventElapsedTime(float* ms, ptr, ptr) { *ms = 0; return 0; }
int hipEventRecord(ptr e, ptr st) { note('R', st, e); return 0; }
int hipEventSynchronize(ptr) { return 0; }
int hipStreamWaitEvent(ptr st, ptr e, unsigned) { note('W', st, e); return 0; }
int hipStreamSynchronize(ptr) { return 0; }
int hipStreamIsCapturing(ptr, int* c) { *c = capturing; return 0; }

int hipDeviceSynchronize() { ++syncs; return 0; }
int hipDeviceGetAttribute(int* v, int, int) { *v = 256; return 0; }
int hipGetDevice(int* d) { *d = 0; return 0; }
int hipSetDevice(int) { return 0; }
int hipFuncGetAttributes(void*, const void*) { return 1; }
int hipFuncSetAttribute(const void*, int, int) { return 0; }
int hipOccupancyMaxActiveBlocksPerMultiprocessor(int* n, const void*, int, size_t) { *n = 1; return 0; }
int hipGetLastError() { const int e = last; last = 0; return e; }
const char* hipGetErrorString(int) { return "error of the stand-in"; }

// ---- for the test

// Notes start anew: launch `at` (from 1 on) fails, 0 none; and so does the `alloc`-th operator new.
void host_start(int at, long alloc, int capture) {
    alloc_fail_at = 0;
    notes.clear();
    notes.reserve(1 << 20);                    // taking notes allocates nothing
    launches = 0;
    fail_at = at;
    allocs = 0;
    alloc_fail_at = alloc;
    capturing = capture;
    last = 0;
    max_malloc = 0;
}
// Lines "L stream 0" (launched), "R stream event" (event recorded behind it), "W stream event" (stream waits).
const char* host_notes() { alloc_fail_at = 0; return notes.c_str(); }
int host_last_error() { return last; }
// From now on the `at`-th hipMalloc fails, 0 none.
void host_fail_malloc(long at) { malloc_fail_at = at; mallocs = 0; }
long host_live() { return live; }
// Calls that wait for the device, and end a capture that is under way.
long host_syncs() { return syncs; }
long long host_largest_malloc() { return max_malloc; }

}  // extern "C"
