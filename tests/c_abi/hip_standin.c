/* The HIP runtime calls of the library's host side, without a GPU: streams that can be captured and released, events, memory from the
 * heap, kernels that are counted and never run.  Loaded globally before the library, its definitions take the runtime's place, and the
 * test asks it what was ordered behind what.
 *
 * A stream is any address; work on it is counted, `done` is how much of it the host has waited for.  An event holds, for every stream,
 * how much of its work lies before it.  A stream that was released must not be named again. */
#include <stdint.h>
#include <stdlib.h>
#include <string.h>

typedef int hipError_t;
enum { kStreams = 16, kOk = 0, kDestroyed = 709, kIsolation = 905, kCapturedEvent = 907 };
typedef struct { uint32_t x, y, z; } dim3_t;
typedef struct { void* handle; int alive; unsigned long long capture; long work[kStreams]; } stream_t;
typedef struct { int recorded; unsigned long long capture; long work[kStreams]; } event_t;

static stream_t streams[kStreams];
static int n_streams;
static long done[kStreams];
static int dead_uses, forbidden;
static hipError_t last;
static dim3_t last_grid, last_block;
static long launches;

static hipError_t fail(hipError_t e) { last = e; return e; }
static int find(void* handle) {
    int i;
    for (i = 0; i < n_streams; ++i)
        if (streams[i].handle == handle) return i;
    if (n_streams == kStreams) abort();
    memset(&streams[n_streams], 0, sizeof streams[0]);
    streams[n_streams].handle = handle;
    streams[n_streams].alive = 1;
    return n_streams++;
}
static int live(void* handle) {
    const int i = find(handle);
    if (streams[i].alive) return i;
    ++dead_uses;
    return -1;
}
static void work_on(int i) { ++streams[i].work[i]; }

/* ---- the test's side ---- */
void standin_capture(void* stream, unsigned long long id) { streams[find(stream)].capture = id; }
void standin_release(void* stream) { streams[find(stream)].alive = 0; }
int standin_dead_uses(void) { return dead_uses; }
int standin_forbidden(void) { return forbidden; }
/* work enqueued on `stream` that the host does not know to be over */
long standin_pending(void* stream) { const int i = find(stream); return streams[i].work[i] - done[i]; }
/* work of `of` that what comes next on `stream` does not wait for */
long standin_unordered(void* stream, void* of) { const int i = find(stream), j = find(of); return streams[j].work[j] - streams[i].work[j]; }
void standin_work(void* stream) { work_on(find(stream)); }
long standin_launches(void) { return launches; }
void standin_grid(uint32_t* out) { out[0] = last_grid.x; out[1] = last_grid.y; out[2] = last_block.x; }

/* ---- the runtime's side ---- */
hipError_t hipStreamGetCaptureInfo(void* s, int* status, unsigned long long* id) {
    const int i = live(s);
    if (i < 0) return fail(kDestroyed);
    *status = streams[i].capture != 0;
    *id = streams[i].capture;
    return kOk;
}
hipError_t hipStreamIsCapturing(void* s, int* status) {
    unsigned long long id;
    return hipStreamGetCaptureInfo(s, status, &id);
}
hipError_t hipStreamCreateWithFlags(void** s, unsigned flags) { (void)flags; *s = malloc(8); find(*s); return kOk; }
hipError_t hipStreamDestroy(void* s) { standin_release(s); return kOk; }
hipError_t hipStreamSynchronize(void* s) {
    int i = live(s), j;
    if (i < 0) return fail(kDestroyed);
    if (streams[i].capture) { ++forbidden; return fail(900); }
    for (j = 0; j < kStreams; ++j) if (streams[i].work[j] > done[j]) done[j] = streams[i].work[j];
    return kOk;
}
hipError_t hipDeviceSynchronize(void) { int i; for (i = 0; i < n_streams; ++i) done[i] = streams[i].work[i]; return kOk; }
hipError_t hipEventCreateWithFlags(void** e, unsigned flags) { (void)flags; *e = calloc(1, sizeof(event_t)); return kOk; }
hipError_t hipEventCreate(void** e) { return hipEventCreateWithFlags(e, 0); }
hipError_t hipEventDestroy(void* e) { free(e); return kOk; }
hipError_t hipEventRecord(void* ev, void* s) {
    event_t* e = ev;
    const int i = live(s);
    if (i < 0) return fail(kDestroyed);
    e->recorded = 1;
    e->capture = streams[i].capture;
    memcpy(e->work, streams[i].work, sizeof e->work);
    return kOk;
}
hipError_t hipEventQuery(void* ev) { (void)ev; return kOk; }
hipError_t hipEventSynchronize(void* ev) {
    event_t* e = ev;
    int j;
    if (!e->recorded) return kOk;
    if (e->capture) return fail(kCapturedEvent);
    for (j = 0; j < kStreams; ++j) if (e->work[j] > done[j]) done[j] = e->work[j];
    return kOk;
}
hipError_t hipEventElapsedTime(float* ms, void* a, void* b) { (void)a; (void)b; *ms = 1.f; return kOk; }
hipError_t hipStreamWaitEvent(void* s, void* ev, unsigned flags) {
    event_t* e = ev;
    int i = live(s), j;
    (void)flags;
    if (i < 0) return fail(kDestroyed);
    if (!e->recorded) return kOk;
    if (e->capture) {
        int going = 0;
        for (j = 0; j < n_streams; ++j) going |= streams[j].capture == e->capture;
        if (!going) return fail(kCapturedEvent);
        if (!streams[i].capture) streams[i].capture = e->capture;             /* joins */
    }
    if (streams[i].capture != e->capture) { ++forbidden; return fail(kIsolation); }
    for (j = 0; j < kStreams; ++j) if (e->work[j] > streams[i].work[j]) streams[i].work[j] = e->work[j];
    return kOk;
}
hipError_t hipMalloc(void** p, size_t n) { *p = aligned_alloc(256, (n + 255) / 256 * 256); return *p ? kOk : fail(2); }
hipError_t hipFree(void* p) { free(p); return kOk; }
hipError_t hipMemset(void* p, int v, size_t n) { memset(p, v, n); return kOk; }
hipError_t hipMemcpy(void* d, const void* s, size_t n, int kind) { (void)kind; memcpy(d, s, n); return kOk; }
hipError_t hipMemcpyAsync(void* d, const void* s, size_t n, int kind, void* st) {
    const int i = live(st);
    (void)kind;
    if (i < 0) return fail(kDestroyed);
    memcpy(d, s, n);
    work_on(i);
    return kOk;
}
/* all memory is page-locked: the attributes start with the type, 1 */
hipError_t hipPointerGetAttributes(void* a, const void* p) { (void)p; *(int*)a = 1; return kOk; }
hipError_t hipFuncSetAttribute(const void* f, int a, int v) { (void)f; (void)a; (void)v; return kOk; }
hipError_t hipGetDevice(int* d) { *d = 0; return kOk; }
hipError_t hipGetSymbolAddress(void** p, const void* s) { (void)s; static char scratch[64]; *p = scratch; return kOk; }
hipError_t hipGetLastError(void) { const hipError_t e = last; last = kOk; return e; }
const char* hipGetErrorString(hipError_t e) { (void)e; return "stand-in"; }
/* what a launch expression hands over */
static dim3_t next_grid, next_block;
static size_t next_lds;
static void* next_stream;
hipError_t __hipPushCallConfiguration(dim3_t grid, dim3_t block, size_t lds, void* s) {
    next_grid = grid; next_block = block; next_lds = lds; next_stream = s;
    return kOk;
}
hipError_t __hipPopCallConfiguration(dim3_t* grid, dim3_t* block, size_t* lds, void** s) {
    *grid = next_grid; *block = next_block; *lds = next_lds; *s = next_stream;
    return kOk;
}
hipError_t hipLaunchKernel(const void* f, dim3_t grid, dim3_t block, void** args, size_t lds, void* s) {
    const int i = live(s);
    (void)f; (void)args; (void)lds;
    if (i < 0) return fail(kDestroyed);
    last_grid = grid;
    last_block = block;
    ++launches;
    work_on(i);
    return kOk;
}
