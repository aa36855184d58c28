// A model of the CUDA runtime in which nothing is computed and everything is ordered: streams, events and waits carry the set of
// the operations that have to be over before.  pool.cu is compiled against it as plain C++, so that a test can ask, on the
// CPU, whether one launch is ordered behind another, what a call does when a runtime function fails, and whether the library
// touches a stream that its caller has destroyed or is capturing.
#include <cuda_runtime.h>

#include <cstdlib>
#include <cstring>
#include <map>
#include <set>
#include <string>
#include <vector>

#include "aafkv_internal.h"
#include "attend_internal.h"

namespace {

typedef std::set<int> Done;
struct Stream {
    unsigned long long id = 0;
    bool alive = true, capturing = false;
    Done done;
};
struct Event {
    bool captured = false;
    Done done;
};
struct Op {
    std::string name;
    cudaStream_t stream;
    bool captured;
    Done before;
};

std::map<cudaStream_t, Stream> streams;
std::map<cudaEvent_t, Event> events;
std::vector<Op> ops;
std::vector<std::string> wrong;
std::map<std::string, int> fail_at;  // calls of a function until the one that fails; -1: all fail
Done host;                           // what the host has waited for
cudaStreamCaptureMode mode = cudaStreamCaptureModeGlobal;  // the calling thread's
unsigned long long ids = 0;
uintptr_t handles = 0x1000;

bool fails(const char *fn) {
    auto f = fail_at.find(fn);
    return f != fail_at.end() && (f->second < 0 || (f->second > 0 && --f->second == 0));
}
Stream &of(cudaStream_t s) {
    auto it = streams.find(s);
    if (it == streams.end()) {
        it = streams.emplace(s, Stream()).first;
        it->second.id = ++ids;
    }
    return it->second;
}
// calls that end a capture of the same thread unless its mode lets them pass
void may_end_a_capture(const char *what) {
    if (mode == cudaStreamCaptureModeRelaxed) return;
    for (const auto &s : streams)
        if (s.second.alive && s.second.capturing) wrong.push_back(std::string(what) + " beside a capture");
}
cudaError_t launch(const char *name, cudaStream_t s) {
    if (fails(name)) return cudaErrorUnknown;
    Stream &st = of(s);
    if (!st.alive) wrong.push_back(std::string(name) + " on a destroyed stream");
    Op op{name, s, st.capturing, st.done};
    op.before.insert(host.begin(), host.end());
    st.done.insert(op.before.begin(), op.before.end());
    st.done.insert((int)ops.size());
    ops.push_back(op);
    return cudaSuccess;
}

}  // namespace

// ------------------------------------------------------------------------------------------ what a test calls
extern "C" {
void order_reset() {
    streams.clear();
    events.clear();
    ops.clear();
    wrong.clear();
    fail_at.clear();
    host.clear();
}
void *order_stream() {
    cudaStream_t s = nullptr;
    cudaStreamCreateWithFlags(&s, cudaStreamNonBlocking);
    return s;
}
// destroys a stream and makes another; same_handle: under the old one's handle
void *order_replace_stream(void *s, int same_handle) {
    of(static_cast<cudaStream_t>(s)).alive = false;
    if (!same_handle) return order_stream();
    Stream fresh;
    fresh.id = ++ids;
    streams[static_cast<cudaStream_t>(s)] = fresh;
    return s;
}
void order_capture(void *s, int on) { of(static_cast<cudaStream_t>(s)).capturing = on != 0; }
void order_fail(const char *fn, int nth) { fail_at[fn] = nth; }
int order_ops() { return (int)ops.size(); }
const char *order_name(int i) { return ops[(size_t)i].name.c_str(); }
void *order_where(int i) { return ops[(size_t)i].stream; }
int order_captured(int i) { return ops[(size_t)i].captured; }
int order_before(int i, int j) { return (int)ops[(size_t)j].before.count(i); }
int order_host_knows(int i) { return (int)host.count(i); }
int order_wrongs() { return (int)wrong.size(); }
const char *order_wrong(int i) { return wrong[(size_t)i].c_str(); }

// ------------------------------------------------------------------------------------------ the runtime's functions
cudaError_t CUDARTAPI cudaStreamCreateWithFlags(cudaStream_t *s, unsigned) {
    *s = reinterpret_cast<cudaStream_t>(handles += 16);
    of(*s);
    return cudaSuccess;
}
cudaError_t CUDARTAPI cudaStreamDestroy(cudaStream_t s) {
    of(s).alive = false;
    return cudaSuccess;
}
cudaError_t CUDARTAPI cudaStreamGetId(cudaStream_t s, unsigned long long *id) {
    if (fails("cudaStreamGetId")) return cudaErrorUnknown;
    if (!of(s).alive) wrong.push_back("the id of a destroyed stream");
    *id = of(s).id;
    return cudaSuccess;
}
cudaError_t CUDARTAPI cudaStreamIsCapturing(cudaStream_t s, cudaStreamCaptureStatus *c) {
    *c = of(s).capturing ? cudaStreamCaptureStatusActive : cudaStreamCaptureStatusNone;
    return cudaSuccess;
}
cudaError_t CUDARTAPI cudaThreadExchangeStreamCaptureMode(cudaStreamCaptureMode *m) {
    std::swap(*m, mode);
    return cudaSuccess;
}
cudaError_t CUDARTAPI cudaStreamSynchronize(cudaStream_t s) {
    if (fails("cudaStreamSynchronize")) return cudaErrorUnknown;
    may_end_a_capture("waiting for a stream");
    if (!of(s).alive) wrong.push_back("the host waits for a destroyed stream");
    if (of(s).capturing) wrong.push_back("the host waits for a stream that is being captured");
    host.insert(of(s).done.begin(), of(s).done.end());
    return cudaSuccess;
}
cudaError_t CUDARTAPI cudaDeviceSynchronize() {
    for (auto &s : streams) host.insert(s.second.done.begin(), s.second.done.end());
    return cudaSuccess;
}
cudaError_t CUDARTAPI cudaStreamWaitEvent(cudaStream_t s, cudaEvent_t e, unsigned) {
    if (fails("cudaStreamWaitEvent")) return cudaErrorUnknown;
    Stream &st = of(s);
    const Event &ev = events[e];
    if (!st.alive) wrong.push_back("a destroyed stream waits for an event");
    if (ev.captured && !st.capturing) {
        wrong.push_back("a stream is pulled into another's capture");
        st.capturing = true;
    }
    st.done.insert(ev.done.begin(), ev.done.end());
    return cudaSuccess;
}
cudaError_t CUDARTAPI cudaEventCreateWithFlags(cudaEvent_t *e, unsigned) {
    *e = reinterpret_cast<cudaEvent_t>(handles += 16);
    events[*e] = Event();
    return cudaSuccess;
}
cudaError_t CUDARTAPI cudaEventCreate(cudaEvent_t *e) { return cudaEventCreateWithFlags(e, 0); }
cudaError_t CUDARTAPI cudaEventDestroy(cudaEvent_t e) {
    events.erase(e);
    return cudaSuccess;
}
cudaError_t CUDARTAPI cudaEventRecord(cudaEvent_t e, cudaStream_t s) {
    if (fails("cudaEventRecord")) return cudaErrorUnknown;
    Stream &st = of(s);
    if (!st.alive) wrong.push_back("an event is recorded on a destroyed stream");
    events[e].captured = st.capturing;
    events[e].done = st.done;
    events[e].done.insert(host.begin(), host.end());
    return cudaSuccess;
}
cudaError_t CUDARTAPI cudaEventQuery(cudaEvent_t) {
    may_end_a_capture("asking for an event");
    return cudaErrorNotReady;  // the device is as slow as it may be
}
cudaError_t CUDARTAPI cudaEventSynchronize(cudaEvent_t e) {
    if (fails("cudaEventSynchronize")) return cudaErrorUnknown;
    may_end_a_capture("waiting for an event");
    if (events[e].captured) wrong.push_back("the host waits for an event of a capture");
    host.insert(events[e].done.begin(), events[e].done.end());
    return cudaSuccess;
}
cudaError_t CUDARTAPI cudaEventElapsedTime(float *ms, cudaEvent_t, cudaEvent_t) {
    *ms = 0.0f;
    return cudaSuccess;
}
cudaError_t CUDARTAPI cudaGetLastError() { return cudaSuccess; }
cudaError_t CUDARTAPI cudaGetDevice(int *d) {
    *d = 0;
    return cudaSuccess;
}
cudaError_t CUDARTAPI cudaSetDevice(int) { return cudaSuccess; }
cudaError_t CUDARTAPI cudaGetDeviceCount(int *n) {
    *n = 1;
    return cudaSuccess;
}
cudaError_t CUDARTAPI cudaDeviceGetAttribute(int *v, cudaDeviceAttr, int) {
    *v = 148;
    return cudaSuccess;
}
cudaError_t CUDARTAPI cudaFuncSetAttribute(const void *, cudaFuncAttribute, int) { return cudaSuccess; }
cudaError_t CUDARTAPI cudaHostAlloc(void **p, size_t n, unsigned) {
    *p = calloc(1, n);
    return *p ? cudaSuccess : cudaErrorMemoryAllocation;
}
cudaError_t CUDARTAPI cudaFreeHost(void *p) {
    free(p);
    return cudaSuccess;
}
cudaError_t CUDARTAPI cudaMemset(void *p, int v, size_t n) {
    memset(p, v, n);
    return cudaSuccess;
}
cudaError_t CUDARTAPI cudaMemcpy(void *d, const void *s, size_t n, cudaMemcpyKind) {
    may_end_a_capture("a copy through the default stream");
    memcpy(d, s, n);
    return cudaSuccess;
}
cudaError_t CUDARTAPI cudaMemcpyAsync(void *d, const void *s, size_t n, cudaMemcpyKind, cudaStream_t st) {
    memcpy(d, s, n);
    return launch("memcpy", st);
}
cudaError_t CUDARTAPI cudaMemcpy2DAsync(void *, size_t, const void *, size_t, size_t, size_t, cudaMemcpyKind, cudaStream_t st) {
    return launch("memcpy2d", st);
}
}

// ------------------------------------------------------------------------------------------ the library's launchers
namespace aafkv {
cudaError_t launch_plan_materialize(const Geom &, const DevState &, int, long long, long long, char *, long long, cudaStream_t st, int) {
    return launch("plan_materialize", st);
}
cudaError_t launch_plan_materialize_batch(const Geom &, const DevState &, const MatEntry *, const SmallMat &, int, int, long long,
                                          cudaStream_t st) {
    return launch("plan_materialize", st);
}
cudaError_t launch_plan_import_batch(const Geom &, const DevState &, const ImpEntry *, const SmallImp &, int, int, long long,
                                     cudaStream_t st) {
    return launch("plan_import", st);
}
cudaError_t launch_plan_import(const Geom &, const DevState &, int, long long, const char *, long long, cudaStream_t st, int) {
    return launch("plan_import", st);
}
cudaError_t launch_fork(const Geom &, const DevState &, int, long long, int, const int *, const SmallInts &, long long, cudaStream_t st) {
    return launch("fork", st);
}
cudaError_t launch_plan_append(const Geom &, const DevState &, const AppendEntry *, const SmallAppend &, int, int, int, int, long long,
                               cudaStream_t st) {
    return launch("plan_append", st);
}
cudaError_t launch_plan_compose(const Geom &, const DevState &, const ComposeSeg *, const SmallCompose &, int, int, int, int, long long,
                                cudaStream_t st) {
    return launch("plan_compose", st);
}
cudaError_t launch_evict(const Geom &, const DevState &, const EvictArgs *, const SmallInts &, int, int, long long, int *n, cudaStream_t st) {
    if (n) *n = 1;
    return launch("evict", st);
}
cudaError_t launch_evict_to_budget(const Geom &, const DevState &, double, double, double, long long, long long, int *, cudaStream_t st) {
    return launch("evict", st);
}
cudaError_t copy_tuning_init(long long, CopyTuning *) { return cudaSuccess; }
cudaError_t launch_expire_wait(const DevState &, long long, cudaStream_t st) { return launch("expire_wait", st); }
cudaError_t launch_copy(int, const CopyTuning &, const Geom &, const DevState &, int, int, int, long long, int, cudaStream_t st) {
    return launch("copy", st);
}
cudaError_t launch_export_catalog(const Geom &, const DevState &, const aaf_kv_catalog_cols &, int, long long, cudaStream_t st) {
    return launch("export", st);
}
int few_rows_limit(int D) { return D <= 64 ? 32 : (D <= 128 ? 16 : 8); }
bool wide_takes(int, int) { return true; }
bool encode_pool_map(const Geom &, PoolMap *) { return true; }
cudaError_t launch_attend_few(const AttnParams &, const SmallSeqs &, int, int, bool, bool, cudaStream_t st) { return launch("attend", st); }
cudaError_t launch_attend_tile(const AttnParams &, const SmallSeqs &, int, int, cudaStream_t st) { return launch("attend", st); }
cudaError_t launch_attend_wide(const AttnParams &, const SmallSeqs &, int, bool, const void *, int, cudaStream_t st) { return launch("attend", st); }
cudaError_t launch_attend_join(const AttnParams &, const SmallSeqs &, int, int, int, int, int, cudaStream_t st) { return launch("join", st); }
cudaError_t launch_attn_mass(const MassParams &, const SmallSeqs &, int, int, cudaStream_t st) { return launch("mass", st); }
cudaError_t launch_attn_mass_wide(const MassParams &, const SmallSeqs &, int, const void *, int, cudaStream_t st) { return launch("mass", st); }
cudaError_t launch_store(const StoreParams &, const SmallStores &, int, int, cudaStream_t st) { return launch("store", st); }
cudaError_t launch_select(const float *, int, int, int, int, int *, float *, cudaStream_t st) { return launch("select", st); }
cudaError_t launch_gather_rows(const Geom &, const int *, const Piece *, const int *, int, int, cudaStream_t st) {
    return launch("gather", st);
}
}  // namespace aafkv
