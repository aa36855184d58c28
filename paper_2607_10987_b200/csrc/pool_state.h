// The host object of a pool and what the entry points' files share: argument checks, the pinned argument ring, the order of
// streams, the records of a batch.
#pragma once
#include <cuda_runtime.h>
#include <stdint.h>
#include <string.h>

#include <algorithm>
#include <atomic>
#include <new>
#include <vector>

#include "aafkv_internal.h"
#include "attend_internal.h"

// Profiler ranges: built with -DAAFKV_NVTX every C-ABI operator call is an NVTX range named after the entry
// point (header-only NVTX 3, no extra library); without the switch the macro is empty.
#ifdef AAFKV_NVTX
#include <nvtx3/nvToolsExt.h>
namespace {
struct ScopedRange {
    explicit ScopedRange(const char *name) { nvtxRangePushA(name); }
    ~ScopedRange() { nvtxRangePop(); }
};
}  // namespace
#define AAF_RANGE(name) ScopedRange aaf_range_(name)
#else
#define AAF_RANGE(name) do { } while (0)
#endif

namespace aafkv {

constexpr int ARG_SLOTS = 16;
constexpr unsigned long long NO_STREAM = ~0ull;  // the id of no stream, or of one whose id could not be had
constexpr size_t ARG_RECORD_BYTES = 96;  // per-record room in a slot of the pinned argument ring
static_assert(sizeof(ComposeSeg) <= ARG_RECORD_BYTES && sizeof(AppendEntry) <= ARG_RECORD_BYTES &&
                  sizeof(MatEntry) <= ARG_RECORD_BYTES && sizeof(ImpEntry) <= ARG_RECORD_BYTES,
              "argument records must fit their room in the pinned ring");

struct Layout {
    size_t ctl, refcount, ring, last_pos, tables, pieces, scratch, cat_len, cat_reuse, cat_last, cat_score, cat_origin, cat_parent, cat_born, cat_parent_born, tile_count, seq_records, total;
    int max_pieces, max_batch;
};

struct TimedLaunch {
    cudaEvent_t start, stop;
    int cls;
};

// The pool's device is the current one meanwhile.  The thread may be capturing another stream, which waiting on the host for the
// pool's own streams and events would end unless it is allowed to pass: they are none of that capture's.
struct DeviceGuard {
    int prev = -1;
    bool switched = false;
    cudaStreamCaptureMode mode = cudaStreamCaptureModeRelaxed;
    explicit DeviceGuard(int dev) {
        cudaThreadExchangeStreamCaptureMode(&mode);
        if (cudaGetDevice(&prev) == cudaSuccess && prev != dev) switched = cudaSetDevice(dev) == cudaSuccess;
    }
    ~DeviceGuard() {
        if (switched) cudaSetDevice(prev);
        cudaThreadExchangeStreamCaptureMode(&mode);
    }
};

}  // namespace aafkv

struct aaf_kv_pool {
    aaf_kv_pool_desc desc;
    aafkv::Geom g;
    aafkv::DevState s;
    aafkv::Layout lay;
    int device = 0, sm_count = 148;
    bool broken = false;  // a CUDA call failed after device state had changed: every later call returns AAF_ERR_CUDA
    aafkv::CopyTuning tuning{};
    std::vector<long long> len;  // tokens per handle, -1 = free
    // first token of a context whose slot no other context can share: what aaf_kv_store may write.  A fork or a sharing
    // merge moves it to the context's end; tokens added later are in blocks that the append copied or took afresh.
    std::vector<long long> own_from;
    // Contexts with the same non-zero fork id hold the same blocks for their first fork_len tokens (whole blocks): set by a
    // fork, in parent and children.  Shared blocks are never written again, so this stays true while both live.
    std::vector<long long> fork_id, fork_len;
    long long last_fork_id = 0;
    int live_ctx = 0;
    long long free_lb = 0;       // guaranteed lower bound of the device's free-block count
    long long clock = 0;         // logical clock: successful state-touching calls so far
    int *result = nullptr;       // pinned, device-writable: result of the scored eviction (max_ctx + 2 ints)
    cudaStream_t last_stream = nullptr;  // the caller's stream of the most recent call (copies run there)
    // Metadata kernels run on their own stream: they touch tables, reference counts, the ring and the piece
    // buffers only, never payload, so the planner of operator i+1 can run while the copy of operator i is
    // still streaming.  Two piece buffers alternate; events order planner -> copy and copy -> buffer reuse.
    cudaStream_t meta_stream = nullptr;
    cudaEvent_t plan_done[2] = {}, copy_done[2] = {};
    int next_buf = 0;
    // Copy launches of a pool share the ticket counter of its control block, so they must never overlap on the
    // device.  Calls on one stream are ordered anyway; when a call arrives on ANOTHER stream than the previous
    // copy launch, that stream is made to wait for the previous operator's last copy launch first.
    cudaEvent_t last_copy_event = nullptr;
    // Kernels that compute with the pool (attention, stores, gathers of a prune) read block tables on the caller's
    // stream: they wait for the metadata launched so far, and the next kernel that changes metadata waits for them.  Streams
    // are told apart by their ids, which are never reused.  read_ev is recorded by each such call itself, while its stream is
    // there and not being captured: who has to wait later has no other use for that stream.
    cudaEvent_t meta_ev = nullptr, read_ev = nullptr;
    long long meta_mark = -1;  // meta_launches when meta_ev was recorded
    bool meta_drained = false; // meta_ev has been seen complete
    bool read_pending = false; // readers that the metadata stream has not been ordered behind,
    std::vector<char> row_read; // and the handles whose table rows they may read
    unsigned long long read_id = aafkv::NO_STREAM, copy_id = aafkv::NO_STREAM;  // streams that are ordered behind the last reader, the last copy launch
    aafkv::PoolMap map;               // tensor map of the pool memory (wide attention kernel)
    bool map_ok = false;
    // pinned argument ring
    char *args = nullptr;
    size_t slot_bytes = 0;
    int next_slot = 0;
    cudaEvent_t slot_ev[aafkv::ARG_SLOTS] = {};
    bool slot_busy[aafkv::ARG_SLOTS] = {};
    int cur_slot = -1;
    // knobs and counters
    int engine = AAF_ENGINE_AUTO;
    bool timing = false;
    long long copy_launches[AAF_OP_CLASSES] = {};
    long long meta_launches = 0;
    double copy_ms[AAF_OP_CLASSES] = {};
    long long timed_launches[AAF_OP_CLASSES] = {};
    std::vector<aafkv::TimedLaunch> pending;
    std::vector<cudaEvent_t> spare_events;
    // chunked host transfers: a second stream for the PCIe copies and ordering events
    // chunked / host-buffer transfers: one library-owned stream per PCIe direction, so that uploads queue behind
    // each other in call order (the first one needed arrives first) while a download runs beside them
    cudaStream_t xfer_stream = nullptr;     // device -> host (aaf_kv_materialize_host_chunked)
    cudaStream_t upload_stream = nullptr;   // host -> device (aaf_kv_import_host_chunked, aaf_kv_append_host)
    // the scatter launches of the last upload call per staging role have read their staging buffer
    cudaEvent_t upload_reader_done = nullptr, import_reader_done = nullptr;
    bool upload_reader_pending = false, import_reader_pending = false;
    std::vector<cudaEvent_t> order_events;  // created on demand, reused round-robin
    size_t next_order_event = 0;
};

namespace aafkv {

inline long long nblk_of(const aaf_kv_pool *p, long long tokens) { return (tokens + p->g.BS - 1) / p->g.BS; }
inline bool is_live(const aaf_kv_pool *p, int c) { return c >= 0 && c < p->g.max_ctx && p->len[c] >= 0; }
// A CUDA runtime call failed after a planner may already have changed the device's metadata: the host mirror
// can no longer be trusted, so the pool refuses all further work.
inline int broke(aaf_kv_pool *p) {
    p->broken = true;
    return AAF_ERR_CUDA;
}
inline bool aligned16(const void *q) { return q && (reinterpret_cast<uintptr_t>(q) & 15u) == 0; }
// next pinned argument slot; waits (host side) until the device has finished reading its last use
inline char *acquire_args(aaf_kv_pool *p) {
    const int sl = p->next_slot;
    p->next_slot = (sl + 1) % ARG_SLOTS;
    if (p->slot_busy[sl]) {
        cudaEventSynchronize(p->slot_ev[sl]);
        p->slot_busy[sl] = false;
    }
    p->cur_slot = sl;
    return p->args + (size_t)sl * p->slot_bytes;
}
inline void release_args(aaf_kv_pool *p, cudaStream_t st) {
    if (p->cur_slot < 0) return;
    cudaEventRecord(p->slot_ev[p->cur_slot], st);
    p->slot_busy[p->cur_slot] = true;
    p->cur_slot = -1;
}
inline unsigned long long stream_id(cudaStream_t st) {
    unsigned long long id = 0;
    if (cudaStreamGetId(st, &id) != cudaSuccess) {
        cudaGetLastError();
        return NO_STREAM;
    }
    return id;
}
inline bool is_stream(unsigned long long known, unsigned long long id) { return known == id && id != NO_STREAM; }
// Before payload work on `st`: the pool's earlier readers and copies on other streams come first.
inline bool after_payload_work(aaf_kv_pool *p, cudaStream_t st) {
    const unsigned long long id = stream_id(st);
    if (!is_stream(p->read_id, id)) {
        if (cudaStreamWaitEvent(st, p->read_ev, 0) != cudaSuccess) return false;
        p->read_id = id;
    }
    if (p->last_copy_event && !is_stream(p->copy_id, id)) {
        if (cudaStreamWaitEvent(st, p->last_copy_event, 0) != cudaSuccess) return false;
        p->copy_id = id;
    }
    return true;
}
// Before a kernel on `st` that reads block tables or payload: it comes after the pool's earlier payload work, whatever
// stream that was on, and after the metadata launched so far.
inline bool begin_read(aaf_kv_pool *p, const int *handles, int n, cudaStream_t st) {
    if (!after_payload_work(p, st)) return false;
    p->read_pending = true;
    for (int i = 0; i < n; ++i) p->row_read[(size_t)handles[i]] = 1;
    if (p->meta_mark != p->meta_launches) {
        if (cudaEventRecord(p->meta_ev, p->meta_stream) != cudaSuccess) return false;
        p->meta_mark = p->meta_launches;
        p->meta_drained = false;
    }
    if (!p->meta_drained) {
        const cudaError_t e = cudaEventQuery(p->meta_ev);
        if (e == cudaSuccess) {
            p->meta_drained = true;
        } else {
            cudaGetLastError();
            if (e != cudaErrorNotReady || cudaStreamWaitEvent(st, p->meta_ev, 0) != cudaSuccess) return false;
        }
    }
    return true;
}
// Behind the last of its launches: what later calls wait for.
inline bool end_read(aaf_kv_pool *p, cudaStream_t st) { return cudaEventRecord(p->read_ev, st) == cudaSuccess; }
// A call reads host arrays and orders the pool's streams, neither of which a replayed graph would do again.
inline bool capturing(cudaStream_t st) {
    cudaStreamCaptureStatus s = cudaStreamCaptureStatusNone;
    if (cudaStreamIsCapturing(st, &s) != cudaSuccess) {
        cudaGetLastError();
        return true;
    }
    return s != cudaStreamCaptureStatusNone;
}

constexpr long long PART_ROWS = 65536;  // rows of partial results that a workspace holds
inline size_t attend_ws_bytes(const aaf_kv_pool *p) { return (size_t)PART_ROWS * ((size_t)p->g.D + 2) * sizeof(float) + 16; }
inline bool dtype_ok(int dtype) { return dtype == AAF_DTYPE_BF16 || dtype == AAF_DTYPE_F16; }
inline bool is_finite(float x) { return x - x == 0.0f; }
inline int log2_of(int v) {
    int s = 0;
    while ((1 << s) < v) ++s;
    return (1 << s) == v ? s : -1;
}
// what attention and attention mass have in common; *total_q, *max_rows describe the batch
inline int attn_check(const aaf_kv_pool *p, int32_t layer, const aaf_kv_attn *a, int32_t n, const aaf_ctx_t *ctxs,
               const int32_t *n_q, const void *q, long long *total_q) {
    if (!a || a->struct_size != sizeof(aaf_kv_attn) || n < 1 || !ctxs || !aligned16(q)) return AAF_ERR_INVALID_ARG;
    if (layer < 0 || layer >= p->g.L || !dtype_ok(a->dtype)) return AAF_ERR_INVALID_ARG;
    if (p->g.E != 2 || p->g.D % 8 != 0 || p->g.D > AAF_ATTN_MAX_HEAD_DIM) return AAF_ERR_INCOMPAT;
    if (a->n_q_heads < 1 || a->n_q_heads % p->g.H != 0 || a->window < 0) return AAF_ERR_INVALID_ARG;
    if ((long long)a->n_q_heads * p->g.D >= 1ll << 31) return AAF_ERR_INVALID_ARG;  // places within a token are ints in the kernels
    if (!is_finite(a->scale * 1.4427f) || !is_finite(a->softcap) || a->softcap < 0.0f) return AAF_ERR_INVALID_ARG;
    if (a->softcap > 0.0f && !is_finite(1.0f / a->softcap)) return AAF_ERR_INVALID_ARG;  // 0 / softcap would be NaN
    if (a->q_stride % 8 != 0 || a->q_stride < (long long)a->n_q_heads * p->g.D) return AAF_ERR_INVALID_ARG;
    if ((reinterpret_cast<uintptr_t>(a->slopes) & 3u) || (reinterpret_cast<uintptr_t>(a->spans) & 3u)) return AAF_ERR_INVALID_ARG;
    if (n > p->lay.max_batch) return AAF_ERR_TOO_MANY;
    long long total = 0;
    for (int i = 0; i < n; ++i) {
        if (!is_live(p, ctxs[i])) return AAF_ERR_BAD_CTX;
        const int nq = n_q ? n_q[i] : 1;
        if (nq < 1 || nq > p->len[ctxs[i]]) return AAF_ERR_INVALID_ARG;
        if (p->len[ctxs[i]] > (1ll << 30)) return AAF_ERR_TOO_LONG;  // token indices are ints in the kernels
        if ((long long)nq * (a->n_q_heads / p->g.H) > (1ll << 30)) return AAF_ERR_TOO_LONG;
        total += nq;
    }
    if (total * a->n_q_heads > (1ll << 31) - 1) return AAF_ERR_TOO_MANY;  // one CTA of the join per token and head
    *total_q = total;
    return AAF_OK;
}
inline AttnParams attn_params(const aaf_kv_pool *p, int layer, const aaf_kv_attn *a, const void *q) {
    AttnParams k{};
    k.q = q;
    k.tables = p->s.tables;
    k.kbase = p->g.pool + (long long)layer * p->g.layer_stride;
    k.slopes = a->slopes;
    k.spans = a->spans;
    k.q_stride = a->q_stride;
    k.run = p->g.run; k.row = p->g.row;
    k.max_blk = p->g.max_blk; k.BS = p->g.BS; k.bs_shift = log2_of(p->g.BS);
    k.H = p->g.H; k.G = a->n_q_heads / p->g.H; k.D = p->g.D;
    k.g_shift = log2_of(k.G);
    k.window = a->window;
    k.scale = a->scale; k.softcap = a->softcap;
    k.inv_cap = a->softcap > 0.0f ? 1.0f / a->softcap : 0.0f;
    return k;
}
// Records of a batch: kernel parameters while they fit, else through the pinned ring into the pool's workspace on `st`
// (the copies and their readers of all calls are ordered by begin_read).
template <typename Rec, typename Small>
bool place_records(aaf_kv_pool *p, const Rec *rec, size_t n, Small &small, const Rec **dev, int which, cudaStream_t st) {
    static_assert(sizeof(Rec) <= sizeof(AttnSeq), "records share the workspace of the attention records");
    *dev = nullptr;
    if (n <= (size_t)SMALL_SEQS) {
        std::copy(rec, rec + n, small.e);
        return true;
    }
    char *pinned = acquire_args(p);
    const size_t bytes = sizeof(Rec) * n;
    memcpy(pinned, rec, bytes);
    char *dst = reinterpret_cast<char *>(p->desc.workspace) + p->lay.seq_records + sizeof(AttnSeq) * (size_t)p->lay.max_batch * which;
    const bool ok = cudaMemcpyAsync(dst, pinned, bytes, cudaMemcpyHostToDevice, st) == cudaSuccess;
    release_args(p, st);
    *dev = reinterpret_cast<const Rec *>(dst);
    return ok;
}
template <typename Rec, typename Small>
bool place_records(aaf_kv_pool *p, const std::vector<Rec> &rec, Small &small, const Rec **dev, int which, cudaStream_t st) {
    return place_records(p, rec.data(), rec.size(), small, dev, which, st);
}

}  // namespace aafkv
