"""ctypes binding of libaafkv.so: the same entry points as include/aaf_kv.h, argument
marshalling only.  Every step of the path runs in the library's kernels; there is no Python
or CPU fallback, and loading fails loudly if the shared library is missing.

``KVPool`` is a convenience holder: it lets PyTorch allocate the pool, the workspace and
transfer buffers (PyTorch is used for device memory and streams only) and forwards to the
C entry points with the current stream.
"""
from __future__ import annotations

import ctypes as C
import os
from array import array

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libaafkv.so")

AAF_KV_ABI_VERSION = 1
AAF_OK = 0
AAF_ERR_INVALID_ARG, AAF_ERR_BAD_CTX, AAF_ERR_OOM_BLOCKS, AAF_ERR_OOM_CTX = -1, -2, -3, -4
AAF_ERR_TOO_LONG, AAF_ERR_INCOMPAT, AAF_ERR_DST_TOO_SMALL, AAF_ERR_CUDA = -5, -6, -7, -8
AAF_ERR_CORRUPT, AAF_ERR_TIMEOUT, AAF_ERR_TOO_MANY, AAF_ERR_SCRATCH_LIMIT = -9, -10, -11, -12
AAF_NOALLOC_MAX_BLOCKS = 4096
AAF_COMPOSE_SHARE, AAF_COMPOSE_COPY_ALL = 0, 1
AAF_POLICY_REUSE, AAF_POLICY_TRANSFER, AAF_POLICY_RECOMPUTE = 0, 1, 2
AAF_ENGINE_AUTO, AAF_ENGINE_VEC, AAF_ENGINE_BULK, AAF_ENGINE_WARP = 0, 1, 2, 3
AAF_OP_MATERIALIZE, AAF_OP_IMPORT, AAF_OP_APPEND, AAF_OP_COMPOSE, AAF_OP_CLASSES = 0, 1, 2, 3, 4
AAF_DTYPE_BF16, AAF_DTYPE_F16 = 0, 1
AAF_ROPE_NONE, AAF_ROPE_LINEAR, AAF_ROPE_BASE, AAF_ROPE_WAVELENGTH, AAF_ROPE_RAMP = 0, 1, 2, 3, 4
AAF_ALL_LAYERS, AAF_LIST_MAX_BLOCKS = -1, 1048576
OP_NAMES = ("materialize", "import", "append", "compose")


class aaf_kv_pool_desc(C.Structure):
    _fields_ = [
        ("struct_size", C.c_uint32), ("abi_version", C.c_uint32),
        ("n_layers", C.c_int32), ("n_kv_heads", C.c_int32), ("head_dim", C.c_int32), ("block_size", C.c_int32),
        ("elt_bytes", C.c_int32), ("n_blocks", C.c_int32), ("max_ctx", C.c_int32),
        ("max_blocks_per_ctx", C.c_int32), ("max_batch", C.c_int32), ("device", C.c_int32),
        ("pool_base", C.c_void_p), ("layer_stride_bytes", C.c_size_t),
        ("workspace", C.c_void_p), ("workspace_bytes", C.c_size_t),
        ("free_order", C.POINTER(C.c_int32)),
        ("model_id", C.c_uint64), ("config_hash", C.c_uint64),
    ]


class aaf_kv_xfer_desc(C.Structure):
    _fields_ = [
        ("model_id", C.c_uint64), ("config_hash", C.c_uint64),
        ("n_layers", C.c_int32), ("n_kv_heads", C.c_int32), ("head_dim", C.c_int32), ("elt_bytes", C.c_int32),
        ("pos_start", C.c_int64), ("n_tokens", C.c_int64),
    ]


class aaf_kv_stats(C.Structure):
    _fields_ = [
        ("free_blocks", C.c_int64), ("live_blocks", C.c_int64), ("peak_live_blocks", C.c_int64),
        ("live_ctx", C.c_int64), ("cow_count", C.c_int64), ("payload_bytes", C.c_int64),
        ("copy_launches", C.c_int64 * AAF_OP_CLASSES), ("meta_launches", C.c_int64),
        ("copy_ms", C.c_double * AAF_OP_CLASSES), ("timed_launches", C.c_int64 * AAF_OP_CLASSES),
    ]


class aaf_kv_catalog_cols(C.Structure):
    _fields_ = [("state_id", C.c_void_p), ("n_tokens", C.c_void_p), ("reuse", C.c_void_p), ("last_access", C.c_void_p),
                ("origin", C.c_void_p), ("parent", C.c_void_p), ("born", C.c_void_p), ("parent_born", C.c_void_p),
                ("block_offsets", C.c_void_p), ("block_id", C.c_void_p), ("pos_begin", C.c_void_p),
                ("pos_end", C.c_void_p), ("refcount", C.c_void_p), ("address", C.c_void_p)]


class aaf_kv_store_desc(C.Structure):
    _fields_ = [("struct_size", C.c_uint32), ("dtype", C.c_int32), ("n_q_heads", C.c_int32), ("rot_dim", C.c_int32),
                ("interleaved", C.c_int32), ("mscale", C.c_float), ("inv_freq", C.c_void_p), ("pos", C.c_void_p),
                ("q", C.c_void_p), ("q_out", C.c_void_p), ("k", C.c_void_p), ("v", C.c_void_p),
                ("q_stride", C.c_int64), ("q_out_stride", C.c_int64), ("k_stride", C.c_int64), ("v_stride", C.c_int64)]


class aaf_kv_rope_scaling(C.Structure):
    _fields_ = [("struct_size", C.c_uint32), ("reserved", C.c_uint32), ("factor", C.c_double), ("low", C.c_double),
                ("high", C.c_double), ("orig_context", C.c_double)]


class aaf_kv_attn(C.Structure):
    _fields_ = [("struct_size", C.c_uint32), ("dtype", C.c_int32), ("n_q_heads", C.c_int32), ("window", C.c_int32),
                ("scale", C.c_float), ("softcap", C.c_float), ("slopes", C.c_void_p), ("spans", C.c_void_p),
                ("q_stride", C.c_int64)]


class aaf_kv_select_desc(C.Structure):
    _fields_ = [("struct_size", C.c_uint32), ("dtype", C.c_int32), ("n_q_heads", C.c_int32), ("keep", C.c_int32),
                ("sink", C.c_int32), ("recent", C.c_int32), ("q_stride", C.c_int64)]


class aaf_kv_batch_desc(C.Structure):
    _fields_ = [("struct_size", C.c_uint32), ("rows", C.c_int32), ("tokens", C.c_int32), ("cols", C.c_int32),
                ("tables", C.c_void_p), ("lens", C.c_void_p), ("offsets", C.c_void_p), ("token_row", C.c_void_p),
                ("positions", C.c_void_p), ("slots", C.c_void_p)]


# every symbol include/aaf_kv.h declares: name -> (restype, argtypes)
_vp, _i32, _i64, _u32, _sz = C.c_void_p, C.c_int32, C.c_int64, C.c_uint32, C.c_size_t
_p32 = C.POINTER(C.c_int32)
SYMBOLS = {
    "aaf_kv_pool_workspace_bytes": (_sz, [C.POINTER(aaf_kv_pool_desc)]),
    "aaf_kv_pool_create": (C.c_int, [C.POINTER(aaf_kv_pool_desc), C.POINTER(_vp)]),
    "aaf_kv_pool_destroy": (C.c_int, [_vp]),
    "aaf_kv_materialize": (C.c_int, [_vp, _i32, _i64, _i64, _vp, _sz, C.POINTER(aaf_kv_xfer_desc), _vp]),
    "aaf_kv_import": (C.c_int, [_vp, _vp, C.POINTER(aaf_kv_xfer_desc), _p32, _vp]),
    "aaf_kv_materialize_batch": (C.c_int, [_vp, _i32, _p32, C.POINTER(_i64), C.POINTER(_i64), C.POINTER(_vp),
                                           C.POINTER(_sz), C.POINTER(aaf_kv_xfer_desc), _vp]),
    "aaf_kv_import_batch": (C.c_int, [_vp, _i32, C.POINTER(_vp), C.POINTER(aaf_kv_xfer_desc), _p32, _vp]),
    "aaf_kv_fork": (C.c_int, [_vp, _i32, _i32, _p32, _vp]),
    "aaf_kv_append": (C.c_int, [_vp, _i32, _p32, _p32, C.POINTER(_vp), _vp]),
    "aaf_kv_compose": (C.c_int, [_vp, _i32, _p32, _u32, _p32, _vp]),
    "aaf_kv_compose_batch": (C.c_int, [_vp, _i32, _p32, _p32, _u32, _p32, _vp]),
    "aaf_kv_evict": (C.c_int, [_vp, _i32, _p32, _vp]),
    "aaf_kv_materialize_host": (C.c_int, [_vp, _i32, _i64, _i64, _vp, _sz, _vp, _sz, C.POINTER(aaf_kv_xfer_desc), _vp]),
    "aaf_kv_import_host": (C.c_int, [_vp, _vp, C.POINTER(aaf_kv_xfer_desc), _vp, _sz, _p32, _vp]),
    "aaf_kv_append_host": (C.c_int, [_vp, _i32, _p32, _p32, C.POINTER(_vp), _vp, _sz, _vp]),
    "aaf_kv_materialize_host_chunked": (C.c_int, [_vp, _i32, _i64, _i64, _vp, _sz, _vp, _sz, _i32, C.POINTER(C.c_uint32),
                                                  _i32, _p32, C.POINTER(aaf_kv_xfer_desc), _vp]),
    "aaf_kv_import_host_chunked": (C.c_int, [_vp, _vp, C.POINTER(aaf_kv_xfer_desc), _vp, _sz, _i32, _p32, _vp]),
    "aaf_kv_evict_to_budget": (C.c_int, [_vp, C.c_double, C.c_double, C.c_double, _i64, _p32, _i32, _p32, _vp]),
    "aaf_kv_reserve": (C.c_int, [_vp, _i32, _p32, _p32, _vp]),
    "aaf_kv_store": (C.c_int, [_vp, _i32, C.POINTER(aaf_kv_store_desc), _i32, _p32, _p32, _vp]),
    "aaf_kv_rope_freqs": (C.c_int, [_i32, C.c_double, _i32, C.POINTER(aaf_kv_rope_scaling), C.POINTER(C.c_double),
                                    C.POINTER(C.c_float)]),
    "aaf_kv_attend_workspace_bytes": (_sz, [_vp]),
    "aaf_kv_attend": (C.c_int, [_vp, _i32, C.POINTER(aaf_kv_attn), _i32, _p32, _p32, _vp, _vp, _vp, _vp, _sz, _vp]),
    "aaf_kv_attn_mass": (C.c_int, [_vp, _i32, C.POINTER(aaf_kv_attn), _i32, _p32, _p32, _vp, _vp, _vp, _vp, _i64, _vp]),
    "aaf_kv_prune": (C.c_int, [_vp, _i32, _vp, _i64, _i64, _i64, _vp, _vp, _p32, _vp]),
    "aaf_kv_summary_bytes": (_sz, [_vp]),
    "aaf_kv_summarize": (C.c_int, [_vp, _i32, _i32, _i32, _p32, _p32, _vp, _sz, _vp]),
    "aaf_kv_select": (C.c_int, [_vp, _i32, C.POINTER(aaf_kv_select_desc), _i32, _p32, _p32, _vp, _vp, _sz, _vp, _vp, _vp, _sz, _vp]),
    "aaf_kv_attend_blocks": (C.c_int, [_vp, _i32, C.POINTER(aaf_kv_attn), _i32, _p32, _p32, _vp, _vp, _i32, _vp, _vp, _vp, _sz, _vp]),
    "aaf_kv_batch_tables": (C.c_int, [_vp, C.POINTER(aaf_kv_batch_desc), _i32, _p32, _p32, _vp]),
    "aaf_kv_catalog_rows": (C.c_int, [_vp, _p32, C.POINTER(_i64)]),
    "aaf_kv_export_catalog": (C.c_int, [_vp, C.POINTER(aaf_kv_catalog_cols), _vp]),
    "aaf_kv_get_catalog": (C.c_int, [_vp, C.POINTER(_i64), C.POINTER(_i64), C.POINTER(_i64)]),
    "aaf_kv_ctx_len": (C.c_int, [_vp, _i32, C.POINTER(_i64)]),
    "aaf_kv_get_table": (C.c_int, [_vp, _i32, _p32, _i32, _p32]),
    "aaf_kv_get_refcounts": (C.c_int, [_vp, _p32]),
    "aaf_kv_get_free_list": (C.c_int, [_vp, _p32, _p32]),
    "aaf_kv_pool_stats": (C.c_int, [_vp, C.POINTER(aaf_kv_stats)]),
    "aaf_kv_sync_status": (C.c_int, [_vp]),
    "aaf_kv_set_copy_engine": (C.c_int, [_vp, C.c_int]),
    "aaf_kv_set_timing": (C.c_int, [_vp, C.c_int]),
    "aaf_kv_materialize_noalloc": (C.c_int, [_vp, _sz, _i32, _i32, _i32, _i32, _i32, _i32, _p32, _i32, _i64, _i64, _vp,
                                             _sz, _vp]),
    "aaf_kv_state_bytes": (C.c_int64, [_i32, _i32, _i32, _i32, _i64]),
    "aaf_kv_transfer_time": (C.c_double, [C.c_double, C.c_double, C.c_double]),
    "aaf_kv_transfer_time_packed": (C.c_double, [C.c_double, C.c_double, C.c_double, C.c_double]),
    "aaf_kv_policy": (C.c_int, [C.c_int, C.c_double, C.c_double]),
    "aaf_kv_debug_expire_wait": (C.c_int, [_vp, C.c_uint64, _vp]),
    "aaf_kv_debug_mark_unusable": (C.c_int, [_vp]),
    "aaf_kv_strerror": (C.c_char_p, [C.c_int]),
}

_lib = None


def load():
    """Loads libaafkv.so (raises if it has not been built: there is no fallback)."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(
                f"{LIB_PATH} is missing: build it with `python -m paper_2607_10987_b200._build` "
                "(nvcc, sm_100a). There is no CPU or PyTorch fallback for the KV operators."
            )
        lib = C.CDLL(LIB_PATH)
        for name, (res, args) in SYMBOLS.items():
            fn = getattr(lib, name)
            fn.restype, fn.argtypes = res, args
        _lib = lib
    return _lib


def _fn(name):
    return getattr(load(), name)


# thin same-name wrappers ---------------------------------------------------------------------
def aaf_kv_pool_workspace_bytes(desc): return _fn("aaf_kv_pool_workspace_bytes")(C.byref(desc))
def aaf_kv_pool_create(desc, out): return _fn("aaf_kv_pool_create")(C.byref(desc), C.byref(out))
def aaf_kv_pool_destroy(pool): return _fn("aaf_kv_pool_destroy")(pool)
def aaf_kv_materialize(pool, ctx, t0, t1, dst, dst_bytes, out_desc, stream):
    return _fn("aaf_kv_materialize")(pool, ctx, t0, t1, dst, dst_bytes, out_desc, stream)
def aaf_kv_import(pool, src, desc, out_ctx, stream): return _fn("aaf_kv_import")(pool, src, desc, out_ctx, stream)
def aaf_kv_materialize_batch(pool, n, ctxs, t0, t1, dsts, dst_bytes, out_descs, stream):
    return _fn("aaf_kv_materialize_batch")(pool, n, ctxs, t0, t1, dsts, dst_bytes, out_descs, stream)
def aaf_kv_import_batch(pool, n, srcs, descs, out_ctxs, stream):
    return _fn("aaf_kv_import_batch")(pool, n, srcs, descs, out_ctxs, stream)
def aaf_kv_fork(pool, parent, k, out_children, stream): return _fn("aaf_kv_fork")(pool, parent, k, out_children, stream)
def aaf_kv_append(pool, n, ctxs, n_new, srcs, stream): return _fn("aaf_kv_append")(pool, n, ctxs, n_new, srcs, stream)
def aaf_kv_compose(pool, m, segs, flags, out_ctx, stream): return _fn("aaf_kv_compose")(pool, m, segs, flags, out_ctx, stream)
def aaf_kv_compose_batch(pool, n_out, seg_off, segs, flags, out_ctxs, stream):
    return _fn("aaf_kv_compose_batch")(pool, n_out, seg_off, segs, flags, out_ctxs, stream)
def aaf_kv_evict(pool, n, ctxs, stream): return _fn("aaf_kv_evict")(pool, n, ctxs, stream)
def aaf_kv_materialize_host(pool, ctx, t0, t1, dst_host, dst_bytes, staging, staging_bytes, out_desc, stream):
    return _fn("aaf_kv_materialize_host")(pool, ctx, t0, t1, dst_host, dst_bytes, staging, staging_bytes, out_desc, stream)
def aaf_kv_import_host(pool, src_host, desc, staging, staging_bytes, out_ctx, stream):
    return _fn("aaf_kv_import_host")(pool, src_host, desc, staging, staging_bytes, out_ctx, stream)
def aaf_kv_append_host(pool, n, ctxs, n_new, srcs_host, staging, staging_bytes, stream):
    return _fn("aaf_kv_append_host")(pool, n, ctxs, n_new, srcs_host, staging, staging_bytes, stream)
def aaf_kv_materialize_host_chunked(pool, ctx, t0, t1, dst_host, dst_bytes, staging, staging_bytes, chunk_tokens,
                                    done_flags, flags_cap, n_chunks_out, out_desc, stream):
    return _fn("aaf_kv_materialize_host_chunked")(pool, ctx, t0, t1, dst_host, dst_bytes, staging, staging_bytes,
                                                  chunk_tokens, done_flags, flags_cap, n_chunks_out, out_desc, stream)
def aaf_kv_import_host_chunked(pool, src_host, desc, staging, staging_bytes, chunk_tokens, out_ctx, stream):
    return _fn("aaf_kv_import_host_chunked")(pool, src_host, desc, staging, staging_bytes, chunk_tokens, out_ctx, stream)
def aaf_kv_evict_to_budget(pool, alpha, beta, gamma, budget, out_victims, cap, n_victims, stream):
    return _fn("aaf_kv_evict_to_budget")(pool, alpha, beta, gamma, budget, out_victims, cap, n_victims, stream)
def aaf_kv_reserve(pool, n, ctxs, n_new, stream): return _fn("aaf_kv_reserve")(pool, n, ctxs, n_new, stream)
def aaf_kv_store(pool, layer, desc, n, ctxs, n_new, stream):
    return _fn("aaf_kv_store")(pool, layer, desc, n, ctxs, n_new, stream)
def aaf_kv_rope_freqs(rot_dim, base, scaling, params, inv_freq, mscale):
    return _fn("aaf_kv_rope_freqs")(rot_dim, base, scaling, params, inv_freq, mscale)
def aaf_kv_attend_workspace_bytes(pool): return _fn("aaf_kv_attend_workspace_bytes")(pool)
def aaf_kv_attend(pool, layer, attn, n, ctxs, n_q, q, out, lse, workspace, workspace_bytes, stream):
    return _fn("aaf_kv_attend")(pool, layer, attn, n, ctxs, n_q, q, out, lse, workspace, workspace_bytes, stream)
def aaf_kv_attn_mass(pool, layer, attn, n, ctxs, n_q, q, lse, prev, mass, mass_stride, stream):
    return _fn("aaf_kv_attn_mass")(pool, layer, attn, n, ctxs, n_q, q, lse, prev, mass, mass_stride, stream)
def aaf_kv_prune(pool, ctx, scores, budget, sink, recent, kept, kept_scores, out_ctx, stream):
    return _fn("aaf_kv_prune")(pool, ctx, scores, budget, sink, recent, kept, kept_scores, out_ctx, stream)
def aaf_kv_summary_bytes(pool): return _fn("aaf_kv_summary_bytes")(pool)
def aaf_kv_summarize(pool, layer, dtype, n, ctxs, n_new, summary, summary_bytes, stream):
    return _fn("aaf_kv_summarize")(pool, layer, dtype, n, ctxs, n_new, summary, summary_bytes, stream)
def aaf_kv_select(pool, layer, desc, n, ctxs, n_q, q, summary, summary_bytes, blocks, scores, workspace, workspace_bytes, stream):
    return _fn("aaf_kv_select")(pool, layer, desc, n, ctxs, n_q, q, summary, summary_bytes, blocks, scores, workspace, workspace_bytes, stream)
def aaf_kv_attend_blocks(pool, layer, attn, n, ctxs, n_q, q, blocks, keep, out, lse, workspace, workspace_bytes, stream):
    return _fn("aaf_kv_attend_blocks")(pool, layer, attn, n, ctxs, n_q, q, blocks, keep, out, lse, workspace, workspace_bytes, stream)
def aaf_kv_batch_tables(pool, desc, n, ctxs, n_new, stream):
    return _fn("aaf_kv_batch_tables")(pool, desc, n, ctxs, n_new, stream)
def aaf_kv_catalog_rows(pool, n_states, n_rows): return _fn("aaf_kv_catalog_rows")(pool, n_states, n_rows)
def aaf_kv_export_catalog(pool, cols, stream): return _fn("aaf_kv_export_catalog")(pool, cols, stream)
def aaf_kv_get_catalog(pool, clock, reuse, last): return _fn("aaf_kv_get_catalog")(pool, clock, reuse, last)
def aaf_kv_ctx_len(pool, ctx, out): return _fn("aaf_kv_ctx_len")(pool, ctx, out)
def aaf_kv_get_table(pool, ctx, out, cap, n_blocks): return _fn("aaf_kv_get_table")(pool, ctx, out, cap, n_blocks)
def aaf_kv_get_refcounts(pool, out): return _fn("aaf_kv_get_refcounts")(pool, out)
def aaf_kv_get_free_list(pool, out, n_free): return _fn("aaf_kv_get_free_list")(pool, out, n_free)
def aaf_kv_pool_stats(pool, out): return _fn("aaf_kv_pool_stats")(pool, out)
def aaf_kv_sync_status(pool): return _fn("aaf_kv_sync_status")(pool)
def aaf_kv_set_copy_engine(pool, engine): return _fn("aaf_kv_set_copy_engine")(pool, engine)
def aaf_kv_set_timing(pool, enable): return _fn("aaf_kv_set_timing")(pool, enable)
def aaf_kv_materialize_noalloc(pool_base, layer_stride, n_layers, n_kv_heads, head_dim, block_size, elt_bytes, n_blocks,
                               block_table_host, n_table_blocks, t0, t1, dst, dst_bytes, stream):
    """Gather without any allocation (see include/aaf_kv.h): for callers that may not call cudaMalloc.
    block_table_host is a ctypes int32 array / pointer in host memory."""
    return _fn("aaf_kv_materialize_noalloc")(pool_base, layer_stride, n_layers, n_kv_heads, head_dim, block_size,
                                             elt_bytes, n_blocks, block_table_host, n_table_blocks, t0, t1, dst,
                                             dst_bytes, stream)
def aaf_kv_state_bytes(n_layers, n_kv_heads, head_dim, elt_bytes, n_tokens):
    return _fn("aaf_kv_state_bytes")(n_layers, n_kv_heads, head_dim, elt_bytes, n_tokens)
def aaf_kv_transfer_time(kv_bytes, bandwidth, latency): return _fn("aaf_kv_transfer_time")(kv_bytes, bandwidth, latency)
def aaf_kv_transfer_time_packed(kv_bytes, bandwidth, latency, pack_rate):
    return _fn("aaf_kv_transfer_time_packed")(kv_bytes, bandwidth, latency, pack_rate)
def aaf_kv_policy(local_and_compatible, t_transfer, t_prefill):
    return _fn("aaf_kv_policy")(1 if local_and_compatible else 0, t_transfer, t_prefill)
def aaf_kv_debug_expire_wait(pool, limit_cycles, stream): return _fn("aaf_kv_debug_expire_wait")(pool, limit_cycles, stream)
def aaf_kv_debug_mark_unusable(pool): return _fn("aaf_kv_debug_mark_unusable")(pool)
def aaf_kv_strerror(status): return _fn("aaf_kv_strerror")(status).decode()


def _ints(v):
    """A list as a C array of int32 (through the buffer protocol: a ctypes array takes its entries one by one)."""
    return C.byref(C.c_int32.from_buffer(array("i", v if len(v) else (0,))))


def _total(counts, n):
    """Tokens of a batch of n contexts (counts None: one each).  The library reads n counts, however many there are."""
    if counts is None:
        return n
    if len(counts) != n:
        raise ValueError(f"{len(counts)} token counts for {n} contexts")
    return sum(counts)


def _fits(*v):
    """Whether numbers are what they are in 32 bits: ctypes drops the bits above."""
    return all(-(1 << 31) <= x < 1 << 31 for x in v)


def make_desc(n_layers, n_kv_heads, head_dim, block_size, elt_bytes, n_blocks, max_ctx, max_blocks_per_ctx,
              max_batch=0, device=0, model_id=0, config_hash=0) -> aaf_kv_pool_desc:
    d = aaf_kv_pool_desc()
    d.struct_size = C.sizeof(aaf_kv_pool_desc)
    d.abi_version = AAF_KV_ABI_VERSION
    d.n_layers, d.n_kv_heads, d.head_dim, d.block_size, d.elt_bytes = n_layers, n_kv_heads, head_dim, block_size, elt_bytes
    d.n_blocks, d.max_ctx, d.max_blocks_per_ctx, d.max_batch, d.device = n_blocks, max_ctx, max_blocks_per_ctx, max_batch, device
    d.model_id, d.config_hash = model_id, config_hash
    return d


def rope_freqs(rot_dim, base=10000.0, scaling=AAF_ROPE_NONE, factor=1.0, low=1.0, high=32.0, orig_context=0.0):
    """Rotary frequencies as aaf_kv_rope_freqs defines them: (list of rot_dim / 2 doubles, mscale)."""
    s = aaf_kv_rope_scaling(C.sizeof(aaf_kv_rope_scaling), 0, factor, low, high, orig_context)
    out = (C.c_double * max(rot_dim // 2, 1))()
    m = C.c_float(1.0)
    st = aaf_kv_rope_freqs(rot_dim, base, scaling, C.byref(s), out, C.byref(m))
    if st != AAF_OK:
        raise ValueError(aaf_kv_strerror(st))
    return list(out[: rot_dim // 2]), m.value


class Rope:
    """Rotary parameters of a model: leading dimensions of a head that turn, their frequencies (float64 device tensor
    of rot_dim / 2 entries), pair layout and factor."""

    def __init__(self, rot_dim, inv_freq, interleaved=False, mscale=1.0):
        import torch

        if inv_freq.dtype != torch.float64 or not inv_freq.is_cuda or not inv_freq.is_contiguous() or 2 * inv_freq.numel() != rot_dim:
            raise ValueError("inv_freq: contiguous float64 CUDA tensor of rot_dim / 2 entries")
        self.rot_dim, self.inv_freq, self.interleaved, self.mscale = rot_dim, inv_freq, interleaved, mscale


class KVPool:
    """Holds the torch-allocated memory of one pool and forwards to the C ABI.

    Methods return (status, result); nothing is computed on the Python side.
    """

    def __init__(self, n_layers, n_kv_heads, head_dim, block_size, elt_bytes, n_blocks, max_ctx,
                 max_blocks_per_ctx, free_order=None, max_batch=0, device=0, model_id=1, config_hash=1,
                 pool_tensor=None):
        import numpy as np
        import torch

        self.torch = torch
        self.device = torch.device("cuda", device)
        self._raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (
            lambda index: torch.cuda.current_stream(index).cuda_stream)
        self._codes = {torch.bfloat16: AAF_DTYPE_BF16, torch.float16: AAF_DTYPE_F16}
        self.L, self.H, self.D, self.BS, self.E, self.NB = n_layers, n_kv_heads, head_dim, block_size, elt_bytes, n_blocks
        self.max_ctx, self.max_blk = max_ctx, max_blocks_per_ctx
        self.row = n_kv_heads * head_dim * elt_bytes
        self.run = block_size * self.row
        self.bpt = 2 * n_layers * self.row
        self.layer_stride = n_blocks * 2 * self.run
        d = make_desc(n_layers, n_kv_heads, head_dim, block_size, elt_bytes, n_blocks, max_ctx, max_blocks_per_ctx,
                      max_batch, device, model_id, config_hash)
        ws_bytes = aaf_kv_pool_workspace_bytes(d)
        if ws_bytes == 0:
            raise ValueError("invalid pool geometry")
        if pool_tensor is None:
            pool_tensor = torch.empty(n_layers * self.layer_stride, dtype=torch.uint8, device=self.device)
        assert pool_tensor.numel() * pool_tensor.element_size() >= n_layers * self.layer_stride
        self.pool = pool_tensor
        self.workspace = torch.empty(ws_bytes, dtype=torch.uint8, device=self.device)
        d.pool_base, d.layer_stride_bytes = self.pool.data_ptr(), self.layer_stride
        d.workspace, d.workspace_bytes = self.workspace.data_ptr(), ws_bytes
        self._fo = None
        if free_order is not None:
            self._fo = np.ascontiguousarray(np.asarray(free_order, dtype=np.int32))
            d.free_order = self._fo.ctypes.data_as(_p32)
        self.desc = d
        self._attend_ws = None  # scratch of attend, allocated by its first call
        self._like = None       # empty tensors of int32 and int64 on the pool's device
        self.h = C.c_void_p()
        st = aaf_kv_pool_create(d, self.h)
        if st != AAF_OK:
            raise RuntimeError(f"aaf_kv_pool_create failed: {aaf_kv_strerror(st)}")

    # ------------------------------------------------------------------ helpers
    def _stream(self):
        """Handle of the current stream of the pool's device."""
        return self._raw_stream(self.device.index)

    def xfer_desc(self, n_tokens, pos_start=0) -> aaf_kv_xfer_desc:
        x = aaf_kv_xfer_desc()
        x.model_id, x.config_hash = self.desc.model_id, self.desc.config_hash
        x.n_layers, x.n_kv_heads, x.head_dim, x.elt_bytes = self.L, self.H, self.D, self.E
        x.pos_start, x.n_tokens = pos_start, n_tokens
        return x

    def close(self):
        if getattr(self, "h", None) and self.h.value:
            aaf_kv_pool_destroy(self.h)
            self.h = C.c_void_p()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    # ------------------------------------------------------------------ operators
    def materialize(self, ctx, t0, t1, out=None):
        n = max(t1 - t0, 0)
        if out is None:
            out = self.torch.empty(max(n * self.bpt, 16), dtype=self.torch.uint8, device=self.device)
        xd = aaf_kv_xfer_desc()
        st = aaf_kv_materialize(self.h, ctx, t0, t1, out.data_ptr(), out.numel() * out.element_size(), C.byref(xd),
                                self._stream())
        return st, (out if st == AAF_OK else None)

    def imp(self, buf, n, desc=None):
        xd = desc if desc is not None else self.xfer_desc(n)
        out = C.c_int32(-1)
        st = aaf_kv_import(self.h, buf.data_ptr(), C.byref(xd), C.byref(out), self._stream())
        return st, (out.value if st == AAF_OK else None)

    def materialize_batch(self, ctxs, t0s, t1s, outs):
        """outs: one device tensor per entry.  Returns the status."""
        n = len(ctxs)
        a = (C.c_int32 * max(n, 1))(*ctxs)
        b0 = (C.c_int64 * max(n, 1))(*t0s)
        b1 = (C.c_int64 * max(n, 1))(*t1s)
        ptrs = (C.c_void_p * max(n, 1))(*[t.data_ptr() for t in outs])
        sizes = (C.c_size_t * max(n, 1))(*[t.numel() * t.element_size() for t in outs])
        return aaf_kv_materialize_batch(self.h, n, a, b0, b1, ptrs, sizes, None, self._stream())

    def import_batch(self, bufs, ns):
        """bufs: one device transfer buffer per entry, ns: its token count.  Returns (status, [handles])."""
        n = len(bufs)
        ptrs = (C.c_void_p * max(n, 1))(*[t.data_ptr() for t in bufs])
        descs = (aaf_kv_xfer_desc * max(n, 1))(*[self.xfer_desc(k) for k in ns])
        out = (C.c_int32 * max(n, 1))()
        st = aaf_kv_import_batch(self.h, n, ptrs, descs, out, self._stream())
        return st, (list(out[:n]) if st == AAF_OK else None)

    def fork(self, parent, k):
        out = (C.c_int32 * max(k, 1))()
        st = aaf_kv_fork(self.h, parent, k, out, self._stream())
        return st, (list(out[:k]) if st == AAF_OK else None)

    def append(self, ctxs, n_new, bufs):
        n = len(ctxs)
        a = (C.c_int32 * max(n, 1))(*ctxs)
        b = (C.c_int32 * max(n, 1))(*n_new)
        ptrs = (C.c_void_p * max(n, 1))(*[t.data_ptr() for t in bufs])
        return aaf_kv_append(self.h, n, a, b, ptrs, self._stream()), None

    def append_host(self, ctxs, n_new, host_bufs, staging):
        """host_bufs: one (pinned) host tensor per entry; staging: device scratch for all of them."""
        n = len(ctxs)
        a = (C.c_int32 * max(n, 1))(*ctxs)
        b = (C.c_int32 * max(n, 1))(*n_new)
        ptrs = (C.c_void_p * max(n, 1))(*[t.data_ptr() for t in host_bufs])
        return aaf_kv_append_host(self.h, n, a, b, ptrs, staging.data_ptr(), staging.numel() * staging.element_size(),
                                  self._stream())

    def compose(self, segs, flags=0):
        m = len(segs)
        a = (C.c_int32 * max(m, 1))(*segs)
        out = C.c_int32(-1)
        st = aaf_kv_compose(self.h, m, a, flags, C.byref(out), self._stream())
        return st, (out.value if st == AAF_OK else None)

    def compose_batch(self, seg_lists, flags=0):
        """seg_lists: one list of segment handles per merge; returns (status, [result handles])."""
        n_out = len(seg_lists)
        offs, flat = [0], []
        for segs in seg_lists:
            flat += list(segs)
            offs.append(len(flat))
        a = (C.c_int32 * (n_out + 1))(*offs)
        b = (C.c_int32 * max(len(flat), 1))(*flat)
        out = (C.c_int32 * max(n_out, 1))()
        st = aaf_kv_compose_batch(self.h, n_out, a, b, flags, out, self._stream())
        return st, (list(out[:n_out]) if st == AAF_OK else None)

    def evict(self, ctxs):
        n = len(ctxs)
        a = (C.c_int32 * max(n, 1))(*ctxs)
        return aaf_kv_evict(self.h, n, a, self._stream()), None

    # ------------------------------------------------------------------ operators that compute with the payload
    # Tensors: q [tokens, q heads, head_dim], k and v [tokens, kv heads, head_dim], bf16 or f16, the heads of a token
    # contiguous; tokens packed in the order of ctxs.  These calls are made once per layer and step: the checks are few
    # and cheap, the library checks the rest.
    def _rows(self, t, tokens, heads, name, dtype):
        """Token stride of a packed per-token tensor."""
        d = self.D
        if t.shape != (tokens, heads, d) or t.dtype != dtype or t.device != self.device:
            raise ValueError(f"{name}: expected a [{tokens}, {heads}, {d}] tensor of {dtype} on {self.device}, "
                             f"got {tuple(t.shape)} {t.dtype} on {t.device}")
        st = t.stride()
        if st[2] != 1 or (heads > 1 and st[1] != d):
            raise ValueError(f"{name}: the heads of a token must be contiguous")
        return st[0] if tokens > 1 else heads * d  # one token: whatever stride the tensor names is not used

    def _flat(self, t, dtype, n, name):
        if t.dtype != dtype or t.numel() != n or not t.is_contiguous() or t.device != self.device:
            raise ValueError(f"{name}: expected a contiguous {dtype} tensor of {n} entries on the pool's device")
        return t.data_ptr()

    def _code(self, t):
        code = self._codes.get(t.dtype)
        if code is None:
            raise ValueError(f"bfloat16 or float16 expected, got {t.dtype}")
        return code

    def reserve(self, ctxs, n_new):
        n = len(ctxs)
        return load().aaf_kv_reserve(self.h, n, (C.c_int32 * (n or 1))(*ctxs), (C.c_int32 * (n or 1))(*n_new),
                                     self._stream()), None

    def store(self, layer, ctxs, n_new, k, v, q=None, q_out=None, rope=None, pos=None):
        """Rotates q (into q_out, default in place) and k, writes k and v into the slots of the contexts' last n_new tokens."""
        n, tokens, dtype = len(ctxs), sum(n_new), k.dtype
        code = self._code(k)
        ks, vs = self._rows(k, tokens, self.H, "k", dtype), self._rows(v, tokens, self.H, "v", dtype)
        heads = qp = op = qs = os = 0
        if q is not None:
            heads = q.shape[1] if q.dim() == 3 else 0
            qs, qp = self._rows(q, tokens, heads, "q", dtype), q.data_ptr()
            os, op = (qs, qp) if q_out is None else (self._rows(q_out, tokens, heads, "q_out", dtype), q_out.data_ptr())
        rot, inter, mscale, inv = 0, 0, 1.0, 0
        if rope is not None:
            if rope.inv_freq.device != self.device:
                raise ValueError("rope: frequencies on another device than the pool")
            rot, inter, mscale, inv = rope.rot_dim, int(rope.interleaved), rope.mscale, rope.inv_freq.data_ptr()
        d = aaf_kv_store_desc(C.sizeof(aaf_kv_store_desc), code, heads, rot, inter, mscale, inv,
                              None if pos is None else self._flat(pos, self.torch.int64, tokens, "pos"),
                              qp, op, k.data_ptr(), v.data_ptr(), qs, os, ks, vs)
        return load().aaf_kv_store(self.h, layer, d, n, (C.c_int32 * (n or 1))(*ctxs), (C.c_int32 * (n or 1))(*n_new),
                                   self._stream()), None

    def _attn(self, q, tokens, scale, softcap, window, slopes, spans):
        heads = q.shape[1] if q.dim() == 3 else 0
        stride = self._rows(q, tokens, heads, "q", q.dtype)
        return aaf_kv_attn(C.sizeof(aaf_kv_attn), self._code(q), heads, window, self.D ** -0.5 if scale is None else scale, softcap,
                           None if slopes is None else self._flat(slopes, self.torch.float32, heads, "slopes"),
                           None if spans is None else self._flat(spans, self.torch.int32, 2 * tokens, "spans"), stride)

    def _attn_out(self, q, tokens, heads, out, lse):
        """Outputs of an attention call and its scratch, None for the latter if it is not there and must not be made."""
        torch = self.torch
        if out is None:
            out = torch.empty_like(q) if q.is_contiguous() else torch.empty_like(q, memory_format=torch.contiguous_format)
        elif self._rows(out, tokens, heads, "out", q.dtype) != heads * self.D:
            raise ValueError("out: dense tensor expected")
        if lse is None:
            lse = q.new_empty((tokens, heads), dtype=torch.float32)
        else:
            self._flat(lse, torch.float32, tokens * heads, "lse")
        return out, lse, self._attend_ws if self._attend_ws is not None else self._scratch()

    def _scratch(self):
        """Workspace of the attention calls, made by the first of them; None if it must not be made now."""
        torch = self.torch
        with torch.cuda.device(self.device):
            if torch.cuda.is_current_stream_capturing():  # refused anyway; kept scratch must not be a graph's memory
                return None
        self._attend_ws = torch.empty(aaf_kv_attend_workspace_bytes(self.h), dtype=torch.uint8, device=self.device)
        return self._attend_ws

    def attend(self, layer, ctxs, n_q, q, out=None, lse=None, scale=None, softcap=0.0, window=0, slopes=None, spans=None):
        """Attention of the contexts' last n_q tokens (None: one each); returns (status, (out, lse))."""
        n = len(ctxs)
        tokens = n if n_q is None else sum(n_q)
        a = self._attn(q, tokens, scale, softcap, window, slopes, spans)
        out, lse, ws = self._attn_out(q, tokens, a.n_q_heads, out, lse)
        if ws is None:
            return AAF_ERR_INVALID_ARG, None
        st = load().aaf_kv_attend(self.h, layer, a, n, (C.c_int32 * (n or 1))(*ctxs),
                                  None if n_q is None else (C.c_int32 * (n or 1))(*n_q), q.data_ptr(), out.data_ptr(),
                                  lse.data_ptr(), ws.data_ptr(), ws.numel(), self._stream())
        return st, ((out, lse) if st == AAF_OK else None)

    def attn_mass(self, layer, ctxs, n_q, q, lse, mass, prev=None, scale=None, softcap=0.0, window=0, slopes=None, spans=None):
        """mass[i, t] = prev[i, t] (default 0; may be mass itself) + what token t of context i received of this attention."""
        n = len(ctxs)
        tokens = n if n_q is None else sum(n_q)
        a = self._attn(q, tokens, scale, softcap, window, slopes, spans)
        for t in (mass,) if prev is None else (mass, prev):
            if t.device != self.device or t.dtype != self.torch.float32 or t.dim() != 2 or t.shape != mass.shape or \
                    t.shape[0] != n or t.stride(1) != 1 or (n > 1 and t.stride(0) != mass.stride(0)):
                raise ValueError("mass, prev: float32 tensors of one row per context, equally strided, on the pool's device")
        # a row's room: up to the next row, or the tensor's width where that is less
        stride = mass.stride(0) if n > 1 else mass.shape[1]
        if mass.shape[1] < stride and any((self.ctx_len(c) or 0) > mass.shape[1] for c in ctxs):
            return AAF_ERR_DST_TOO_SMALL, None
        st = load().aaf_kv_attn_mass(self.h, layer, a, n, (C.c_int32 * (n or 1))(*ctxs),
                                     None if n_q is None else (C.c_int32 * (n or 1))(*n_q), q.data_ptr(),
                                     self._flat(lse, self.torch.float32, tokens * a.n_q_heads, "lse"),
                                     None if prev is None else prev.data_ptr(), mass.data_ptr(), stride, self._stream())
        return st, (mass if st == AAF_OK else None)

    def prune(self, ctx, scores, budget, sink=0, recent=0, kept=None, kept_scores=None):
        """New context of `budget` tokens of ctx; kept (int32) and kept_scores (float32) receive which ones.
        Returns (status, handle)."""
        torch = self.torch
        n = self.ctx_len(ctx)
        if kept is None:
            kept = torch.empty(max(budget, 1), dtype=torch.int32, device=self.device)
        out = C.c_int32(-1)
        st = load().aaf_kv_prune(self.h, ctx, self._flat(scores, torch.float32, scores.numel() if n is None else n, "scores"), budget,
                                 sink, recent, self._flat(kept, torch.int32, max(budget, 1), "kept"),
                                 None if kept_scores is None else self._flat(kept_scores, torch.float32, max(budget, 1), "kept_scores"),
                                 C.byref(out), self._stream())
        return st, (out.value if st == AAF_OK else None)

    # Sparse attention: summaries (int8, a tensor of aaf_kv_summary_bytes entries of any shape, see new_summary), the choice of
    # blocks for every query token and kv head (int32 [tokens, kv heads, keep]), attention over them.
    def summary_bytes(self):
        return aaf_kv_summary_bytes(self.h)

    def new_summary(self):
        """Room for the summaries of all blocks: int8 [layers, blocks, bytes of a record]; not initialised."""
        size = self.summary_bytes()
        if not size:
            raise ValueError("a pool of 16-bit elements with a head_dim that is a multiple of 8 and at most 256 has summaries")
        return self.torch.empty((self.L, self.NB, size // (self.L * self.NB)), dtype=self.torch.int8, device=self.device)

    def summarize(self, layer, ctxs, n_new, summary, dtype):
        """Sums up the blocks of the contexts' last n_new tokens (None: all blocks) in one layer (None: in all).  dtype: torch type of the
        pool's elements."""
        n = len(ctxs)
        _total(n_new, n)
        code = self._codes.get(dtype)
        if code is None:
            raise ValueError(f"bfloat16 or float16 expected, got {dtype}")
        if layer is not None and not _fits(layer):
            return AAF_ERR_INVALID_ARG, None
        return load().aaf_kv_summarize(self.h, AAF_ALL_LAYERS if layer is None else layer, code, n, _ints(ctxs),
                                       None if n_new is None else _ints(n_new),
                                       self._flat(summary, self.torch.int8, self.summary_bytes(), "summary"), summary.numel(),
                                       self._stream()), None

    def select(self, layer, ctxs, n_q, q, summary, keep, sink=1, recent=1, blocks=None, scores=None):
        """For every query token and kv head the `keep` blocks with the largest bound on a score, the first `sink` and the last `recent`
        among them: (status, blocks), int32 [tokens, kv heads, keep], -1 behind the last.  scores: float32 tensor of the same shape."""
        n = len(ctxs)
        tokens = _total(n_q, n)
        if not _fits(layer, keep, sink, recent):
            return AAF_ERR_INVALID_ARG, None
        heads = q.shape[1] if q.dim() == 3 else 0
        d = aaf_kv_select_desc(C.sizeof(aaf_kv_select_desc), self._code(q), heads, keep, sink, recent, self._rows(q, tokens, heads, "q", q.dtype))
        if blocks is None:
            blocks = q.new_empty((tokens, self.H, max(keep, 0)), dtype=self.torch.int32)
        size = tokens * self.H * max(keep, 0)
        ws = self._attend_ws if self._attend_ws is not None else self._scratch()
        if ws is None:
            return AAF_ERR_INVALID_ARG, None
        st = load().aaf_kv_select(self.h, layer, d, n, _ints(ctxs), None if n_q is None else _ints(n_q),
                                  q.data_ptr(), self._flat(summary, self.torch.int8, self.summary_bytes(), "summary"), summary.numel(),
                                  self._flat(blocks, self.torch.int32, size, "blocks"),
                                  None if scores is None else self._flat(scores, self.torch.float32, size, "scores"), ws.data_ptr(), ws.numel(),
                                  self._stream())
        return st, (blocks if st == AAF_OK else None)

    def attend_blocks(self, layer, ctxs, n_q, q, blocks, out=None, lse=None, scale=None, softcap=0.0, window=0, slopes=None, spans=None):
        """attend over the listed blocks alone: blocks is int32 [tokens, kv heads, keep]; returns (status, (out, lse))."""
        n = len(ctxs)
        tokens = _total(n_q, n)
        if not _fits(layer, window):
            return AAF_ERR_INVALID_ARG, None
        a = self._attn(q, tokens, scale, softcap, window, slopes, spans)
        if blocks.dim() != 3 or blocks.shape[:2] != (tokens, self.H):
            raise ValueError(f"blocks: expected [{tokens}, {self.H}, keep], got {tuple(blocks.shape)}")
        keep = blocks.shape[2]
        out, lse, ws = self._attn_out(q, tokens, a.n_q_heads, out, lse)
        if ws is None:
            return AAF_ERR_INVALID_ARG, None
        st = load().aaf_kv_attend_blocks(self.h, layer, a, n, _ints(ctxs),
                                         None if n_q is None else _ints(n_q), q.data_ptr(),
                                         self._flat(blocks, self.torch.int32, blocks.numel(), "blocks"), keep, out.data_ptr(), lse.data_ptr(),
                                         ws.data_ptr(), ws.numel(), self._stream())
        return st, ((out, lse) if st == AAF_OK else None)

    def batch_tables(self, ctxs, n_new=None, rows=None, tokens=None, cols=None, out=None):
        """Device arrays of a batch for kernels of one's own (see aaf_kv_batch_tables): (status, dict of tables, lens, offsets,
        token_row (int32), positions, slots (int64)).  rows, tokens, cols: the arrays' sizes, by default the batch's own.  out: a dict of
        some or all of them to be filled instead."""
        torch = self.torch
        n = len(ctxs)
        total = _total(n_new, n)
        rows, tokens = n if rows is None else rows, total if tokens is None else tokens
        if cols is None:
            if out is not None and "tables" in out:
                cols = out["tables"].shape[-1]
            else:
                cols = max([-(-(self.ctx_len(c) or 0) // self.BS) for c in ctxs], default=0)
        if not _fits(rows, tokens, cols):
            return AAF_ERR_TOO_MANY, None
        i32, i64 = torch.int32, torch.int64
        if out is None:
            if rows < 0 or tokens < 0 or cols < 0:
                return AAF_ERR_DST_TOO_SMALL, None
            if self._like is None:  # new_empty of a tensor of the same kind is the cheapest allocation
                self._like = torch.empty(0, dtype=i32, device=self.device), torch.empty(0, dtype=i64, device=self.device)
            e32, e64 = self._like[0].new_empty, self._like[1].new_empty
            out = {"tables": e32((rows, cols)), "lens": e32((rows,)), "offsets": e32((rows + 1,)), "token_row": e32((tokens,)),
                   "positions": e64((tokens,)), "slots": e64((tokens,))}
            ptrs = [x.data_ptr() for x in out.values()]
        else:
            shapes = {"tables": (rows, cols), "lens": (rows,), "offsets": (rows + 1,), "token_row": (tokens,), "positions": (tokens,),
                      "slots": (tokens,)}
            if set(out) - set(shapes) or any(x.shape != shapes[k] for k, x in out.items()):
                raise ValueError(f"out: expected some of {shapes}")
            ptrs = [self._flat(out[k], i64 if k in ("positions", "slots") else i32, out[k].numel(), k) if k in out else None for k in shapes]
        d = aaf_kv_batch_desc(C.sizeof(aaf_kv_batch_desc), rows, tokens, cols, *ptrs)
        st = load().aaf_kv_batch_tables(self.h, d, n, _ints(ctxs), None if n_new is None else _ints(n_new), self._stream())
        return st, (out if st == AAF_OK else None)

    def materialize_host(self, ctx, t0, t1, dst_host, staging):
        return aaf_kv_materialize_host(self.h, ctx, t0, t1, dst_host.data_ptr(),
                                       dst_host.numel() * dst_host.element_size(), staging.data_ptr(),
                                       staging.numel() * staging.element_size(), None, self._stream())

    def import_host(self, src_host, n, staging):
        xd = self.xfer_desc(n)
        out = C.c_int32(-1)
        st = aaf_kv_import_host(self.h, src_host.data_ptr(), C.byref(xd), staging.data_ptr(),
                                staging.numel() * staging.element_size(), C.byref(out), self._stream())
        return st, (out.value if st == AAF_OK else None)

    def evict_to_budget(self, alpha, beta, gamma, budget_blocks):
        out = (C.c_int32 * self.max_ctx)()
        nv = C.c_int32(0)
        st = aaf_kv_evict_to_budget(self.h, alpha, beta, gamma, budget_blocks, out, self.max_ctx, C.byref(nv),
                                    self._stream())
        return st, (list(out[: nv.value]) if st == AAF_OK else None)

    def catalog(self):
        import numpy as np

        clock = C.c_int64(0)
        reuse = np.empty(self.max_ctx, dtype=np.int64)
        last = np.empty(self.max_ctx, dtype=np.int64)
        st = aaf_kv_get_catalog(self.h, C.byref(clock), reuse.ctypes.data_as(C.POINTER(C.c_int64)),
                                last.ctypes.data_as(C.POINTER(C.c_int64)))
        if st != AAF_OK:
            raise RuntimeError(aaf_kv_strerror(st))
        return {"clock": clock.value, "reuse": reuse.tolist(), "last_access": last.tolist()}

    def export_catalog(self) -> dict:
        """Runs the columnar export into torch-allocated device buffers; returns the columns as torch tensors
        (still on the device) trimmed to their row counts."""
        torch = self.torch
        ns, nr = C.c_int32(0), C.c_int64(0)
        aaf_kv_catalog_rows(self.h, C.byref(ns), C.byref(nr))
        i32 = lambda n: torch.empty(max(n, 1), dtype=torch.int32, device=self.device)
        i64 = lambda n: torch.empty(max(n, 1), dtype=torch.int64, device=self.device)
        t = {"state_id": i32(ns.value), "n_tokens": i64(ns.value), "reuse": i64(ns.value), "last_access": i64(ns.value),
             "origin": i32(ns.value), "parent": i32(ns.value), "born": i64(ns.value), "parent_born": i64(ns.value),
             "block_offsets": i32(ns.value + 1), "block_id": i32(nr.value), "pos_begin": i64(nr.value),
             "pos_end": i64(nr.value), "refcount": i32(nr.value), "address": i64(nr.value)}
        cols = aaf_kv_catalog_cols(**{k: v.data_ptr() for k, v in t.items()})
        st = aaf_kv_export_catalog(self.h, C.byref(cols), self._stream())
        if st != AAF_OK:
            raise RuntimeError(aaf_kv_strerror(st))
        n_of = lambda k: ns.value + 1 if k == "block_offsets" else (
            ns.value if k in ("state_id", "n_tokens", "reuse", "last_access", "origin", "parent", "born",
                              "parent_born") else nr.value)
        return {k: v[: n_of(k)] for k, v in t.items()}

    def materialize_host_chunked(self, ctx, t0, t1, dst_host, staging, chunk_tokens, flags=None):
        """flags: pinned torch int32 tensor receiving one completion flag per chunk (or None)."""
        nch = C.c_int32(0)
        fptr = C.cast(flags.data_ptr(), C.POINTER(C.c_uint32)) if flags is not None else None
        st = aaf_kv_materialize_host_chunked(self.h, ctx, t0, t1, dst_host.data_ptr(),
                                             dst_host.numel() * dst_host.element_size(), staging.data_ptr(),
                                             staging.numel() * staging.element_size(), chunk_tokens, fptr,
                                             flags.numel() if flags is not None else 0, C.byref(nch), None,
                                             self._stream())
        return st, nch.value

    def import_host_chunked(self, src_host, n, staging, chunk_tokens):
        xd = self.xfer_desc(n)
        out = C.c_int32(-1)
        st = aaf_kv_import_host_chunked(self.h, src_host.data_ptr(), C.byref(xd), staging.data_ptr(),
                                        staging.numel() * staging.element_size(), chunk_tokens, C.byref(out),
                                        self._stream())
        return st, (out.value if st == AAF_OK else None)

    # ------------------------------------------------------------------ introspection
    def ctx_len(self, ctx):
        v = C.c_int64(-1)
        return v.value if aaf_kv_ctx_len(self.h, ctx, C.byref(v)) == AAF_OK else None

    def table(self, ctx):
        import numpy as np

        out = np.empty(self.max_blk, dtype=np.int32)
        nb = C.c_int32(0)
        st = aaf_kv_get_table(self.h, ctx, out.ctypes.data_as(_p32), self.max_blk, C.byref(nb))
        if st != AAF_OK:
            raise RuntimeError(aaf_kv_strerror(st))
        return out[: nb.value].copy()

    def refcounts(self):
        import numpy as np

        out = np.empty(self.NB, dtype=np.int32)
        st = aaf_kv_get_refcounts(self.h, out.ctypes.data_as(_p32))
        if st != AAF_OK:
            raise RuntimeError(aaf_kv_strerror(st))
        return out

    def free_list(self):
        import numpy as np

        out = np.empty(self.NB, dtype=np.int32)
        nf = C.c_int32(0)
        st = aaf_kv_get_free_list(self.h, out.ctypes.data_as(_p32), C.byref(nf))
        if st != AAF_OK:
            raise RuntimeError(aaf_kv_strerror(st))
        return out[: nf.value].copy()

    def live_ctxs(self):
        return [c for c in range(self.max_ctx) if self.ctx_len(c) is not None]

    def stats(self) -> dict:
        s = aaf_kv_stats()
        st = aaf_kv_pool_stats(self.h, C.byref(s))
        if st != AAF_OK:
            raise RuntimeError(aaf_kv_strerror(st))
        d = {k: getattr(s, k) for k in ("free_blocks", "live_blocks", "peak_live_blocks", "live_ctx", "cow_count",
                                        "payload_bytes", "meta_launches")}
        d["copy_launches"] = dict(zip(OP_NAMES, list(s.copy_launches)))
        d["copy_ms"] = dict(zip(OP_NAMES, list(s.copy_ms)))
        d["timed_launches"] = dict(zip(OP_NAMES, list(s.timed_launches)))
        return d

    def sync_status(self):
        return aaf_kv_sync_status(self.h)

    def set_copy_engine(self, engine):
        return aaf_kv_set_copy_engine(self.h, engine)

    def set_timing(self, enable):
        return aaf_kv_set_timing(self.h, 1 if enable else 0)
