"""ctypes binding of libkvswap.so, the C-ABI library declared in include/kvswap.h.

Argument marshalling only: every byte is moved by the HIP kernels / HIP copies
inside the library.  The functions carry the names of the C entry points; the
`KVPool` class bundles a handle with the tensors it points into so that they
stay alive.  There is no fallback: importing this module without a built
library raises.
"""
import ctypes as C
import os
import struct

import numpy as np
import torch  # noqa: F401  -- first, so that the library binds to the HIP runtime torch has loaded:
#                               two runtimes in one process do not see each other's allocations

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libkvswap.so")

KV_OK, KV_EINVAL, KV_ERANGE, KV_EDUP, KV_ENOENT = 0, -1, -2, -3, -4
KV_EEXIST, KV_ENOSPC, KV_EHIP, KV_ESTATE, KV_ENOMEM, KV_E2BIG = -5, -6, -7, -8, -9, -10
KV_NOALLOC_MAX_BLOCKS = 65536
KV_PATH_AUTO, KV_PATH_DMA, KV_PATH_ZEROCOPY, KV_STAGING_DEVICE, KV_PLAN_ONLY, KV_REQ_EVENTS = 0, 1, 2, 4, 8, 16
KV_DELTA_INCLUDE_TAIL = 1
KV_KEEP_STAGING = 1
KV_TUNE_MAX_WGS_DEVICE, KV_TUNE_MAX_WGS_LINK, KV_TUNE_KERNEL_VARIANT, KV_TUNE_DMA_SLICE_BLOCKS = 1, 2, 3, 4
KV_TUNE_SEGMENT_BYTES = 5
KV_TUNE_SCALE_LDS = 6
KV_TUNE_SEGMENT_MAX_BYTES = 7
KV_TUNE_SCATTER_ORDER = 8
KV_TUNE_PHASE_BYTES, KV_TUNE_PHASE_WGS_OUT, KV_TUNE_PHASE_WGS_IN = 9, 10, 11
KV_TUNE_KERNEL_EVENTS = 12
KV_TUNE_HOST_STORES = 13
KV_TUNE_LINK_IN_WGS, KV_TUNE_LINK_IN_UNROLL = 14, 15
KV_F16, KV_BF16, KV_FP8_E4M3 = 0, 1, 2
KV_ROPE_PLAIN, KV_ROPE_LINEAR, KV_ROPE_BASE, KV_ROPE_PARTS, KV_ROPE_YARN = 0, 1, 2, 3, 4

EXPORTS = ["kv_pool_create", "kv_pool_destroy", "kv_swap_out", "kv_swap_out_delta", "kv_swap_in", "kv_evict_and_load", "kv_sync",
           "kv_move_blocks", "kv_move_blocks_noalloc", "kv_req_reserve", "kv_req_release", "kv_req_query", "kv_last_stats",
           "kv_slot_bytes", "kv_last_plan", "kv_pool_tune", "kv_last_hip_error", "kv_strerror",
           "kv_io_stats_get", "kv_budget_blocks", "kv_req_poll", "kv_req_wait", "kv_last_timeline",
           "kv_swap_out_delta_timed", "kv_bench_copy", "kv_bench_copy_scrambled", "kv_bench_link", "kv_bench_link_bidir",
           "kv_wq_post", "kv_wq_drain", "kv_wq_remove", "kv_wq_pending",
           "kv_batch_create", "kv_batch_destroy", "kv_batch_set", "kv_batch_query", "kv_rope_freqs", "kv_append", "kv_attn", "kv_evict"]


class kv_pool_config(C.Structure):
    _fields_ = [("struct_size", C.c_uint32),
                ("num_layers", C.c_int32), ("num_kv_heads", C.c_int32), ("head_dim", C.c_int32),
                ("block_size", C.c_int32), ("dtype", C.c_int32), ("num_blocks", C.c_int64),
                ("pool_dev", C.c_void_p),
                ("layer_stride", C.c_int64), ("kv_stride", C.c_int64), ("block_stride", C.c_int64),
                ("scale_dev", C.c_void_p),
                ("scale_layer_stride", C.c_int64), ("scale_kv_stride", C.c_int64),
                ("scale_block_stride", C.c_int64),
                ("staging_host", C.c_void_p), ("staging_bytes", C.c_int64),
                ("bounce_dev", C.c_void_p), ("bounce_bytes", C.c_int64),
                ("evict_stream", C.c_void_p), ("load_stream", C.c_void_p),
                ("flags", C.c_uint32)]


class kv_stats(C.Structure):
    _fields_ = [("struct_size", C.c_uint32), ("op", C.c_int32), ("path", C.c_int32), ("launches", C.c_int32),
                ("copies", C.c_int32), ("grid", C.c_int32), ("blocks", C.c_int64), ("bytes", C.c_int64),
                ("plan_us", C.c_double), ("enqueue_us", C.c_double), ("ms_total", C.c_float),
                ("ms_kernel", C.c_float), ("scatter_order", C.c_int32), ("reserved", C.c_int32)]

    def as_dict(self):
        return {k: getattr(self, k) for k, _ in self._fields_ if k not in ("struct_size", "reserved")}


class kv_io_stats(C.Structure):
    _fields_ = [("struct_size", C.c_uint32), ("inflight_calls", C.c_int32 * 2), ("inflight_bytes", C.c_int64 * 2),
                ("total_calls", C.c_int64 * 2), ("total_bytes", C.c_int64 * 2), ("ewma_gbps", C.c_double * 2),
                ("ewma_small_us", C.c_double * 2)]

    def as_dict(self):
        return {k: list(getattr(self, k)) for k, _ in self._fields_ if k != "struct_size"}


class kv_batch_info(C.Structure):
    _fields_ = [("struct_size", C.c_uint32), ("rows", C.c_int32), ("items", C.c_int32), ("partial_rows", C.c_int32),
                ("cached_tokens", C.c_int64), ("read_tokens", C.c_int64)]

    def as_dict(self):
        return {k: getattr(self, k) for k, _ in self._fields_ if k != "struct_size"}


class kv_append_args(C.Structure):
    _fields_ = [("struct_size", C.c_uint32), ("layer", C.c_int32), ("io_dtype", C.c_int32), ("rot", C.c_int32),
                ("interleaved", C.c_int32), ("magnitude", C.c_float), ("q", C.c_void_p), ("k", C.c_void_p), ("v", C.c_void_p),
                ("q_out", C.c_void_p), ("q_strides", C.c_int64 * 2), ("k_strides", C.c_int64 * 2), ("v_strides", C.c_int64 * 2),
                ("q_out_strides", C.c_int64 * 2), ("turns", C.c_void_p), ("positions", C.c_void_p), ("k_scale", C.c_void_p),
                ("v_scale", C.c_void_p)]


class kv_attn_args(C.Structure):
    _fields_ = [("struct_size", C.c_uint32), ("layer", C.c_int32), ("io_dtype", C.c_int32), ("scale", C.c_float),
                ("q", C.c_void_p), ("out", C.c_void_p), ("q_strides", C.c_int64 * 2), ("out_strides", C.c_int64 * 2),
                ("lse", C.c_void_p), ("lse_stride", C.c_int64), ("weights", C.c_void_p), ("weights_strides", C.c_int64 * 2),
                ("weights_cap", C.c_int64)]


class kv_evict_args(C.Structure):
    _fields_ = [("struct_size", C.c_uint32), ("layer", C.c_int32), ("num_layers", C.c_int32), ("keep", C.c_int32),
                ("keep_first", C.c_int32), ("keep_last", C.c_int32), ("weights", C.c_void_p), ("weights_out", C.c_void_p),
                ("weights_strides", C.c_int64 * 3), ("weights_cap", C.c_int64), ("kept", C.c_void_p), ("kept_strides", C.c_int64 * 3),
                ("req_ids", C.c_void_p)]


if not os.path.exists(LIB_PATH):
    raise ImportError("libkvswap.so is not built: run `python -c 'import __graft_entry__ as g; g.build()'` "
                      "(hipcc --offload-arch=gfx950) first; there is no fallback path")
_lib = C.CDLL(LIB_PATH)

_vp, _i32, _i64, _u32, _u64 = C.c_void_p, C.c_int32, C.c_int64, C.c_uint32, C.c_uint64
_sig = {
    "kv_pool_create": (C.c_int, [C.POINTER(kv_pool_config), C.POINTER(_vp)]),
    "kv_pool_destroy": (C.c_int, [_vp]),
    "kv_swap_out": (C.c_int, [_vp, _i32, _vp, _vp, _vp, _vp, _vp]),
    "kv_swap_out_delta": (C.c_int, [_vp, _i32, _vp, _vp, _vp, _vp, _i64, _u32, _vp, _vp]),
    "kv_swap_out_delta_timed": (C.c_int, [_vp, _i32, _vp, _vp, _vp, _vp, _vp, C.c_double, _u32, _vp, _vp, _vp]),
    "kv_swap_in": (C.c_int, [_vp, _i32, _vp, _vp, _vp, _u32, _vp]),
    "kv_evict_and_load": (C.c_int, [_vp, _i32, _vp, _vp, _vp, _vp, _i32, _vp, _vp, _vp, _u32, _vp]),
    "kv_sync": (C.c_int, [_vp]),
    "kv_move_blocks": (C.c_int, [_vp, _i64, _vp, _vp, _vp]),
    "kv_move_blocks_noalloc": (C.c_int, [_vp, _i64, _vp, _vp, _vp]),
    "kv_req_reserve": (C.c_int, [_vp, _u64, _i32]),
    "kv_req_release": (C.c_int, [_vp, _u64]),
    "kv_req_query": (C.c_int, [_vp, _u64, _vp, _vp, _vp, _vp, _vp]),
    "kv_last_stats": (C.c_int, [_vp, C.POINTER(kv_stats)]),
    "kv_slot_bytes": (_i64, [_vp]),
    "kv_last_plan": (_i64, [_vp, _vp, _vp, _i64]),
    "kv_pool_tune": (C.c_int, [_vp, _i32, _i64]),
    "kv_last_hip_error": (C.c_int, [_vp]),
    "kv_strerror": (C.c_char_p, [C.c_int]),
    "kv_req_poll": (C.c_int, [_vp, _u64]),
    "kv_req_wait": (C.c_int, [_vp, _u64]),
    "kv_last_timeline": (_i64, [_vp, _vp, _vp, _i64]),
    "kv_io_stats_get": (C.c_int, [_vp, C.POINTER(kv_io_stats)]),
    "kv_budget_blocks": (_i64, [_vp, _i32, C.c_double]),
    "kv_bench_copy": (C.c_double, [_vp, _vp, _i64, _i32, _i32, _vp]),
    "kv_bench_copy_scrambled": (C.c_double, [_vp, _vp, _i64, _i64, _i32, _i32, _vp]),
    "kv_bench_link": (C.c_double, [_vp, _vp, _i64, _i32, _i32, _vp]),
    "kv_bench_link_bidir": (C.c_double, [_vp, _vp, _vp, _vp, _i64, _i32]),
    "kv_wq_post": (C.c_int, [_vp, _i32, _vp, _vp, _vp, _vp, _vp]),
    "kv_wq_drain": (C.c_int, [_vp, C.c_double, _i64, _u32, _vp, _vp, _vp, _vp]),
    "kv_wq_remove": (C.c_int, [_vp, _u64]),
    "kv_wq_pending": (C.c_int, [_vp, _vp, _vp]),
    "kv_batch_create": (C.c_int, [_vp, C.POINTER(_vp)]),
    "kv_batch_destroy": (C.c_int, [_vp]),
    "kv_batch_set": (C.c_int, [_vp, _i32, _vp, _vp, _vp, _vp, _i32, _vp]),
    "kv_batch_query": (C.c_int, [_vp, C.POINTER(kv_batch_info)]),
    "kv_rope_freqs": (C.c_int, [_i32, C.c_double, _i32, C.c_double, C.c_double, C.c_double, C.c_double, _vp, _vp]),
    "kv_append": (C.c_int, [_vp, _vp, _vp]),
    "kv_attn": (C.c_int, [_vp, _vp, _vp]),
    "kv_evict": (C.c_int, [_vp, _vp, _vp]),
}
for _name, (_res, _args) in _sig.items():
    _f = getattr(_lib, _name)
    _f.restype, _f.argtypes = _res, _args


_at = (C.c_char * 0).from_buffer


def _p(a):
    """The array as a pointer argument.  A ctypes view of its memory, 0.25 us against 1.2 for its ctypes.data; an array that cannot be
    written to has no such view.  (Two calls with seven arrays
    together, nothing enqueued: 15.7 us and 9.9; 1 MiB to a device arena and back, queued, 23.2 and 19.8, a short move 7.0 and 6.1.)"""
    if a is None:
        return None
    try:
        return _at(a)
    except TypeError:
        return a.ctypes.data


_I32, _U64 = np.dtype(np.int32), np.dtype(np.uint64)


def _i32a(a):
    if type(a) is np.ndarray and a.ndim and a.dtype == _I32 and a.flags.c_contiguous:
        return a
    return np.ascontiguousarray(np.asarray(a, dtype=np.int32))


def _u64a(a):
    if type(a) is np.ndarray and a.ndim and a.dtype == _U64 and a.flags.c_contiguous:
        return a
    return np.ascontiguousarray(np.asarray(a, dtype=np.uint64))


def _csr_ok(n, offsets, block_ids, *per_request):
    """The C side trusts the array lengths the CSR implies: check them here, where they are known."""
    if len(offsets) != n + 1 or any(len(a) != n for a in per_request):
        return False
    return n == 0 or int(offsets.max()) <= len(block_ids)


def _rows_ok(n, offsets, block_ids, *per_request):
    """_csr_ok for the calls that refuse offsets which go down before they read a block id: the last one is then the
    largest."""
    if len(offsets) != n + 1:
        return False
    for a in per_request:
        if len(a) != n:
            return False
    return n == 0 or (offsets[n] if offsets.ndim == 1 else offsets.max()) <= len(block_ids)


def kv_strerror(code):
    return _lib.kv_strerror(int(code)).decode()


def kv_pool_create(cfg):
    """cfg: kv_pool_config -> (rc, handle)"""
    cfg.struct_size = C.sizeof(kv_pool_config)
    h = _vp()
    rc = _lib.kv_pool_create(C.byref(cfg), C.byref(h))
    return rc, h


def kv_pool_destroy(h):
    return _lib.kv_pool_destroy(h)


def kv_swap_out(h, req_ids, offsets, block_ids, num_tokens, wait_event=None):
    r, o, b, t = _u64a(req_ids), _i32a(offsets), _i32a(block_ids), _i32a(num_tokens)
    if not _rows_ok(len(r), o, b, t):
        return KV_EINVAL
    return _lib.kv_swap_out(h, len(r), _p(r), _p(o), _p(b), _p(t), wait_event)


def kv_swap_out_delta(h, req_ids, offsets, block_ids, num_tokens, block_budget=0, flags=0, wait_event=None):
    """-> (rc, blocks_moved int32[n])"""
    r, o, b, t = _u64a(req_ids), _i32a(offsets), _i32a(block_ids), _i32a(num_tokens)
    moved = np.zeros(len(r), dtype=np.int32)
    if not _rows_ok(len(r), o, b, t):
        return KV_EINVAL, moved
    rc = _lib.kv_swap_out_delta(h, len(r), _p(r), _p(o), _p(b), _p(t), int(block_budget), int(flags),
                                _p(moved), wait_event)
    return rc, moved


def kv_swap_out_delta_timed(h, req_ids, offsets, block_ids, num_tokens, priority, interval_us, flags=0,
                            wait_event=None):
    """-> (rc, blocks_moved int32[n] in the caller's order, budget applied)"""
    r, o, b, t = _u64a(req_ids), _i32a(offsets), _i32a(block_ids), _i32a(num_tokens)
    pr = None if priority is None else np.ascontiguousarray(np.asarray(priority, dtype=np.float32))
    moved = np.zeros(len(r), dtype=np.int32)
    if not _csr_ok(len(r), o, b, t) or (pr is not None and len(pr) != len(r)):
        return KV_EINVAL, moved, 0
    used = _i64(0)
    rc = _lib.kv_swap_out_delta_timed(h, len(r), _p(r), _p(o), _p(b), _p(t), _p(pr), float(interval_us), int(flags),
                                      _p(moved), C.byref(used), wait_event)
    return rc, moved, used.value


def kv_wq_post(h, req_ids, offsets, block_ids, num_tokens, priority=None):
    r, o, b, t = _u64a(req_ids), _i32a(offsets), _i32a(block_ids), _i32a(num_tokens)
    pr = None if priority is None else np.ascontiguousarray(np.asarray(priority, dtype=np.float64))
    if not _csr_ok(len(r), o, b, t) or (pr is not None and len(pr) != len(r)):
        return KV_EINVAL
    return _lib.kv_wq_post(h, len(r), _p(r), _p(o), _p(b), _p(t), _p(pr))


def kv_wq_drain(h, interval_us=0.0, block_budget=0, flags=0, wait_event=None):
    """-> (rc, blocks written, full blocks still pending, budget applied)"""
    w, pend, used = _i64(0), _i64(0), _i64(0)
    rc = _lib.kv_wq_drain(h, float(interval_us), int(block_budget), int(flags), C.byref(w), C.byref(pend),
                          C.byref(used), wait_event)
    return rc, w.value, pend.value, used.value


def kv_wq_remove(h, req_id):
    return _lib.kv_wq_remove(h, int(req_id))


def kv_wq_pending(h):
    """-> (rc, full blocks not yet written through, requests that have some)"""
    nb, nr = _i64(0), _i32(0)
    rc = _lib.kv_wq_pending(h, C.byref(nb), C.byref(nr))
    return rc, nb.value, nr.value


def kv_swap_in(h, req_ids, offsets, new_block_ids, flags=0, wait_event=None):
    r, o, b = _u64a(req_ids), _i32a(offsets), _i32a(new_block_ids)
    if not _rows_ok(len(r), o, b):
        return KV_EINVAL
    return _lib.kv_swap_in(h, len(r), _p(r), _p(o), _p(b), int(flags), wait_event)


def kv_evict_and_load(h, out_ids, out_offsets, out_block_ids, out_tokens, in_ids, in_offsets, in_block_ids, in_flags=0,
                      wait_event=None):
    r, o, b, t = _u64a(out_ids), _i32a(out_offsets), _i32a(out_block_ids), _i32a(out_tokens)
    r2, o2, b2 = _u64a(in_ids), _i32a(in_offsets), _i32a(in_block_ids)
    if not _rows_ok(len(r), o, b, t) or not _rows_ok(len(r2), o2, b2):
        return KV_EINVAL
    return _lib.kv_evict_and_load(h, len(r), _p(r), _p(o), _p(b), _p(t), len(r2), _p(r2), _p(o2), _p(b2), int(in_flags),
                                  wait_event)


def kv_sync(h):
    return _lib.kv_sync(h)


def kv_move_blocks(h, src_ids, dst_ids, wait_event=None):
    s, d = _i32a(src_ids), _i32a(dst_ids)
    if len(s) != len(d):
        return KV_EINVAL
    return _lib.kv_move_blocks(h, len(s), _p(s), _p(d), wait_event)


def kv_move_blocks_noalloc(h, src_ids, dst_ids, wait_event=None):
    s, d = _i32a(src_ids), _i32a(dst_ids)
    if len(s) != len(d):
        return KV_EINVAL
    return _lib.kv_move_blocks_noalloc(h, len(s), _p(s), _p(d), wait_event)


def kv_req_reserve(h, req_id, max_blocks):
    return _lib.kv_req_reserve(h, int(req_id), int(max_blocks))


def kv_req_release(h, req_id):
    return _lib.kv_req_release(h, int(req_id))


def kv_req_query(h, req_id):
    """-> (rc, dict(offset, cap, staged, wm, swapped))"""
    off = _i64()
    cap, st, wm, sw = _i32(), _i32(), _i32(), _i32()
    rc = _lib.kv_req_query(h, int(req_id), C.byref(off), C.byref(cap), C.byref(st), C.byref(wm), C.byref(sw))
    return rc, dict(offset=off.value, cap=cap.value, staged=st.value, wm=wm.value, swapped=sw.value)


def kv_last_stats(h):
    st = kv_stats()
    st.struct_size = C.sizeof(kv_stats)
    rc = _lib.kv_last_stats(h, C.byref(st))
    return rc, st.as_dict()


def kv_slot_bytes(h):
    return _lib.kv_slot_bytes(h)


def kv_last_plan(h):
    """-> (phys int32[n], slot int64[n]) of the most recent swap call"""
    n = _lib.kv_last_plan(h, None, None, 0)
    phys, slot = np.zeros(n, np.int32), np.zeros(n, np.int64)
    if n:
        _lib.kv_last_plan(h, _p(phys), _p(slot), n)
    return phys, slot


def kv_req_poll(h, req_id):
    return _lib.kv_req_poll(h, int(req_id))


def kv_req_wait(h, req_id):
    return _lib.kv_req_wait(h, int(req_id))


def kv_last_timeline(h):
    """-> (req_ids uint64[n], done_ms float32[n]) of the most recent swap call"""
    n = _lib.kv_last_timeline(h, None, None, 0)
    if n < 0:
        raise KVSwapError(n, "kv_last_timeline")
    ids, ms = np.zeros(n, np.uint64), np.zeros(n, np.float32)
    if n:
        _lib.kv_last_timeline(h, _p(ids), _p(ms), n)
    return ids, ms


def kv_io_stats_get(h):
    """-> (rc, dict of 2-element lists: index 0 evict stream, 1 load stream)"""
    st = kv_io_stats()
    rc = _lib.kv_io_stats_get(h, C.byref(st))
    return rc, st.as_dict()


def kv_budget_blocks(h, direction, interval_us):
    return _lib.kv_budget_blocks(h, int(direction), float(interval_us))


def kv_pool_tune(h, what, value):
    return _lib.kv_pool_tune(h, int(what), int(value))


def kv_last_hip_error(h):
    return _lib.kv_last_hip_error(h)


def kv_bench_copy(dst_ptr, src_ptr, nbytes, grid, iters, stream=None):
    return _lib.kv_bench_copy(dst_ptr, src_ptr, int(nbytes), int(grid), int(iters), stream)


def kv_bench_copy_scrambled(dst_ptr, src_ptr, nbytes, chunk_bytes, which, iters, stream=None):
    return _lib.kv_bench_copy_scrambled(dst_ptr, src_ptr, int(nbytes), int(chunk_bytes), int(which), int(iters), stream)


def kv_bench_link(host_ptr, dev_ptr, nbytes, direction, iters, stream=None):
    return _lib.kv_bench_link(host_ptr, dev_ptr, int(nbytes), int(direction), int(iters), stream)


def kv_bench_link_bidir(host_a, dev_a, host_b, dev_b, nbytes, iters):
    return _lib.kv_bench_link_bidir(host_a, dev_a, host_b, dev_b, int(nbytes), int(iters))


class KVSwapError(RuntimeError):
    def __init__(self, code, what):
        super().__init__("%s: %s (%d)" % (what, kv_strerror(code), code))
        self.code = code


class KVPool:
    """A handle plus references to the memory it points into.

    pool / scale / bounce are torch uint8 device tensors, staging a pinned uint8
    host tensor (or a device tensor with KV_STAGING_DEVICE); under KV_PLAN_ONLY
    all of them may be None.  Strides default to the layer-major layout.
    """

    def __init__(self, geom, pool=None, staging=None, scale=None, bounce=None, strides=None, scale_strides=None,
                 flags=0, evict_stream=None, load_stream=None, staging_bytes=None, dtype_code=None):
        from .workloads import DTYPE_CODE
        self.geom = geom
        self._keep = (pool, staging, scale, bounce, evict_stream, load_stream)
        cfg = kv_pool_config()
        cfg.num_layers, cfg.num_kv_heads, cfg.head_dim, cfg.block_size = geom.L, geom.H, geom.D, geom.B
        cfg.dtype = DTYPE_CODE[geom.dtype] if dtype_code is None else dtype_code
        cfg.num_blocks = geom.N
        cfg.pool_dev = pool.data_ptr() if pool is not None else None
        cfg.layer_stride, cfg.kv_stride, cfg.block_stride = strides or geom.strides
        if geom.scales:
            cfg.scale_dev = scale.data_ptr() if scale is not None else None
            cfg.scale_layer_stride, cfg.scale_kv_stride, cfg.scale_block_stride = scale_strides or geom.scale_strides
        cfg.staging_host = staging.data_ptr() if staging is not None else None
        cfg.staging_bytes = staging.numel() if staging is not None else int(staging_bytes or 0)
        cfg.bounce_dev = bounce.data_ptr() if bounce is not None else None
        cfg.bounce_bytes = bounce.numel() if bounce is not None else 0
        cfg.evict_stream = evict_stream.cuda_stream if evict_stream is not None else None
        cfg.load_stream = load_stream.cuda_stream if load_stream is not None else None
        cfg.flags = flags
        rc, self.h = kv_pool_create(cfg)
        if rc:
            self.h = None
            raise KVSwapError(rc, "kv_pool_create")
        self.slot_bytes = kv_slot_bytes(self.h)

    def close(self):
        if getattr(self, "h", None):
            rc = kv_pool_destroy(self.h)
            self.h = None
            return rc
        return KV_OK

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def __enter__(self):
        return self

    def __exit__(self, *exc):
        self.close()
        return False

    # thin pass-throughs returning the C status codes
    def swap_out(self, req_ids, offsets, block_ids, num_tokens, wait_event=None):
        return kv_swap_out(self.h, req_ids, offsets, block_ids, num_tokens, wait_event)

    def swap_out_delta(self, req_ids, offsets, block_ids, num_tokens, budget=0, flags=0, wait_event=None):
        return kv_swap_out_delta(self.h, req_ids, offsets, block_ids, num_tokens, budget, flags, wait_event)

    def swap_out_delta_timed(self, req_ids, offsets, block_ids, num_tokens, priority, interval_us, flags=0,
                             wait_event=None):
        return kv_swap_out_delta_timed(self.h, req_ids, offsets, block_ids, num_tokens, priority, interval_us, flags,
                                       wait_event)

    def wq_post(self, req_ids, offsets, block_ids, num_tokens, priority=None):
        return kv_wq_post(self.h, req_ids, offsets, block_ids, num_tokens, priority)

    def wq_drain(self, interval_us=0.0, block_budget=0, flags=0, wait_event=None):
        return kv_wq_drain(self.h, interval_us, block_budget, flags, wait_event)

    def wq_remove(self, req_id):
        return kv_wq_remove(self.h, req_id)

    def wq_pending(self):
        return kv_wq_pending(self.h)

    def swap_in(self, req_ids, offsets, new_block_ids, flags=0, wait_event=None):
        return kv_swap_in(self.h, req_ids, offsets, new_block_ids, flags, wait_event)

    def move_blocks(self, src_ids, dst_ids, wait_event=None):
        return kv_move_blocks(self.h, src_ids, dst_ids, wait_event)

    def move_blocks_noalloc(self, src_ids, dst_ids, wait_event=None):
        return kv_move_blocks_noalloc(self.h, src_ids, dst_ids, wait_event)

    def evict_and_load(self, out_ids, out_offsets, out_block_ids, out_tokens, in_ids, in_offsets, in_block_ids, in_flags=0,
                       wait_event=None):
        return kv_evict_and_load(self.h, out_ids, out_offsets, out_block_ids, out_tokens, in_ids, in_offsets,
                                 in_block_ids, in_flags, wait_event)

    def sync(self):
        return kv_sync(self.h)

    def reserve(self, req_id, max_blocks):
        return kv_req_reserve(self.h, req_id, max_blocks)

    def release(self, req_id):
        return kv_req_release(self.h, req_id)

    def query(self, req_id):
        return kv_req_query(self.h, req_id)

    def stats(self):
        rc, st = kv_last_stats(self.h)
        if rc:
            raise KVSwapError(rc, "kv_last_stats")
        return st

    def last_plan(self):
        return kv_last_plan(self.h)

    def req_poll(self, req_id):
        return kv_req_poll(self.h, req_id)

    def req_wait(self, req_id):
        return kv_req_wait(self.h, req_id)

    def timeline(self):
        return kv_last_timeline(self.h)

    def io_stats(self):
        rc, st = kv_io_stats_get(self.h)
        if rc:
            raise KVSwapError(rc, "kv_io_stats_get")
        return st

    def budget_blocks(self, direction, interval_us):
        return kv_budget_blocks(self.h, direction, interval_us)

    def tune(self, what, value):
        return kv_pool_tune(self.h, what, value)


# ------------------------------------------------------------------ operators on the pool's contents

def kv_batch_create(h):
    """-> (rc, batch handle)"""
    b = _vp()
    rc = _lib.kv_batch_create(h, C.byref(b))
    return rc, b


def kv_batch_destroy(b):
    return _lib.kv_batch_destroy(b)


def kv_batch_set(b, offsets, block_ids, num_tokens, q_lens, num_q_heads, stream=None):
    o, ids, t, q = _i32a(offsets), _i32a(block_ids), _i32a(num_tokens), _i32a(q_lens)
    if not _rows_ok(len(t), o, ids, q):
        return KV_EINVAL
    return _lib.kv_batch_set(b, len(t), _p(o), _p(ids), _p(t), _p(q), int(num_q_heads), stream)


def kv_batch_query(b):
    """-> (rc, dict)"""
    st = kv_batch_info()
    st.struct_size = C.sizeof(kv_batch_info)
    rc = _lib.kv_batch_query(b, C.byref(st))
    return rc, st.as_dict()


def kv_rope_freqs(rot, base=10000.0, kind=KV_ROPE_PLAIN, factor=1.0, trained=0.0, low=1.0, high=4.0):
    """-> (rc, turns int64[rot/2], magnitude)"""
    turns, magnitude = np.zeros(max(0, int(rot)) // 2, np.int64), C.c_float(0)
    rc = _lib.kv_rope_freqs(int(rot), float(base), int(kind), float(factor), float(trained), float(low), float(high),
                            turns.ctypes.data, C.byref(magnitude))
    return rc, turns, magnitude.value


def kv_append(b, args, stream=None):
    """args: kv_append_args"""
    args.struct_size = C.sizeof(kv_append_args)
    return _lib.kv_append(b, C.addressof(args), stream)


def kv_attn(b, args, stream=None):
    """args: kv_attn_args"""
    args.struct_size = C.sizeof(kv_attn_args)
    return _lib.kv_attn(b, C.addressof(args), stream)


def kv_evict(b, args, stream=None):
    """args: kv_evict_args"""
    args.struct_size = C.sizeof(kv_evict_args)
    return _lib.kv_evict(b, C.addressof(args), stream)


def kv_check(rc, what="kvswap"):
    """Raises KVSwapError unless rc is KV_OK."""
    if rc != KV_OK:
        raise KVSwapError(rc, what)


_IO = {torch.float16: KV_F16, torch.bfloat16: KV_BF16}
# The argument structures as one packing each, and checks that ask a tensor for as little as possible: the host's share of an append
# with all its tensors, launch excluded, 5.3 us so, 10.3 with the fields set one by one.
_APPEND, _ATTN, _EVICT = struct.Struct("@IiiiifPPPPqqqqqqqqPPPP"), struct.Struct("@IiifPPqqqqPqPqqq"), struct.Struct("@IiiiiiPPqqqqPqqqP")
assert [s.size for s in (_APPEND, _ATTN, _EVICT)] == [C.sizeof(s) for s in (kv_append_args, kv_attn_args, kv_evict_args)]


class KVBatch:
    """The requests of one step on a KVPool, and the operators on them: append, attn, evict.

    Tensors are torch tensors on the pool's GPU.  q, q_out, out are [T, num_q_heads, D] and k, v [T, H, D], of any strides with
    a contiguous last dimension; T counts the new tokens of all requests in order.  Calls are enqueued on `stream`
    (default: torch's current stream of the device) and return the C status codes; shapes, types and devices that the C side cannot
    see are checked here (KV_EINVAL).  A batch is used by one thread at a time.
    """

    def __init__(self, pool):
        self.pool = pool
        self.geom = pool.geom
        data = pool._keep[0]
        self.device = data.device if data is not None else None
        self._dev = data.get_device() if data is not None else -1
        self._describe(0, 0, 0, 0)
        self._args = C.create_string_buffer(max(s.size for s in (_APPEND, _ATTN, _EVICT)))
        self._at = C.addressof(self._args)
        rc, self.h = kv_batch_create(pool.h)
        if rc:
            self.h = None
            raise KVSwapError(rc, "kv_batch_create")

    def _describe(self, n, T, Hq, max_len):
        self.n, self.T, self.Hq, self.max_len = n, T, Hq, max_len
        self._q_shape, self._kv_shape = (T, Hq, self.geom.D), (T, self.geom.H, self.geom.D)

    def close(self):
        if getattr(self, "h", None):
            rc = kv_batch_destroy(self.h)
            self.h = None
            return rc
        return KV_OK

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def __enter__(self):
        return self

    def __exit__(self, *exc):
        self.close()
        return False

    def _stream(self, stream):
        if stream is not None:
            return stream.cuda_stream
        return torch._C._cuda_getCurrentRawStream(self.device.index) if self.device is not None else None

    def _fits(self, x, dtype, shape):
        """Type, device and shape, and a contiguous last dimension."""
        return x.dtype is dtype and x.shape == shape and x.get_device() == self._dev and (shape[-1] <= 1 or x.stride(-1) == 1)

    def set(self, offsets, block_ids, num_tokens, q_lens, num_q_heads, stream=None):
        if not self.h or not self.pool.h:
            return KV_EINVAL
        t, q = _i32a(num_tokens), _i32a(q_lens)
        rc = kv_batch_set(self.h, offsets, block_ids, t, q, num_q_heads, self._stream(stream))
        if rc in (KV_ENOMEM, KV_EHIP):
            self._describe(0, 0, 0, 0)
        if rc == KV_OK:
            self._describe(len(t), int(q.sum()), int(num_q_heads), int(t.max()) if len(t) else 0)
        return rc

    def query(self):
        rc, st = kv_batch_query(self.h)
        if rc:
            raise KVSwapError(rc, "kv_batch_query")
        return st

    def append(self, layer, q, k, v, q_out=None, turns=None, interleaved=False, magnitude=1.0, positions=None, k_scale=None, v_scale=None, stream=None):
        """q may be None; q_out defaults to q itself.  turns: int64 [rot/2] on the device (None: nothing is turned), positions: int32 [T]."""
        dtype, dev, shape, ks, vs = k.dtype, self._dev, self._kv_shape, k.stride(), v.stride()
        io = _IO.get(dtype)
        if not (self.h and self.pool.h and io is not None and k.shape == shape and v.shape == shape and v.dtype is dtype and
                ks[2] == 1 and vs[2] == 1 and k.get_device() == dev and v.get_device() == dev):
            return KV_EINVAL
        qp, op, qs, qo, rot, tp, pp, kp, vp = 0, 0, (0, 0), (0, 0), 0, 0, 0, 0, 0
        if q is not None:
            q_out = q if q_out is None else q_out
            shape, qs, qo = self._q_shape, q.stride(), q_out.stride()
            if not (q.shape == shape and q_out.shape == shape and q.dtype is dtype and q_out.dtype is dtype and qs[2] == 1 and qo[2] == 1 and
                    q.get_device() == dev and q_out.get_device() == dev):
                return KV_EINVAL
            qp, op = q.data_ptr(), q_out.data_ptr()
        if turns is not None:
            rot, tp = 2 * turns.numel(), turns.data_ptr()
            if turns.dtype is not torch.int64 or turns.get_device() != dev or not turns.is_contiguous():
                return KV_EINVAL
        if positions is not None:
            pp = positions.data_ptr()
            if positions.dtype is not torch.int32 or positions.shape != (self.T,) or positions.get_device() != dev or not positions.is_contiguous():
                return KV_EINVAL
        if k_scale is not None:
            kp = k_scale.data_ptr()
            if not self._fits(k_scale, torch.float32, (self.geom.H,)):
                return KV_EINVAL
        if v_scale is not None:
            vp = v_scale.data_ptr()
            if not self._fits(v_scale, torch.float32, (self.geom.H,)):
                return KV_EINVAL
        _APPEND.pack_into(self._args, 0, _APPEND.size, layer, io, rot, 1 if interleaved else 0, magnitude, qp, k.data_ptr(), v.data_ptr(), op,
                          qs[0], qs[1], ks[0], ks[1], vs[0], vs[1], qo[0], qo[1], tp, pp, kp, vp)
        return _lib.kv_append(self.h, self._at, self._stream(stream))

    def attn(self, layer, q, out, scale, lse=None, weights=None, stream=None):
        """lse: float32 [T, num_q_heads]; weights: float32 [n, H, cap] with cap no less than the longest request's tokens."""
        dtype, dev, shape, qs, os_ = q.dtype, self._dev, self._q_shape, q.stride(), out.stride()
        io = _IO.get(dtype)
        if not (self.h and self.pool.h and io is not None and q.shape == shape and out.shape == shape and out.dtype is dtype and
                qs[2] == 1 and os_[2] == 1 and q.get_device() == dev and out.get_device() == dev):
            return KV_EINVAL
        lp, ls, wp, ws, cap = 0, 0, 0, (0, 0), 0
        if lse is not None:
            if not self._fits(lse, torch.float32, (self.T, self.Hq)):
                return KV_EINVAL
            lp, ls = lse.data_ptr(), lse.stride(0)
        if weights is not None:
            if weights.dim() != 3 or not self._fits(weights, torch.float32, (self.n, self.geom.H, weights.shape[2])):
                return KV_EINVAL
            wp, ws, cap = weights.data_ptr(), weights.stride(), weights.shape[2]
        _ATTN.pack_into(self._args, 0, _ATTN.size, layer, io, scale, q.data_ptr(), out.data_ptr(), qs[0], qs[1], os_[0], os_[1], lp, ls, wp,
                        ws[0], ws[1], cap)
        return _lib.kv_attn(self.h, self._at, self._stream(stream))

    def evict(self, layer, num_layers, weights, kept, keep, keep_first=0, keep_last=0, weights_out=None, req_ids=None, stream=None):
        """weights, weights_out (default: weights itself): float32 [num_layers, n, H, cap] of the same strides; kept: int32
        [num_layers, n, H, keep or more]; req_ids: host uint64 [n].  In a pool with scales that differ from block to block keep has to be a
        multiple of the block size, so that the next append begins a block."""
        if not self.h or not self.pool.h or weights.dim() != 4 or kept.dim() != 4 or kept.shape[3] < min(keep, self.max_len):
            return KV_EINVAL
        lead, ws, ks, out, ids = (num_layers, self.n, self.geom.H), weights.stride(), kept.stride(), 0, 0
        if not self._fits(weights, torch.float32, lead + (weights.shape[3],)) or not self._fits(kept, torch.int32, lead + (kept.shape[3],)):
            return KV_EINVAL
        if weights_out is not None:
            if not self._fits(weights_out, torch.float32, weights.shape) or weights_out.stride() != ws:
                return KV_EINVAL
            out = weights_out.data_ptr()
        if req_ids is not None:
            req_ids = _u64a(req_ids)
            if len(req_ids) != self.n:
                return KV_EINVAL
            ids = req_ids.ctypes.data
        _EVICT.pack_into(self._args, 0, _EVICT.size, layer, num_layers, keep, keep_first, keep_last, weights.data_ptr(), out,
                         ws[0], ws[1], ws[2], weights.shape[3], kept.data_ptr(), ks[0], ks[1], ks[2], ids)
        return _lib.kv_evict(self.h, self._at, self._stream(stream))
