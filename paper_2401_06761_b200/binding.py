"""ctypes binding of libapar.so: the same names and arguments as include/apar.h.

Argument marshalling only.  Device buffers are passed as integer addresses (for example
`tensor.data_ptr()`), host arrays as sequences of ints.  There is no fallback: if the
library has not been built, importing this module raises.
"""
from __future__ import annotations

import ctypes as C
import functools
import os
import struct

import numpy as np

_LIB_PATH = os.path.join(os.path.dirname(os.path.abspath(__file__)), "libapar.so")
if not os.path.exists(_LIB_PATH):
    raise ImportError(f"{_LIB_PATH} is missing: run `python -m paper_2401_06761_b200.build`")
lib = C.CDLL(_LIB_PATH)

APAR_OK = 0
APAR_ERR_INVALID_ARG = -1
STATUS = {0: "OK", -1: "INVALID_ARG", -2: "BAD_THREAD", -3: "NO_BLOCKS", -4: "NO_THREADS",
          -5: "TABLE_FULL", -6: "EMPTY_CONTEXT", -7: "WORKSPACE_TOO_SMALL", -8: "CUDA",
          -9: "UNSUPPORTED"}


class AparError(RuntimeError):
    def __init__(self, status: int):
        self.status = status
        self.code = STATUS.get(status, "UNKNOWN")
        super().__init__(lib.apar_status_string(status).decode())


class apar_config(C.Structure):
    _fields_ = [("num_blocks", C.c_int32), ("block_size", C.c_int32),
                ("num_q_heads", C.c_int32), ("num_kv_heads", C.c_int32),
                ("head_dim", C.c_int32), ("max_threads", C.c_int32),
                ("max_blocks_per_thread", C.c_int32), ("num_layers", C.c_int32),
                ("k_pool", C.c_void_p), ("v_pool", C.c_void_p),
                ("workspace", C.c_void_p), ("workspace_bytes", C.c_size_t)]


class apar_rope_config(C.Structure):
    _fields_ = [("head_dim", C.c_int32), ("rotary_dim", C.c_int32), ("layout", C.c_int32),
                ("scaling", C.c_int32), ("original_len", C.c_int32), ("reserved", C.c_int32),
                ("base", C.c_double), ("factor", C.c_double), ("low", C.c_double),
                ("high", C.c_double), ("attn_scale", C.c_double)]


KV_FORMATS = {"bf16": 0, "q4": 1}
ROPE_LAYOUTS = {"half": 0, "interleaved": 1}
ROPE_SCALINGS = {"none": 0, "linear": 1, "bands": 2, "yarn": 3}


class apar_stats(C.Structure):
    _fields_ = [(n, C.c_int64) for n in (
        "live_threads", "free_blocks", "used_blocks", "forks", "cow_blocks", "cow_rows",
        "attn_threads", "attn_attended_tokens", "attn_unique_tokens", "attn_work_items",
        "attn_partials", "attn_kernels", "attn_plan_reused", "attn_vec_items",
        "attn_mma_items", "kernels_total", "peak_used_blocks", "device_wait_timeouts",
        "attn_plan_host_us", "attn_upload_bytes")]

    def as_dict(self):
        return {n: getattr(self, n) for n, _ in self._fields_}


_i32p = C.POINTER(C.c_int32)
_ctx = C.c_void_p
_cfgp = C.POINTER(apar_config)

_SIGS = {
    "apar_workspace_bytes": (C.c_size_t, [_cfgp]),
    "apar_create": (C.c_int32, [_cfgp, C.POINTER(_ctx)]),
    "apar_create_host_only": (C.c_int32, [_cfgp, C.POINTER(_ctx)]),
    "apar_create_kv": (C.c_int32, [_cfgp, C.c_int32, C.POINTER(_ctx)]),
    "apar_kv_pool_bytes": (C.c_size_t, [_cfgp, C.c_int32]),
    "apar_read_kv": (C.c_int32, [_ctx, C.c_int32, C.c_int32, _i32p, _i32p, _i32p, C.c_void_p,
                                 C.c_void_p, C.c_void_p]),
    "apar_rope": (C.c_int32, [C.POINTER(apar_rope_config), C.c_int32, C.c_void_p, C.c_int32,
                              C.c_void_p, C.c_int64, C.c_void_p, C.c_int64, C.c_int32, C.c_void_p,
                              C.c_int64, C.c_void_p, C.c_int64, C.c_void_p]),
    "apar_destroy": (C.c_int32, [_ctx]),
    "apar_new_threads": (C.c_int32, [_ctx, C.c_int32, _i32p]),
    "apar_fork": (C.c_int32, [_ctx, C.c_int32, _i32p, _i32p, C.c_void_p]),
    "apar_append_kv": (C.c_int32, [_ctx, C.c_int32, _i32p, _i32p, C.c_void_p, C.c_void_p,
                                   C.c_void_p]),
    "apar_tree_decode_attention": (C.c_int32, [_ctx, C.c_int32, _i32p, C.c_void_p, C.c_void_p,
                                               C.c_float, C.c_void_p]),
    "apar_tree_prefix_attention": (C.c_int32, [_ctx, C.c_int32, _i32p, _i32p, C.c_void_p,
                                               C.c_void_p, C.c_float, C.c_void_p]),
    "apar_tree_verify_attention": (C.c_int32, [_ctx, C.c_int32, _i32p, _i32p,
                                               C.POINTER(C.c_uint64), C.c_void_p, C.c_void_p,
                                               C.c_float, C.c_void_p]),
    "apar_accept_candidates": (C.c_int32, [_ctx, C.c_int32, _i32p, _i32p, _i32p, _i32p,
                                           C.c_void_p]),
    "apar_tree_prefill_attention": (C.c_int32, [_ctx, C.c_int32, C.c_int32, _i32p, _i32p, _i32p,
                                                C.c_void_p, C.c_void_p, C.c_float, C.c_void_p]),
    "apar_append_kv_layer": (C.c_int32, [_ctx, C.c_int32, C.c_void_p, C.c_void_p, C.c_void_p]),
    "apar_tree_decode_attention_layer": (C.c_int32, [_ctx, C.c_int32, C.c_void_p, C.c_void_p,
                                                     C.c_float, C.c_void_p]),
    "apar_decode_step": (C.c_int32, [_ctx, C.c_int32, _i32p, C.c_void_p, C.c_void_p, C.c_void_p,
                                     C.c_void_p, C.c_float, C.c_void_p]),
    "apar_steps_before_new_block": (C.c_int32, [_ctx, _i32p]),
    "apar_note_step_replay": (C.c_int32, [_ctx]),
    "apar_release": (C.c_int32, [_ctx, C.c_int32, _i32p]),
    "apar_tree_decode_attention_tables": (C.c_int32, [_cfgp, C.c_int32, _i32p, _i32p,
                                                      C.c_void_p, C.c_void_p, C.c_float,
                                                      C.c_void_p]),
    "apar_tree_decode_attention_static": (C.c_int32, [C.c_void_p, C.c_void_p, C.c_int32, C.c_int32,
                                                      C.c_int32, C.c_int32, C.c_void_p, C.c_void_p,
                                                      C.c_int32, C.c_void_p, C.c_void_p, C.c_float,
                                                      C.c_void_p]),
    "apar_paragraph_root": (C.c_int32, [_ctx, C.c_int32]),
    "apar_restore": (C.c_int32, [_ctx, C.c_int32, _i32p, C.c_int32, _i32p]),
    "apar_get_thread": (C.c_int32, [_ctx, C.c_int32, _i32p, _i32p, _i32p, C.c_int32]),
    "apar_get_refcounts": (C.c_int32, [_ctx, _i32p]),
    "apar_get_free_list": (C.c_int32, [_ctx, _i32p, C.c_int32, _i32p]),
    "apar_get_stats": (C.c_int32, [_ctx, C.POINTER(apar_stats)]),
    "apar_check_invariants": (C.c_int32, [_ctx]),
    "apar_debug_plan": (C.c_int32, [C.c_int32, C.c_int32, C.c_int32, C.c_int32, C.c_int32, _i32p,
                                    _i32p, C.c_int32, C.c_int32, _i32p, C.c_int32, _i32p,
                                    C.c_int32, _i32p, C.c_int32, C.POINTER(C.c_int64)]),
    "apar_debug_plan_threads": (C.c_int32, [_ctx, C.c_int32, _i32p, C.c_int32, C.c_int32,
                                            C.c_int32, _i32p, C.c_int32, _i32p, C.c_int32, _i32p,
                                            C.c_int32, C.POINTER(C.c_int64)]),
    "apar_stream_read": (C.c_int32, [C.c_void_p, C.c_size_t, C.c_void_p, C.c_void_p]),
    "apar_set_timing_events": (C.c_int32, [_ctx, C.c_void_p, C.c_void_p]),
    "apar_last_cuda_error": (C.c_int32, [_ctx]),
    "apar_status_string": (C.c_char_p, [C.c_int32]),
}
for _name, (_res, _args) in _SIGS.items():
    _f = getattr(lib, _name)
    _f.restype, _f.argtypes = _res, _args

EXPORTS = tuple(_SIGS)


@functools.lru_cache(256)
def _packer(n):
    return struct.Struct(f"{n}i")


def _arr(xs):
    if isinstance(xs, tuple) and len(xs) == 2 and isinstance(xs[0], C.Array):
        return xs          # already marshalled by int32_array()
    if not isinstance(xs, np.ndarray):
        xs = xs if isinstance(xs, (list, tuple)) else list(xs)
        n = len(xs)
        try:                           # (several times as fast as numpy for short lists)
            raw = _packer(max(n, 1)).pack(*(xs or (0,)))
        except (struct.error, TypeError):   # not plain 32-bit ints: numpy's conversions and errors
            raw = np.fromiter(xs, dtype=np.int32).tobytes()
        return (C.c_int32 * max(n, 1)).from_buffer_copy(raw), n
    a = np.ascontiguousarray(xs.astype(np.int32, copy=False))
    buf = (C.c_int32 * max(a.size, 1)).from_buffer_copy(a.tobytes() if a.size else b"\0" * 4)
    return buf, int(a.size)


def _arr_for(n, xs):
    """The array of a list that has an entry for each of n threads (the library reads that many)."""
    buf, m = _arr(xs)
    if m < n:
        raise AparError(APAR_ERR_INVALID_ARG)
    return buf


def _check(status: int):
    if status != APAR_OK:
        raise AparError(status)


def make_config(num_blocks, num_q_heads, num_kv_heads, max_threads, max_blocks_per_thread,
                k_pool=0, v_pool=0, workspace=0, workspace_bytes=0, block_size=16, head_dim=128,
                num_layers=1):
    return apar_config(num_blocks, block_size, num_q_heads, num_kv_heads, head_dim, max_threads,
                       max_blocks_per_thread, num_layers, k_pool, v_pool, workspace,
                       workspace_bytes)


def apar_workspace_bytes(cfg: apar_config) -> int:
    return lib.apar_workspace_bytes(C.byref(cfg))


def apar_create(cfg: apar_config):
    ctx = _ctx()
    _check(lib.apar_create(C.byref(cfg), C.byref(ctx)))
    return ctx


def apar_create_host_only(cfg: apar_config):
    ctx = _ctx()
    _check(lib.apar_create_host_only(C.byref(cfg), C.byref(ctx)))
    return ctx


def apar_create_kv(cfg: apar_config, kv_format: int):
    """kv_format: a value of KV_FORMATS."""
    ctx = _ctx()
    _check(lib.apar_create_kv(C.byref(cfg), kv_format, C.byref(ctx)))
    return ctx


def apar_kv_pool_bytes(cfg: apar_config, kv_format: int) -> int:
    return lib.apar_kv_pool_bytes(C.byref(cfg), kv_format)


def apar_destroy(ctx):
    _check(lib.apar_destroy(ctx))


def apar_new_threads(ctx, n: int):
    out = (C.c_int32 * max(n, 1))()
    _check(lib.apar_new_threads(ctx, n, out))
    return list(out[:n])


def apar_fork(ctx, parent_tid, stream=0):
    parents, n = _arr(parent_tid)
    out = (C.c_int32 * max(n, 1))()
    _check(lib.apar_fork(ctx, n, parents, out, stream))
    return list(out[:n])


def apar_append_kv(ctx, tid, n_tok, k_new: int, v_new: int, stream=0):
    tids, n = _arr(tid)
    counts = _arr_for(n, n_tok) if n_tok is not None else None
    _check(lib.apar_append_kv(ctx, n, tids, counts, k_new, v_new, stream))


def apar_tree_decode_attention(ctx, tid, q: int, out: int, sm_scale: float, stream=0):
    tids, n = _arr(tid)
    _check(lib.apar_tree_decode_attention(ctx, n, tids, q, out, sm_scale, stream))


def apar_tree_prefix_attention(ctx, tid, attend_len, q: int, out: int, sm_scale: float, stream=0):
    tids, n = _arr(tid)
    lens = _arr_for(n, attend_len)
    _check(lib.apar_tree_prefix_attention(ctx, n, tids, lens, q, out, sm_scale, stream))


def apar_tree_verify_attention(ctx, tid, n_cand, anc_mask, q: int, out: int, sm_scale: float,
                               stream=0):
    """anc_mask: a sequence of ints (uint64 bit masks), one per candidate, all threads' in order."""
    tids, n = _arr(tid)
    cands = _arr_for(n, n_cand)
    if len(anc_mask) < sum(cands[:n]):
        raise AparError(APAR_ERR_INVALID_ARG)
    m = max(len(anc_mask), 1)
    try:
        masks = (C.c_uint64 * m).from_buffer_copy(struct.pack(f"{m}Q", *(anc_mask if len(anc_mask) else (0,))))
    except struct.error:               # (a negative int stands for its 64 low bits)
        masks = (C.c_uint64 * m)(*anc_mask)
    _check(lib.apar_tree_verify_attention(ctx, n, tids, cands, masks, q, out, sm_scale, stream))


def apar_accept_candidates(ctx, tid, n_cand, keep, stream=0):
    """keep: per thread, the list of candidate indices that stay (increasing)."""
    tids, n = _arr(tid)
    cands = _arr_for(n, n_cand)
    counts = _arr_for(n, [len(k) for k in keep])
    flat, _ = _arr([x for k in keep for x in k])
    _check(lib.apar_accept_candidates(ctx, n, tids, cands, counts, flat, stream))


def apar_tree_prefill_attention(ctx, layer: int, tid, q_begin, q_count, q: int, out: int,
                                sm_scale: float, stream=0):
    tids, n = _arr(tid)
    begins, counts = _arr_for(n, q_begin), _arr_for(n, q_count)
    _check(lib.apar_tree_prefill_attention(ctx, layer, n, tids, begins, counts, q, out, sm_scale,
                                           stream))


def apar_append_kv_layer(ctx, layer: int, k_new: int, v_new: int, stream=0):
    _check(lib.apar_append_kv_layer(ctx, layer, k_new, v_new, stream))


def apar_tree_decode_attention_layer(ctx, layer: int, q: int, out: int, sm_scale: float, stream=0):
    _check(lib.apar_tree_decode_attention_layer(ctx, layer, q, out, sm_scale, stream))


def apar_decode_step(ctx, tid, k_new: int, v_new: int, q: int, out: int, sm_scale: float,
                     stream=0):
    tids, n = _arr(tid)
    _check(lib.apar_decode_step(ctx, n, tids, k_new, v_new, q, out, sm_scale, stream))


def apar_steps_before_new_block(ctx) -> int:
    steps = C.c_int32()
    _check(lib.apar_steps_before_new_block(ctx, C.byref(steps)))
    return steps.value


def apar_note_step_replay(ctx):
    _check(lib.apar_note_step_replay(ctx))


def apar_read_kv(ctx, layer: int, tid, begin, count, k_out: int, v_out: int, stream=0):
    tids, n = _arr(tid)
    begins, n_begin = _arr(begin)
    counts, n_count = _arr(count)
    if n_begin != n or n_count != n:   # (the library takes n entries of each)
        raise AparError(APAR_ERR_INVALID_ARG)
    _check(lib.apar_read_kv(ctx, layer, n, tids, begins, counts, k_out, v_out, stream))


def make_rope_config(rotary_dim=128, layout="half", base=10000.0, scaling="none", factor=1.0,
                     original_len=0, low=1.0, high=4.0, attn_scale=1.0, head_dim=128):
    return apar_rope_config(head_dim, rotary_dim, ROPE_LAYOUTS[layout], ROPE_SCALINGS[scaling],
                            original_len, 0, base, factor, low, high, attn_scale)


def apar_rope(cfg: apar_rope_config, n: int, positions: int, num_q_heads: int, q: int,
              q_stride: int, q_out: int, q_out_stride: int, num_kv_heads: int, k: int,
              k_stride: int, k_out: int, k_out_stride: int, stream=0):
    _check(lib.apar_rope(C.byref(cfg), n, positions, num_q_heads, q, q_stride, q_out, q_out_stride,
                         num_kv_heads, k, k_stride, k_out, k_out_stride, stream))


def apar_release(ctx, tid):
    tids, n = _arr(tid)
    _check(lib.apar_release(ctx, n, tids))


def apar_tree_decode_attention_tables(cfg, block_tables, ctx_lens, q: int, out: int,
                                      sm_scale: float, stream=0):
    """block_tables: n rows, each padded by the caller to cfg.max_blocks_per_thread ints."""
    lens, n = _arr(ctx_lens)
    flat = _arr_for(n * cfg.max_blocks_per_thread, [x for row in block_tables for x in row])
    _check(lib.apar_tree_decode_attention_tables(C.byref(cfg), n, flat, lens, q, out,
                                                 sm_scale, stream))


def apar_tree_decode_attention_static(k_pool: int, v_pool: int, num_q_heads: int,
                                      num_kv_heads: int, n_threads: int,
                                      max_blocks_per_thread: int, block_tables: int,
                                      ctx_lens: int, max_ctx_len: int, q: int, out: int,
                                      sm_scale: float, stream=0):
    """Allocation-free variant: block_tables and ctx_lens are DEVICE addresses here."""
    _check(lib.apar_tree_decode_attention_static(k_pool, v_pool, num_q_heads, num_kv_heads,
                                                 n_threads, max_blocks_per_thread, block_tables,
                                                 ctx_lens, max_ctx_len, q, out, sm_scale, stream))


def apar_paragraph_root(ctx, tid: int):
    _check(lib.apar_paragraph_root(ctx, tid))


def apar_restore(ctx, root_tid: int):
    """Slices (tid, start, end) of the response in reading order."""
    n = C.c_int32()
    _check(lib.apar_restore(ctx, root_tid, None, 0, C.byref(n)))
    buf = (C.c_int32 * max(3 * n.value, 1))()
    _check(lib.apar_restore(ctx, root_tid, buf, n.value, C.byref(n)))
    return [tuple(buf[3 * i:3 * i + 3]) for i in range(n.value)]


def apar_get_thread(ctx, tid: int, cap: int = 0):
    """Returns (len, blocks)."""
    ln, nb = C.c_int32(), C.c_int32()
    _check(lib.apar_get_thread(ctx, tid, C.byref(ln), C.byref(nb), None, 0))
    blocks = (C.c_int32 * max(nb.value, 1))()
    _check(lib.apar_get_thread(ctx, tid, None, None, blocks, nb.value))
    return ln.value, list(blocks[:nb.value])


def apar_get_refcounts(ctx, num_blocks: int):
    out = (C.c_int32 * num_blocks)()
    _check(lib.apar_get_refcounts(ctx, out))
    return list(out)


def apar_get_free_list(ctx, num_blocks: int):
    out = (C.c_int32 * max(num_blocks, 1))()
    n = C.c_int32()
    _check(lib.apar_get_free_list(ctx, out, num_blocks, C.byref(n)))
    return list(out[:min(n.value, num_blocks)])


def apar_get_stats(ctx) -> dict:
    s = apar_stats()
    _check(lib.apar_get_stats(ctx, C.byref(s)))
    return s.as_dict()


def apar_check_invariants(ctx):
    _check(lib.apar_check_invariants(ctx))


def apar_debug_plan(num_blocks, num_q_heads, num_kv_heads, tables, lens, mma_min_rows=2,
                    fuse_final=True):
    """Host-only planning of one attention call; `tables` is an [n][max_blocks] int32 array.
    Returns (items [k][8], users [m][2], merges [j][3], counts dict) as numpy arrays."""
    tables = np.ascontiguousarray(tables, dtype=np.int32)
    lens = np.ascontiguousarray(lens, dtype=np.int32)
    n, mb = tables.shape
    cap_users = int(sum((int(l) + 15) // 16 for l in lens)) + 1
    cap_items = 4 * cap_users + 16
    items = np.zeros((cap_items, 8), dtype=np.int32)
    users = np.zeros((cap_users, 2), dtype=np.int32)
    merges = np.zeros((n + 1, 3), dtype=np.int32)
    counts = (C.c_int64 * 6)()
    p = lambda a: a.ctypes.data_as(_i32p)
    _check(lib.apar_debug_plan(num_blocks, num_q_heads, num_kv_heads, n, mb, p(tables), p(lens),
                               mma_min_rows, int(bool(fuse_final)), p(items), cap_items,
                               p(users), cap_users, p(merges), n + 1, counts))
    names = ("items", "users", "merges", "partial_slots", "unique_tokens", "attended_tokens")
    c = dict(zip(names, (int(x) for x in counts)))
    return items[:c["items"]], users[:c["users"]], merges[:c["merges"]], c


def apar_debug_plan_threads(ctx, tid, by_groups: bool, mma_min_rows=2, fuse_final=True):
    """Host-only planning for threads of a context; same return value as apar_debug_plan."""
    tids, n = _arr(tid)
    lens = [apar_get_thread(ctx, t)[0] for t in tid]
    cap_users = int(sum((int(l) + 15) // 16 for l in lens)) + 1
    cap_items = 4 * cap_users + 16
    items = np.zeros((cap_items, 8), dtype=np.int32)
    users = np.zeros((cap_users, 2), dtype=np.int32)
    merges = np.zeros((n + 1, 3), dtype=np.int32)
    counts = (C.c_int64 * 6)()
    p = lambda a: a.ctypes.data_as(_i32p)
    _check(lib.apar_debug_plan_threads(ctx, n, tids, int(bool(by_groups)), mma_min_rows,
                                       int(bool(fuse_final)), p(items), cap_items, p(users),
                                       cap_users, p(merges), n + 1, counts))
    names = ("items", "users", "merges", "partial_slots", "unique_tokens", "attended_tokens")
    c = dict(zip(names, (int(x) for x in counts)))
    return items[:c["items"]], users[:c["users"]], merges[:c["merges"]], c


def apar_stream_read(src: int, nbytes: int, sink: int, stream=0):
    _check(lib.apar_stream_read(src, nbytes, sink, stream))


def apar_set_timing_events(ctx, start: int, stop: int):
    """cudaEvent_t handles (integers), or 0, 0 to turn the recording off."""
    _check(lib.apar_set_timing_events(ctx, start or None, stop or None))


def apar_last_cuda_error(ctx) -> int:
    return lib.apar_last_cuda_error(ctx)


def int32_array(xs):
    """Pre-marshalled id list for repeated calls of apar_tree_decode_attention."""
    return _arr(xs)
