"""A pool plus a library context: device memory from PyTorch, every operation through the
C-ABI binding.  Used by the tests, the benchmark and the smoke entry."""
from __future__ import annotations

import math

import numpy as np
import torch

from . import binding as B
from .synth import ForestSpec, LayerShape


# torch.cuda.current_stream().cuda_stream without its 3 us of wrapping; not part of torch's public
# interface, so that its absence must not matter
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)


def pool_requirements(spec: ForestSpec, slack: float = 0.05):
    """(num_blocks, max_threads, max_blocks_per_thread) that hold `spec`."""
    bs = spec.shape.block_size
    blocks = sum(-(-n.n_tok // bs) + 1 for n in spec.nodes)
    longest = max(spec.attended_tokens(n) for n in spec.nodes)
    depth = max(n.depth for n in spec.nodes) + 1
    return (int(blocks * (1 + slack)) + 16, len(spec.nodes) + 8, -(-longest // bs) + depth + 1)


class Rope:
    """Rotary positions of a model: the parameters of apar_rope_config, applied by calling.

    q [n][heads][128] and k (or None) are bf16 and may be views with any stride between tokens
    (rows that overlap are refused; one row expanded to all tokens is copied out first, and refused
    in place); positions is int32 [n].  Returns rotated (q, k): new contiguous tensors, or the
    inputs themselves with inplace=True."""

    def __init__(self, **params):
        self.cfg = B.make_rope_config(**params)

    @staticmethod
    def _rows(x: torch.Tensor, inplace: bool) -> torch.Tensor:
        # (apar_rope takes a stride of 0 for contiguous rows)
        if x.shape[0] > 1 and x.stride(0) == 0:
            if inplace:
                raise ValueError("the tokens of an expanded tensor share one row: not in place")
            x = x.contiguous()
        return x

    def __call__(self, q: torch.Tensor, k: torch.Tensor, positions: torch.Tensor, inplace=False):
        n = q.shape[0]
        assert positions.dtype == torch.int32 and positions.is_contiguous() and positions.is_cuda
        assert positions.shape == (n,)
        here = torch.cuda.current_device()             # (the launch goes to its current stream)
        assert positions.get_device() == here
        outs, sides, held = [], [], []                 # (held: copies live until the launch)
        for x in (q, k):
            if x is None:
                outs.append(None)
                sides += [0, 0, 0, 0, 0]
                continue
            assert x.get_device() == here and x.dtype == torch.bfloat16
            assert x.dim() == 3 and x.shape[0] == n
            assert x.shape[2] == self.cfg.head_dim
            assert x.stride(2) == 1 and (x.shape[1] == 1 or x.stride(1) == x.shape[2])
            x = self._rows(x, inplace)
            held.append(x)
            out = x if inplace else torch.empty_like(x, memory_format=torch.contiguous_format)
            stride = x.stride(0) if n > 1 else 0       # (0: contiguous)
            outs.append(out)
            sides += [x.shape[1], x.data_ptr(), stride, out.data_ptr(), stride if inplace else 0]
        B.apar_rope(self.cfg, n, positions.data_ptr(), *sides, PagedSession._stream())
        return tuple(outs)


class PagedSession:
    def __init__(self, shape: LayerShape, num_blocks: int, max_threads: int,
                 max_blocks_per_thread: int, device="cuda", poison: bool = False,
                 num_layers: int = 1, kv_format: str = "bf16"):
        if not torch.cuda.is_available():
            raise RuntimeError("the APAR library needs a CUDA device; there is no CPU path")
        self.shape, self.device = shape, torch.device(device)
        self.num_blocks = num_blocks
        self.num_layers = num_layers
        self.kv_format = kv_format
        cfg = B.make_config(num_blocks, shape.num_q_heads, shape.num_kv_heads, max_threads,
                            max_blocks_per_thread, num_layers=num_layers)
        pool_shape = (num_layers * num_blocks, shape.num_kv_heads, shape.block_size,
                      shape.head_dim)
        if kv_format != "bf16":   # rows of a library-defined layout, as bytes
            nbytes = B.apar_kv_pool_bytes(cfg, B.KV_FORMATS[kv_format])
            # (0xFF: the scales of unwritten rows are NaN)
            fill = 0xFF if poison else 0
            self.k_pool = torch.full((nbytes,), fill, dtype=torch.uint8, device=device)
            self.v_pool = torch.full((nbytes,), fill, dtype=torch.uint8, device=device)
        elif poison:   # NaN bit patterns everywhere: any read of an unwritten row shows up
            self.k_pool = torch.full(pool_shape, float("nan"), dtype=torch.bfloat16, device=device)
            self.v_pool = torch.full(pool_shape, float("nan"), dtype=torch.bfloat16, device=device)
        else:
            self.k_pool = torch.zeros(pool_shape, dtype=torch.bfloat16, device=device)
            self.v_pool = torch.zeros(pool_shape, dtype=torch.bfloat16, device=device)
        ws_bytes = B.apar_workspace_bytes(cfg)
        self.workspace = torch.empty(ws_bytes, dtype=torch.uint8, device=device)
        cfg.k_pool, cfg.v_pool = self.k_pool.data_ptr(), self.v_pool.data_ptr()
        cfg.workspace, cfg.workspace_bytes = self.workspace.data_ptr(), ws_bytes
        self.cfg = cfg
        self.ctx = None
        self.ctx = (B.apar_create(cfg) if kv_format == "bf16" else
                    B.apar_create_kv(cfg, B.KV_FORMATS[kv_format]))
        self.sm_scale = 1.0 / math.sqrt(shape.head_dim)

    @classmethod
    def for_spec(cls, spec: ForestSpec, device="cuda", poison=False, extra_blocks=0,
                 kv_format="bf16"):
        nb, nt, mb = pool_requirements(spec)
        return cls(spec.shape, nb + extra_blocks, nt, mb, device, poison, kv_format=kv_format)

    def close(self):
        if self.ctx is not None:
            torch.cuda.synchronize()
            B.apar_destroy(self.ctx)
            self.ctx = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    @staticmethod
    def _stream() -> int:
        if _raw_stream is None:
            return torch.cuda.current_stream().cuda_stream
        return _raw_stream(torch.cuda.current_device())

    # the replay protocol of synth.build_forest
    def new_threads(self, n):
        return B.apar_new_threads(self.ctx, n)

    def fork(self, parents):
        return B.apar_fork(self.ctx, parents, self._stream())

    def append(self, tids, counts, k_rows: torch.Tensor, v_rows: torch.Tensor):
        assert k_rows.is_cuda and k_rows.is_contiguous() and v_rows.is_contiguous()
        assert k_rows.dtype == torch.bfloat16 and k_rows.shape == v_rows.shape
        assert k_rows.shape[0] == (sum(counts) if counts is not None else len(tids))
        B.apar_append_kv(self.ctx, tids, counts, k_rows.data_ptr(), v_rows.data_ptr(),
                         self._stream())

    def attention(self, tids, q: torch.Tensor, out: torch.Tensor = None, sm_scale=None):
        assert q.is_cuda and q.is_contiguous() and q.dtype == torch.bfloat16
        if out is None:
            out = torch.empty_like(q)
        B.apar_tree_decode_attention(self.ctx, tids, q.data_ptr(), out.data_ptr(),
                                     self.sm_scale if sm_scale is None else sm_scale,
                                     self._stream())
        return out

    def decode_step(self, tids, k_rows: torch.Tensor, v_rows: torch.Tensor, q: torch.Tensor,
                    out: torch.Tensor = None, sm_scale=None):
        assert k_rows.is_cuda and k_rows.is_contiguous() and v_rows.is_contiguous()
        assert q.is_cuda and q.is_contiguous() and q.dtype == torch.bfloat16
        if out is None:
            out = torch.empty_like(q)
        B.apar_decode_step(self.ctx, tids, k_rows.data_ptr(), v_rows.data_ptr(), q.data_ptr(),
                           out.data_ptr(), self.sm_scale if sm_scale is None else sm_scale,
                           self._stream())
        return out

    def prefix_attention(self, tids, attend_len, q: torch.Tensor, sm_scale=None):
        assert q.is_cuda and q.is_contiguous() and q.dtype == torch.bfloat16
        out = torch.empty_like(q)
        B.apar_tree_prefix_attention(self.ctx, tids, attend_len, q.data_ptr(), out.data_ptr(),
                                     self.sm_scale if sm_scale is None else sm_scale,
                                     self._stream())
        return out

    def verify_attention(self, tids, n_cand, anc_mask, q: torch.Tensor, sm_scale=None):
        assert q.is_cuda and q.is_contiguous() and q.dtype == torch.bfloat16
        out = torch.empty_like(q)
        B.apar_tree_verify_attention(self.ctx, tids, n_cand, anc_mask, q.data_ptr(),
                                     out.data_ptr(),
                                     self.sm_scale if sm_scale is None else sm_scale,
                                     self._stream())
        return out

    def accept(self, tids, n_cand, keep):
        B.apar_accept_candidates(self.ctx, tids, n_cand, keep, self._stream())

    def prefill_attention(self, tids, q_begin, q_count, q: torch.Tensor, out: torch.Tensor = None,
                          layer: int = 0, sm_scale=None):
        assert q.is_cuda and q.is_contiguous() and q.dtype == torch.bfloat16
        if out is None:
            out = torch.empty_like(q)
        B.apar_tree_prefill_attention(self.ctx, layer, tids, q_begin, q_count, q.data_ptr(),
                                      out.data_ptr(),
                                      self.sm_scale if sm_scale is None else sm_scale,
                                      self._stream())
        return out

    def append_layer(self, layer: int, k_rows: torch.Tensor, v_rows: torch.Tensor):
        assert k_rows.is_cuda and k_rows.is_contiguous() and v_rows.is_contiguous()
        B.apar_append_kv_layer(self.ctx, layer, k_rows.data_ptr(), v_rows.data_ptr(),
                               self._stream())

    def attention_layer(self, layer: int, q: torch.Tensor, out: torch.Tensor = None,
                        sm_scale=None):
        assert q.is_cuda and q.is_contiguous() and q.dtype == torch.bfloat16
        if out is None:
            out = torch.empty_like(q)
        B.apar_tree_decode_attention_layer(self.ctx, layer, q.data_ptr(), out.data_ptr(),
                                           self.sm_scale if sm_scale is None else sm_scale,
                                           self._stream())
        return out

    def read_kv(self, tids, begin, count, layer: int = 0):
        """Rows begin[i] .. begin[i] + count[i] - 1 of each thread's chain, as bf16 (k, v)."""
        count = B.int32_array(count)
        # (negative counts are the library's to refuse)
        rows = max(0, int(np.frombuffer(count[0], np.int32, count[1]).sum(dtype=np.int64)))
        shape = (rows, self.shape.num_kv_heads, self.shape.head_dim)
        k = torch.empty(shape, dtype=torch.bfloat16, device=self.device)
        v = torch.empty(shape, dtype=torch.bfloat16, device=self.device)
        B.apar_read_kv(self.ctx, layer, tids, begin, count, k.data_ptr(), v.data_ptr(),
                       self._stream())
        return k, v

    def release(self, tids):
        B.apar_release(self.ctx, tids)

    def stats(self):
        return B.apar_get_stats(self.ctx)

    def thread(self, tid):
        return B.apar_get_thread(self.ctx, tid)
