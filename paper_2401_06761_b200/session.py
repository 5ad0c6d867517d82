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


class BeamSelect:
    """Beam search's selection: the parameters of apar_beam_config, applied by calling.

    logits [n][beams][vocab] is bf16, f16 or f32 and may be a view with any strides of its first two
    dims; scores is f32 [n][beams]; finished is None or a bool or uint8 tensor [n][beams] (then eos is
    needed).  Returns (scores f32, beams int32, tokens int32), each [n][select], best first."""

    def __init__(self, beams: int, vocab: int, select: int, eos=None):
        self.beams, self.vocab, self.select = beams, vocab, select
        self.cfgs = {t: B.make_beam_config(vocab, beams, select, str(t).rpartition(".")[2], eos)
                     for t in (torch.bfloat16, torch.float16, torch.float32)}
        self._bytes = {}                               # scratch by number of sequences and type

    def __call__(self, logits: torch.Tensor, scores: torch.Tensor, finished: torch.Tensor = None):
        n = logits.shape[0]
        here = torch.cuda.current_device()             # (the launches go to its current stream)
        assert logits.shape == (n, self.beams, self.vocab) and logits.dtype in self.cfgs
        assert scores.shape == (n, self.beams) and scores.dtype == torch.float32
        assert logits.get_device() == here and scores.get_device() == here and scores.is_contiguous()
        if finished is not None:
            assert finished.shape == (n, self.beams) and finished.dtype in (torch.bool, torch.uint8)
            assert finished.get_device() == here and finished.is_contiguous()
        by_seq, by_beam, by_token = logits.stride()
        if (by_token != 1 and self.vocab > 1) or by_seq == 0 or by_beam == 0:
            logits = logits.contiguous()               # (a stride of 0 stands for contiguous rows)
            by_seq, by_beam, _ = logits.stride()
        cfg = self.cfgs[logits.dtype]
        nbytes = self._bytes.get((n, logits.dtype))
        if nbytes is None:
            nbytes = self._bytes[n, logits.dtype] = B.apar_beam_workspace_bytes(cfg, n)
        held = scores.new_empty((nbytes + 3) // 4)
        best = scores.new_empty((n, self.select))
        beams = best.new_empty((n, self.select), dtype=torch.int32)
        tokens = beams.new_empty((n, self.select))
        B.apar_beam_select(cfg, n, logits.data_ptr(), by_seq, by_beam, scores.data_ptr(),
                           0 if finished is None else finished.data_ptr(), best.data_ptr(),
                           beams.data_ptr(), tokens.data_ptr(), held.data_ptr(), nbytes,
                           PagedSession._stream())
        return best, beams, tokens


class PagedSession:
    def __init__(self, shape: LayerShape, num_blocks: int, max_threads: int,
                 max_blocks_per_thread: int, device="cuda", poison: bool = False,
                 num_layers: int = 1, kv_format: str = "bf16", weights: bool = False):
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
        self._close_left()
        self.ctx = (B.apar_create(cfg) if kv_format == "bf16" else
                    B.apar_create_kv(cfg, B.KV_FORMATS[kv_format]))
        self.sm_scale = 1.0 / math.sqrt(shape.head_dim)
        # accumulated weight of every cached row: [layers][blocks][kv heads][16]
        self.weights = None
        if weights:
            nbytes = B.apar_weights_bytes(cfg)
            self._weights_memory = torch.zeros(nbytes, dtype=torch.uint8, device=device)
            rows = num_layers * num_blocks * shape.num_kv_heads * shape.block_size
            self.weights = self._weights_memory[:4 * rows].view(torch.float32).view(
                num_layers, num_blocks, shape.num_kv_heads, shape.block_size)
            B.apar_attach_weights(self.ctx, self._weights_memory.data_ptr(), nbytes)

    @classmethod
    def for_spec(cls, spec: ForestSpec, device="cuda", poison=False, extra_blocks=0,
                 kv_format="bf16"):
        nb, nt, mb = pool_requirements(spec)
        return cls(spec.shape, nb + extra_blocks, nt, mb, device, poison, kv_format=kv_format)

    # what sessions held that went while a graph was being captured, when nothing may wait for the device
    _left = []

    def close(self):
        if self.ctx is None:
            return
        self._left.append(dict(vars(self)))
        self.ctx = None
        self._close_left()

    @classmethod
    def _close_left(cls):
        if cls._left and not torch.cuda.is_current_stream_capturing():
            torch.cuda.synchronize()
            while cls._left:
                B.apar_destroy(cls._left.pop()["ctx"])

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

    def _attend(self, lse, q, call, *args):
        """One attention call, which also writes lse [queries][heads] if one is given."""
        if lse is None:
            return call(self.ctx, *args)
        assert lse.is_cuda and lse.is_contiguous() and lse.dtype == torch.float32
        assert lse.shape == q.shape[:2]
        B.apar_set_lse_output(self.ctx, lse.data_ptr())
        try:
            return call(self.ctx, *args)
        finally:
            B.apar_set_lse_output(self.ctx, 0)

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

    def attention(self, tids, q: torch.Tensor, out: torch.Tensor = None, sm_scale=None, lse=None):
        """lse (here and below): a float tensor [n][heads] that takes the log of each row's softmax
        denominator, for add_weights."""
        assert q.is_cuda and q.is_contiguous() and q.dtype == torch.bfloat16
        if out is None:
            out = torch.empty_like(q)
        self._attend(lse, q, B.apar_tree_decode_attention, tids, q.data_ptr(),
                     out.data_ptr(), self.sm_scale if sm_scale is None else sm_scale,
                     self._stream())
        return out

    def decode_step(self, tids, k_rows: torch.Tensor, v_rows: torch.Tensor, q: torch.Tensor,
                    out: torch.Tensor = None, sm_scale=None, lse=None):
        assert k_rows.is_cuda and k_rows.is_contiguous() and v_rows.is_contiguous()
        assert q.is_cuda and q.is_contiguous() and q.dtype == torch.bfloat16
        if out is None:
            out = torch.empty_like(q)
        self._attend(lse, q, B.apar_decode_step, tids, k_rows.data_ptr(), v_rows.data_ptr(),
                     q.data_ptr(), out.data_ptr(), self.sm_scale if sm_scale is None else
                     sm_scale, self._stream())
        return out

    def prefix_attention(self, tids, attend_len, q: torch.Tensor, sm_scale=None, lse=None):
        assert q.is_cuda and q.is_contiguous() and q.dtype == torch.bfloat16
        out = torch.empty_like(q)
        self._attend(lse, q, B.apar_tree_prefix_attention, tids, attend_len, q.data_ptr(),
                     out.data_ptr(), self.sm_scale if sm_scale is None else sm_scale,
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
                          layer: int = 0, sm_scale=None, lse=None):
        assert q.is_cuda and q.is_contiguous() and q.dtype == torch.bfloat16
        if out is None:
            out = torch.empty_like(q)
        self._attend(lse, q, B.apar_tree_prefill_attention, layer, tids, q_begin, q_count,
                     q.data_ptr(), out.data_ptr(), self.sm_scale if sm_scale is None else
                     sm_scale, self._stream())
        return out

    def append_layer(self, layer: int, k_rows: torch.Tensor, v_rows: torch.Tensor):
        assert k_rows.is_cuda and k_rows.is_contiguous() and v_rows.is_contiguous()
        B.apar_append_kv_layer(self.ctx, layer, k_rows.data_ptr(), v_rows.data_ptr(),
                               self._stream())

    def attention_layer(self, layer: int, q: torch.Tensor, out: torch.Tensor = None,
                        sm_scale=None, lse=None):
        assert q.is_cuda and q.is_contiguous() and q.dtype == torch.bfloat16
        if out is None:
            out = torch.empty_like(q)
        self._attend(lse, q, B.apar_tree_decode_attention_layer, layer, q.data_ptr(),
                     out.data_ptr(), self.sm_scale if sm_scale is None else sm_scale,
                     self._stream())
        return out

    @staticmethod
    def _counts(count):
        """Counts as the library takes them, and their total (negative ones are the library's to refuse)."""
        count = B.int32_array(count)
        buf, n = count
        rows = sum(buf[:n]) if n <= 64 else int(np.frombuffer(buf, np.int32, n).sum(dtype=np.int64))
        return count, max(0, rows)

    def read_kv(self, tids, begin, count, layer: int = 0):
        """Rows begin[i] .. begin[i] + count[i] - 1 of each thread's chain, as bf16 (k, v)."""
        count, rows = self._counts(count)
        k = self.workspace.new_empty((rows, self.shape.num_kv_heads, self.shape.head_dim),
                                     dtype=torch.bfloat16)
        v = torch.empty_like(k)
        B.apar_read_kv(self.ctx, layer, tids, begin, count, k.data_ptr(), v.data_ptr(),
                       self._stream())
        return k, v

    def reorder(self, tids, sources):
        """Thread tids[i] goes on with the chain that sources[i] held (beam search)."""
        B.apar_reorder(self.ctx, tids, sources, self._stream())

    def add_weights(self, q: torch.Tensor, lse: torch.Tensor, layer: int = 0, sm_scale=None,
                    replace: bool = False):
        """Adds to each cached row the weight that the queries of the most recent decode attention
        gave it: q and lse are that call's (of this layer)."""
        assert q.is_cuda and q.is_contiguous() and q.dtype == torch.bfloat16
        assert lse.is_cuda and lse.is_contiguous() and lse.dtype == torch.float32
        assert lse.shape == q.shape[:2]
        B.apar_add_weights(self.ctx, layer, q.data_ptr(), lse.data_ptr(),
                           self.sm_scale if sm_scale is None else sm_scale, replace, self._stream())

    def add_weights_prefill(self, tids, q_begin, q_count, q: torch.Tensor, lse: torch.Tensor,
                            layer: int = 0, sm_scale=None, replace: bool = False):
        """The same for runs of queries, as prefill_attention takes them."""
        assert q.is_cuda and q.is_contiguous() and q.dtype == torch.bfloat16
        assert lse.is_cuda and lse.is_contiguous() and lse.dtype == torch.float32
        q_count, total = self._counts(q_count)
        assert lse.shape == q.shape[:2] and q.shape[0] == total
        B.apar_add_weights_prefill(self.ctx, layer, tids, q_begin, q_count, q.data_ptr(),
                                   lse.data_ptr(), self.sm_scale if sm_scale is None else sm_scale,
                                   replace, self._stream())

    def read_weights(self, tids, begin, count, layer: int = 0):
        """Weights [rows][kv heads] of rows begin[i] .. begin[i] + count[i] - 1 of each chain."""
        count, rows = self._counts(count)
        out = self.workspace.new_empty((rows, self.shape.num_kv_heads), dtype=torch.float32)
        B.apar_read_weights(self.ctx, layer, tids, begin, count, out.data_ptr(), self._stream())
        return out

    def evict(self, tids, begin, end, keep):
        """Of rows begin[i] .. end[i] - 1 of each chain only the keep[i] heaviest stay, per layer and
        kv head."""
        B.apar_evict(self.ctx, tids, begin, end, keep, self._stream())

    def release(self, tids):
        B.apar_release(self.ctx, tids)

    def stats(self):
        return B.apar_get_stats(self.ctx)

    def thread(self, tid):
        return B.apar_get_thread(self.ctx, tid)
