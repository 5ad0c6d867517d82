"""Replay of one event list on a 4-bit session and on checkers that hold the values of its rows."""
import numpy as np
import torch

from oracle import kv4
from helpers import OracleBackend, assert_same_bookkeeping
from paper_2401_06761_b200.session import PagedSession
from paper_2401_06761_b200.synth import LayerShape


def host(t):
    return t.detach().float().cpu().numpy()


class Kv4Pair:
    """A 4-bit PagedSession with two checkers: one holds the rows' values, the other has the
    values' height over the lowest of their group, s c, in place of V (what the rounding of the
    weights is relative to)."""

    def __init__(self, hq, hk, num_blocks=256, max_threads=64, max_blocks=64, num_layers=1):
        self.shape = LayerShape(hq, hk)
        self.sess = PagedSession(self.shape, num_blocks, max_threads, max_blocks, poison=True,
                                 num_layers=num_layers, kv_format="q4")
        args = (self.shape, num_blocks, max_threads, max_blocks)
        self.ref, self.mid = OracleBackend(*args), OracleBackend(*args)

    def new_threads(self, n):
        tids = self.sess.new_threads(n)
        assert tids == self.ref.new_threads(n) == self.mid.new_threads(n)
        return tids

    def fork(self, parents):
        kids = self.sess.fork(parents)
        assert kids == self.ref.fork(parents) == self.mid.fork(parents)
        return kids

    def note_append(self, tids, counts, k, v):
        """The checkers' side of an append."""
        kc, vc = kv4.quantise(host(k)), kv4.quantise(host(v))
        kv = torch.from_numpy(kv4.values(*kc))
        self.ref.append(tids, counts, kv, torch.from_numpy(kv4.values(*vc)))
        self.mid.append(tids, counts, kv, torch.from_numpy(kv4.spread(*vc[:2])))

    def append(self, tids, counts, k, v):
        self.sess.append(tids, counts, k, v)
        self.note_append(tids, counts, k, v)

    def release(self, tids):
        for x in (self.sess, self.ref, self.mid):
            x.release(tids)

    def expected(self, tids, q, scale):
        return self.ref.attention(tids, q, scale), self.mid.attention(tids, q, scale)

    def check_attention(self, tids, q, scale=None, what=""):
        got = self.sess.attention(tids, q, sm_scale=scale)
        scale = self.sess.sm_scale if scale is None else scale
        check(got, *self.expected(tids, q, scale), what)
        return got

    def check_books(self):
        live = [t for t in self.ref.node_of if t in self.ref.model.lens]
        assert_same_bookkeeping(self.sess, self.ref.model, live)

    def close(self):
        self.sess.close()


def check(got, ref, mid, what=""):
    """got bf16 against the 64-bit result ref.  The output is rounded to bf16 (half a step is 2^-8
    of it).  The weights are rounded to f16 after their scale: half a step is 2^-11 of each term,
    and for terms below 2^-20 of the largest 2^-31 of that (2^18 of them add up to no more than
    2^-13); they multiply s c, whose weighted mean is mid.  Sums and scores are in 32 bits.  The
    kernel for many rows rounds the values to f16 instead, which is no more, and K too: 128
    independent errors of 2^-12 of a product each shift a score by some 2^-12 of its spread, a
    tenth of what is left of 2^-10."""
    got = host(got).astype(np.float64)
    assert np.isfinite(got).all(), f"{what}: non-finite output"
    err = np.abs(got - ref)
    tol = 2.0 ** -8 * np.abs(ref) + 2.0 ** -10 * mid + 1e-30
    worst = np.unravel_index(np.argmax(err / tol), err.shape)
    assert (err <= tol).all(), f"{what}: {worst}: {got[worst]} for {ref[worst]}, allowed {tol[worst]}"


def rows(n, heads, seed, spread=1.0):
    g = torch.Generator(device="cpu").manual_seed(seed)
    return (torch.randn(n, heads, 128, generator=g) * spread).to(torch.bfloat16).cuda()
