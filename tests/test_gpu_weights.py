"""Log-sum-exps from attention, accumulated weights, and eviction, against plain 64-bit versions."""
import math
import random

import numpy as np
import pytest
import torch

from paper_2401_06761_b200 import binding as B
from paper_2401_06761_b200.session import PagedSession
from paper_2401_06761_b200.synth import LayerShape

pytestmark = pytest.mark.gpu
DIM = 128
SCALE = 1 / math.sqrt(DIM)


def rows(n, heads, seed, spread=1.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return (torch.randn(n, heads, DIM, generator=g, device="cuda") * spread).to(torch.bfloat16)


class Forest:
    """A session whose threads' keys are also kept here: per thread a list of (row name, key) and
    what each name's weight should be, [layers][kv heads]."""

    def __init__(self, hq, hk, blocks=600, threads=64, per_thread=300, layers=1, poison=True):
        self.hq, self.hk, self.layers = hq, hk, layers
        self.s = PagedSession(LayerShape(hq, hk), blocks, threads, per_thread, poison=poison,
                              num_layers=layers, weights=True)
        self.s.weights.fill_(float("nan"))               # (rows start at zero by being appended)
        self.names, self.k, self.v, self.w = {}, {}, {}, {}
        self.n = 0
        self.seed = 0

    def new(self, n):
        tids = self.s.new_threads(n)
        for t in tids:
            self.names[t] = []
        return tids

    def append(self, tids, counts, spread=1.0):
        total = sum(counts)
        kv = []
        for l in range(self.layers):
            self.seed += 1
            kv.append((rows(total, self.hk, 2 * self.seed, spread), rows(total, self.hk, 2 * self.seed + 1)))
        self.s.append(tids, counts, *kv[0])
        for l in range(1, self.layers):
            self.s.append_layer(l, *kv[l])
        host = [(a.double().cpu().numpy(), b.double().cpu().numpy()) for a, b in kv]
        at = 0
        for t, c in zip(tids, counts):
            for _ in range(c):
                name = self.n
                self.n += 1
                self.names[t].append(name)
                self.k[name] = np.stack([host[l][0][at] for l in range(self.layers)])   # [layers][hk][128]
                self.v[name] = np.stack([host[l][1][at] for l in range(self.layers)])
                self.w[name] = np.zeros((self.layers, self.hk))
                at += 1

    def fork(self, parents):
        kids = self.s.fork(parents)
        for c, p in zip(kids, parents):
            self.names[c] = self.copied(self.names[p])
        return kids

    def copied(self, names):
        full = len(names) // 16 * 16
        out = list(names[:full])
        for x in names[full:]:                           # a partial block's rows are rows of their own
            self.n += 1
            out.append(-self.n)
            self.k[-self.n], self.v[-self.n], self.w[-self.n] = self.k[x], self.v[x], self.w[x].copy()
        return out

    def probabilities(self, t, q, layer, lim=None):
        """exp(scale <q, k> - lse) [hq][keys], lse [hq], and the largest sum of |q k| products."""
        k = np.stack([self.k[x][layer] for x in self.names[t][:lim]], 1)                # [hk][n][128]
        k = np.repeat(k, self.hq // self.hk, 0)
        s = SCALE * np.einsum("hd,hnd->hn", q, k)
        lse = np.logaddexp.reduce(s, 1)
        size = SCALE * np.einsum("hd,hnd->hn", np.abs(q), np.abs(k)).max()
        return np.exp(s - lse[:, None]), lse, size

    def add(self, tids, q, layer=0, lims=None, replace=False):
        """The definition; returns lse [n][hq] and a bound on relative errors."""
        qq = q.double().cpu().numpy()
        if replace:
            for i, t in enumerate(tids):
                for x in self.names[t][:lims[i] if lims else None]:
                    self.w[x][layer] = 0
        lse, size = [], 1.0
        for i, t in enumerate(tids):
            p, l, z = self.probabilities(t, qq[i], layer, lims[i] if lims else None)
            p = p.reshape(self.hk, -1, p.shape[1]).sum(1)
            for j, x in enumerate(self.names[t][:p.shape[1]]):
                self.w[x][layer] += p[:, j]
            lse.append(l)
            size = max(size, z, np.abs(l).max())
        # a score goes through sixteen roundings at most, each 2^-23 of the sum of its products at most;
        # the exponent and the log-sum-exp through a few more, relative to their size
        return np.stack(lse), size * 24 * 2.0 ** -23 + 2.0 ** -20

    def check_weights(self, tids, rel, layer=0):
        counts = [len(self.names[t]) for t in tids]
        got = self.s.read_weights(tids, [0] * len(tids), counts, layer=layer).cpu().numpy()
        want = np.concatenate([np.stack([self.w[x][layer] for x in self.names[t]])
                               for t in tids if self.names[t]])
        assert np.isfinite(got).all()
        assert (np.abs(got - want) <= rel * want + 1e-12).all(), np.abs(got - want).max()

    def check_rows(self, tids, layer=0):
        counts = [len(self.names[t]) for t in tids]
        k, v = self.s.read_kv(tids, [0] * len(tids), counts, layer=layer)
        for got, held in ((k, self.k), (v, self.v)):
            want = np.concatenate([np.stack([held[x][layer] for x in self.names[t]])
                                   for t in tids if self.names[t]])
            assert np.array_equal(got.double().cpu().numpy(), want)


def small_forest(hq, hk, layers=1, prompt=70):
    f = Forest(hq, hk, layers=layers)
    a, b = f.new(2)
    f.append([a, b], [prompt, 33])
    kids = f.fork([a, a, a, b])
    f.append(kids, [1, 16, 40, 5])
    grand = f.fork([kids[2]])
    f.append(grand, [9])
    return f, [a, b, *kids, *grand]


HEADS = [(8, 2), (32, 32), (40, 40), (64, 8), (32, 8), (4, 4), (64, 1), (6, 2)]


@pytest.mark.parametrize("hq,hk", HEADS)
def test_lse_and_weights_of_a_forest(hq, hk):
    f, tids = small_forest(hq, hk)
    q = rows(len(tids), hq, 1000)
    plain = f.s.attention(tids, q)
    lse = torch.full((len(tids), hq), float("nan"), device="cuda")
    assert torch.equal(f.s.attention(tids, q, lse=lse), plain)
    want, rel = f.add(tids, q)
    assert np.abs(lse.cpu().numpy() - want).max() <= rel
    f.s.add_weights(q, lse)
    f.check_weights(tids, rel)
    f.s.add_weights(q, lse)                              # twice as much
    f.add(tids, q)
    f.check_weights(tids, rel)
    f.s.add_weights(q, lse, replace=True)
    f.add(tids, q, replace=True)
    f.check_weights(tids, rel)


@pytest.mark.parametrize("path", ["vec", "ws", "umma", "auto"])
@pytest.mark.parametrize("mode", ["grid", "persist"])
@pytest.mark.parametrize("hq,hk", [(8, 8), (32, 4), (64, 2)])
def test_lse_of_every_attention_kernel(path, mode, hq, hk, monkeypatch):
    monkeypatch.setenv("APAR_ATTN_PATH", path)
    monkeypatch.setenv("APAR_UMMA_MODE", mode)
    monkeypatch.setenv("APAR_WS_MODE", mode)
    f = Forest(hq, hk, blocks=900, threads=40)
    a, b = f.new(2)
    f.append([a, b], [700, 20])
    tids = f.fork([a] * 9 + [b])
    f.append(tids, [3, 17, 100, 1, 5, 64, 30, 200, 8, 2])
    q = rows(len(tids), hq, 7)
    for scale in (SCALE, -0.05):
        lse = torch.full((len(tids), hq), float("nan"), device="cuda")
        f.s.attention(tids, q, lse=lse, sm_scale=scale)
        for i, t in enumerate(tids):
            k = np.stack([f.k[x][0] for x in f.names[t]], 1)
            s = scale * np.einsum("hd,hnd->hn", q[i].double().cpu().numpy(), np.repeat(k, hq // hk, 0))
            want = np.logaddexp.reduce(s, 1)
            # (products of at most 128 * 25 in size; see Forest.add)
            assert np.abs(lse[i].cpu().numpy() - want).max() <= 2e-4, (path, mode, i)
    torch.cuda.synchronize()


def test_lse_of_prefill_prefix_layers_and_verification():
    f, tids = small_forest(16, 4, layers=2)
    n = [len(f.names[t]) for t in tids]
    q = rows(sum(n), 16, 5)
    lse = torch.full((sum(n), 16), float("nan"), device="cuda")
    f.s.prefill_attention(tids, [0] * len(tids), n, q, layer=1, lse=lse)
    at, qq = 0, q.double().cpu().numpy()
    for t, c in zip(tids, n):
        for p in range(c):
            _, want, size = f.probabilities(t, qq[at + p], 1, p + 1)
            assert np.abs(lse[at + p].cpu().numpy() - want).max() <= (size + 10) * 24 * 2.0 ** -23
        at += c
    two = rows(2, 16, 6)
    lse2 = torch.full((2, 16), float("nan"), device="cuda")
    f.s.prefix_attention([tids[0]] * 2, [1, 50], two, lse=lse2)
    for i, lim in enumerate((1, 50)):
        _, want, size = f.probabilities(tids[0], two[i].double().cpu().numpy(), 0, lim)
        assert np.abs(lse2[i].cpu().numpy() - want).max() <= (size + 10) * 24 * 2.0 ** -23
    lse3 = torch.full((2, 16), float("nan"), device="cuda")
    B.apar_set_lse_output(f.s.ctx, lse3.data_ptr())
    f.s.verify_attention([tids[3]], [2], [1, 3], two)
    B.apar_set_lse_output(f.s.ctx, 0)
    m = len(f.names[tids[3]])
    for i in range(2):
        _, want, size = f.probabilities(tids[3], two[i].double().cpu().numpy(), 0, m - 1 + i)
        assert np.abs(lse3[i].cpu().numpy() - want).max() <= (size + 10) * 24 * 2.0 ** -23


@pytest.mark.parametrize("hq,hk", [(8, 2), (40, 40)])
def test_weights_over_steps_forks_layers_and_prefixes(hq, hk):
    f, tids = small_forest(hq, hk, layers=2)
    rel = 0
    for step in range(20):                               # (blocks are opened on the way)
        new = [rows(len(tids), hk, 9000 + 10 * step + l) for l in range(4)]
        q = [rows(len(tids), hq, 5000 + 2 * step + l) for l in range(2)]
        lse = [torch.empty(len(tids), hq, device="cuda") for _ in range(2)]
        f.s.decode_step(tids, new[0], new[1], q[0], lse=lse[0])
        f.s.append_layer(1, new[2], new[3])
        f.s.attention_layer(1, q[1], lse=lse[1])
        host = [x.double().cpu().numpy() for x in new]
        for i, t in enumerate(tids):
            f.names[t].append(f.n)
            f.k[f.n], f.v[f.n] = np.stack([host[0][i], host[2][i]]), np.stack([host[1][i], host[3][i]])
            f.w[f.n] = np.zeros((2, hk))
            f.n += 1
        for l in range(2):
            f.s.add_weights(q[l], lse[l], layer=l)
            rel = max(rel, f.add(tids, q[l], l)[1])
        if step in (4, 11):
            tids = tids + f.fork([tids[1], tids[-1]])
            f.append(tids[-2:], [2, 0])
    for l in range(2):
        f.check_weights(tids, rel, l)
        f.check_rows(tids, l)
    # queries that see part of a chain, a thread listed twice
    some, lims = [tids[0], tids[0], tids[1]], [17, 64, 3]
    q = rows(3, hq, 77)
    lse = torch.empty(3, hq, device="cuda")
    f.s.prefix_attention(some, lims, q, lse=lse)
    f.s.add_weights(q, lse)
    f.check_weights(tids, max(rel, f.add(some, q, lims=lims)[1]))


def test_weights_of_wide_shared_runs_and_long_chains():
    f = Forest(8, 2, blocks=1200, threads=64, per_thread=700)
    (a,) = f.new(1)
    f.append([a], [4111])
    tids = f.fork([a] * 21)
    f.append(tids, [1 + 3 * i for i in range(21)])
    q = rows(21, 8, 3)
    lse = torch.empty(21, 8, device="cuda")
    f.s.attention(tids, q, lse=lse)
    f.s.add_weights(q, lse)
    f.check_weights(tids, f.add(tids, q)[1])


def test_captured_step_with_weights():
    f, tids = small_forest(8, 2)
    f.append(tids, [16 - len(f.names[t]) % 16 + 1 for t in tids])     # room for fifteen steps
    q = rows(len(tids), 8, 50)
    k, v = rows(len(tids), 2, 51), rows(len(tids), 2, 52)
    lse, out = torch.empty(len(tids), 8, device="cuda"), torch.empty_like(q)

    def step():
        f.s.decode_step(tids, k, v, q, out=out, lse=lse)
        f.s.add_weights(q, lse)

    def follow():
        host = k.double().cpu().numpy(), v.double().cpu().numpy()
        for i, t in enumerate(tids):
            f.names[t].append(f.n)
            f.k[f.n], f.v[f.n], f.w[f.n] = host[0][i][None], host[1][i][None], np.zeros((1, 2))
            f.n += 1
        return f.add(tids, q)[1]

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
        rel = follow()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=side):
            step()
        g.replay()
        follow()
        for _ in range(3):
            B.apar_note_step_replay(f.s.ctx)
            g.replay()
            rel = follow()
        with pytest.raises(B.AparError):                 # a plan has to be made: not while capturing
            g2 = torch.cuda.CUDAGraph()
            f.s.attention(tids[:2], q[:2].contiguous(), lse=lse[:2].contiguous())
            with torch.cuda.graph(g2, stream=side):
                f.s.add_weights(q[:2].contiguous(), lse[:2].contiguous())
        side.synchronize()
    f.check_weights(tids, rel)


def test_replays_between_other_plans():
    """A captured step with weights is replayed after a prompt's weights and after another step's plan of
    the same threads took the place of the captured one's."""
    f, tids = small_forest(8, 2)
    f.append(tids, [16 - len(f.names[t]) % 16 + 1 for t in tids])
    q = rows(len(tids), 8, 50)
    k, v = rows(len(tids), 2, 51), rows(len(tids), 2, 52)
    lse, out = torch.empty(len(tids), 8, device="cuda"), torch.empty_like(q)

    def step():
        f.s.decode_step(tids, k, v, q, out=out, lse=lse)
        f.s.add_weights(q, lse)

    def follow():
        host = k.double().cpu().numpy(), v.double().cpu().numpy()
        for i, t in enumerate(tids):
            f.names[t].append(f.n)
            f.k[f.n], f.v[f.n], f.w[f.n] = host[0][i][None], host[1][i][None], np.zeros((1, 2))
            f.n += 1
        return f.add(tids, q)[1]

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
        follow()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=side):
            step()
        g.replay()
        rel = follow()
        n = len(f.names[tids[0]])
        p, pl = rows(20, 8, 60), torch.empty(20, 8, device="cuda")
        # (the lse of a thread's last rows, without an attention call in between, from its definition)
        want, _ = add_segments(f, [(tids[0], n - 20, 20)], p)
        pl.copy_(torch.from_numpy(want).float())
        f.s.add_weights_prefill([tids[0]], [n - 20], [20], p, pl)
        B.apar_note_step_replay(f.s.ctx)
        g.replay()
        follow()
        some = tids[:3]
        q3, lse3 = rows(3, 8, 70), torch.empty(3, 8, device="cuda")
        f.s.attention(some, q3, lse=lse3)
        f.s.add_weights(q3, lse3)
        f.add(some, q3)
        with pytest.raises(B.AparError):                 # (the plan is another's)
            B.apar_note_step_replay(f.s.ctx)
        f.s.attention(tids, q, lse=lse)
        f.s.add_weights(q, lse)
        rel = max(rel, f.add(tids, q)[1])
        side.synchronize()
    f.check_weights(tids, 2 * rel)                       # (lse rounded once more)


def test_rows_that_move_take_their_weights_along():
    f, tids = small_forest(8, 2)
    t = tids[4]
    f.append([t], [6])
    q, lse = rows(1, 8, 60), torch.empty(1, 8, device="cuda")
    f.s.attention([t], q, lse=lse)
    f.s.add_weights(q, lse)
    rel = f.add([t], q)[1]
    f.s.accept([t], [6], [[1, 4, 5]])
    f.names[t] = f.names[t][:-6] + [f.names[t][-6 + x] for x in (1, 4, 5)]
    f.check_weights([t], rel)
    f.check_rows([t])


def test_reorder_moves_chains():
    f, tids = small_forest(8, 2, layers=2)
    q = [rows(len(tids), 8, 90 + l) for l in range(2)]
    lse = torch.empty(len(tids), 8, device="cuda")
    f.s.attention(tids, q[0], lse=lse)
    f.s.add_weights(q[0], lse)
    rel = f.add(tids, q[0])[1]
    rng = random.Random(1)
    for _ in range(12):
        some = rng.sample(tids, rng.randint(1, len(tids)))
        sources = [rng.choice(some if rng.random() < 0.8 else tids) for _ in some]
        f.s.reorder(some, sources)
        old = dict(f.names)
        kept = {s: s for t, s in zip(some, sources) if t == s}
        kept.update({s: s for s in sources if s not in some})
        for t, s in zip(some, sources):
            if t != s:
                f.names[t] = f.copied(old[s]) if s in kept else old[s]
                kept.setdefault(s, t)
        f.append(tids, [rng.choice([0, 1, 2]) for _ in tids])
        B.apar_check_invariants(f.s.ctx)
        for l in range(2):
            f.check_rows(tids, l)
        f.check_weights(tids, rel)
        out = f.s.attention(tids, q[0])
        for i, t in enumerate(tids):
            p, _, _ = f.probabilities(t, q[0][i].double().cpu().numpy(), 0)
            v = np.repeat(np.stack([f.v[x][0] for x in f.names[t]], 1), 4, 0)
            assert np.abs(out[i].double().cpu().numpy() - np.einsum("hn,hnd->hd", p, v)).max() <= 2e-2


def add_segments(f, segments, q, layer=0, replace=False):
    """The definition for runs of queries (thread, first, count); returns lse and the bound."""
    qq = q.double().cpu().numpy()
    if replace:
        for t, b, c in segments:
            for x in f.names[t][:b + c]:
                f.w[x][layer] = 0
    lse, size, at = [], 1.0, 0
    for t, b, c in segments:
        k = np.stack([f.k[x][layer] for x in f.names[t][:b + c]], 1)
        k = np.repeat(k, f.hq // f.hk, 0)
        s = SCALE * np.einsum("qhd,hnd->hqn", qq[at:at + c], k)
        s[:, np.arange(b + c)[None, :] > b + np.arange(c)[:, None]] = -np.inf
        l = np.logaddexp.reduce(s, 2)
        p = np.exp(s - l[..., None]).sum(1).reshape(f.hk, -1, b + c).sum(1)
        for j, x in enumerate(f.names[t][:b + c]):
            f.w[x][layer] += p[:, j]
        lse.append(l.T)
        big = SCALE * np.einsum("qhd,hnd->hqn", np.abs(qq[at:at + c]), np.abs(k)).max()
        size, at = max(size, big, np.abs(l).max()), at + c
    return np.concatenate(lse), size * 24 * 2.0 ** -23 + 2.0 ** -20


@pytest.mark.parametrize("hq,hk", HEADS + [(5, 1)])
def test_weights_of_prompts(hq, hk):
    f, tids = small_forest(hq, hk, layers=2, prompt=301)
    n = [len(f.names[t]) for t in tids]
    # whole prompts; children from their own first row on; windows, one query, the same thread twice
    segments = [(tids[0], 0, n[0]), (tids[1], 0, n[1])]
    segments += [(t, 301, m - 301) for t, m in zip(tids[2:5], n[2:5])]
    segments += [(tids[6], n[6] - 3, 3), (tids[5], n[5] - 1, 1), (tids[0], 100, 7), (tids[0], 0, 1)]
    q = rows(sum(c for _, _, c in segments), hq, 21)
    ids, begin, count = (list(x) for x in zip(*segments))
    for layer in (0, 1):
        lse = torch.empty(q.shape[:2], device="cuda")
        f.s.prefill_attention(ids, begin, count, q, layer=layer, lse=lse)
        want, rel = add_segments(f, segments, q, layer)
        assert np.abs(lse.cpu().numpy() - want).max() <= rel
        f.s.add_weights_prefill(ids, begin, count, q, lse, layer=layer)
        f.check_weights(tids, rel, layer)
        some = segments[2:4]
        part = q[n[0] + n[1]:][:sum(c for _, _, c in some)].contiguous()
        lse2 = lse[n[0] + n[1]:][:len(part)].contiguous()
        f.s.add_weights_prefill(*(list(x) for x in zip(*some)), part, lse2, layer=layer, replace=True)
        add_segments(f, some, part, layer, replace=True)
        f.check_weights(tids, rel, layer)
    assert B.apar_get_stats(f.s.ctx)["device_wait_timeouts"] == 0


@pytest.mark.parametrize("n,count", [(1, 1), (16, 16), (17, 17), (128, 128), (129, 2), (256, 256),
                                     (257, 257), (400, 130), (1025, 1025), (2000, 1), (2000, 33)])
@pytest.mark.parametrize("hq,hk", [(8, 1), (2, 2)])
def test_weights_of_prompts_of_many_lengths(n, count, hq, hk):
    f = Forest(hq, hk)
    (t,) = f.new(1)
    f.append([t], [n])
    q = rows(count, hq, n)
    segments = [(t, n - count, count)]
    lse = torch.empty(count, hq, device="cuda")
    f.s.prefill_attention([t], [n - count], [count], q, lse=lse)
    _, rel = add_segments(f, segments, q)
    f.s.add_weights_prefill([t], [n - count], [count], q, lse)
    f.check_weights([t], rel)
    # a decode step's weights after it: each has a plan of its own
    q1, lse1 = rows(1, hq, n + 1), torch.empty(1, hq, device="cuda")
    f.s.attention([t], q1, lse=lse1)
    f.s.add_weights(q1, lse1)
    f.s.add_weights_prefill([t], [n - count], [count], q, lse)
    f.s.add_weights(q1, lse1)
    f.add([t], q1)
    f.add([t], q1)
    add_segments(f, segments, q)
    f.check_weights([t], rel)
    assert B.apar_get_stats(f.s.ctx)["device_wait_timeouts"] == 0


def test_weights_of_prompts_in_many_units():
    """More units than CTAs, of different lengths; the same bits every time; the sum of a query's
    weights is the number of heads of a group."""
    s = PagedSession(LayerShape(32, 8), 1500, 16, 200, weights=True)
    tids = s.new_threads(9)
    n = [2100, 1, 700, 1999, 64, 333, 16, 2500, 1300]
    s.append(tids, n, rows(sum(n), 8, 1, 2.0), rows(sum(n), 8, 2))
    q = rows(sum(n), 32, 3)
    lse = torch.empty(sum(n), 32, device="cuda")
    zero = [0] * 9
    s.prefill_attention(tids, zero, n, q, lse=lse)
    s.add_weights_prefill(tids, zero, n, q, lse)
    first = s.read_weights(tids, zero, n)
    at = 0
    for m in n:
        total = first[at:at + m].double().sum(0).cpu().numpy()
        # every weight within 1e-4 of its own (scores are below 2^6 here; see Forest.add)
        assert np.abs(total - 4 * m).max() <= 4 * m * 1e-4
        at += m
    for _ in range(3):
        s.add_weights_prefill(tids, zero, n, q, lse, replace=True)
        assert torch.equal(s.read_weights(tids, zero, n), first)
    assert B.apar_get_stats(s.ctx)["device_wait_timeouts"] == 0


@pytest.mark.parametrize("hq,hk", [(32, 32), (32, 8)])
def test_weights_of_prompts_have_the_same_bits_in_many_runs(hq, hk):
    """Units with even and odd numbers of query tiles after each other, many of them per CTA."""
    s = PagedSession(LayerShape(hq, hk), 1100, 16, 200, weights=True)
    n = [2040, 1910, 1777, 1650, 2001, 1523, 1999, 1801]
    tids = s.new_threads(8)
    s.append(tids, n, rows(sum(n), hk, 1), rows(sum(n), hk, 2))
    q = rows(sum(n), hq, 3)
    lse = torch.empty(sum(n), hq, device="cuda")
    zero = [0] * 8
    s.prefill_attention(tids, zero, n, q, lse=lse)
    s.add_weights_prefill(tids, zero, n, q, lse, replace=True)
    first = s.read_weights(tids, zero, n)
    wrong = torch.zeros((), dtype=torch.int64, device="cuda")
    for _ in range(300):
        s.add_weights_prefill(tids, zero, n, q, lse, replace=True)
        wrong += (s.read_weights(tids, zero, n) != first).sum()
    assert wrong.item() == 0
    assert B.apar_get_stats(s.ctx)["device_wait_timeouts"] == 0


def place(w, keep):
    """Rows that stay, by place, of weights w [n]: NaN first, then by weight, ties to the earlier."""
    key = [(not math.isnan(x), 0 if math.isnan(x) else -x, i) for i, x in enumerate(w)]
    kept = sorted(i for _, _, i in sorted(key)[:keep])
    move = iter([i for i in kept if i >= keep])
    stay = {i for i in kept if i < keep}
    return [i if i in stay else next(move) for i in range(keep)]


def set_weights(f, t, w):
    """w [layers][rows][hk] into the memory of thread t's rows."""
    _, blocks = f.s.thread(t)
    full = np.zeros((w.shape[0], len(blocks) * 16, f.hk), np.float32)
    full[:, :w.shape[1]] = w
    x = torch.from_numpy(full).cuda().unflatten(1, (-1, 16)).transpose(2, 3)
    f.s.weights[:, torch.tensor(blocks, device="cuda")] = x


def check_evicted(f, t, w, k, v, begin, end, keep):
    """Rows and weights of t after eviction; w, k, v are [layers][rows][hk](128) from before."""
    n = w.shape[1]
    for l in range(f.layers):
        total = n - (end - begin) + keep
        gk, gv = f.s.read_kv([t], [0], [total], layer=l)
        gw = f.s.read_weights([t], [0], [total], layer=l).cpu().numpy()
        for h in range(f.hk):
            src = list(range(begin)) + [begin + i for i in place(w[l, begin:end, h], keep)] + list(range(end, n))
            assert torch.equal(gk[:, h], k[l][src, h]) and torch.equal(gv[:, h], v[l][src, h]), (l, h)
            assert np.array_equal(gw[:, h], w[l, src, h], equal_nan=True), (l, h)


KINDS = ["plain", "equal", "few", "special", "tiny"]


def some_weights(rng, kind, layers, n, hk):
    if kind == "plain":
        return np.exp(2 * rng.standard_normal((layers, n, hk))).astype(np.float32)
    if kind == "equal":
        return np.ones((layers, n, hk), np.float32)
    if kind == "few":
        return rng.integers(0, 3, (layers, n, hk)).astype(np.float32)
    if kind == "tiny":                                   # neighbours in the last bits
        return (np.float32(1) + rng.integers(0, 5, (layers, n, hk)).astype(np.float32) * np.float32(2 ** -23))
    w = rng.standard_normal((layers, n, hk)).astype(np.float32)
    for x in (np.nan, np.inf, -np.inf, 0.0, -0.0):
        w[rng.random(w.shape) < 0.1] = x
    return w


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("n,begin,end,keep", [
    (1, 0, 1, 0), (17, 0, 17, 1), (17, 16, 17, 0), (100, 0, 100, 99), (100, 16, 100, 50), (96, 32, 64, 16),
    (200, 0, 192, 64), (700, 16, 700, 333), (513, 0, 513, 512), (1500, 0, 1488, 16), (40, 16, 32, 0)])
def test_eviction(n, begin, end, keep, kind):
    f = Forest(8, 2, layers=2)
    (t,) = f.new(1)
    f.append([t], [n])
    w = some_weights(np.random.default_rng(n + keep), kind, 2, n, 2)
    set_weights(f, t, w)
    kv = [f.s.read_kv([t], [0], [n], layer=l) for l in range(2)]
    f.s.evict([t], [begin], [end], [keep])
    B.apar_check_invariants(f.s.ctx)
    check_evicted(f, t, w, [x[0] for x in kv], [x[1] for x in kv], begin, end, keep)


@pytest.mark.parametrize("hq,hk", [(8, 2), (40, 40), (64, 1)])
def test_eviction_of_several_threads_shared_and_copied(hq, hk):
    f = Forest(hq, hk, blocks=2000)
    a, b, c = f.new(3)
    f.append([a, b, c], [640, 333, 64])
    kids = f.fork([a, a, b])
    f.append(kids, [0, 0, 50])
    rng = np.random.default_rng(5)
    held = {}
    for t in (a, b, c, *kids):
        m = f.s.thread(t)[0]
        if t in (a, b, c, kids[2]):
            set_weights(f, t, some_weights(rng, "plain", 1, m, hk))
    for t in (a, b, c, *kids):
        m = f.s.thread(t)[0]
        w = f.s.read_weights([t], [0], [m]).cpu().numpy()[None]
        held[t] = (w, *[[x] for x in f.s.read_kv([t], [0], [m])])
    # a stays whole, its two children share what they keep; b and its child part; c in place
    tids = [kids[0], b, kids[1], c]
    f.s.evict(tids, [16, 0, 16, 0], [640, 333, 640, 48], [160, 100, 160, 32])
    B.apar_check_invariants(f.s.ctx)
    check_evicted(f, kids[0], *held[kids[0]], 16, 640, 160)
    check_evicted(f, kids[1], *held[kids[1]], 16, 640, 160)
    check_evicted(f, b, *held[b], 0, 333, 100)
    check_evicted(f, c, *held[c], 0, 48, 32)
    check_evicted(f, a, *held[a], 0, 640, 640)
    check_evicted(f, kids[2], *held[kids[2]], 0, 383, 383)
    assert f.s.thread(kids[0])[1] == f.s.thread(kids[1])[1]
    # all of them go on
    q, lse = rows(6, hq, 8), torch.empty(6, hq, device="cuda")
    k = rows(6, hk, 9)
    f.s.decode_step([a, b, c, *kids], k, k, q, lse=lse)
    f.s.add_weights(q, lse)
    B.apar_check_invariants(f.s.ctx)


@pytest.mark.parametrize("n", [16384, 16400, 33000, 70000, 131072, 140001])
def test_eviction_of_a_long_stretch(n):
    f = Forest(4, 1, blocks=13000, per_thread=8800, poison=False)
    (t,) = f.new(1)
    k, v = rows(n, 1, 1), rows(n, 1, 2)
    f.s.append([t], [n], k, v)
    w = some_weights(np.random.default_rng(3), "plain" if n % 16 else "few", 1, n, 1)
    set_weights(f, t, w)
    keep = n * 3 // 7
    (c,) = f.s.fork([t])
    f.s.evict([c], [16], [n], [keep])                    # copied: the parent keeps its rows
    check_evicted(f, c, w, [k], [v], 16, n, keep)
    f.s.release([c])
    f.s.evict([t], [0], [n], [keep])
    check_evicted(f, t, w, [k], [v], 0, n, keep)


@pytest.mark.parametrize("n_threads,n,keep,hk", [
    (1, 512, 200, 2), (1, 513, 200, 2), (1, 2048, 2047, 1), (1, 2049, 30, 1), (1, 8192, 5000, 2),
    (1, 8193, 8000, 2), (8, 300, 200, 2), (9, 300, 200, 2), (1, 10241, 10240, 1), (1, 10257, 10256, 1),
    (40, 600, 333, 4), (40, 2048, 100, 4)])
def test_eviction_of_stretches_that_are_few_and_many(n_threads, n, keep, hk):
    f = Forest(2 * hk, hk, blocks=n_threads * 2 * (n // 16 + 2) + 64, threads=2 * n_threads + 8,
               per_thread=n // 16 + 8, poison=False)
    tids = f.new(n_threads)
    k, v = rows(n * n_threads, hk, 1), rows(n * n_threads, hk, 2)
    f.s.append(tids, [n] * n_threads, k, v)
    ws = []
    for i, t in enumerate(tids):
        kind = KINDS[i % len(KINDS)] if n_threads > 1 else "few"
        ws.append(some_weights(np.random.default_rng(i), kind, 1, n, hk))
        set_weights(f, t, ws[-1])
    kids = f.s.fork(tids)
    for who in (kids, tids):                             # copied, then in place
        f.s.evict(who, [0] * n_threads, [n] * n_threads, [keep] * n_threads)
        B.apar_check_invariants(f.s.ctx)
        for i, t in enumerate(who):
            check_evicted(f, t, ws[i], [k[i * n:i * n + n]], [v[i * n:i * n + n]], 0, n, keep)
        if who is kids:
            f.s.release(kids)


@pytest.mark.parametrize("hq,hk,n_threads,prompt,kids", [
    (8, 1, 1, 1025, 0), (8, 1, 3, 2100, 0), (8, 1, 1, 5000, 1), (4, 1, 2, 700, 9), (32, 32, 6, 130, 1)])
def test_weights_of_runs_cut_into_even_units(hq, hk, n_threads, prompt, kids):
    f = Forest(hq, hk, blocks=2000, per_thread=400)
    tids = f.new(n_threads)
    f.append(tids, [prompt + 37 * i for i in range(n_threads)])
    if kids:
        tids = tids + f.fork(tids * kids)
    q, lse = rows(len(tids), hq, 3), torch.empty(len(tids), hq, device="cuda")
    f.s.attention(tids, q, lse=lse)
    f.s.add_weights(q, lse)
    _, rel = f.add(tids, q)
    f.check_weights(tids, rel)


def test_beam_search_with_a_bounded_cache():
    """Selection, reordering, decode steps with weights and evictions, as they are used together:
    the library's threads against plain lists of rows."""
    from paper_2401_06761_b200.session import BeamSelect
    beams, vocab, hq, hk = 4, 500, 8, 2
    f = Forest(hq, hk)
    (root,) = f.new(1)
    f.append([root], [48])
    tids = f.fork([root] * beams)
    f.s.release([root])
    select = BeamSelect(beams, vocab, beams)
    scores = torch.tensor([[0.0] + [-math.inf] * (beams - 1)], device="cuda")
    g = torch.Generator(device="cuda").manual_seed(5)
    proj = torch.randn(hq * DIM, vocab, generator=g, device="cuda") * 0.05
    rel = 2.0 ** -20
    for step in range(40):
        q = rows(beams, hq, 300 + step)
        k, v = rows(beams, hk, 700 + step), rows(beams, hk, 800 + step)
        lse = torch.empty(beams, hq, device="cuda")
        out = f.s.decode_step(tids, k, v, q, lse=lse)
        hk_, hv_ = k.double().cpu().numpy(), v.double().cpu().numpy()
        for i, t in enumerate(tids):
            f.names[t].append(f.n)
            f.k[f.n], f.v[f.n], f.w[f.n] = hk_[i][None], hv_[i][None], np.zeros((1, hk))
            f.n += 1
        f.s.add_weights(q, lse)
        rel = max(rel, f.add(tids, q)[1])
        logits = (out.float().flatten(1) @ proj)[None]
        scores, source, _ = select(logits, scores)
        sources = [tids[b] for b in source[0].tolist()]
        f.s.reorder(tids, sources)
        old, kept = dict(f.names), {s: s for t, s in zip(tids, sources) if t == s}
        for t, s in zip(tids, sources):
            if t != s:
                f.names[t] = f.copied(old[s]) if s in kept else old[s]
                kept.setdefault(s, t)
        if step in (7, 15):                              # the shared prompt shrinks for all at once
            end = 48 if step == 7 else 32
            got = f.s.read_weights([tids[0]], [0], [end]).cpu().numpy()
            keep = end - 16
            f.s.evict(tids, [0] * beams, [end] * beams, [keep] * beams)
            # (each kv head keeps rows of its own: a place is a new row made of them)
            names = f.names[tids[0]][:end]
            new = []
            src = [place(got[:, h], keep) for h in range(hk)]
            for j in range(keep):
                f.k[f.n], f.v[f.n], f.w[f.n] = (np.stack([x[names[src[h][j]]][0, h] for h in range(hk)])[None]
                                                for x in (f.k, f.v, f.w))
                new.append(f.n)
                f.n += 1
            for t in tids:
                f.names[t] = new + f.names[t][end:]
        B.apar_check_invariants(f.s.ctx)
        f.check_rows(tids)
        f.check_weights(tids, rel)
    assert B.apar_get_stats(f.s.ctx)["device_wait_timeouts"] == 0


def test_refusals():
    f, tids = small_forest(8, 2)
    s = f.s
    q, lse = rows(len(tids), 8, 1), torch.empty(len(tids), 8, device="cuda")

    def refused(code, call, *args, **kw):
        with pytest.raises(B.AparError) as e:
            call(*args, **kw)
        assert e.value.code == code

    refused("INVALID_ARG", s.add_weights, q, lse)        # no attention yet
    s.attention(tids, q, lse=lse)
    refused("INVALID_ARG", s.add_weights, q, lse, layer=1)
    refused("INVALID_ARG", B.apar_add_weights, s.ctx, 0, q.data_ptr() + 2, lse.data_ptr(), 1.0, False)
    refused("INVALID_ARG", B.apar_add_weights, s.ctx, 0, q.data_ptr(), 0, 1.0, False)
    f.append([tids[0]], [1])
    refused("INVALID_ARG", s.add_weights, q, lse)        # bookkeeping since
    s.verify_attention([tids[0]], [1], [1], q[:1].contiguous())
    refused("INVALID_ARG", s.add_weights, q[:1].contiguous(), lse[:1].contiguous())
    refused("INVALID_ARG", s.read_weights, [tids[0]], [0], [9999])
    refused("BAD_THREAD", s.read_weights, [999], [0], [1])
    refused("INVALID_ARG", s.read_weights, [tids[0]], [0], [1], layer=1)
    assert s.read_weights([tids[0]], [3], [0]).shape == (0, 2)
    m = len(f.names[tids[0]])
    for begin, count in ((0, 0), (-1, 2), (m, 1), (m - 1, 2)):
        refused("INVALID_ARG", B.apar_add_weights_prefill, s.ctx, 0, [tids[0]], [begin], [count],
                q.data_ptr(), lse.data_ptr(), 1.0, False)
    refused("BAD_THREAD", B.apar_add_weights_prefill, s.ctx, 0, [999], [0], [1], q.data_ptr(),
            lse.data_ptr(), 1.0, False)
    refused("INVALID_ARG", B.apar_add_weights_prefill, s.ctx, 0, [tids[0]], [0], [1],
            q.data_ptr() + 2, lse.data_ptr(), 1.0, False)
    refused("INVALID_ARG", B.apar_attach_weights, s.ctx, s._weights_memory.data_ptr() + 16, 1 << 40)
    refused("WORKSPACE_TOO_SMALL", B.apar_attach_weights, s.ctx, s._weights_memory.data_ptr(), 1024)
    B.apar_attach_weights(s.ctx, 0, 0)
    s.attention(tids, q, lse=lse)
    refused("INVALID_ARG", s.add_weights, q, lse)
    refused("INVALID_ARG", s.evict, [tids[0]], [0], [16], [0])
    refused("INVALID_ARG", s.read_weights, [tids[0]], [0], [1])
    q4 = PagedSession(LayerShape(8, 2), 50, 4, 10, kv_format="q4")
    refused("UNSUPPORTED", B.apar_attach_weights, q4.ctx, 0, 0)
    refused("UNSUPPORTED", B.apar_set_lse_output, q4.ctx, 0)
    refused("UNSUPPORTED", q4.evict, [], [], [], [])


def test_reorder_of_a_4_bit_cache():
    s = PagedSession(LayerShape(8, 2), 200, 16, 40, kv_format="q4")
    tids = s.new_threads(3)
    s.append(tids, [20, 35, 16], rows(71, 2, 1), rows(71, 2, 2))
    was = [s.read_kv([t], [0], [s.thread(t)[0]]) for t in tids]
    s.reorder(tids, [tids[1], tids[2], tids[1]])
    for t, i in zip(tids, (1, 2, 1)):
        for got, want in zip(s.read_kv([t], [0], [s.thread(t)[0]]), was[i]):
            assert torch.equal(got, want)
    s.append(tids, [3, 3, 3], rows(9, 2, 3), rows(9, 2, 4))
    for got, want in zip(s.read_kv([tids[0]], [0], [35]), was[1]):
        assert torch.equal(got, want)
    B.apar_check_invariants(s.ctx)


def test_calls_while_capturing_are_refused():
    f, tids = small_forest(8, 2)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    g = torch.cuda.CUDAGraph()
    codes = []
    with torch.cuda.graph(g, stream=side):
        for call in (lambda: f.s.evict([tids[0]], [0], [64], [16]),
                     lambda: f.s.reorder([tids[0]], [tids[2]]),
                     lambda: f.s.read_weights([tids[0]], [0], [4])):
            try:
                call()
                codes.append("ok")
            except B.AparError as e:
                codes.append(e.code)
        f.s.weights.add_(0)                              # (something to capture)
    assert codes == ["INVALID_ARG"] * 3
    B.apar_check_invariants(f.s.ctx)
    f.check_rows(tids)


def test_a_refused_attention_call_leaves_the_one_before_it():
    """Queries of so many lengths that their partial results do not fit are refused; the weights, the layer
    calls and the plan of the call before are then still there."""
    f = Forest(8, 2, layers=2)
    (a, b) = f.new(2)
    f.append([a, b], [64 * 16, 40])
    tids = f.fork([a, a]) + [b]
    q = [rows(3, 8, 40 + l) for l in range(2)]
    lse = [torch.empty(3, 8, device="cuda") for _ in range(2)]
    plain = f.s.attention(tids, q[0], lse=lse[0])
    plain1 = f.s.attention_layer(1, q[1], lse=lse[1])

    def refused():
        many = rows(64, 8, 44)
        before = B.apar_get_stats(f.s.ctx)
        with pytest.raises(B.AparError) as e:
            f.s.prefix_attention([a] * 64, [16 * (i + 1) for i in range(64)], many)
        assert e.value.code == "WORKSPACE_TOO_SMALL"
        with pytest.raises(B.AparError) as e:            # (a prompt's queries that begin between boundaries)
            B.apar_tree_prefill_attention(f.s.ctx, 0, [a], [0], [4], many.data_ptr() + 2, many.data_ptr(), SCALE)
        assert e.value.code == "INVALID_ARG"
        assert B.apar_get_stats(f.s.ctx) == before

    refused()
    f.s.add_weights(q[0], lse[0])                        # (its plan is made after the refusal)
    rel = f.add(tids, q[0])[1]
    refused()
    f.s.add_weights(q[1], lse[1], layer=1)               # (and was there before it)
    rel = max(rel, f.add(tids, q[1], 1)[1])
    assert torch.equal(f.s.attention_layer(1, q[1]), plain1)
    refused()
    assert torch.equal(f.s.attention(tids, q[0]), plain)
    for l in range(2):
        f.check_weights([*tids, a], rel, l)
    assert f.s.stats()["device_wait_timeouts"] == 0


def test_prompt_attention_ends_what_weights_can_be_added():
    f, tids = small_forest(8, 2)
    q, lse = rows(len(tids), 8, 1), torch.empty(len(tids), 8, device="cuda")
    f.s.attention(tids, q, lse=lse)
    f.s.prefill_attention([tids[0]], [0], [4], rows(4, 8, 2))
    with pytest.raises(B.AparError) as e:
        f.s.add_weights(q, lse)
    assert e.value.code == "INVALID_ARG"
    f.s.attention(tids, q, lse=lse)
    f.s.add_weights(q, lse)
    f.check_weights(tids, f.add(tids, q)[1])


def test_no_replay_over_other_queries_weights():
    """A captured apar_add_weights follows the units on the device: while those are another call's (whose
    queries may be more than the captured call has), no replay is announced."""
    f, tids = small_forest(8, 2)
    f.append(tids, [16 - len(f.names[t]) % 16 + 1 for t in tids])
    some = tids[:2]
    q, k = rows(2, 8, 50), rows(2, 2, 51)
    lse, out = torch.empty(2, 8, device="cuda"), torch.empty_like(q)
    all_q, all_lse = rows(len(tids), 8, 52), torch.empty(len(tids), 8, device="cuda")

    def step():
        f.s.decode_step(some, k, k, q, out=out, lse=lse)
        f.s.add_weights(q, lse)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=side):
            step()
        g.replay()
        B.apar_note_step_replay(f.s.ctx)
        g.replay()
        f.s.attention(tids, all_q, lse=all_lse)
        f.s.add_weights(all_q, all_lse)
        f.s.attention(some, q, lse=lse)                  # the step's plan again, but not its weights'
        with pytest.raises(B.AparError) as e:
            B.apar_note_step_replay(f.s.ctx)
        assert e.value.code == "INVALID_ARG"
        f.s.add_weights(q, lse)
        B.apar_note_step_replay(f.s.ctx)
        g.replay()
        side.synchronize()
    # of every query each kv head's weights sum up to its heads: four steps and an attention call of two
    # threads, one call of all (a weight is off by less than 1e-4 of itself, see Forest.add)
    total = f.s.weights[0].nan_to_num(0).double().sum((0, 2)).cpu().numpy()
    assert np.abs(total - 4 * (5 * 2 + len(tids))).max() <= 4 * (10 + len(tids)) * 1e-4


def test_lists_may_be_made_beforehand():
    """Lists that int32_array made, and arrays, as the prompt's attention takes them."""
    f, tids = small_forest(8, 2)
    n = [len(f.names[t]) for t in tids[:2]]
    q, lse = rows(sum(n), 8, 5), torch.empty(sum(n), 8, device="cuda")
    lists = [tids[:2], [0, 0], n]
    f.s.prefill_attention(*lists, q, lse=lse)
    f.s.add_weights_prefill(*lists, q, lse, replace=True)
    want = f.s.read_weights(*lists)
    for made in (B.int32_array, np.array):
        args = [made(x) for x in lists]
        f.s.prefill_attention(*args, q, lse=lse)
        f.s.add_weights_prefill(*args, q, lse, replace=True)
        assert torch.equal(f.s.read_weights(*args), want)


def test_a_table_row_larger_than_the_staging_area():
    """A thread whose new blocks' ids do not fit one upload is refused; the call before it stays."""
    s = PagedSession(LayerShape(1, 1), 170020, 2, 170000, weights=True)
    a, b = s.new_threads(2)
    k = rows(1 << 16, 1, 1)
    s.append([a], [100], k[:100], k[:100])
    for _ in range(41):
        s.append([b], [1 << 16], k, k)                   # 167936 blocks
    q, lse = rows(1, 1, 2), torch.empty(1, 1, device="cuda")
    plain = s.attention([a], q, lse=lse)
    before = s.stats()
    with pytest.raises(B.AparError) as e:
        s.attention([b], q)
    assert e.value.code == "WORKSPACE_TOO_SMALL" and s.stats() == before
    s.add_weights(q, lse)
    # (weights of one query and head sum up to one; every one is off by less than 1e-4 of itself)
    assert abs(s.read_weights([a], [0], [100]).double().sum().item() - 1) <= 1e-4
    assert torch.equal(s.attention([a], q), plain)
