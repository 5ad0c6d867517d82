"""Beam search's selection against its definition in 64 bits, ties included."""
import numpy as np
import pytest
import torch

from paper_2401_06761_b200 import binding as B
from paper_2401_06761_b200.session import BeamSelect

pytestmark = pytest.mark.gpu

# A sum of exponentials is taken in 32 bits: a lane adds at most 130 terms one after the other in
# the cases here (each at most 2^-24 off), an exponential is at most 2^-22 off, and the lanes' sums
# go through some ten more roundings: below 150 * 2^-24 = 9e-6 of the sum, so of the logarithm.
LSE_TOL = 1e-5


def reference(logits, scores, finished, eos):
    """Values [n][beams * vocab] in 64 bits; -inf where there is no pair."""
    x = logits.double().cpu().numpy()
    n, b, v = x.shape
    s = scores.double().cpu().numpy()
    with np.errstate(all="ignore"):
        top = x.max(-1, keepdims=True)
        lse = top + np.log(np.exp(x - top).sum(-1, keepdims=True))
        value = s[..., None] + x - lse
    ok = np.isfinite(lse[..., 0]) & np.isfinite(s)
    value[~ok] = -np.inf
    if finished is not None:
        done = finished.cpu().numpy().astype(bool)
        value[done] = -np.inf
        alive = done & np.isfinite(s)
        value[..., eos][alive] = s[alive]
    return value.reshape(n, b * v)


def check(logits, scores, select, finished=None, eos=None, exact_order=False):
    n, beams, vocab = logits.shape
    got = BeamSelect(beams, vocab, select, eos)(logits, scores, finished)
    torch.cuda.synchronize()
    best, at_beam, at_token = (x.cpu().numpy() for x in got)
    value = reference(logits, scores, finished, eos)
    for i in range(n):
        order = np.lexsort((np.arange(beams * vocab), -value[i]))[:select]
        want = value[i][order]
        none = ~np.isfinite(want)
        k = int((~none).sum())
        assert np.all(best[i, k:] == -np.inf) and np.all(at_beam[i, k:] == -1) and np.all(at_token[i, k:] == -1)
        tol = LSE_TOL + np.abs(want[:k]) * 2.0 ** -24
        assert np.all(np.abs(best[i, :k] - want[:k]) <= tol), (i, best[i], want)
        flat = at_beam[i, :k].astype(np.int64) * vocab + at_token[i, :k]
        assert len(set(flat.tolist())) == k
        # the pair at a rank has that rank's value (two beams' sums may be off in opposite directions)
        assert np.all(np.abs(value[i][flat] - want[:k]) <= 2 * tol), (i, flat, order)
        if exact_order:
            assert np.array_equal(flat, order[:k]), (i, flat, order)
        else:            # equal logits of one beam: the lower token first, none left out between them
            for b in range(beams):
                mine = flat[at_beam[i, :k] == b]
                ref = [o for o in np.lexsort((np.arange(vocab), -value[i, b * vocab:(b + 1) * vocab]))[:len(mine)]]
                assert np.array_equal(mine - b * vocab, ref), (i, b, mine, ref)


def random_inputs(n, beams, vocab, dtype, seed, pad=0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    x = torch.randn(n, beams, vocab + pad, generator=g, device="cuda") * 3
    s = -10 * torch.rand(n, beams, generator=g, device="cuda")
    return x.to(dtype)[..., pad // 2:pad // 2 + vocab], s, g


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16, torch.float32])
@pytest.mark.parametrize("n,beams,vocab,select,pad", [
    (1, 1, 1, 1, 0), (2, 3, 7, 5, 0), (1, 4, 33, 64, 3), (3, 2, 255, 4, 1), (2, 4, 2049, 8, 9),
    (1, 4, 32000, 8, 0), (5, 5, 5003, 10, 6), (1, 64, 700, 64, 0), (2, 32, 1200, 64, 2),
    (70, 8, 1001, 16, 7), (1, 1, 262144, 64, 0), (300, 2, 513, 2, 0)])
def test_selection(n, beams, vocab, select, pad, dtype):
    x, s, _ = random_inputs(n, beams, vocab, dtype, n + vocab, pad)
    check(x, s, select)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_ties_go_to_the_lower_beam_then_the_lower_token(dtype):
    for vocab in (50, 4100, 20000):
        x = torch.zeros(2, 3, vocab, device="cuda", dtype=dtype)
        x[1, :, 1::2] = -0.0                             # (equal to zero)
        s = torch.zeros(2, 3, device="cuda")
        check(x, s, 40, exact_order=True)                # every value equal
        x = (torch.arange(vocab, device="cuda") % 7).to(dtype).expand(2, 3, vocab).contiguous()
        check(x, s, 64, exact_order=True)


@pytest.mark.parametrize("order", ["rising", "falling", "late"])
def test_rows_in_awkward_order(order):
    vocab = 30011
    x = torch.linspace(-5, 5, vocab, device="cuda").expand(2, 2, vocab).contiguous()
    if order == "falling":
        x = x.flip(-1).contiguous()
    elif order == "late":                                # the largest values in the last elements
        x = torch.zeros_like(x)
        x[..., -37:] = torch.arange(37, device="cuda").float() / 8
    s = torch.tensor([[0.0, -1.0], [-3.0, -3.0]], device="cuda")
    check(x, s, 64)


def test_finished_beams_and_dead_beams():
    x, s, g = random_inputs(6, 5, 901, torch.bfloat16, 3)
    done = torch.rand(6, 5, generator=g, device="cuda") < 0.4
    done[0] = True                                       # five pairs in all
    s[1, 1:] = -float("inf")                             # a search's first step: one live beam
    s[2, 0], s[2, 1], s[2, 2] = float("nan"), float("inf"), -float("inf")
    done[1:3] = False
    s[3] = -float("inf")                                 # nothing left
    check(x, s, 10, done, eos=17)
    check(x, s, 10, done.to(torch.uint8) * 3, eos=17)
    check(x, s, 10)


def test_masked_and_spoiled_logits():
    x, s, _ = random_inputs(5, 3, 4000, torch.float32, 4)
    x[0, :, 3:] = -float("inf")                          # nine pairs
    x[1, 0] = -float("inf")
    x[2, 1, 77] = float("nan")
    x[3, 2, 3999] = float("inf")
    x[4, :, ::2] = -float("inf")
    check(x, s, 16)


def test_large_and_small_logits():
    x, s, _ = random_inputs(2, 2, 3001, torch.float32, 5)
    check(x * 1e4, s, 8)
    check(x * 1e-6 + 500, s * 1e3, 8)
    check(x, s * 1e-3, 3)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16, torch.float32])
def test_masks_of_the_lowest_and_logits_of_the_largest_value(dtype):
    """A row whose logits all lie at the type's lowest value is as good as one of zeros."""
    low, high = torch.finfo(dtype).min, torch.finfo(dtype).max
    x, s, _ = random_inputs(5, 2, 9000, dtype, 11)
    x[0, :, 40:] = low                                   # most of a row, whole threads of it
    x[1, 0] = low
    x[2, 1] = high
    x[3, 0, :4500], x[3, 0, 4500:] = low, high
    x[4, 1] = low
    x[4, 1, 8999] = 0
    x = x.contiguous()
    best, beam, token = (t.cpu().numpy() for t in BeamSelect(2, 9000, 12)(x, s))
    d = x.double().cpu().numpy()
    less = d - d.max(-1, keepdims=True)                  # (before anything else: it is exact)
    value = s.double().cpu().numpy()[..., None] + (less - np.log(np.exp(less).sum(-1, keepdims=True)))
    value = value.reshape(5, -1)
    for i in range(5):
        order = np.lexsort((np.arange(18000), -value[i]))[:12]
        want = value[i][order]
        tol = LSE_TOL + np.abs(want) * 2.0 ** -24
        assert np.all(np.abs(best[i] - want) <= tol), (i, best[i], want)
        flat = beam[i].astype(np.int64) * 9000 + token[i]
        assert np.all(np.abs(value[i][flat] - want) <= 2 * tol) and len(set(flat.tolist())) == 12
        for b in range(2):                               # equal logits: the lower token first
            mine = token[i][beam[i] == b]
            ref = np.lexsort((np.arange(9000), -d[i, b]))[:len(mine)]
            assert np.array_equal(mine, ref), (i, b, mine, ref)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16, torch.float32])
def test_many_rows_whose_pieces_take_several_rounds(dtype):
    x, s, g = random_inputs(225, 8, 17003, dtype, 12, pad=5)
    x[3, :, 11:13000] = 1.0                              # more equal ones than are collected
    x[3] = x[3].clamp(max=1.0)
    x[4] = 0.0
    done = torch.rand(225, 8, generator=g, device="cuda") < 0.2
    check(x[:40], s[:40], 16, done[:40].contiguous(), eos=3)
    sel = BeamSelect(8, 17003, 16, 3)
    whole = sel(x, s, done)
    for i in range(0, 225, 45):                          # few rows are cut into pieces, many are not
        part = sel(x[i:i + 45], s[i:i + 45], done[i:i + 45])
        assert all(torch.equal(u[i:i + 45], v) for u, v in zip(whole[1:], part[1:]))
        assert torch.allclose(whole[0][i:i + 45], part[0], rtol=2.0 ** -23, atol=2 * LSE_TOL)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("beams,vocab,spread", [(32, 10000, 1.0), (64, 3000, 30.0), (16, 20000, 0.0), (64, 9000, 0.1)])
def test_wide_beams_of_different_scores(beams, vocab, spread, dtype):
    x, s, _ = random_inputs(3, beams, vocab, dtype, beams)
    check(x, s * spread, 64)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16, torch.float32])
@pytest.mark.parametrize("n,beams,vocab,select,pad", [
    (300, 2, 1, 1, 0), (200, 3, 33, 4, 1), (150, 4, 257, 64, 0), (100, 8, 1000, 64, 3), (80, 8, 2047, 16, 2),
    (600, 1, 2048, 64, 0), (40, 16, 2048, 32, 8)])
def test_many_short_rows(n, beams, vocab, select, pad, dtype):
    x, s, g = random_inputs(n, beams, vocab, dtype, n + vocab, pad)
    check(x, s, select)
    low = torch.finfo(dtype).min
    x = x.clone()
    x[0] = 1.0                                           # equal ones
    x[1, 0] = low
    x[2, :, vocab // 2:] = -float("inf")
    x[3, 0] = -float("inf")
    x[4, 0, -1] = float("nan")
    x[5, 0, 0] = float("inf")
    x[6, :, ::2] = low
    done = torch.rand(n, beams, generator=g, device="cuda") < 0.3
    done[:7] = False
    sel = BeamSelect(beams, vocab, select, 0)
    many = sel(x, s, done)
    for i in (0, 2, 3, 4, 5, 6, 7, n - 1):               # one sequence's rows take the other way
        one = sel(x[i:i + 1], s[i:i + 1], done[i:i + 1])
        assert all(torch.equal(u[i:i + 1], v) for u, v in zip(many[1:], one[1:])), i
        assert torch.allclose(many[0][i:i + 1], one[0], rtol=2.0 ** -23, atol=2 * LSE_TOL)
    rows_ok = [i for i in range(n) if i not in (1, 6)][:60]
    check(x[rows_ok].contiguous(), s[rows_ok].contiguous(), select, done[rows_ok].contiguous(), eos=0)


def test_strided_views_and_other_streams():
    x, s, _ = random_inputs(4, 3, 1000, torch.float16, 6)
    swapped = x.transpose(0, 1).contiguous().transpose(0, 1)       # beams outermost in memory
    a = BeamSelect(3, 1000, 6)(x, s)
    b = BeamSelect(3, 1000, 6)(swapped, s)
    wide = x[:1].expand(4, 3, 1000)
    c = BeamSelect(3, 1000, 6)(wide, s)
    d = BeamSelect(3, 1000, 6)(wide.contiguous(), s)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        e = BeamSelect(3, 1000, 6)(x, s)
    side.synchronize()
    torch.cuda.synchronize()
    for p, q in ((a, b), (c, d), (a, e)):
        for u, v in zip(p, q):
            assert torch.equal(u, v)


def test_two_captured_graphs_do_not_share_scratch():
    x1, s1, _ = random_inputs(2, 4, 5000, torch.bfloat16, 7)
    x2, s2, _ = random_inputs(3, 4, 5000, torch.bfloat16, 8)
    sel = BeamSelect(4, 5000, 8)
    want = [[t.clone() for t in sel(x, s)] for x, s in ((x1, s1), (x2, s2))]
    graphs, outs = [], []
    for x, s in ((x1, s1), (x2, s2)):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            outs.append(sel(x, s))
        graphs.append(g)
    streams = [torch.cuda.Stream() for _ in graphs]
    for _ in range(20):
        for g, st in zip(graphs, streams):
            with torch.cuda.stream(st):
                g.replay()
    torch.cuda.synchronize()
    for o, w in zip(outs, want):
        for u, v in zip(o, w):
            assert torch.equal(u, v)


def test_same_bits_every_time():
    x, s, _ = random_inputs(3, 8, 40000, torch.float32, 9)
    sel = BeamSelect(8, 40000, 16)
    first = sel(x, s)
    for _ in range(5):
        for u, v in zip(first, sel(x, s)):
            assert torch.equal(u, v)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_sums_of_very_long_rows(dtype):
    """Rows of 2^22 logits in two pieces: a thread adds up 8192 exponentials, all but a few of them the same, so
    that in a running 32-bit sum they round the same way (off by up to 1e-4 in the end).  LSE_TOL holds: no
    more than 64 are added up one after the other in 32 bits."""
    vocab, beams = 1 << 22, 64
    x = torch.empty(1, beams, vocab, dtype=dtype, device="cuda")
    low = -(torch.arange(beams, device="cuda") + 1).to(dtype) / 64           # (exact)
    x[:] = low[None, :, None]
    zeros = 0
    for at in range(0, vocab, vocab // 4):
        x[:, :, at:at + 65536] = 0
        zeros += 65536
    select = BeamSelect(beams, vocab, 3)
    for b in range(0, beams, 3):
        s = torch.full((1, beams), -float("inf"), device="cuda")
        s[0, b] = 0.0
        best, beam, token = select(x, s)
        want = -np.log(zeros + (vocab - zeros) * np.exp(-(b + 1) / 64))
        assert beam.tolist() == [[b] * 3] and token.tolist() == [[0, 1, 2]]
        got = best.double().cpu().numpy()
        assert np.abs(got - want).max() <= LSE_TOL + abs(want) * 2.0 ** -24, (b, got - want)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16, torch.float32])
@pytest.mark.parametrize("rise", [0.01, 3.0, 9.0])
def test_rows_that_rise_with_every_step(rise, dtype):
    """The reference of a thread's sum moves a little, by steps, or at each: rows of 100003 logits in one piece."""
    vocab, rows = 100003, 1500
    at = torch.arange(vocab, device="cuda")
    x = ((at // 1024) * rise - (at % 1024) / 512.0).to(dtype).expand(rows // 4, 4, vocab)
    scores = -0.3 * torch.arange(4, device="cuda", dtype=torch.float32).expand(rows // 4, 4).contiguous()
    best, beam, token = BeamSelect(4, vocab, 5)(x.contiguous(), scores)
    assert all(torch.equal(t, t[:1].expand_as(t)) for t in (best, beam, token))
    value = reference(x[:1], scores[:1], None, None)[0]
    order = np.lexsort((np.arange(4 * vocab), -value))[:5]
    assert beam[0].tolist() == (order // vocab).tolist() and token[0].tolist() == (order % vocab).tolist()
    tol = LSE_TOL + np.abs(value[order]) * 2.0 ** -24
    assert np.all(np.abs(best[0].cpu().numpy() - value[order]) <= tol)
