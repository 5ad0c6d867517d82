"""4-bit cache: store and read back, forks, tree attention, verification, decode steps."""
import numpy as np
import pytest
import torch

from oracle import kv4
from kv4_helpers import Kv4Pair, check, host, rows
from paper_2401_06761_b200 import binding as B
from paper_2401_06761_b200.session import PagedSession, Rope
from paper_2401_06761_b200.synth import LayerShape

pytestmark = pytest.mark.gpu


def _expect_rows(x):
    with np.errstate(all="ignore"):
        return kv4.round_bf16(kv4.values(*kv4.quantise(host(x))).astype(np.float32))


def _read_equal(sess, tids, begin, count, k, v, layer=0):
    gk, gv = sess.read_kv(tids, begin, count, layer)
    np.testing.assert_array_equal(host(gk), _expect_rows(k))
    np.testing.assert_array_equal(host(gv), _expect_rows(v))


# ------------------------------------------------------------------------------ store, read back
@pytest.mark.parametrize("hk,counts", [(1, [1]), (2, [1, 3, 0, 16]), (5, [17, 15]),
                                       (8, [33, 1, 64]), (32, [7])])
def test_rows_read_back_as_their_values(hk, counts):
    sess = PagedSession(LayerShape(hk * 2, hk), 64, 8, 16, poison=True, kv_format="q4")
    tids = sess.new_threads(len(counts))
    held = rows(5 * len(counts), hk, 1)
    sess.append(tids, [5] * len(counts), held, held)           # rows start inside a block
    k, v = rows(sum(counts), hk, 2), rows(sum(counts), hk, 3, 30.0)
    sess.append(tids, counts, k, v)
    _read_equal(sess, tids, [5] * len(counts), counts, k, v)
    _read_equal(sess, tids, [0] * len(counts), [5] * len(counts), held, held)


def _odd_rows(hk):
    """Rows whose groups are hard: equal values, ties, tiny and huge ranges, one outlier."""
    x = torch.zeros(12, hk, 128)
    g = torch.Generator().manual_seed(5)
    x[0] = 3.0                                                 # no range
    x[1] = torch.randint(0, 31, (hk, 128), generator=g) * 0.5  # s = 1 where 0 and 15 occur: ties
    x[1, :, 0::32], x[1, :, 1::32] = 0.0, 15.0
    x[2] = torch.randn(hk, 128, generator=g) * 2.0 ** -98       # scales around the smallest one kept
    x[3] = torch.randn(hk, 128, generator=g) * 1e37
    x[4, :, 7::32] = 1000.0
    x[5] = torch.randn(hk, 128, generator=g) * 1e-5
    x[5, :, 3::32] = -1.0
    x[6] = -0.0
    x[6, :, 64:] = 0.0
    x[7] = torch.randn(hk, 128, generator=g) * 1e-40           # subnormal inputs
    x[8] = torch.randint(-127, 128, (hk, 128), generator=g).float()
    x[9] = 1.0 + torch.randint(0, 3, (hk, 128), generator=g) * 2.0 ** -7   # one or two bf16 steps
    x[10] = torch.randn(hk, 128, generator=g).exp() ** 5
    x[11] = torch.randn(hk, 128, generator=g)
    return x.to(torch.bfloat16).cuda()


def test_hard_groups():
    sess = PagedSession(LayerShape(3, 3), 8, 2, 4, poison=True, kv_format="q4")
    t = sess.new_threads(1)
    x = _odd_rows(3)
    sess.append(t, [12], x, x.flip(0).contiguous())
    _read_equal(sess, t, [0], [12], x, x.flip(0))


def test_groups_that_are_not_finite_read_as_nan_and_alone():
    sess = PagedSession(LayerShape(2, 2), 8, 2, 4, poison=True, kv_format="q4")
    t = sess.new_threads(1)
    x = rows(20, 2, 9)
    x[3, 0, 40] = float("nan")
    x[4, 1, 0] = float("inf")
    x[5, 1, 127] = float("-inf")
    x[6, 0, 64], x[6, 0, 65] = 3e38, -3e38                     # the range overflows
    sess.append(t, [20], x, x)
    k, v = sess.read_kv(t, [0], [20])
    want = _expect_rows(x)
    assert np.isnan(want).sum() == 4 * 32
    np.testing.assert_array_equal(host(k), want)
    np.testing.assert_array_equal(host(v), want)


def test_read_kv_on_a_bf16_context_and_in_pieces():
    sess = PagedSession(LayerShape(4, 2), 40, 4, 20, poison=True, num_layers=2)
    t = sess.new_threads(2)
    k, v = rows(70, 2, 11), rows(70, 2, 12)
    sess.append(t, [30, 40], k, v)
    sess.append_layer(1, v, k)
    gk, gv = sess.read_kv([t[1], t[0], t[1], t[0]], [3, 29, 0, 5], [37, 1, 0, 0], layer=1)
    assert torch.equal(gk, torch.cat([v[33:70], v[29:30]]))
    assert torch.equal(gv, torch.cat([k[33:70], k[29:30]]))


def test_layers_and_forks_keep_every_row():
    """A fork copies the partial block in 4 bits, in every layer; later rows are the child's own."""
    sess = PagedSession(LayerShape(6, 3), 64, 8, 16, poison=True, num_layers=3, kv_format="q4")
    (root,) = sess.new_threads(1)
    k, v = rows(21, 3, 21), rows(21, 3, 22)
    sess.append([root], [21], k, v)
    for layer in (1, 2):
        sess.append_layer(layer, k + layer, v - layer)
    a, b = sess.fork([root, root])
    k2, v2 = rows(9, 3, 23), rows(9, 3, 24)
    sess.append([a, root], [4, 5], k2, v2)
    for layer in (1, 2):
        sess.append_layer(layer, k2 + layer, v2 - layer)
    for layer in (0, 1, 2):
        kk, vv = torch.cat([k, k2]) + layer, torch.cat([v, v2]) - layer
        _read_equal(sess, [b], [0], [21], kk[:21], vv[:21], layer)
        _read_equal(sess, [a], [0], [25], kk[:25], vv[:25], layer)
        _read_equal(sess, [root], [0], [26], torch.cat([kk[:21], kk[25:]]),
                    torch.cat([vv[:21], vv[25:]]), layer)


# ------------------------------------------------------------------------------------- attention
# query heads per kv head of a single thread decide which kernel takes it: up to four rows, up to
# eight, more
WIDTHS = [(4, 2), (16, 2), (32, 2)]


@pytest.mark.parametrize("hq,hk", [(2, 2), (8, 2), (6, 1), (32, 8), (40, 40), (64, 1), (24, 2)])
@pytest.mark.parametrize("length", [1, 15, 16, 17, 63, 130, 600])
def test_single_threads(hq, hk, length):
    p = Kv4Pair(hq, hk)
    tids = p.new_threads(2)
    p.append(tids, [length, 1], rows(length + 1, hk, length), rows(length + 1, hk, length + 1))
    p.check_attention(tids, rows(2, hq, 7))
    p.check_books()
    p.close()


@pytest.mark.parametrize("hq,hk,children,prompt", [(8, 2, 3, 64), (4, 4, 4, 70), (16, 2, 9, 200),
                                                   (8, 1, 17, 33), (3, 3, 33, 48), (64, 8, 8, 300)])
def test_forest(hq, hk, children, prompt):
    p = Kv4Pair(hq, hk, num_blocks=1024, max_threads=128)
    roots = p.new_threads(2)
    p.append(roots, [prompt, prompt + 5], rows(2 * prompt + 5, hk, 31), rows(2 * prompt + 5, hk, 32))
    kids = p.fork([roots[i % 2] for i in range(2 * children)])
    counts = [1 + (i * 7) % 40 for i in range(len(kids))]
    p.append(kids, counts, rows(sum(counts), hk, 33), rows(sum(counts), hk, 34))
    grand = p.fork(kids[:3])
    p.append(grand, [1, 20, 16], rows(37, hk, 35), rows(37, hk, 36))
    live = kids + grand
    p.check_attention(live, rows(len(live), hq, 37))
    # a thread listed twice, and the parents among the queries
    some = [live[0], roots[0], live[0], grand[1]]
    p.check_attention(some, rows(4, hq, 38))
    p.release(kids[1:4])
    live = [t for t in live if t not in kids[1:4]]
    p.check_attention(live, rows(len(live), hq, 39))
    p.check_books()
    p.close()


@pytest.mark.parametrize("hq,hk", WIDTHS)
@pytest.mark.parametrize("scale", [0.0, -0.11, 0.7])
def test_scale_argument(scale, hq, hk):
    p = Kv4Pair(hq, hk)
    tids = p.new_threads(2)
    p.append(tids, [77, 200], rows(277, hk, 41), rows(277, hk, 42))
    p.check_attention(tids, rows(2, hq, 43), scale=scale)
    p.close()


@pytest.mark.parametrize("hq,hk", WIDTHS)
def test_scores_that_grow_along_the_chain(hq, hk):
    """The reference of the softmax has to move again and again."""
    p = Kv4Pair(hq, hk, num_blocks=128)
    (t,) = p.new_threads(1)
    k = rows(700, 2, 44) * 0.1 + torch.linspace(0, 4, 700, device="cuda")[:, None, None]
    q = torch.ones(1, hq, 128, device="cuda")
    q[:, hq // 2:] = -1.0
    p.append([t], [700], k.to(torch.bfloat16), rows(700, 2, 45))
    p.check_attention([t], q.to(torch.bfloat16))
    p.close()


@pytest.mark.parametrize("hq,hk", WIDTHS)
@pytest.mark.parametrize("order", ["rising", "falling", "mixed"])
def test_v_rows_of_very_different_size(order, hq, hk):
    """Scales of V from 2^-75 to 2^30: the reference follows score and scale together."""
    p = Kv4Pair(hq, hk, num_blocks=128)
    (t,) = p.new_threads(1)
    n = 180
    e = torch.linspace(-75, 30, n)
    if order == "falling":
        e = e.flip(0)
    if order == "mixed":
        e = e[torch.randperm(n, generator=torch.Generator().manual_seed(3))]
    v = rows(n, 2, 46).float() * torch.exp2(e).cuda()[:, None, None]
    v[::9] = v[::9, :, :1]                                     # rows of equal values: scale 0
    p.append([t], [n], rows(n, 2, 47), v.to(torch.bfloat16))
    p.check_attention([t], rows(1, hq, 48))
    p.close()


@pytest.mark.parametrize("hq,hk", WIDTHS)
def test_small_v_rows_with_all_the_weight(hq, hk):
    """The large rows have next to no weight: what remains is small and has to be exact."""
    p = Kv4Pair(hq, hk, num_blocks=64)
    (t,) = p.new_threads(1)
    k = torch.zeros(200, 2, 128)
    k[100:, :, 0::2] = 1.0
    v = rows(200, 2, 49).float()
    v[:100] *= 1024.0
    v[100:] *= 2.0 ** -12
    q = torch.full((1, hq, 128), 16.0)
    p.append([t], [200], k.to(torch.bfloat16).cuda(), v.to(torch.bfloat16))
    p.check_attention([t], q.to(torch.bfloat16).cuda())
    p.close()


@pytest.mark.parametrize("hq,hk", WIDTHS)
def test_a_nan_row_reaches_only_the_threads_that_see_it(hq, hk):
    for side in ("k", "v"):
        p = Kv4Pair(hq, hk)
        (root,) = p.new_threads(1)
        p.append([root], [40], rows(40, 2, 51), rows(40, 2, 52))
        a, b = p.fork([root, root])
        k, v = rows(12, 2, 53), rows(12, 2, 54)
        p.append([a], [6], k[:6], v[:6])
        bad = k.clone() if side == "k" else v.clone()
        bad[8, 1, 35] = float("nan")
        p.sess.append([b], [6], (bad if side == "k" else k)[6:].contiguous(),
                      (bad if side == "v" else v)[6:].contiguous())
        q = rows(2, hq, 55)
        out = p.sess.attention([a, b], q)
        check(out[:1], *p.expected([a], q[:1], p.sess.sm_scale))
        got, h = torch.isnan(out[1].float()), hq // 2
        assert not got[:h].any()                               # the other kv head
        if side == "k":
            assert got[h:].all()
        else:                                                  # the other groups are untouched
            assert got[h:, 32:64].all() and not got[h:, :32].any() and not got[h:, 64:].any()
        p.close()


def test_prefix_attention():
    p = Kv4Pair(8, 2)
    (t,) = p.new_threads(1)
    n = 50
    k, v = rows(n, 2, 61), rows(n, 2, 62)
    p.append([t], [n], k, v)
    q = rows(n, 8, 63)
    got = p.sess.prefix_attention([t] * n, list(range(1, n + 1)), q)
    for i in (0, 1, 14, 15, 16, 17, 31, 32, 49):
        ref = Kv4Pair(8, 2)
        (u,) = ref.new_threads(1)
        ref.note_append([u], [i + 1], k[:i + 1], v[:i + 1])
        check(got[i:i + 1], *ref.expected([u], q[i:i + 1], p.sess.sm_scale), f"position {i}")
        ref.close()
    p.close()


@pytest.mark.parametrize("hq,hk,held", [(8, 2, 37), (4, 4, 0), (32, 8, 160)])
def test_verification_and_acceptance(hq, hk, held):
    """Each candidate is a thread of its own in the checker, forked from its parent candidate."""
    p = Kv4Pair(hq, hk, num_blocks=512, max_threads=128)
    roots = p.new_threads(1)
    if held:
        p.append(roots, [held], rows(held, hk, 71), rows(held, hk, 72))
    tids = p.sess.fork([roots[0], roots[0]])
    parents = [[-1, 0, 0, 1, 3, -1, 5], [-1, -1, 1]]
    counts = [len(x) for x in parents]
    k, v = rows(10, hk, 73), rows(10, hk, 74)
    p.sess.append(tids, counts, k, v)
    masks, refs, at = [], [], 0
    for mine in parents:
        node, bits = [], []
        for j, par in enumerate(mine):
            src = roots[0] if par < 0 else node[par]
            node.append(p.ref.fork([src])[0])
            assert p.mid.fork([src])[0] == node[-1]
            p.note_append([node[-1]], [1], k[at + j:at + j + 1], v[at + j:at + j + 1])
            bits.append((1 << j) | (bits[par] if par >= 0 else 0))
        masks += bits
        refs += node
        at += len(mine)
    q = rows(10, hq, 75)
    for _ in range(2):                                         # the call changes nothing
        got = p.sess.verify_attention(tids, counts, masks, q)
        check(got, *p.expected(refs, q, p.sess.sm_scale))
    p.sess.accept(tids, counts, [[1, 3, 4], [2]])
    _read_equal(p.sess, tids, [held, held], [3, 1], k[[1, 3, 4, 9]], v[[1, 3, 4, 9]])
    assert [p.sess.thread(t)[0] for t in tids] == [held + 3, held + 1]
    p.close()


def test_sixty_four_candidates():
    p = Kv4Pair(8, 2, num_blocks=64, max_threads=128)
    (t,) = p.new_threads(1)
    k, v = rows(64, 2, 81), rows(64, 2, 82)
    p.append([t], [64], k, v)
    q = rows(64, 8, 83)
    got = p.sess.verify_attention([t], [64], [(1 << (j + 1)) - 1 for j in range(64)], q)
    want = p.sess.prefix_attention([t] * 64, list(range(1, 65)), q)
    # two kernels for the same sums: each within half a bf16 step of the same number, so one step
    assert (got.float() - want.float()).abs().max() <= 2.0 ** -7 * want.float().abs().max()
    p.close()


# ------------------------------------------------------------- steps, layers, graphs, all together
def _positions(p, tids):
    return torch.tensor([p.ref.model.lens[t] for t in tids], dtype=torch.int32, device="cuda")


def test_decode_steps_with_rotary_positions_over_layers_and_forks():
    """What a decode loop does: rotate, one step over all threads, the other layers, fork, again;
    and the rows of the cache read back at the end."""
    layers, hq, hk = 2, 16, 4
    rope = Rope(rotary_dim=64, layout="interleaved", base=10000.0)
    pairs = [Kv4Pair(hq, hk, num_blocks=256, num_layers=layers if i == 0 else 1) for i in range(layers)]
    sess = pairs[0].sess
    for p in pairs:
        (root,) = p.new_threads(1)
    prompt = [(rows(37, hk, 90 + i), rows(37, hk, 95 + i)) for i in range(layers)]
    pos = torch.arange(37, dtype=torch.int32, device="cuda")
    turned = [rope(k, None, pos)[0] for k, _ in prompt]
    sess.append([root], [37], turned[0], prompt[0][1])
    sess.append_layer(1, turned[1], prompt[1][1])
    for i, p in enumerate(pairs):
        p.note_append([root], [37], turned[i], prompt[i][1])
    tids = [root]
    for step in range(20):
        if step in (0, 3, 12):
            tids = tids + sess.fork(tids)
            for i, p in enumerate(pairs):
                kids = p.ref.fork(tids[:len(tids) // 2])
                assert kids == p.mid.fork(tids[:len(tids) // 2]) == tids[len(tids) // 2:]
        n = len(tids)
        pos = _positions(pairs[0], tids)
        for i, p in enumerate(pairs):
            qkv = rows(n, hq + 2 * hk, 1000 + 10 * step + i)
            q, k = rope(qkv[:, :hq], qkv[:, hq:hq + hk], pos)
            v = qkv[:, hq + hk:].contiguous()
            if i == 0:
                out = sess.decode_step(tids, k, v, q)
            else:
                sess.append_layer(i, k, v)
                out = sess.attention_layer(i, q)
            p.note_append(tids, [1] * n, k, v)
            check(out, *p.expected(tids, q, sess.sm_scale), f"step {step} layer {i}")
    pairs[0].check_books()
    for p in pairs:
        p.close()


@pytest.mark.parametrize("hq,hk", WIDTHS)
def test_captured_step_replays(hq, hk):
    n = 5
    p = Kv4Pair(hq, hk, num_blocks=64)
    tids = p.new_threads(n)
    k, v = rows(18 * n, hk, 101), rows(18 * n, hk, 102)
    p.append(tids, [18] * n, k, v)
    kb, vb, qb = rows(n, hk, 103), rows(n, hk, 104), rows(n, hq, 105)
    out = p.sess.decode_step(tids, kb, vb, qb)                 # the list becomes resident
    p.note_append(tids, [1] * n, kb, vb)
    check(out, *p.expected(tids, qb, p.sess.sm_scale))
    stream, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=stream):
        p.sess.decode_step(tids, kb, vb, qb, out=out)
    for step in range(4):
        for buf, seed in ((kb, 110), (vb, 120), (qb, 130)):
            buf.copy_(rows(n, buf.shape[1], seed + step))
        if step:
            B.apar_note_step_replay(p.sess.ctx)
        graph.replay()
        torch.cuda.synchronize()
        p.note_append(tids, [1] * n, kb, vb)
        check(out, *p.expected(tids, qb, p.sess.sm_scale), f"replay {step}")
    with pytest.raises(B.AparError):                           # staging is needed: not capturable
        with torch.cuda.graph(torch.cuda.CUDAGraph(), stream=stream):
            p.sess.read_kv(tids, [0] * n, [1] * n)
    torch.cuda.synchronize()
    del graph
    p.close()


def test_offsets_past_32_bits():
    """A pool above 4 GiB: threads whose blocks lie at its end."""
    hq, hk, blocks = 32, 32, 106000
    sess = PagedSession(LayerShape(hq, hk), blocks, 4, 105000, kv_format="q4")
    assert sess.k_pool.numel() > 2 ** 32
    filler, t = sess.new_threads(2)
    junk = rows(8192, hk, 141)
    for _ in range(105000 * 16 // 8192):
        sess.append([filler], [8192], junk, junk)
    k, v, q = rows(300, hk, 142), rows(300, hk, 143), rows(1, hq, 144)
    sess.append([t], [300], k, v)
    assert min(sess.thread(t)[1]) * hk * 1280 > 2 ** 32
    (c,) = sess.fork([t])
    _read_equal(sess, [c], [0], [300], k, v)
    small = Kv4Pair(hq, hk)
    (u,) = small.new_threads(1)
    small.note_append([u], [300], k, v)
    for x in (t, c):
        check(sess.attention([x], q), *small.expected([u], q, sess.sm_scale))
    small.close()
    sess.close()


def test_large_groups_of_items_and_long_chains():
    """Chunked long chains, partial results merged; more than 16 tiles of items."""
    p = Kv4Pair(16, 2, num_blocks=4096, max_threads=64, max_blocks=1024)
    tids = p.new_threads(3)
    counts = [9001, 130, 4096]
    p.append(tids, counts, rows(sum(counts), 2, 151), rows(sum(counts), 2, 152))
    p.check_attention(tids, rows(3, 16, 153))
    kids = p.fork([tids[0]] * 20)
    p.append(kids, [3] * 20, rows(60, 2, 154), rows(60, 2, 155))
    p.check_attention(kids, rows(20, 16, 156))
    p.close()


@pytest.mark.parametrize("hq,hk,requests,children", [(64, 16, 40, 4), (128, 16, 30, 4), (40, 40, 16, 3)])
def test_more_units_than_one_round(hq, hk, requests, children):
    """Every warp and every CTA works through several units, forwards and backwards: shared
    prompts on the wide kernel, tails of four, eight and one row."""
    p = Kv4Pair(hq, hk, num_blocks=2048, max_threads=256, max_blocks=32)
    roots = p.new_threads(requests)
    lens = [97 + 16 * (i % 5) + i for i in range(requests)]
    p.append(roots, lens, rows(sum(lens), hk, 171), rows(sum(lens), hk, 172))
    kids = p.fork([r for r in roots for _ in range(children)])
    counts = [1 + (11 * i) % 70 for i in range(len(kids))]
    p.append(kids, counts, rows(sum(counts), hk, 173), rows(sum(counts), hk, 174))
    q = rows(len(kids), hq, 175)
    got = p.sess.attention(kids, q)
    again = p.sess.attention(kids, q)
    assert torch.equal(got, again)                             # the same sums in the same order
    some = list(range(0, len(kids), 7)) + [len(kids) - 1]
    check(got[some], *p.expected([kids[i] for i in some], q[some], p.sess.sm_scale))
    p.check_books()
    p.close()


@pytest.mark.parametrize("children", [6, 7, 18, 22, 23])
def test_runs_whose_rows_fill_wide_units_and_leave_a_rest(children):
    """24, 28, 64 + 8, 64 + 24 and 64 + 28 rows on a shared prompt, with work enough for wide units."""
    hq, hk, requests, held = 64, 16, 6, 401
    p = Kv4Pair(hq, hk, num_blocks=1024, max_threads=256, max_blocks=32)
    roots = p.new_threads(requests)
    p.append(roots, [held] * requests, rows(held * requests, hk, 191), rows(held * requests, hk, 192))
    kids = p.fork([r for r in roots for _ in range(children)])
    n = len(kids)
    p.append(kids, [2] * n, rows(2 * n, hk, 193), rows(2 * n, hk, 194))
    q = rows(n, hq, 195)
    got = p.sess.attention(kids, q)
    some = [i for i in range(n) if i % children in (0, 1, 15, 16, 17, 21, children - 1)][:2 * children]
    check(got[some], *p.expected([kids[i] for i in some], q[some], p.sess.sm_scale))
    p.close()


@pytest.mark.parametrize("hq,hk", WIDTHS)
def test_a_thread_listed_several_times(hq, hk):
    p = Kv4Pair(hq, hk)
    t, u = p.new_threads(2)
    p.append([t, u], [70, 33], rows(103, hk, 201), rows(103, hk, 202))
    p.check_attention([t, u, t, t, u] * 3, rows(15, hq, 203))
    (c,) = p.fork([t])
    p.append([c], [1], rows(1, hk, 204), rows(1, hk, 205))
    p.check_attention([c, t, c], rows(3, hq, 206))
    p.close()


def test_one_long_chain_on_one_kv_head():
    """More chunks than partial-result rows: the chunks grow until they fit."""
    p = Kv4Pair(4, 1, num_blocks=20000, max_threads=4, max_blocks=20000)
    (t,) = p.new_threads(1)
    n = 250007
    k, v, q = rows(n, 1, 181), rows(n, 1, 182), rows(1, 4, 183)
    p.append([t], [n], k, v)
    got = p.sess.attention([t], q)
    check(got, *p.expected([t], q, p.sess.sm_scale))
    p.close()


# -------------------------------------------------------------------------------------- refusals
def test_refusals():
    sess = PagedSession(LayerShape(8, 2), 16, 4, 4, kv_format="q4")
    (t,) = sess.new_threads(1)
    k, q = rows(20, 2, 161), rows(1, 8, 162)
    sess.append([t], [20], k, k)
    before = sess.stats()["kernels_total"]

    def refused(code, f, *args):
        with pytest.raises(B.AparError) as e:
            f(*args)
        assert e.value.code == code

    out = torch.empty_like(q)
    odd = out.data_ptr() + 2
    refused("UNSUPPORTED", sess.prefill_attention, [t], [0], [20], rows(20, 8, 163))
    refused("INVALID_ARG", B.apar_tree_decode_attention, sess.ctx, [t], odd, out.data_ptr(), 1.0)
    refused("INVALID_ARG", B.apar_tree_decode_attention, sess.ctx, [t], q.data_ptr(), odd, 1.0)
    refused("INVALID_ARG", B.apar_append_kv, sess.ctx, [t], [1], odd, k.data_ptr())
    refused("INVALID_ARG", B.apar_append_kv_layer, sess.ctx, 0, k.data_ptr(), odd)
    refused("INVALID_ARG", B.apar_append_kv_layer, sess.ctx, 1, k.data_ptr(), k.data_ptr())
    refused("INVALID_ARG", B.apar_read_kv, sess.ctx, 0, [t], [0], [21], out.data_ptr(), out.data_ptr())
    refused("INVALID_ARG", B.apar_read_kv, sess.ctx, 0, [t], [-1], [1], out.data_ptr(), out.data_ptr())
    refused("INVALID_ARG", B.apar_read_kv, sess.ctx, 0, [t], [0], [1], odd, out.data_ptr())
    refused("INVALID_ARG", B.apar_read_kv, sess.ctx, 1, [t], [0], [1], out.data_ptr(), out.data_ptr())
    refused("BAD_THREAD", B.apar_read_kv, sess.ctx, 0, [t + 1], [0], [1], out.data_ptr(), out.data_ptr())
    refused("TABLE_FULL", sess.append, [t], [60], rows(60, 2, 164), rows(60, 2, 165))
    assert sess.stats()["kernels_total"] == before
    with pytest.raises(B.AparError):
        B.apar_create_kv(sess.cfg, 2)
    sess.close()


def test_read_kv_refuses_lists_of_different_lengths_and_negative_counts():
    sess = PagedSession(LayerShape(4, 2), 16, 4, 4, kv_format="q4")
    t, u = sess.new_threads(2)
    k = rows(10, 2, 221)
    sess.append([t, u], [5, 5], k, k)
    for args in (([t, u], [0], [5, 5]), ([t, u], [0, 0], [5]), ([t], [0, 0], [5, 5]), ([t, u], [0, 0], [5, -1]),
                 ([t, u], [0, 0], [-5, -5])):
        with pytest.raises(B.AparError) as e:
            sess.read_kv(*args)
        assert e.value.code == "INVALID_ARG"
    sess.close()


@pytest.mark.parametrize("fmt", ["q4", "bf16"])
def test_read_kv_of_no_rows(fmt):
    sess = PagedSession(LayerShape(4, 2), 16, 4, 4, kv_format=fmt)
    t, u = sess.new_threads(2)
    k = rows(5, 2, 231)
    sess.append([t], [5], k, k)
    for args in (([], [], []), ([t], [5], [0]), ([u, t], [0, 2], [0, 0])):
        gk, gv = sess.read_kv(*args)
        assert gk.shape == gv.shape == (0, 2, 128)
    for args in (([t], [6], [0]), ([t], [0], [6])):
        with pytest.raises(B.AparError):
            sess.read_kv(*args)
    with pytest.raises(B.AparError):
        B.apar_read_kv(sess.ctx, 0, [t], [0], [1], 0, 0)
    sess.close()


@pytest.mark.parametrize("fmt", ["q4", "bf16"])
def test_read_kv_of_more_rows_than_one_upload_lists(fmt):
    """2^18 rows go to a launch; the next one begins inside an entry."""
    sess = PagedSession(LayerShape(1, 1), 160, 4, 140, kv_format=fmt)
    (t,) = sess.new_threads(1)
    n, times = 2000, 140
    k, v = rows(n, 1, 232), rows(n, 1, 233)
    sess.append([t], [n], k, v)
    gk, gv = sess.read_kv([t] * times, [0] * times, [n] * times)
    for got, x in ((gk, k), (gv, v)):
        want = torch.from_numpy(_expect_rows(x)).to(torch.bfloat16).cuda() if fmt == "q4" else x
        assert torch.equal(got.view(times, n, 1, 128), want.expand(times, n, 1, 128))
    sess.close()


def test_the_current_stream_with_and_without_the_short_way(monkeypatch):
    from paper_2401_06761_b200 import session
    for short in (session._raw_stream, None):
        monkeypatch.setattr(session, "_raw_stream", short)
        stream = torch.cuda.Stream()
        assert PagedSession._stream() == torch.cuda.current_stream().cuda_stream
        with torch.cuda.stream(stream):
            assert PagedSession._stream() == stream.cuda_stream
