"""Calls on a 4-bit cache large enough that runs of more than three 8-row units go to the kernel for
wide items: verification, prefix attention, several rounds of shared prompts."""
import numpy as np
import pytest
import torch

from kv4_helpers import Kv4Pair, check, rows
from oracle import dense_attention

pytestmark = pytest.mark.gpu


def _candidate_tree(rng, n):
    """Parents (-1: the thread's last token) and ancestor masks of n candidates."""
    parents = [int(rng.integers(-1, j)) if j else -1 for j in range(n)]
    masks = []
    for j, par in enumerate(parents):
        masks.append((1 << j) | (masks[par] if par >= 0 else 0))
    return parents, masks


def _check_candidates(p, root, got, parents, k, v, q):
    """Each candidate is a thread of its own in the oracle, forked from its parent candidate."""
    node = []
    for j, par in enumerate(parents):
        src = root if par < 0 else node[par]
        node.append(p.ref.fork([src])[0])
        assert p.mid.fork([src])[0] == node[-1]
        p.note_append([node[-1]], [1], k[j:j + 1], v[j:j + 1])
    check(got, *p.expected(node, q, p.sess.sm_scale))
    p.ref.release(node[::-1])
    p.mid.release(node[::-1])


@pytest.mark.parametrize("hq,hk,requests,prompt,children,cands", [
    (32, 8, 4, 200, 2, 26), (64, 8, 3, 130, 2, 13), (16, 4, 4, 0, 2, 64), (8, 8, 8, 300, 3, 64),
    (32, 2, 6, 500, 2, 9)])
def test_verification_packs_candidates_of_several_threads(hq, hk, requests, prompt, children, cands):
    rng = np.random.default_rng(7)
    p = Kv4Pair(hq, hk, num_blocks=4096, max_threads=requests * (children * cands + 1 + children) + 64,
                max_blocks=128)
    roots = p.new_threads(requests)
    if prompt:
        p.append(roots, [prompt] * requests, rows(requests * prompt, hk, 11), rows(requests * prompt, hk, 12))
    tids = p.fork([r for r in roots for _ in range(children)])
    held = [70 + 13 * i for i in range(len(tids))]
    if not prompt:
        held = [h + 240 for h in held]
    p.append(tids, held, rows(sum(held), hk, 13), rows(sum(held), hk, 14))
    n = len(tids) * cands
    k, v, q = rows(n, hk, 15), rows(n, hk, 16), rows(n, hq, 17)
    p.sess.append(tids, [cands] * len(tids), k, v)
    trees = [_candidate_tree(rng, cands) for _ in tids]
    if cands == 64:                                            # one long chain among them
        trees[1] = (list(range(-1, 63)), [(1 << (j + 1)) - 1 for j in range(64)])
    masks = [m for _, mine in trees for m in mine]
    got = p.sess.verify_attention(tids, [cands] * len(tids), masks, q)
    assert torch.equal(got, p.sess.verify_attention(tids, [cands] * len(tids), masks, q))
    st = p.sess.stats()
    # wide items and the merge at least; fewer items than 8-row units say that rows were packed wider
    assert st["attn_kernels"] >= 2 and st["device_wait_timeouts"] == 0
    units = sum(-(-c * cands * (hq // hk) // 8) for c in [children] * requests * bool(prompt) + [1] * len(tids))
    assert st["attn_work_items"] < units
    for i in (0, 1, len(tids) - 1):
        at = slice(i * cands, (i + 1) * cands)
        _check_candidates(p, tids[i], got[at], trees[i][0], k[at], v[at], q[at])
    p.close()


@pytest.mark.parametrize("hq,hk", [(32, 8), (64, 8), (8, 8)])
def test_prefix_attention_at_many_positions(hq, hk):
    p = Kv4Pair(hq, hk, num_blocks=256, max_threads=512, max_blocks=64)
    (root,) = p.new_threads(1)
    p.append([root], [333], rows(333, hk, 21), rows(333, hk, 22))
    (kid,) = p.fork([root])
    p.append([kid], [100], rows(100, hk, 23), rows(100, hk, 24))
    tids = [root] * 120 + [kid] * 380
    lens = list(range(214, 334)) + list(range(54, 434))
    q = rows(500, hq, 25)
    got = p.sess.prefix_attention(tids, lens, q)
    assert torch.equal(got, p.sess.prefix_attention(tids, lens, q))        # (tables are there by now)
    st = p.sess.stats()
    assert st["attn_kernels"] == 3 and st["device_wait_timeouts"] == 0     # wide, narrow, merge
    for i in (0, 1, 119, 120, 121, 130, 131, 398, 399, 400, 401, 499):
        K, V = p.ref.forest.chain(p.ref.node_of[tids[i]])
        _, M = p.mid.forest.chain(p.mid.node_of[tids[i]])
        qi = q[i].detach().double().cpu().numpy()
        n = lens[i]
        check(got[i:i + 1], dense_attention(qi, K[:n], V[:n], p.sess.sm_scale)[None],
              dense_attention(qi, K[:n], M[:n], p.sess.sm_scale)[None], f"query {i}")
    p.close()


@pytest.mark.parametrize("hq,hk,requests,children", [(64, 16, 40, 12), (128, 16, 30, 12), (40, 40, 8, 40)])
def test_shared_prompts_over_several_rounds_of_wide_units(hq, hk, requests, children):
    p = Kv4Pair(hq, hk, num_blocks=4096, max_threads=1024, max_blocks=32)
    roots = p.new_threads(requests)
    lens = [97 + 16 * (i % 5) + i for i in range(requests)]
    p.append(roots, lens, rows(sum(lens), hk, 31), rows(sum(lens), hk, 32))
    kids = p.fork([r for r in roots for _ in range(children)])
    counts = [1 + (11 * i) % 70 for i in range(len(kids))]
    p.append(kids, counts, rows(sum(counts), hk, 33), rows(sum(counts), hk, 34))
    q = rows(len(kids), hq, 35)
    got = p.sess.attention(kids, q)
    assert torch.equal(got, p.sess.attention(kids, q))
    st = p.sess.stats()
    assert st["attn_kernels"] == 3 and st["device_wait_timeouts"] == 0     # wide, narrow, merge
    some = list(range(0, len(kids), 37)) + [len(kids) - 1]
    check(got[some], *p.expected([kids[i] for i in some], q[some], p.sess.sm_scale))
    p.check_books()
    p.close()
