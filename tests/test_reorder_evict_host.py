"""Bookkeeping of apar_reorder and apar_evict against a plain model of chains: no GPU needed."""
import random

import pytest

from paper_2401_06761_b200 import binding as B


class Model:
    """A thread is a list of blocks; a block is a list of row names, the same object where shared."""

    def __init__(self):
        self.chain = {}
        self.rows = 0

    def new(self, tids):
        for t in tids:
            self.chain[t] = []

    def fresh(self):
        self.rows += 1
        return self.rows

    def append(self, t, n):
        for _ in range(n):
            if not self.chain[t] or len(self.chain[t][-1]) == 16:
                self.chain[t].append([])
            self.chain[t][-1].append(self.fresh())

    def copy(self, t):
        return [b if len(b) == 16 else list(b) for b in self.chain[t]]

    def reorder(self, tids, sources):
        old = {t: self.chain[t] for t in self.chain}
        kept = {s: s for t, s in zip(tids, sources) if t == s}
        kept.update({s: s for s in sources if s not in tids})
        for t, s in zip(tids, sources):
            if t == s:
                continue
            if s in kept:
                self.chain[t] = [b if len(b) == 16 else list(b) for b in old[s]]
            else:
                kept[s] = t
                self.chain[t] = old[s]

    def length(self, t):
        return sum(len(b) for b in self.chain[t])


def context(blocks=4000, threads=64, per_thread=200):
    return B.apar_create_host_only(B.make_config(blocks, 8, 2, threads, per_thread))


def compare(ctx, m):
    """Lengths, and which threads share which blocks."""
    B.apar_check_invariants(ctx)
    ids = {}
    used = set()
    for t, chain in m.chain.items():
        n, blocks = B.apar_get_thread(ctx, t)
        assert n == m.length(t) and len(blocks) == len(chain)
        for b, mine in zip(blocks, chain):
            assert ids.setdefault(id(mine), b) == b, (t, b)
            used.add(b)
    assert len(used) == len(ids)                        # two different blocks never have one id
    stats = B.apar_get_stats(ctx)
    assert stats["used_blocks"] == len(used)


def plans_agree(ctx, tids):
    live = [t for t in tids if B.apar_get_thread(ctx, t)[0] > 0]
    if not live:
        return
    a, b = (B.apar_debug_plan_threads(ctx, live, by) for by in (True, False))
    assert a[3] == b[3]
    assert (a[0] == b[0]).all() and (a[1] == b[1]).all() and (a[2] == b[2]).all()


@pytest.mark.parametrize("seed", range(12))
def test_random_calls(seed):
    rng = random.Random(seed)
    ctx, m = context(), Model()
    tids = B.apar_new_threads(ctx, 3)
    m.new(tids)
    for _ in range(150):
        live = list(m.chain)
        what = rng.choice(["append", "append", "fork", "reorder", "reorder", "evict", "evict", "release"])
        if what == "append":
            some = rng.sample(live, rng.randint(1, len(live)))
            counts = [rng.choice([0, 1, 3, 16, 40]) for _ in some]
            B.apar_append_kv(ctx, some, counts, 0, 0)
            for t, n in zip(some, counts):
                m.append(t, n)
        elif what == "fork" and len(live) < 30:
            parents = [rng.choice(live) for _ in range(rng.randint(1, 3))]
            for k, p in zip(B.apar_fork(ctx, parents), parents):
                m.chain[k] = m.copy(p)
        elif what == "reorder":
            some = rng.sample(live, rng.randint(1, len(live)))
            sources = [rng.choice(live if rng.random() < 0.3 else some) for _ in some]
            B.apar_reorder(ctx, some, sources)
            m.reorder(some, sources)
        elif what == "release" and len(live) > 4:
            t = rng.choice(live)
            B.apar_release(ctx, [t])
            del m.chain[t]
        elif what == "evict":
            random_evict(ctx, m, rng)
        compare(ctx, m)
        plans_agree(ctx, m.chain)


def random_evict(ctx, m, rng):
    """A stretch of one thread and, at times, of all threads that hold its blocks."""
    t = rng.choice(list(m.chain))
    n = m.length(t)
    if n == 0:
        return
    b0 = rng.randrange(0, (n - 1) // 16 + 1)
    to_end = rng.random() < 0.5
    b1 = len(m.chain[t]) if to_end else rng.randint(b0, n // 16)
    end = n if to_end else 16 * b1
    if end <= 16 * b0:
        return
    stretch = [id(b) for b in m.chain[t][b0:b1]]
    holders = [x for x, c in m.chain.items() if [id(b) for b in c[b0:b1]] == stretch
               and (not to_end or len(c) >= b1)]
    partial = [x for x, c in m.chain.items() if x not in holders and any(id(b) in stretch for b in c)]
    listed = holders if rng.random() < 0.6 else [t]
    if to_end:
        listed = [x for x in listed if m.length(x) == end]
    in_place = not partial and set(listed) == set(holders)
    keep = rng.randint(0, end - 16 * b0)
    if end < n or len(listed) > 1 or any(m.length(x) > end for x in listed):
        keep = keep // 16 * 16
    args = (listed, [16 * b0] * len(listed), [end] * len(listed), [keep] * len(listed))
    if keep == end - 16 * b0:
        before = {x: B.apar_get_thread(ctx, x) for x in m.chain}
        B.apar_evict(ctx, *args)
        assert before == {x: B.apar_get_thread(ctx, x) for x in m.chain}
        return
    if not in_place and any(m.length(x) != end for x in listed):
        with pytest.raises(B.AparError) as e:
            B.apar_evict(ctx, *args)
        assert e.value.code == "INVALID_ARG"
        return
    old = B.apar_get_thread(ctx, t)[1]
    B.apar_evict(ctx, *args)
    kb = -(-keep // 16)
    new = [[m.fresh() for _ in range(min(16, keep - 16 * j))] for j in range(kb)]
    for x in listed:
        m.chain[x] = m.chain[x][:b0] + new + m.chain[x][b1:]
    now = B.apar_get_thread(ctx, t)[1]
    if in_place:
        assert now == old[:b0 + kb] + old[b1:]
    else:
        assert not set(now[b0:]) & set(old[b0:b1])


def test_refusals_of_reorder():
    ctx = context(blocks=12)
    a, b, c = B.apar_new_threads(ctx, 3)
    B.apar_append_kv(ctx, [a, b, c], [20, 20, 120], 0, 0)      # all twelve blocks
    before = [B.apar_get_thread(ctx, t) for t in (a, b, c)]
    for args, code in (((([a, 99], [a, a])), "BAD_THREAD"), (([a], [99]), "BAD_THREAD"),
                       (([a, a], [b, b]), "INVALID_ARG"), (([a], [a, b]), "INVALID_ARG"),
                       (([a], [b]), "NO_BLOCKS")):
        with pytest.raises(B.AparError) as e:
            B.apar_reorder(ctx, *args)
        assert e.value.code == code
        assert before == [B.apar_get_thread(ctx, t) for t in (a, b, c)]
    B.apar_reorder(ctx, [a, b], [b, a])                 # no copy: the ids change places
    assert [B.apar_get_thread(ctx, t) for t in (b, a, c)] == before
    B.apar_reorder(ctx, [], [])
    B.apar_paragraph_root(ctx, c)
    for args in (([c], [a]), ([a], [c])):
        with pytest.raises(B.AparError) as e:
            B.apar_reorder(ctx, *args)
        assert e.value.code == "INVALID_ARG"


def test_refusals_of_evict():
    ctx = context()
    a, b = B.apar_new_threads(ctx, 2)
    B.apar_append_kv(ctx, [a, b], [100, 64], 0, 0)
    (c,) = B.apar_fork(ctx, [b])                        # shares all four blocks with b
    (d,) = B.apar_fork(ctx, [a])
    B.apar_release(ctx, [d])
    before = [B.apar_get_thread(ctx, t) for t in (a, b, c)]
    bad = "INVALID_ARG"
    for args, code in ((([9], [0], [1], [0]), "BAD_THREAD"), (([a, a], [0, 0], [16, 16], [0, 0]), bad),
                       (([a], [8], [100], [50]), bad), (([a], [0], [101], [50]), bad),
                       (([a], [-16], [100], [50]), bad), (([a], [32], [16], [0]), bad),
                       (([a], [0], [100], [101]), bad), (([a], [0], [100], [-1]), bad),
                       (([a], [0], [90], [32]), bad), (([a], [0], [96], [30]), bad),
                       (([b], [0], [32], [16]), bad),              # c holds the blocks, and rows follow
                       (([b, c], [0, 0], [64, 64], [30, 30]), bad),  # a partial block of two threads
                       (([b, c], [0, 0], [64, 64], [32, 16]), bad),
                       (([b, c], [0, 16], [64, 64], [32, 32]), bad),
                       (([a], [0], [100], []), bad)):
        with pytest.raises(B.AparError) as e:
            B.apar_evict(ctx, *args)
        assert e.value.code == code, args
        assert before == [B.apar_get_thread(ctx, t) for t in (a, b, c)]
    B.apar_evict(ctx, [a, b], [0, 64], [100, 64], [100, 0])    # nothing goes
    assert before == [B.apar_get_thread(ctx, t) for t in (a, b, c)]
    B.apar_evict(ctx, [b, c], [0, 0], [64, 64], [32, 32])
    assert B.apar_get_thread(ctx, b) == (32, before[1][1][:2]) == B.apar_get_thread(ctx, c)
    B.apar_check_invariants(ctx)


def test_evict_without_blocks_for_a_copy():
    ctx = context(blocks=8)
    (a,) = B.apar_new_threads(ctx, 1)
    B.apar_append_kv(ctx, [a], [96], 0, 0)
    (b,) = B.apar_fork(ctx, [a])
    with pytest.raises(B.AparError) as e:
        B.apar_evict(ctx, [b], [0], [96], [33])         # three blocks, two are free
    assert e.value.code == "NO_BLOCKS"
    B.apar_evict(ctx, [b], [0], [96], [32])
    assert B.apar_get_thread(ctx, a)[0] == 96 and B.apar_get_thread(ctx, b) == (32, [6, 7])
    B.apar_check_invariants(ctx)
