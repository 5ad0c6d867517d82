"""Measured cases of beam search's selection, the weights that cached keys receive, and eviction by them.

Five kinds of case.  All but the first run on attention layers with 128-dim heads.

  beam     one step of beam search: of all (beam, token) pairs of a sequence those with the highest
           score, a pair's score being its beam's score plus the token's log-probability.
  reorder  the chosen pairs' beams go on: every beam takes over the cached rows of the beam that its
           new token was chosen for, and the new tokens' queries attend over them.
  weights  decode attention's probabilities, summed per key over the queries that see it: one query
           per live thread of a forest of forked threads, prompts shared between the threads forked
           from them.  The log-sum-exps of the scores are at hand from the attention itself.
  prompt   the same sums for runs of consecutive queries, each of which sees the keys up to its own
           position: whole prompts, or a window of queries at the end of a long context.
  evict    of the rows of a stretch of each thread's cache, per layer and kv head, those with the
           largest weights are kept and moved up into one stretch.

Order of kept rows: a kept row that lies within the first `keep` of the stretch stays at its place;
the others, in order, take the places of the rows that go.  Equal weights: the earlier row is kept.
Equal scores: the lower beam first, then the lower token.  A finished beam has one continuation, the
end token, at its own score.

Shapes of heads and trees are those of the benchmark's configurations (GQA 8/2, MHA 32, MHA 40,
GQA 64/8, GQA 32/8) at request counts that keep one pass short; values are random.
"""
import math
import random

import torch

own = False

DIM = 128
HEADS = ((8, 2), (32, 32), (40, 40), (64, 8), (32, 8))
TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
SCALE = 1.0 / math.sqrt(DIM)


# ------------------------------------------------------------------------------------- the cases
def listed():
    return [
        # one request with four beams: only latency counts
        {"name": "beam_1x4", "kind": "beam", "seqs": 1, "beams": 4, "vocab": 32000, "select": 8,
         "type": "bf16", "pad": 0, "finished": 0.0},
        # a serving batch over a large vocabulary
        {"name": "beam_32x4_large_vocab", "kind": "beam", "seqs": 32, "beams": 4, "vocab": 131072,
         "select": 8, "type": "bf16", "pad": 0, "finished": 0.0},
        # many sequences with wide beams, logits in 32 bits, an odd vocabulary whose rows lie in a
        # padded array, some beams at their end already
        {"name": "beam_256x8_f32_odd", "kind": "beam", "seqs": 256, "beams": 8, "vocab": 32003,
         "select": 16, "type": "f32", "pad": 13, "finished": 0.2},
        # the step after a selection: two of four beams go on, and the new tokens attend
        {"name": "reorder_1x4", "kind": "reorder", "seqs": 1, "beams": 4, "prompt": 61,
         "tail_min": 40, "tail_max": 40, "hq": 8, "hk": 2, "shape_seed": 9},
        {"name": "reorder_48x8", "kind": "reorder", "seqs": 48, "beams": 8, "prompt": 1500,
         "tail_min": 50, "tail_max": 400, "hq": 32, "hk": 8, "shape_seed": 10},
        # the threads of one short request
        {"name": "weights_3", "kind": "weights", "requests": 1, "prompt": 64, "children": 3,
         "tail_min": 20, "tail_max": 40, "hq": 8, "hk": 2, "shape_seed": 1},
        # a serving batch: prompts shared by four threads each
        {"name": "weights_64x4", "kind": "weights", "requests": 64, "prompt": 2048, "children": 4,
         "tail_min": 128, "tail_max": 512, "hq": 32, "hk": 8, "shape_seed": 2},
        # whole prompts, as many kv heads as query heads
        {"name": "prompt_8x2048", "kind": "prompt", "threads": 8, "len_min": 1500, "len_max": 2048,
         "window": 0, "hq": 32, "hk": 32, "shape_seed": 4},
        # a window of 32 queries at the end of long contexts
        {"name": "prompt_window32", "kind": "prompt", "threads": 8, "len_min": 9000,
         "len_max": 16000, "window": 32, "hq": 64, "hk": 8, "shape_seed": 5},
        # a short thread, where only latency counts
        {"name": "evict_1x300", "kind": "evict", "threads": 1, "len_min": 300, "len_max": 300,
         "keep": 130, "begin": 16, "layers": 1, "hq": 8, "hk": 2, "shape_seed": 6},
        # a batch brought back to half its rows, in every layer at once
        {"name": "evict_32x2048", "kind": "evict", "threads": 32, "len_min": 1800, "len_max": 2048,
         "keep": 900, "begin": 16, "layers": 2, "hq": 32, "hk": 8, "shape_seed": 7},
        # one very long context of which little stays
        {"name": "evict_long", "kind": "evict", "threads": 1, "len_min": 131000, "len_max": 131000,
         "keep": 8192, "begin": 0, "layers": 1, "hq": 64, "hk": 8, "shape_seed": 8},
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["beam", "reorder", "weights", "prompt", "evict"])
    seed = rng.randrange(1, 1 << 30)
    if kind == "beam":
        beams, vocab = rng.choice([1, 2, 3, 4, 5, 8, 16, 32]), _log_int(rng, 500, 262144)
        seqs = _log_int(rng, 1, max(1, 65000000 // (beams * vocab)))
        return {"kind": kind, "seqs": min(seqs, 2000), "beams": beams, "vocab": vocab,
                "select": rng.choice([beams, 2 * beams]), "type": rng.choice(["bf16", "f16", "f32"]),
                "pad": rng.choice([0, 0, 1, 8, 24]), "finished": rng.choice([0.0, 0.0, 0.25])}
    hq, hk = HEADS[rng.randrange(len(HEADS))]
    if kind == "reorder":
        seqs, beams = _log_int(rng, 1, 48), rng.choice([2, 3, 4, 5, 8])
        # rows times kv heads, and rows times query heads that see them, stay below the largest's
        rows = min(1000000 // hk, 18000000 // (hq * beams)) // seqs
        prompt = 0 if rng.random() < 0.1 else _log_int(rng, 1, max(2, min(rows // 2, 16000)))
        tail_max = _log_int(rng, 1, max(2, min((rows - prompt) // beams, 4000)))
        return {"kind": kind, "seqs": seqs, "beams": beams, "prompt": prompt,
                "tail_min": max(1, tail_max // rng.choice([1, 2, 4])), "tail_max": tail_max,
                "hq": hq, "hk": hk, "shape_seed": seed}
    if kind == "weights":
        requests, children = _log_int(rng, 1, 64), rng.choice([1, 2, 3, 4, 8])
        # (the same bound)
        rows = min(1500000 // hk, 18000000 // hq) // requests
        prompt = 0 if rng.random() < 0.2 else _log_int(rng, 1, max(2, min(rows // (2 * children), 16000)))
        tail_max = _log_int(rng, 1, max(2, min((rows - prompt * children) // children, 130000)))
        return {"kind": kind, "requests": requests, "prompt": prompt, "children": children,
                "tail_min": max(1, tail_max // rng.choice([1, 2, 4])), "tail_max": tail_max,
                "hq": hq, "hk": hk, "shape_seed": seed}
    if kind == "prompt":
        window = rng.choice([0, 0, 1, 5, 16, 64, 130])
        threads = _log_int(rng, 1, 16)
        if window:
            longest = _log_int(rng, 17, min(20000, 800000 // (threads * hk),
                                            200000000 // (threads * hq * window)))
        else:
            longest = _log_int(rng, 17, int(math.sqrt(600000000 / (threads * hq))))
        return {"kind": kind, "threads": threads, "len_min": max(1, longest // rng.choice([1, 2])),
                "len_max": longest, "window": window, "hq": hq, "hk": hk, "shape_seed": seed}
    threads, layers = _log_int(rng, 1, 64), rng.choice([1, 1, 2, 3])
    longest = _log_int(rng, 40, min(130000, max(80, 1000000 // (threads * layers * hk))))
    len_min = max(24, longest // rng.choice([1, 1, 2]))
    begin = rng.choice([0, 0, 16])
    keep = rng.randint(1, min(len_min - begin, max(8, 400000 // (threads * layers * hk))))
    return {"kind": kind, "threads": threads, "len_min": len_min, "len_max": longest, "keep": keep,
            "begin": begin, "layers": layers, "hq": hq, "hk": hk, "shape_seed": seed}


# ------------------------------------------------------------------------- shapes, from the case
def _forest(case):
    """Row ranges of the cache: prompts [(begin, end)] and live threads [(request, begin, end)]."""
    rng = random.Random(case["shape_seed"])
    prompts, threads, at = [], [], 0
    for r in range(case["requests"]):
        prompts.append((at, at + case["prompt"]))
        at += case["prompt"]
        for _ in range(case["children"]):
            n = rng.randint(case["tail_min"], case["tail_max"])
            threads.append((r, at, at + n))
            at += n
    return prompts, threads, at


def _beams(case):
    """Row ranges of prompts and beams' tails, and for each beam the beam that it goes on from."""
    rng = random.Random(case["shape_seed"])
    prompts, tails, source, at = [], [], [], 0
    for i in range(case["seqs"]):
        prompts.append((at, at + case["prompt"]))
        at += case["prompt"]
        n = rng.randint(case["tail_min"], case["tail_max"])
        go_on = rng.sample(range(case["beams"]), max(1, case["beams"] // 2))
        for b in range(case["beams"]):
            tails.append((i, at, at + n))
            at += n
            source.append(i * case["beams"] + (b if b in go_on else rng.choice(go_on)))
    return prompts, tails, source, at


def _lengths(case):
    rng = random.Random(case["shape_seed"])
    return [rng.randint(case["len_min"], case["len_max"]) for _ in range(case["threads"])]


def _queries(case, length):
    return min(length, case["window"]) if case["window"] else length


def work(case):
    if case["kind"] == "beam":
        rows = case["seqs"] * case["beams"]
        size = 4 if case["type"] == "f32" else 2
        return {"bytes": rows * (case["vocab"] * size + 5) + case["seqs"] * case["select"] * 12,
                "flops": 4 * rows * case["vocab"]}
    hq, hk = case["hq"], case["hk"]
    if case["kind"] == "reorder":
        _, tails, source, _ = _beams(case)
        rows = case["seqs"] * case["prompt"] + sum(tails[b][2] - tails[b][1] for b in set(source))
        attended = sum(case["prompt"] + e - b for _, b, e in tails)
        # the rows of the beams that go on read once, queries read, results written
        return {"bytes": rows * hk * 4 * DIM + len(tails) * hq * 4 * DIM, "flops": 4 * DIM * hq * attended}
    if case["kind"] == "weights":
        _, threads, total = _forest(case)
        attended = sum(case["prompt"] + e - b for _, b, e in threads)
        # keys, queries and their log-sum-exps read, one weight per key and kv head written
        return {"bytes": total * hk * (2 * DIM + 4) + len(threads) * hq * (2 * DIM + 4),
                "flops": hq * attended * (2 * DIM + 3)}
    if case["kind"] == "prompt":
        total = queries = attended = 0
        for n in _lengths(case):
            c = _queries(case, n)
            total, queries = total + n, queries + c
            attended += c * (n - c) + c * (c + 1) // 2
        return {"bytes": total * hk * (2 * DIM + 4) + queries * hq * (2 * DIM + 4),
                "flops": hq * attended * (2 * DIM + 3)}
    rows = sum(n - case["begin"] for n in _lengths(case))
    kept = case["threads"] * case["keep"]
    # all weights read; kept rows of K and V and their weights read and written
    return {"bytes": case["layers"] * hk * (4 * rows + kept * 2 * (4 * DIM + 4)), "flops": 0}


# --------------------------------------------------------------------------------------- inputs
def _generator(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _rows(n, heads, g):
    """K or V rows: normal values, with dims of larger and smaller spread as projections have them."""
    spread = torch.exp(0.5 * torch.randn(heads, DIM, generator=g, device="cuda"))
    out = torch.empty(n, heads, DIM, dtype=torch.bfloat16, device="cuda")
    step = max(1, (1 << 26) // (heads * DIM))
    for b in range(0, n, step):
        e = min(n, b + step)
        out[b:e] = torch.randn(e - b, heads, DIM, generator=g, device="cuda") * spread
    return out


def _chains(case):
    """Of each query thread, the row ranges of its chain."""
    prompts, threads, _ = _forest(case)
    return [[p for p in (prompts[r], (b, e)) if p[1] > p[0]] for r, b, e in threads]


def _grouped(q, hk):
    """[n][hq][128] as [hk][n * group][128] in 32 bits, rows ordered by query, then head."""
    n, hq = q.shape[0], q.shape[1]
    return q.float().reshape(n, hk, hq // hk, DIM).permute(1, 0, 2, 3).reshape(hk, -1, DIM)


def _lse(q, k, first=None):
    """Natural log-sum-exps [n][hq] of the scaled scores; query i sees keys 0..first + i, or all."""
    n, hq, hk = q.shape[0], q.shape[1], k.shape[1]
    out = torch.empty(n, hq, device=q.device)
    step = max(1, (1 << 27) // (hq * k.shape[0]))
    keys = k.float().permute(1, 2, 0)
    for b in range(0, n, step):
        e = min(n, b + step)
        s = (_grouped(q[b:e], hk) @ keys) * SCALE
        if first is not None:
            s = s.masked_fill(_unseen(first + b, first + e, k.shape[0], hq // hk, s.device), -math.inf)
        out[b:e] = torch.logsumexp(s, -1).reshape(hk, e - b, hq // hk).permute(1, 0, 2).reshape(e - b, hq)
    return out


def _unseen(p0, p1, keys, group, device):
    at = torch.arange(p0, p1, device=device).repeat_interleave(group)
    return torch.arange(keys, device=device)[None, :] > at[:, None]


def _session(case, blocks, threads, longest, layers=1):
    from paper_2401_06761_b200.session import PagedSession
    from paper_2401_06761_b200.synth import LayerShape
    return PagedSession(LayerShape(case["hq"], case["hk"]), blocks, threads, -(-longest // 16) + 1,
                        num_layers=layers, weights=True)


def _forked(sess, prompts, threads, k, v):
    """Threads forked from their prompts, then grown by their own rows."""
    roots = sess.new_threads(len(prompts))
    for r, (b, e) in zip(roots, prompts):
        if e > b:
            sess.append([r], [e - b], k[b:e], v[b:e])
    tids = sess.fork([roots[r] for r, _, _ in threads])
    for t, (_, b, e) in zip(tids, threads):
        sess.append([t], [e - b], k[b:e], v[b:e])
    sess.release(roots)
    return tids


def prepare(case, seed):
    g = _generator(seed)
    state = {"case": case}
    if case["kind"] == "beam":
        return _prepare_beam(case, state, g)
    hq, hk = case["hq"], case["hk"]
    if case["kind"] == "reorder":
        prompts, tails, source, total = _beams(case)
        k, v = _rows(total, hk, g), _rows(total, hk, g)
        state["q"] = torch.randn(len(tails), hq, DIM, generator=g, device="cuda", dtype=torch.bfloat16)
        if not own:
            state.update(k=k, v=v, prompts=prompts, tails=tails, source=source)
            return state
        blocks = sum(-(-(e - b) // 16) for b, e in prompts) + sum(-(-(e - b) // 16) + 2 for _, b, e in tails)
        sess = _session(case, blocks, len(tails) + len(prompts),
                        case["prompt"] + max(e - b for _, b, e in tails))
        tids = _forked(sess, prompts, tails, k, v)
        state.update(sess=sess, tids=tids, sources=[tids[b] for b in source])
        return state
    if case["kind"] == "weights":
        prompts, threads, total = _forest(case)
        k = _rows(total, hk, g)
        q = torch.randn(len(threads), hq, DIM, generator=g, device="cuda", dtype=torch.bfloat16)
        chains = _chains(case)
        lse = torch.cat([_lse(q[i:i + 1], torch.cat([k[b:e] for b, e in c])) for i, c in enumerate(chains)])
        state.update(q=q, lse=lse)
        if not own:
            state.update(k=k, chains=chains)
            return state
        blocks = sum(-(-(e - b) // 16) for b, e in prompts) + sum(-(-(e - b) // 16) + 1 for _, b, e in threads)
        sess = _session(case, blocks, len(threads) + len(prompts),
                        case["prompt"] + max(e - b for _, b, e in threads))
        tids = _forked(sess, prompts, threads, k, k)
        sess.attention(tids, q)               # (the step whose weights are summed)
        # each row once: a prompt through the first of its threads; and behind all of them what the other
        # threads' copies of a prompt's last, partial block have received
        where = {}
        for t, (r, b, e) in zip(tids, threads):
            if case["prompt"]:
                where.setdefault(prompts[r][0], (t, 0, case["prompt"]))
            where[b] = (t, case["prompt"], e - b)
        rows = [where[at] for at in sorted(where)]
        part = case["prompt"] % 16
        state["copied"] = None
        if part and case["children"] > 1:
            for c in range(1, case["children"]):
                rows += [(t, case["prompt"] - part, part) for t in tids[c::case["children"]]]
            state["copied"] = torch.cat([torch.arange(e - part, e) for _, e in prompts]).cuda()
            state["total"] = total
        state.update(sess=sess, tids=[x[0] for x in rows], begin=[x[1] for x in rows],
                     count=[x[2] for x in rows])
        return state
    lengths = _lengths(case)
    if case["kind"] == "prompt":
        k = _rows(sum(lengths), hk, g)
        counts = [_queries(case, n) for n in lengths]
        q = torch.randn(sum(counts), hq, DIM, generator=g, device="cuda", dtype=torch.bfloat16)
        lse, kb, qb = [], 0, 0
        for n, c in zip(lengths, counts):
            lse.append(_lse(q[qb:qb + c], k[kb:kb + n], n - c))
            kb, qb = kb + n, qb + c
        state.update(q=q, lse=torch.cat(lse), lengths=lengths, counts=counts)
        if not own:
            state.update(k=k)
            return state
        sess = _session(case, sum(-(-n // 16) for n in lengths), len(lengths), max(lengths))
        tids = sess.new_threads(len(lengths))
        sess.append(tids, lengths, k, k)
        state.update(sess=sess, tids=tids, first=[n - c for n, c in zip(lengths, counts)],
                     zeros=[0] * len(tids))
        return state
    total, layers = sum(lengths), case["layers"]
    k = [_rows(total, hk, g) for _ in range(layers)]
    v = [_rows(total, hk, g) for _ in range(layers)]
    w = _weights_of_rows(layers, total, hk, g)
    if not own:
        state.update(k=k, v=v, w=w, lengths=lengths)
        return state
    held = -(-(case["begin"] + case["keep"]) // 16) + 1
    sess = _session(case, sum(-(-n // 16) + held for n in lengths), 2 * len(lengths), max(lengths), layers)
    tids = sess.new_threads(len(lengths))
    sess.append(tids, lengths, k[0], v[0])
    for l in range(1, layers):
        sess.append_layer(l, k[l], v[l])
    at = 0
    for t, n in zip(tids, lengths):
        _, blocks = sess.thread(t)
        rows = torch.zeros(layers, len(blocks) * 16, hk, device="cuda")
        rows[:, :n] = w[:, at:at + n]
        sess.weights[:, torch.tensor(blocks, device="cuda")] = rows.unflatten(1, (-1, 16)).transpose(2, 3)
        at += n
    state.update(sess=sess, tids=tids, lengths=lengths)
    return state


def _prepare_beam(case, state, g):
    seqs, beams, vocab = case["seqs"], case["beams"], case["vocab"]
    dtype = TYPES[case["type"]]
    logits = torch.empty(seqs * beams, vocab + case["pad"], dtype=dtype, device="cuda")
    # a head's logits: most of the mass on few tokens, each row with its own sharpness
    sharp = 0.5 + 3.0 * torch.rand(seqs * beams, 1, generator=g, device="cuda")
    step = max(1, (1 << 26) // (vocab + case["pad"]))
    for b in range(0, seqs * beams, step):
        e = min(seqs * beams, b + step)
        logits[b:e] = torch.randn(e - b, vocab + case["pad"], generator=g, device="cuda") * sharp[b:e]
    state["logits"] = logits.view(seqs, beams, -1)[:, :, :vocab]
    scores = -20.0 * torch.rand(seqs, beams, generator=g, device="cuda")
    state["scores"] = torch.sort(scores, dim=1, descending=True).values
    state["finished"] = None
    if case["finished"]:
        state["finished"] = torch.rand(seqs, beams, generator=g, device="cuda") < case["finished"]
    state["eos"] = 2
    if own:
        from paper_2401_06761_b200.session import BeamSelect
        state["beam"] = BeamSelect(beams, vocab, case["select"], eos=2)
    return state


def _weights_of_rows(layers, total, hk, g):
    """Accumulated weights [layers][total][hk]: a few heavy rows, many light ones, some never seen."""
    w = torch.exp(2.0 * torch.randn(layers, total, hk, generator=g, device="cuda"))
    return w * (torch.rand(layers, total, hk, generator=g, device="cuda") > 0.05)


# ----------------------------------------------------------------------------------------- a pass
def run(state):
    kind = state["case"]["kind"]
    if kind == "beam":
        if own:
            return state["beam"](state["logits"], state["scores"], state["finished"])
        return _plain_beam(state)
    if kind == "reorder":
        if own:
            state["sess"].reorder(state["tids"], state["sources"])
            return state["sess"].attention(state["tids"], state["q"])
        return _plain_reorder(state)
    if kind == "weights":
        if own:
            state["sess"].add_weights(state["q"], state["lse"], replace=True)
            w = state["sess"].read_weights(state["tids"], state["begin"], state["count"])
            if state["copied"] is None:
                return w
            w, copies = w[:state["total"]], w[state["total"]:]
            w[state["copied"]] += copies.view(-1, len(state["copied"]), w.shape[1]).sum(0)
            return w
        return _plain_weights(state)
    if kind == "prompt":
        if own:
            state["sess"].add_weights_prefill(state["tids"], state["first"], state["counts"],
                                              state["q"], state["lse"], replace=True)
            return state["sess"].read_weights(state["tids"], state["zeros"], state["lengths"])
        return _plain_prompt(state)
    if own:
        return _own_evict(state)
    return _plain_evict(state)


def _own_evict(state):
    """A continuation forked from each thread keeps the heavy rows; the thread keeps all of its own."""
    case, sess = state["case"], state["sess"]
    n, begin, keep = len(state["tids"]), case["begin"], case["keep"]
    kids = sess.fork(state["tids"])
    sess.evict(kids, [begin] * n, state["lengths"], [keep] * n)
    first, count = [begin] * n, [keep] * n
    kv = [sess.read_kv(kids, first, count, layer=l) for l in range(case["layers"])]
    w = [sess.read_weights(kids, first, count, layer=l) for l in range(case["layers"])]
    sess.release(kids)
    return {"k": [x[0] for x in kv], "v": [x[1] for x in kv], "w": w}


# ----------------------------------------------------------------------------------- plain forms
def _plain_beam(state):
    case = state["case"]
    vocab, select = case["vocab"], case["select"]
    # (64 bits: pairs of different beams are compared through their rows' log-sum-exps)
    scores, beams, tokens = [], [], []
    step = max(1, (1 << 26) // (case["beams"] * vocab))
    for b in range(0, case["seqs"], step):
        x = state["logits"][b:b + step].double()
        top = x.amax(-1, keepdim=True)
        logp = x - (top + torch.exp(x - top).sum(-1, keepdim=True).log())
        total = state["scores"][b:b + step].double()[..., None] + logp
        if state["finished"] is not None:
            done = state["finished"][b:b + step]
            only = torch.full_like(total, -math.inf)
            only[..., state["eos"]] = state["scores"][b:b + step].double()
            total = torch.where(done[..., None], only, total)
        best, at = torch.sort(total.flatten(1), dim=1, descending=True, stable=True)
        best, at = best[:, :select], at[:, :select]
        scores.append(best.float())
        beams.append((at // vocab).int())
        tokens.append((at % vocab).int())
    return torch.cat(scores), torch.cat(beams), torch.cat(tokens)


def _plain_reorder(state):
    k, v, q, tails = state["k"], state["v"], state["q"], state["tails"]
    hk, group = k.shape[1], q.shape[1] // k.shape[1]
    out = torch.empty_like(q)
    for i, b in enumerate(state["source"]):
        parts = [state["prompts"][tails[b][0]], tails[b][1:]]
        keys, values = (torch.cat([x[b:e] for b, e in parts]).float() for x in (k, v))
        s = (q[i].float().view(hk, group, DIM) @ keys.permute(1, 2, 0)) * SCALE
        p = torch.exp(s - s.amax(-1, keepdim=True))
        o = (p @ values.transpose(0, 1)) / p.sum(-1, keepdim=True)
        out[i] = o.reshape(-1, DIM).to(q.dtype)
    return out


def _plain_weights(state):
    k, q, lse = state["k"], state["q"], state["lse"]
    hk, group = k.shape[1], q.shape[1] // k.shape[1]
    out = torch.zeros(k.shape[0], hk, device=k.device)
    for i, chain in enumerate(state["chains"]):
        qi, li = q[i].float().view(hk, group, DIM), lse[i].view(hk, group, 1)
        for b, e in chain:
            s = (qi @ k[b:e].float().permute(1, 2, 0)) * SCALE
            out[b:e] += torch.exp(s - li).sum(1).T
    return out


def _plain_prompt(state):
    k, q, lse = state["k"], state["q"], state["lse"]
    hk, group = k.shape[1], q.shape[1] // k.shape[1]
    out = torch.zeros(k.shape[0], hk, device=k.device)
    kb = qb = 0
    for n, c in zip(state["lengths"], state["counts"]):
        keys = k[kb:kb + n].float().permute(1, 2, 0)
        step = max(1, (1 << 27) // (q.shape[1] * n))
        for b in range(0, c, step):
            e = min(c, b + step)
            s = (_grouped(q[qb + b:qb + e], hk) @ keys) * SCALE
            l = lse[qb + b:qb + e].view(e - b, hk, group).permute(1, 0, 2).reshape(hk, -1, 1)
            p = torch.exp(s - l).masked_fill(_unseen(n - c + b, n - c + e, n, group, s.device), 0.0)
            out[kb:kb + n] += p.sum(1).T
        kb, qb = kb + n, qb + c
    return out


def _plain_evict(state):
    case = state["case"]
    begin, keep = case["begin"], case["keep"]
    out = {"k": [], "v": [], "w": []}
    for l in range(case["layers"]):
        parts, at = [], 0
        for n in state["lengths"]:
            w = state["w"][l, at + begin:at + n].T                       # [hk][rows]
            order = torch.sort(w, dim=1, descending=True, stable=True).indices[:, :keep]
            kept = torch.sort(order, dim=1).values
            place = torch.arange(keep, device=w.device).expand_as(kept).clone()
            hole = torch.ones_like(w, dtype=torch.bool).scatter_(1, kept, False)[:, :keep]
            place[hole] = kept[kept >= keep]
            heads = torch.arange(w.shape[0], device=w.device)[:, None]
            rows = place + at + begin
            parts.append((state["k"][l][rows, heads].transpose(0, 1), state["v"][l][rows, heads].transpose(0, 1),
                          w.gather(1, place).T))
            at += n
        for name, x in zip(("k", "v", "w"), zip(*parts)):
            out[name].append(torch.cat(x))
    return out


# ------------------------------------------------------------------------- definitions in 64 bits
def exact(case, seed):
    global own
    was, own = own, False
    try:
        state = prepare(case, seed)
    finally:
        own = was
    if case["kind"] == "beam":
        return _exact_beam(case, state)
    if case["kind"] == "reorder":
        out = torch.empty(state["q"].shape, dtype=torch.float64, device="cuda")
        for i, b in enumerate(state["source"]):
            (p0, p1), (_, t0, t1) = state["prompts"][state["tails"][b][0]], state["tails"][b]
            at = torch.cat([torch.arange(p0, p1, device="cuda"), torch.arange(t0, t1, device="cuda")])
            heads = torch.arange(case["hq"], device="cuda") // (case["hq"] // case["hk"])
            k, v = (state[x][at].double()[:, heads] for x in ("k", "v"))
            s = torch.einsum("hd,nhd->hn", state["q"][i].double(), k) / math.sqrt(DIM)
            out[i] = torch.einsum("hn,nhd->hd", torch.softmax(s, 1), v)
        return out
    if case["kind"] == "weights":
        out = torch.zeros(state["k"].shape[0], case["hk"], dtype=torch.float64, device="cuda")
        for i, chain in enumerate(state["chains"]):
            at = torch.cat([torch.arange(b, e, device="cuda") for b, e in chain])
            out.index_add_(0, at, _exact_sums(case, state["q"][i:i + 1], state["lse"][i:i + 1], state["k"][at], None))
        return out
    if case["kind"] == "prompt":
        parts, kb, qb = [], 0, 0
        for n, c in zip(state["lengths"], state["counts"]):
            parts.append(_exact_sums(case, state["q"][qb:qb + c], state["lse"][qb:qb + c],
                                     state["k"][kb:kb + n], n - c))
            kb, qb = kb + n, qb + c
        return torch.cat(parts)
    return _exact_evict(case, state)


def _exact_sums(case, q, lse, k, first):
    """sum over queries and the heads of a group of exp(scale * <q, k> - lse), head by head."""
    n, group = k.shape[0], case["hq"] // case["hk"]
    out = torch.zeros(n, case["hk"], dtype=torch.float64, device="cuda")
    pos = torch.arange(n, device="cuda")
    step = max(1, (1 << 26) // n)
    for h in range(case["hq"]):
        kh = k[:, h // group].double()
        for b in range(0, q.shape[0], step):
            s = torch.einsum("kd,qd->kq", kh, q[b:b + step, h].double()) / math.sqrt(DIM)
            p = (s - lse[b:b + step, h].double()).exp()
            if first is not None:
                see = first + b + torch.arange(p.shape[1], device="cuda")
                p = p * (pos[:, None] <= see[None, :])
            out[:, h // group] += p.sum(1)
    return out


def _exact_beam(case, state):
    best = []
    for i in range(case["seqs"]):
        found = []
        x = state["logits"][i].double()
        for b in range(case["beams"]):
            score = state["scores"][i, b].double()
            if state["finished"] is not None and bool(state["finished"][i, b]):
                found.append((score.view(1), torch.tensor([b * case["vocab"] + state["eos"]], device="cuda")))
                continue
            value = torch.log_softmax(x[b], 0) + score
            # everything at least as high as the row's last wanted value
            last = torch.topk(value, min(case["select"], case["vocab"])).values[-1]
            at = torch.nonzero(value >= last).flatten()
            found.append((value[at], at + b * case["vocab"]))
        value, at = torch.cat([f[0] for f in found]), torch.cat([f[1] for f in found])
        order = torch.argsort(value, descending=True, stable=True)[:case["select"]]
        best.append((value[order], at[order]))
    values, at = torch.stack([b[0] for b in best]), torch.stack([b[1] for b in best])
    return values, (at // case["vocab"]).int(), (at % case["vocab"]).int()


def _exact_evict(case, state):
    """The kept rows chosen by rank: how many rows of the stretch are heavier, or as heavy and earlier."""
    begin, keep = case["begin"], case["keep"]
    k, v, w = ([[] for _ in range(case["layers"])] for _ in range(3))
    for l in range(case["layers"]):
        at = 0
        for n in state["lengths"]:
            picks = []
            for h in range(case["hk"]):
                x = state["w"][l, at + begin:at + n, h].cpu().numpy()
                by_rank = sorted(range(len(x)), key=lambda i: (-x[i], i))[:keep]
                stay = {i for i in by_rank if i < keep}
                moved = iter(sorted(i for i in by_rank if i >= keep))
                picks.append([j if j in stay else next(moved) for j in range(keep)])
            rows = torch.tensor(picks, device="cuda").T + at + begin              # [keep][hk]
            heads = torch.arange(case["hk"], device="cuda")[None, :]
            k[l].append(state["k"][l][rows, heads])
            v[l].append(state["v"][l][rows, heads])
            w[l].append(state["w"][l][rows, heads])
            at += n
        k[l], v[l], w[l] = torch.cat(k[l]), torch.cat(v[l]), torch.cat(w[l])
    return {"k": k, "v": v, "w": w}
