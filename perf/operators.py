"""Measured cases of the rotary and 4-bit-cache operators: inputs, plain forms, the calls a user makes.

Four kinds of case.  All of them run on the rows of one attention layer with 128-dim heads.

  rope    rotary positions applied to the query and key rows of a batch of tokens, taken as views
          out of the projection's fused output.
  store   new K and V rows quantised into a 4-bit paged cache (the scatter of one layer), and the
          same rows read back from it as values.
  decode  one query per live thread of a forest of forked threads, over a 4-bit cache whose
          prompts are shared between the threads forked from them.
  verify  several speculated tokens per thread with a tree mask among them, over a 4-bit cache.

A 4-bit row: 128 values in four groups of 32 consecutive ones.  Of each group lo = min(x) and
s = bf16((max(x) - lo) / 15) are kept, and x is held as the integer c = min(15, round((x - lo) / s)),
ties to even, which stands for lo + s * c.  A group of equal values has s = 0 and c = 0.

Shapes of heads and trees are those of the benchmark's configurations (GQA 8/2, MHA 32, MHA 40,
GQA 64/8, GQA 32/8) at request counts that keep one pass short; values are random.
"""
import math
import random

import torch

own = False

DIM = 128
GROUP = 32

HEADS = ((8, 2), (32, 32), (40, 40), (64, 8), (32, 8))


# ------------------------------------------------------------------------------------- the cases
def listed():
    return [
        # the smallest step: three threads of one request, where only latency counts
        {"name": "rope_step3", "kind": "rope", "n": 3, "hq": 8, "hk": 2, "rotary": 128,
         "layout": "half", "scaling": "none", "base": 10000.0, "factor": 1.0, "max_pos": 128},
        # one decode step of a large batch, interleaved pairs in half of each head, positions far
        # beyond the trained length with banded scaling
        {"name": "rope_step4096_interleaved", "kind": "rope", "n": 4095, "hq": 64, "hk": 8,
         "rotary": 64, "layout": "interleaved", "scaling": "bands", "base": 500000.0,
         "factor": 8.0, "max_pos": 131072},
        # prompts of a batch, whole heads
        {"name": "rope_prompts", "kind": "rope", "n": 16384, "hq": 40, "hk": 40, "rotary": 128,
         "layout": "half", "scaling": "yarn", "base": 10000.0, "factor": 4.0, "max_pos": 16384},
        # one new row for each of three threads
        {"name": "store_step3", "kind": "store", "threads": 3, "held": 37, "new_min": 1,
         "new_max": 1, "hq": 8, "hk": 2, "shape_seed": 1},
        # one new row for each thread of a large batch
        {"name": "store_step4096", "kind": "store", "threads": 4096, "held": 21, "new_min": 1,
         "new_max": 1, "hq": 64, "hk": 8, "shape_seed": 2},
        # ragged prompts
        {"name": "store_prompts", "kind": "store", "threads": 17, "held": 0, "new_min": 500,
         "new_max": 2048, "hq": 32, "hk": 32, "shape_seed": 3},
        # a single request: prompt of 64, three children
        {"name": "decode_one_request", "kind": "decode", "requests": 1, "prompt": 64,
         "children": 3, "tail_min": 17, "tail_max": 40, "hq": 8, "hk": 2, "shape_seed": 4},
        # a small MHA batch: single-row tails and four-row prompts
        {"name": "decode_mha", "kind": "decode", "requests": 32, "prompt": 512, "children": 4,
         "tail_min": 128, "tail_max": 256, "hq": 32, "hk": 32, "shape_seed": 5},
        # long prompts shared by eight children with eight query heads to a kv head
        {"name": "decode_gqa_shared", "kind": "decode", "requests": 64, "prompt": 2048,
         "children": 8, "tail_min": 128, "tail_max": 512, "hq": 64, "hk": 8, "shape_seed": 6},
        # a few very long contexts without forks
        {"name": "decode_long", "kind": "decode", "requests": 4, "prompt": 0, "children": 1,
         "tail_min": 120001, "tail_max": 131071, "hq": 32, "hk": 8, "shape_seed": 7},
        # five candidates of one thread
        {"name": "verify_one", "kind": "verify", "requests": 1, "prompt": 100, "children": 1,
         "tail_min": 9, "tail_max": 9, "candidates": 5, "hq": 8, "hk": 2, "shape_seed": 8},
        # a batch of predict-verify steps, two children to a prompt
        {"name": "verify_batch", "kind": "verify", "requests": 48, "prompt": 512, "children": 2,
         "tail_min": 65, "tail_max": 700, "candidates": 26, "hq": 32, "hk": 8, "shape_seed": 9},
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["rope", "store", "decode", "decode", "verify"])
    hq, hk = rng.choice(HEADS)
    if kind == "rope":
        return {"kind": kind, "n": _log_int(rng, 1, 16384 * 80 // (hq + hk) // 2), "hq": hq, "hk": hk,
                "rotary": rng.choice([128, 128, 64, 32, 96, 20, 2]),
                "layout": rng.choice(["half", "interleaved"]),
                "scaling": rng.choice(["none", "linear", "bands", "yarn"]),
                "base": rng.choice([10000.0, 500000.0, 1000000.0]),
                "factor": rng.choice([2.0, 4.0, 8.0, 32.0]), "max_pos": _log_int(rng, 2, 1 << 20)}
    seed = rng.randrange(1 << 30)
    if kind == "store":
        threads = _log_int(rng, 1, 2048)
        most = max(1, min(2048, 20000 * 32 // hk // threads))
        new_max = _log_int(rng, 1, most)
        return {"kind": kind, "threads": threads, "held": rng.randrange(0, 40),
                "new_min": rng.randint(max(1, new_max // 4), new_max), "new_max": new_max,
                "hq": hq, "hk": hk, "shape_seed": seed}
    requests, children = _log_int(rng, 1, 48), rng.choice([1, 2, 3, 4, 8])
    # unique rows times kv heads stay below those of the largest listed case
    rows = min(2500000, 60000 * requests) // hk // requests
    prompt = 0 if rng.random() < 0.15 else _log_int(rng, 1, max(2, min(rows // 2, 16000)))
    tail_max = _log_int(rng, 1, max(2, min((rows - prompt) // children, 30000 // children)))
    case = {"kind": kind, "requests": requests, "prompt": prompt, "children": children,
            "tail_min": max(1, tail_max // rng.choice([1, 2, 4])), "tail_max": tail_max,
            "hq": hq, "hk": hk, "shape_seed": seed}
    if kind == "verify":
        case["candidates"] = rng.choice([1, 2, 5, 13, 26, 64])
        # products stay below those of the largest listed case
        while case["candidates"] > 1 and (case["candidates"] * requests * children * hq
                                          * (prompt + tail_max)) > 50000000:
            case["candidates"] //= 2
        case["tail_max"] = max(case["tail_max"], 2 * case["candidates"])
        case["tail_min"] = max(case["tail_min"], case["candidates"])
    return case


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


def _new_counts(case):
    rng = random.Random(case["shape_seed"])
    return [rng.randint(case["new_min"], case["new_max"]) for _ in range(case["threads"])]


def _candidate_masks(case, n_threads):
    """For each candidate the candidates of its thread that it sees: its ancestors and itself."""
    rng = random.Random(case["shape_seed"] + 1)
    k, masks = case["candidates"], []
    for _ in range(n_threads):
        mine = []
        for j in range(k):
            parent = rng.randint(-1, j - 1)
            mine.append((1 << j) | (mine[parent] if parent >= 0 else 0))
        masks.append(mine)
    return masks


def work(case):
    hq, hk = case["hq"], case["hk"]
    if case["kind"] == "rope":
        elems = case["n"] * (hq + hk) * DIM
        return {"bytes": 4 * elems + 4 * case["n"],
                "flops": 3 * case["n"] * (hq + hk) * case["rotary"]}
    row = DIM // 2 + DIM // GROUP * 4                       # one 4-bit row of K or of V
    if case["kind"] == "store":
        rows = 2 * sum(_new_counts(case)) * hk
        # read the rows, write the cache, read the cache, write the values
        return {"bytes": rows * (2 * DIM + row + row + 2 * DIM), "flops": 8 * rows * DIM}
    prompts, threads, total = _forest(case)
    queries, attended = 0, 0
    if case["kind"] == "decode":
        queries = len(threads)
        attended = sum(case["prompt"] + e - b for _, b, e in threads)
    else:
        k = case["candidates"]
        queries = k * len(threads)
        attended = sum(k * (case["prompt"] + e - b - k) for _, b, e in threads)
        attended += sum(bin(m).count("1") for mine in _candidate_masks(case, len(threads)) for m in mine)
    return {"bytes": total * hk * 2 * row + queries * hq * DIM * 4,
            "flops": 4 * DIM * hq * attended}


# --------------------------------------------------------------------------------------- inputs
def _generator(seed, device="cuda"):
    g = torch.Generator(device=device)
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


def _inv_freq(case, dtype=torch.float64):
    """Angle per position of each pair of dims."""
    rd, base, f = case["rotary"], case["base"], case["factor"]
    theta = base ** (-2.0 * torch.arange(rd // 2, dtype=dtype) / rd)
    kind = case["scaling"]
    if kind == "linear":
        theta = theta / f
    elif kind == "bands":                     # long wavelengths are stretched, short ones kept
        low, high, trained = 1.0, 4.0, 8192.0
        turns = trained * theta / (2 * math.pi)
        t = ((turns - low) / (high - low)).clamp(0, 1)
        theta = (1 - t) * theta / f + t * theta
    elif kind == "yarn":                      # a ramp over the index of the pair
        fast, slow, trained = 32.0, 1.0, 4096.0

        def index(turns):
            return rd * math.log(trained / (turns * 2 * math.pi)) / (2 * math.log(base))
        low, high = max(0, math.floor(index(fast))), min(rd - 1, math.ceil(index(slow)))
        ramp = ((torch.arange(rd // 2, dtype=dtype) - low) / max(high - low, 0.001)).clamp(0, 1)
        theta = theta / f * ramp + theta * (1 - ramp)
    return theta


def _magnitude(case):
    return 0.1 * math.log(case["factor"]) + 1.0 if case["scaling"] == "yarn" else 1.0


def _session(case, blocks, threads, longest):
    from paper_2401_06761_b200.session import PagedSession
    from paper_2401_06761_b200.synth import LayerShape
    return PagedSession(LayerShape(case["hq"], case["hk"]), blocks, threads, -(-longest // 16) + 1,
                        kv_format="q4")


def prepare(case, seed):
    g = _generator(seed)
    hq, hk = case["hq"], case["hk"]
    state = {"case": case}
    if case["kind"] == "rope":
        n = case["n"]
        qkv = torch.randn(n, hq + 2 * hk, DIM, generator=g, device="cuda", dtype=torch.bfloat16)
        state["q"], state["k"] = qkv[:, :hq], qkv[:, hq:hq + hk]
        state["pos"] = torch.randint(0, case["max_pos"], (n,), generator=g, device="cuda",
                                     dtype=torch.int32)
        if own:
            from paper_2401_06761_b200 import session
            state["rope"] = session.Rope(
                rotary_dim=case["rotary"], layout=case["layout"], base=case["base"],
                scaling=case["scaling"], factor=case["factor"], attn_scale=_magnitude(case),
                original_len=4096 if case["scaling"] == "yarn" else 8192,
                low=1.0, high=32.0 if case["scaling"] == "yarn" else 4.0)
        else:
            state["theta"] = _inv_freq(case).cuda()
        return state
    if case["kind"] == "store":
        counts = _new_counts(case)
        total = sum(counts)
        state["k"], state["v"] = _rows(total, hk, g), _rows(total, hk, g)
        if own:
            held = case["held"]
            sess = _session(case, sum(-(-(held + c) // 16) for c in counts), len(counts),
                            held + max(counts))
            tids = sess.new_threads(len(counts))
            if held:
                zeros = torch.zeros(held * len(counts), hk, DIM, dtype=torch.bfloat16, device="cuda")
                sess.append(tids, [held] * len(counts), zeros, zeros)
            sess.append(tids, counts, state["k"], state["v"])
            state.update(sess=sess, tids=tids, begin=[held] * len(counts), counts=counts)
        return state
    prompts, threads, total = _forest(case)
    k, v = _rows(total, hk, g), _rows(total, hk, g)
    per_thread = case["candidates"] if case["kind"] == "verify" else 1
    state["q"] = torch.randn(per_thread * len(threads), hq, DIM, generator=g, device="cuda",
                             dtype=torch.bfloat16)
    if case["kind"] == "verify":
        state["masks"] = _candidate_masks(case, len(threads))
    if own:
        blocks = sum(-(-(e - b) // 16) for b, e in prompts) + sum(-(-(e - b) // 16) + 1 for _, b, e in threads)
        sess = _session(case, blocks, max(len(state["q"]), len(threads) + len(prompts)),
                        case["prompt"] + max(e - b for _, b, e in threads))
        roots = sess.new_threads(len(prompts))
        if case["prompt"]:
            for r, (b, e) in zip(roots, prompts):
                sess.append([r], [e - b], k[b:e], v[b:e])
        tids = sess.fork([roots[r] for r, _, _ in threads])
        for t, (_, b, e) in zip(tids, threads):
            sess.append([t], [e - b], k[b:e], v[b:e])
        sess.release(roots)
        state.update(sess=sess, tids=tids)
        if case["kind"] == "verify":
            state.update(counts=[per_thread] * len(tids), bits=[m for mine in state["masks"] for m in mine])
    else:
        state.update(prompts=prompts, threads=threads, k=_quantise(k), v=_quantise(v))
    return state


# ----------------------------------------------------------------------------------- plain forms
def _quantise(x):
    """Codes [n][heads][4][32] as bytes, scales and lowest values [n][heads][4][1] as bf16."""
    codes = torch.empty(x.shape[0], x.shape[1], DIM // GROUP, GROUP, dtype=torch.uint8, device=x.device)
    s = torch.empty(x.shape[0], x.shape[1], DIM // GROUP, 1, dtype=torch.bfloat16, device=x.device)
    lo = torch.empty_like(s)
    step = max(1, (1 << 26) // (x.shape[1] * DIM))
    for b in range(0, x.shape[0], step):
        part = x[b:b + step].float().unflatten(-1, (DIM // GROUP, GROUP))
        low = part.amin(-1, keepdim=True)
        scale = ((part.amax(-1, keepdim=True) - low) / 15.0).bfloat16().float()
        c = torch.round((part - low) / scale.where(scale > 0, torch.ones_like(scale))).clamp(max=15)
        codes[b:b + step] = c.where(scale > 0, torch.zeros_like(c)).to(torch.uint8)
        s[b:b + step], lo[b:b + step] = scale.bfloat16(), low.bfloat16()
    return codes, s, lo


def _values(held, b, e):
    codes, s, lo = held
    return (lo[b:e].float() + s[b:e].float() * codes[b:e].float()).flatten(-2)


def _rotate(x, cos, sin, rd, layout):
    head = x[..., :rd].float()
    if layout == "half":
        a, b = head[..., :rd // 2], head[..., rd // 2:]
        turned = torch.cat([a * cos - b * sin, b * cos + a * sin], -1)
    else:
        a, b = head[..., 0::2], head[..., 1::2]
        turned = torch.stack([a * cos - b * sin, b * cos + a * sin], -1).flatten(-2)
    return torch.cat([turned.to(x.dtype), x[..., rd:]], -1)


def _attend(q, k, v, seen=None):
    """q [n][hq][128], k and v [tokens][hk][128], seen [n][tokens] or None; all in 32 bits."""
    n, hq, hk = q.shape[0], q.shape[1], k.shape[1]
    q = q.reshape(n, hk, hq // hk, DIM).permute(1, 0, 2, 3).reshape(hk, -1, DIM)
    s = (q @ k.permute(1, 2, 0)) * (1.0 / math.sqrt(DIM))              # [hk][n * group][tokens]
    if seen is not None:
        rows = seen.repeat_interleave(hq // hk, 0)
        s = s.masked_fill(~rows, float("-inf"))
    p = torch.exp(s - s.amax(-1, keepdim=True))
    o = (p @ v.permute(1, 0, 2)) / p.sum(-1, keepdim=True)
    return o.reshape(hk, n, hq // hk, DIM).permute(1, 0, 2, 3).reshape(n, hq, DIM)


def _seen(masks, committed, device):
    k = len(masks)
    seen = torch.ones(k, committed + k, dtype=torch.bool)
    for j, m in enumerate(masks):
        for x in range(k):
            seen[j, committed + x] = bool((m >> x) & 1)
    return seen.to(device)


def _run_plain(state):
    case = state["case"]
    if case["kind"] == "rope":
        # angles in 64 bits: at position 2^20 a 32-bit product is off by a sixteenth of a radian
        angle = state["pos"].double()[:, None] * state["theta"]
        cos = (torch.cos(angle) * _magnitude(case)).float()[:, None]
        sin = (torch.sin(angle) * _magnitude(case)).float()[:, None]
        return {"q": _rotate(state["q"], cos, sin, case["rotary"], case["layout"]),
                "k": _rotate(state["k"], cos, sin, case["rotary"], case["layout"])}
    if case["kind"] == "store":
        out = {}
        for name in ("k", "v"):
            held = _quantise(state[name])
            out[name] = _values(held, 0, len(state[name])).bfloat16()
        return out
    outs, per = [], len(state["q"]) // len(state["threads"])
    for i, (r, b, e) in enumerate(state["threads"]):
        p0, p1 = state["prompts"][r]
        k = torch.cat([_values(state["k"], p0, p1), _values(state["k"], b, e)])
        v = torch.cat([_values(state["v"], p0, p1), _values(state["v"], b, e)])
        seen = None
        if case["kind"] == "verify":
            seen = _seen(state["masks"][i], len(k) - per, k.device)
        outs.append(_attend(state["q"][i * per:(i + 1) * per].float(), k, v, seen))
    return {"out": torch.cat(outs).bfloat16()}


def _run_own(state):
    case = state["case"]
    if case["kind"] == "rope":
        q, k = state["rope"](state["q"], state["k"], state["pos"])
        return {"q": q, "k": k}
    sess = state["sess"]
    if case["kind"] == "store":
        sess.append_layer(0, state["k"], state["v"])
        k, v = sess.read_kv(state["tids"], state["begin"], state["counts"])
        return {"k": k, "v": v}
    if case["kind"] == "decode":
        return {"out": sess.attention(state["tids"], state["q"])}
    return {"out": sess.verify_attention(state["tids"], state["counts"], state["bits"], state["q"])}


def run(state):
    return _run_own(state) if own else _run_plain(state)


# ------------------------------------------------------------------------ the definition, 64 bits
def _exact_values(x):
    """What the rows of x stand for once held in 4 bits, from the definition in 64 bits."""
    out = torch.empty(x.shape, dtype=torch.float64, device=x.device)
    step = max(1, (1 << 24) // (x.shape[1] * DIM))
    for b in range(0, len(x), step):
        d = x[b:b + step].double()
        for g in range(0, DIM, GROUP):
            part = d[..., g:g + GROUP]
            low, high = part.min(-1, keepdim=True).values, part.max(-1, keepdim=True).values
            # the scale rounded to eight significant bits, ties to even
            mant, expo = torch.frexp((high - low) / 15.0)
            s = torch.ldexp(torch.round(mant * 256.0) / 256.0, expo)
            c = torch.where(s > 0, torch.round((part - low) / torch.where(s > 0, s, 1.0)), 0.0)
            out[b:b + step, :, g:g + GROUP] = low + s * torch.minimum(c, torch.full_like(c, 15.0))
    return out


def _exact_heads(q, k, v, hidden):
    """Queries [m][128] of the heads of one kv head over its rows: softmax(K q / sqrt(128)) V, with the
    weights as exp of scores less the logarithm of their sum; hidden: [m][tokens] or None."""
    s = torch.einsum("td,md->mt", k, q) / math.sqrt(float(DIM))
    if hidden is not None:
        s[hidden] = -math.inf
    w = torch.exp(s - torch.logsumexp(s, 1)[:, None])
    return torch.einsum("mt,td->md", w, v)


def exact(case, seed):
    global own
    was, own = own, False
    try:
        if case["kind"] in ("rope", "store"):
            state = prepare(case, seed)
        else:
            # the same draws as in prepare, in the same order
            g = _generator(seed)
            prompts, threads, total = _forest(case)
            k, v = _rows(total, case["hk"], g), _rows(total, case["hk"], g)
            per = case.get("candidates", 1)
            q = torch.randn(per * len(threads), case["hq"], DIM, generator=g, device="cuda",
                            dtype=torch.bfloat16)
    finally:
        own = was
    if case["kind"] == "rope":
        rd, m = case["rotary"], _magnitude(case)
        angle = state["pos"].double()[:, None, None] * _inv_freq(case).cuda()
        turn = torch.polar(torch.full_like(angle, m), angle)          # a complex turn for each pair
        out = {}
        for name in ("q", "k"):
            x = state[name].double()
            y = x.clone()
            if case["layout"] == "half":
                z = torch.complex(x[..., :rd // 2].contiguous(), x[..., rd // 2:rd].contiguous()) * turn
                y[..., :rd // 2], y[..., rd // 2:rd] = z.real, z.imag
            else:
                z = torch.complex(x[..., 0:rd:2].contiguous(), x[..., 1:rd:2].contiguous()) * turn
                y[..., 0:rd:2], y[..., 1:rd:2] = z.real, z.imag
            out[name] = y
        return out
    if case["kind"] == "store":
        return {"k": _exact_values(state["k"]), "v": _exact_values(state["v"])}
    k, v = _exact_values(k), _exact_values(v)
    masks = _candidate_masks(case, len(threads)) if case["kind"] == "verify" else None
    out = torch.empty(q.shape, dtype=torch.float64, device="cuda")
    group = case["hq"] // case["hk"]
    for i, (r, b, e) in enumerate(threads):
        p0, p1 = prompts[r]
        kk, vv = torch.cat([k[p0:p1], k[b:e]]), torch.cat([v[p0:p1], v[b:e]])
        mine = q[i * per:(i + 1) * per].double()
        hidden = None
        if masks is not None:
            unseen = torch.tensor([[not (m >> x) & 1 for x in range(per)] for m in masks[i]], device="cuda")
            hidden = torch.zeros(per, group, len(kk), dtype=torch.bool, device="cuda")
            hidden[:, :, len(kk) - per:] = unseen[:, None]
            hidden = hidden.flatten(0, 1)
        for h in range(case["hk"]):
            heads = mine[:, h * group:(h + 1) * group].flatten(0, 1)
            got = _exact_heads(heads, kk[:, h], vv[:, h], hidden)
            out[i * per:(i + 1) * per, h * group:(h + 1) * group] = got.unflatten(0, (per, group))
    return {"out": out}
