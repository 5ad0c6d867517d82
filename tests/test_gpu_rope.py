"""Rotary positions against a 64-bit evaluation of the formula."""
import math

import numpy as np
import pytest
import torch

from kv4_helpers import host
from paper_2401_06761_b200 import binding as B
from paper_2401_06761_b200.session import Rope

pytestmark = pytest.mark.gpu


def _theta(rd, base=10000.0, scaling="none", factor=1.0, original_len=0, low=1.0, high=4.0, **_):
    out = []
    for i in range(rd // 2):
        t = base ** (-2.0 * i / rd)
        if scaling == "linear":
            t /= factor
        elif scaling == "bands":
            turns = original_len * t / (2 * math.pi)
            w = min(1.0, max(0.0, (turns - low) / (high - low)))
            t = (1 - w) * t / factor + w * t
        elif scaling == "yarn":
            at = lambda n: rd * math.log(original_len / (n * 2 * math.pi)) / (2 * math.log(base))
            a, b = max(0, math.floor(at(high))), min(rd - 1, math.ceil(at(low)))
            r = min(1.0, max(0.0, (i - a) / max(b - a, 0.001)))
            t = r * t / factor + (1 - r) * t
        out.append(t)
    return np.array(out)


def _expect(x, pos, rd, layout, attn_scale=1.0, **scaling):
    x = host(x).astype(np.float64)
    ang = pos.cpu().numpy().astype(np.float64)[:, None] * _theta(rd, **scaling)
    c, s = np.cos(ang)[:, None] * attn_scale, np.sin(ang)[:, None] * attn_scale
    y = x.copy()
    a = slice(0, rd // 2) if layout == "half" else slice(0, rd, 2)
    b = slice(rd // 2, rd) if layout == "half" else slice(1, rd, 2)
    y[..., a], y[..., b] = x[..., a] * c - x[..., b] * s, x[..., b] * c + x[..., a] * s
    size = np.abs(x)
    size[..., a] = size[..., b] = abs(attn_scale) * (np.abs(x[..., a]) + np.abs(x[..., b]))
    return y, size


def _check(got, x, pos, rd, layout, **kw):
    """Half a bf16 step of the result, and 32-bit arithmetic on the two products: cos and sin are
    good to 2^-22 (a reduced angle below 4 rounded to 32 bits, 2^-23 absolute, and the function's
    own two units), the products and their sum add 2^-23 of their size."""
    ref, size = _expect(x, pos, rd, layout, **kw)
    err = np.abs(host(got).astype(np.float64) - ref)
    assert (err <= 2.0 ** -8 * np.abs(ref) + 2.0 ** -20 * size).all(), err.max()
    if rd < 128:
        assert torch.equal(got[..., rd:], x[..., rd:])


def _inputs(n, hq, hk, seed, max_pos=100000):
    g = torch.Generator(device="cuda").manual_seed(seed)
    qkv = torch.randn(n, hq + 2 * hk, 128, generator=g, device="cuda").to(torch.bfloat16)
    pos = torch.randint(0, max_pos, (n,), generator=g, device="cuda", dtype=torch.int32)
    return qkv, pos


@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("rd", [2, 6, 16, 20, 32, 64, 96, 126, 128])
@pytest.mark.parametrize("n,hq,hk", [(1, 1, 1), (3, 8, 2), (130, 5, 3)])
def test_against_formula(layout, rd, n, hq, hk):
    qkv, pos = _inputs(n, hq, hk, rd)
    rope = Rope(rotary_dim=rd, layout=layout)
    keep = qkv.clone()
    q, k = rope(qkv[:, :hq], qkv[:, hq:hq + hk], pos)
    _check(q, qkv[:, :hq], pos, rd, layout)
    _check(k, qkv[:, hq:hq + hk], pos, rd, layout)
    assert torch.equal(qkv, keep)
    rope(qkv[:, :hq], qkv[:, hq:hq + hk], pos, inplace=True)
    assert torch.equal(qkv[:, :hq], q) and torch.equal(qkv[:, hq:hq + hk], k)
    assert torch.equal(qkv[:, hq + hk:], keep[:, hq + hk:])          # V of the fused rows


@pytest.mark.parametrize("kw", [
    dict(scaling="linear", factor=8.0),
    dict(scaling="bands", factor=8.0, original_len=8192, low=1.0, high=4.0, base=500000.0),
    dict(scaling="yarn", factor=4.0, original_len=4096, low=1.0, high=32.0, attn_scale=1.1386),
    dict(scaling="yarn", factor=32.0, original_len=2048, low=1.0, high=32.0, base=1e6),
    dict(attn_scale=-0.5), dict(base=0.5)])
@pytest.mark.parametrize("rd", [64, 128])
def test_scalings(kw, rd):
    qkv, pos = _inputs(200, 4, 2, 5, 1 << 20)
    q, k = Rope(rotary_dim=rd, **kw)(qkv[:, :4], qkv[:, 4:6], pos)
    _check(q, qkv[:, :4], pos, rd, "half", **kw)
    _check(k, qkv[:, 4:6], pos, rd, "half", **kw)


def test_extreme_positions():
    pos = torch.tensor([0, -1, 1, 2 ** 31 - 1, -2 ** 31, 1 << 20], dtype=torch.int32, device="cuda")
    x = torch.randn(6, 2, 128, device="cuda").to(torch.bfloat16)
    (q, none) = Rope()(x, None, pos)
    assert none is None
    _check(q, x, pos, 128, "half")
    assert torch.equal(q[0], x[0])


def test_many_tokens_and_only_one_side():
    """Enough tokens for several to a CTA, a last CTA that is not full."""
    qkv, pos = _inputs(4099, 3, 2, 9)
    q, _ = Rope(layout="interleaved")(qkv[:, :3], None, pos)
    _check(q, qkv[:, :3], pos, 128, "interleaved")
    q2, k2 = Rope(layout="interleaved")(qkv[:, :3], qkv[:, 3:5], pos)
    assert torch.equal(q, q2)
    _check(k2, qkv[:, 3:5], pos, 128, "interleaved")


@pytest.mark.parametrize("layout", ["half", "interleaved"])
def test_rows_off_the_sixteen_byte_grid(layout):
    """Odd offsets and strides take the element-wise kernel and give the same numbers."""
    n, h = 9, 3
    x = torch.randn(n, h, 128, device="cuda").to(torch.bfloat16)
    pos = torch.arange(n, dtype=torch.int32, device="cuda") * 1001
    want, _ = Rope(layout=layout)(x, None, pos)
    buf = torch.zeros(n * (h * 128 + 3) + 1, dtype=torch.bfloat16, device="cuda")
    view = buf[1:].as_strided((n, h, 128), (h * 128 + 3, 128, 1), 1)
    view.copy_(x)
    got, _ = Rope(layout=layout)(view, None, pos)
    assert torch.equal(got, want)


def test_captured_in_a_graph():
    x = torch.randn(5, 4, 128, device="cuda").to(torch.bfloat16)
    pos = torch.arange(5, dtype=torch.int32, device="cuda")
    out = torch.empty_like(x)
    rope = Rope()
    stream, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()

    def call():
        B.apar_rope(rope.cfg, 5, pos.data_ptr(), 4, x.data_ptr(), 0, out.data_ptr(), 0, 0, 0, 0, 0, 0,
                    torch.cuda.current_stream().cuda_stream)
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=stream):
        call()
        pos.add_(1)
    for step in range(3):
        graph.replay()
        torch.cuda.synchronize()
        _check(out, x, pos - 1, 128, "half")
    assert int(pos[0]) == 3


def test_one_row_expanded_to_all_tokens():
    x = torch.randn(1, 3, 128, device="cuda").to(torch.bfloat16)
    pos = torch.arange(7, dtype=torch.int32, device="cuda")
    many, before = x.expand(7, 3, 128), x.clone()
    rope = Rope()
    q, k = rope(many, many[:, :1], pos)
    _check(q, many, pos, 128, "half")
    assert torch.equal(k, q[:, :1])
    with pytest.raises(ValueError):
        rope(many, None, pos, inplace=True)
    with pytest.raises(B.AparError):                           # rows that overlap
        rope(torch.zeros(20 * 128, dtype=torch.bfloat16, device="cuda").as_strided((7, 3, 128), (128, 128, 1)),
             None, pos)
    assert torch.equal(x, before)
