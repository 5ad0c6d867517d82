"""4-bit attention where rounding could add up: long units, keys with channel offsets, rows whose
groups and blocks whose tokens differ in size.

Two measures.  `check` of kv4_helpers bounds every element.  `check_norm` bounds the error of a whole
result against its norm: an output rounded to bf16 is off by an even spread over half a step, which
is 2^-8 / sqrt(3) of a number at the bottom of its binade and 0.72 of that on average, 0.0016; all
else - weights rounded to 11 bits, each multiplying a deviation from the middle of its group, values
rounded to 11 bits, 32-bit sums - gets 2^-10 together, and the two are independent:
sqrt(0.0016^2 + 2^-20) < 2^-9."""
import numpy as np
import pytest
import torch

from oracle import kv4
from kv4_helpers import Kv4Pair, check, host, rows
from paper_2401_06761_b200 import binding as B
from paper_2401_06761_b200.session import PagedSession
from paper_2401_06761_b200.synth import LayerShape

pytestmark = pytest.mark.gpu

# query heads per kv head of a single thread decide which kernel takes it: up to four rows, up to
# eight, more
WIDTHS = [(4, 2), (16, 2), (32, 2)]


def check_norm(got, ref, what=""):
    got = host(got).astype(np.float64)
    assert np.isfinite(got).all(), f"{what}: non-finite output"
    err = np.linalg.norm(got - ref) / np.linalg.norm(ref)
    assert err <= 2.0 ** -9, f"{what}: error {err} of the result"


def _attention(q, k, v, scale):
    """q [heads][128] over k, v [tokens][kv heads][128] (values), in 64 bits on the device."""
    q = q.double().reshape(k.shape[1], -1, 128)
    w = torch.softmax(torch.einsum("hgd,thd->hgt", q, k) * scale, -1)
    return torch.einsum("hgt,thd->hgd", w, v).reshape(-1, 128).cpu().numpy()


@pytest.mark.parametrize("group", [1, 4, 8, 16])
def test_flat_scores_over_long_units(group):
    """Enough threads that none is cut into pieces: 32768 tokens to one unit, every weight alike, so
    that the result is hundreds of times smaller than what is summed."""
    hk, threads, n = 8, 256, 32768
    sess = PagedSession(LayerShape(hk * group, hk), threads * (n // 16) + 16, threads, n // 16 + 1,
                        kv_format="q4")
    tids = sess.new_threads(threads)
    g = torch.Generator(device="cuda").manual_seed(1)
    k, v = (torch.randn(n, 2, 128, generator=g, device="cuda").to(torch.bfloat16) for _ in range(2))
    k_all, v_all = k.repeat(1, hk // 2, 1), v.repeat(1, hk // 2, 1)
    for t in tids:
        sess.append([t], [n], k_all, v_all)
    q = (torch.randn(threads, hk * group, 128, generator=g, device="cuda") * 0.02).to(torch.bfloat16)
    q[1] = 0.0                                                 # every weight the same number
    got = sess.attention(tids, q)
    assert torch.equal(got, sess.attention(tids, q))
    assert sess.stats()["attn_work_items"] == threads          # (none is cut)
    kv, vv = (torch.from_numpy(kv4.values(*kv4.quantise(host(x)))).cuda() for x in (k, v))
    for i in (0, 1, 100, 255):
        check_norm(got[i, :2 * group], _attention(q[i, :2 * group], kv, vv, sess.sm_scale), f"thread {i}")
    sess.close()


@pytest.mark.parametrize("hq,hk", WIDTHS)
@pytest.mark.parametrize("offset,query", [(0, 1), (16, 4), (40, 8), (100, 10), (200, 20)])
def test_keys_with_channel_offsets(offset, query, hq, hk):
    """Two channels with an offset each, whose shares of a score cancel but for their spread."""
    p = Kv4Pair(hq, hk, num_blocks=256, max_blocks=200)
    (t,) = p.new_threads(1)
    n = 1500
    k = rows(n, hk, 11).float()
    k[..., 5] += offset
    k[..., 70] += offset
    q = rows(1, hq, 12)
    q[..., 5], q[..., 70] = query, -query
    p.append([t], [n], k.to(torch.bfloat16), rows(n, hk, 13))
    got = p.sess.attention([t], q)
    check_norm(got, p.expected([t], q, p.sess.sm_scale)[0])
    p.close()


@pytest.mark.parametrize("hq,hk", WIDTHS)
@pytest.mark.parametrize("bits", [2, 4, 8, 10, 12])
def test_one_large_key_row_in_a_block(bits, hq, hk):
    """Its neighbours' scores stay what they are.  (The large row's own score is made very low.)"""
    p = Kv4Pair(hq, hk, num_blocks=64)
    (t,) = p.new_threads(1)
    n = 200
    k, q = rows(n, hk, 21).float(), rows(1, hq, 22)
    for i in range(3, n, 16):
        k[i] = -(2.0 ** bits) * q[0, ::hq // hk].float()
    p.append([t], [n], k.to(torch.bfloat16), rows(n, hk, 23))
    p.check_attention([t], q)
    p.close()


@pytest.mark.parametrize("hq,hk", WIDTHS)
@pytest.mark.parametrize("bits", [4, 8, 10, 16, 20])
@pytest.mark.parametrize("n", [1, 64, 500])
def test_groups_of_a_v_row_of_different_size(n, bits, hq, hk):
    p = Kv4Pair(hq, hk, num_blocks=64)
    (t,) = p.new_threads(1)
    v = rows(n, hk, 31).float()
    v[..., 32:64] *= 2.0 ** bits
    v[..., 64:96] *= 2.0 ** (bits // 2)
    p.append([t], [n], rows(n, hk, 32), v.to(torch.bfloat16))
    p.check_attention([t], rows(1, hq, 33))
    p.close()


@pytest.mark.parametrize("hq,hk", WIDTHS)
def test_rows_of_zeros_beside_a_large_one_keep_their_weight(hq, hk):
    """3000 rows of V that are zero, each with 2^-12 of the weight of a row of size 2^24."""
    p = Kv4Pair(hq, hk, num_blocks=256, max_blocks=200)
    (t,) = p.new_threads(1)
    n = 3001
    k, v = torch.zeros(n, hk, 128), torch.zeros(n, hk, 128)
    k[777, :, 0] = 12.0
    v[777] = rows(1, hk, 41)[0].float().cpu() * 2.0 ** 24
    q = torch.zeros(1, hq, 128)
    q[..., 0] = 1.0
    p.append([t], [n], k.to(torch.bfloat16).cuda(), v.to(torch.bfloat16).cuda())
    p.check_attention([t], q.to(torch.bfloat16).cuda(), scale=float(np.log(2.0)))
    p.close()


@pytest.mark.parametrize("hq,hk", WIDTHS)
def test_keys_whose_groups_are_flat(hq, hk):
    """Scales of 0: all of a score is in the offsets.  And rows that mix flat groups with others."""
    p = Kv4Pair(hq, hk, num_blocks=64)
    (t,) = p.new_threads(1)
    n = 150
    k = rows(n, hk, 51).float().reshape(n, hk, 4, 32)
    k[:100] = k[:100, ..., :1]
    k[100:120, :, 1] = k[100:120, :, 1, :1] * 64.0
    k[140:] = 0.0
    p.append([t], [n], k.reshape(n, hk, 128).to(torch.bfloat16), rows(n, hk, 52))
    p.check_attention([t], rows(1, hq, 53))
    p.close()


@pytest.mark.parametrize("hq,hk", WIDTHS)
@pytest.mark.parametrize("bits", [100, 60, -60, -90])
def test_keys_and_queries_far_from_one(bits, hq, hk):
    """Keys of size 2^bits under queries of 2^-bits: ordinary scores."""
    p = Kv4Pair(hq, hk, num_blocks=64)
    (t,) = p.new_threads(1)
    k, q = rows(130, hk, 61).float() * 2.0 ** bits, rows(1, hq, 62).float() * 2.0 ** -bits
    p.append([t], [130], k.to(torch.bfloat16), rows(130, hk, 63))
    p.check_attention([t], q.to(torch.bfloat16))
    p.close()


@pytest.mark.parametrize("hq,hk", WIDTHS)
@pytest.mark.parametrize("offset", [1000, 4000])
def test_one_channel_of_the_keys_far_above_the_rest(offset, hq, hk):
    """The other groups' scales are hundreds of times smaller and decide the scores."""
    p = Kv4Pair(hq, hk, num_blocks=256, max_blocks=200)
    (t,) = p.new_threads(1)
    n = 1500
    k = rows(n, hk, 71).float()
    k[..., 40] = offset
    q = rows(1, hq, 72)
    q[..., 40] = 0.0
    p.append([t], [n], k.to(torch.bfloat16), rows(n, hk, 73))
    got = p.sess.attention([t], q)
    check_norm(got, p.expected([t], q, p.sess.sm_scale)[0])
    p.close()
