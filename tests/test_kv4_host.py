"""What of the 4-bit cache and the rotary operator can be checked without a GPU."""
import ctypes as C

import numpy as np
import pytest

from oracle import kv4
from paper_2401_06761_b200 import binding as B


def test_pool_bytes():
    cfg = B.make_config(1000, 32, 8, 64, 40, num_layers=3)
    assert B.apar_kv_pool_bytes(cfg, B.KV_FORMATS["bf16"]) == 3 * 1000 * 8 * 16 * 256
    assert B.apar_kv_pool_bytes(cfg, B.KV_FORMATS["q4"]) == 3 * 1000 * 8 * 16 * 80
    assert B.apar_kv_pool_bytes(cfg, 2) == 0 and B.apar_kv_pool_bytes(cfg, -1) == 0
    assert B.apar_kv_pool_bytes(B.make_config(1000, 32, 8, 64, 40, head_dim=64), 1) == 0


def test_create_refusals():
    cfg = B.make_config(1000, 32, 8, 64, 40)
    for fmt in (0, 1, 2, -1):
        with pytest.raises(B.AparError) as e:
            B.apar_create_kv(cfg, fmt)                 # no pools
        assert e.value.code == "INVALID_ARG"
    bad = B.make_config(1000, 32, 8, 64, 40, block_size=32)
    with pytest.raises(B.AparError) as e:
        B.apar_create_kv(bad, 1)
    assert e.value.code == "UNSUPPORTED"


def test_read_kv_needs_a_device():
    ctx = B.apar_create_host_only(B.make_config(100, 8, 2, 4, 10))
    (t,) = B.apar_new_threads(ctx, 1)
    B.apar_append_kv(ctx, [t], [5], 0, 0)
    with pytest.raises(B.AparError) as e:
        B.apar_read_kv(ctx, 0, [t], [0], [5], 256, 256)
    assert e.value.code == "UNSUPPORTED"
    B.apar_destroy(ctx)


def test_checker_of_the_format():
    """Hand-worked groups, the half-step bound, and its own rounding."""
    x = np.zeros((1, 128), dtype=np.float32)
    x[0, :16] = np.arange(16)
    x[0, 16:32] = [0.5, 1.5, 2.5, 14.5] * 4                    # s = 1: ties go to the even code
    x[0, 32:64] = 7.0
    x[0, 64:96] = np.linspace(-3, 4.5, 32).astype(np.float16)  # s = 0.5
    c, s, lo = kv4.quantise(kv4.round_bf16(x))
    assert s[0, 0] == 1 and lo[0, 0] == 0 and list(c[0, 0, :16]) == list(range(16))
    assert list(c[0, 0, 16:20]) == [0, 2, 2, 14]
    assert s[0, 1] == 0 and lo[0, 1] == 7 and not c[0, 1].any()
    assert s[0, 2] == 0.5 and lo[0, 2] == -3
    rng = np.random.default_rng(0)
    y = kv4.round_bf16(rng.normal(size=(500, 128)))
    c, s, lo = kv4.quantise(y)
    err = np.abs(kv4.values(c, s, lo) - y).reshape(500, 4, 32)
    # half a step, and at the top of the range what rounding s to eight bits costs
    assert (err <= s[..., None] * (0.5 + 15 * 2.0 ** -8)).all()
    assert kv4.round_bf16(np.float32(1 + 2.0 ** -8)) == 1.0
    assert kv4.round_bf16(np.float32(1 + 3 * 2.0 ** -8)) == np.float32(1 + 2.0 ** -6)


ROPE_REFUSED = [dict(rotary_dim=3), dict(rotary_dim=0), dict(rotary_dim=130), dict(base=0.0),
                dict(base=float("nan")), dict(base=float("inf")), dict(scaling="linear", factor=0.0),
                dict(scaling="linear", factor=-2.0), dict(scaling="bands", factor=2.0),
                dict(scaling="bands", factor=2.0, original_len=100, low=4.0, high=4.0),
                dict(scaling="yarn", factor=2.0, original_len=100, base=1.0, high=32.0),
                dict(scaling="yarn", factor=2.0, original_len=100, low=0.0, high=32.0),
                dict(attn_scale=float("nan"))]


@pytest.mark.parametrize("params", ROPE_REFUSED)
def test_rope_parameters_refused(params):
    cfg = B.make_rope_config(**params)
    with pytest.raises(B.AparError) as e:
        B.apar_rope(cfg, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0)
    assert e.value.code == "INVALID_ARG"


def test_rope_arguments_refused():
    """Every refusal comes before a launch: the addresses are never used."""
    cfg, p = B.make_rope_config(), 1 << 20

    def refused(code, *args):
        with pytest.raises(B.AparError) as e:
            B.apar_rope(*args)
        assert e.value.code == code

    refused("UNSUPPORTED", B.make_rope_config(head_dim=64, rotary_dim=64), 1, p, 1, p, 0, p, 0, 0, 0, 0, 0, 0)
    refused("INVALID_ARG", cfg, -1, p, 1, p, 0, p, 0, 0, 0, 0, 0, 0)
    refused("INVALID_ARG", cfg, 1, 0, 1, p, 0, p, 0, 0, 0, 0, 0, 0)                # no positions
    refused("INVALID_ARG", cfg, 1, p + 2, 1, p, 0, p, 0, 0, 0, 0, 0, 0)            # positions off 4 bytes
    refused("INVALID_ARG", cfg, 1, p, 1, 0, 0, p, 0, 0, 0, 0, 0, 0)                # no q
    refused("INVALID_ARG", cfg, 1, p, 0, 0, 0, 0, 0, 2, p, 0, 0, 0)                # no k_out
    refused("INVALID_ARG", cfg, 4, p, 2, p, 255, 2 * p, 0, 0, 0, 0, 0, 0)          # stride below a row
    refused("INVALID_ARG", cfg, 4, p, 2, p + 1, 0, 2 * p, 0, 0, 0, 0, 0, 0)        # odd address
    refused("INVALID_ARG", cfg, 4, p, 2, p, 0, p + 256, 0, 0, 0, 0, 0, 0)          # overlap
    refused("INVALID_ARG", cfg, 4, p, 2, p, 0, p, 512, 0, 0, 0, 0, 0)              # in place, other stride
    refused("INVALID_ARG", cfg, 4, p, 40000, p, 0, 4 * p, 0, 40000, p, 0, 8 * p, 0)
    B.apar_rope(cfg, 0, 0, 4, 0, 0, 0, 0, 4, 0, 0, 0, 0)                           # nothing to do
    B.apar_rope(cfg, 5, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0)


def test_rope_config_layout():
    assert C.sizeof(B.apar_rope_config) == 64


def test_argument_lists():
    """Lists of anything numpy turns into 32-bit ints, as before lists of plain ints got a faster way."""
    for xs in ([3, -1, 2**31 - 1], (x for x in (3, -1, 2**31 - 1)), [3.0, np.float32(-1), 2**31 - 1],
               np.array([3, -1, 2**31 - 1]), [np.int64(3), -1, 2**31 - 1]):
        buf, n = B._arr(xs)
        assert n == 3 and list(buf) == [3, -1, 2**31 - 1]
    assert B._arr([])[1] == 0 and B._arr(range(2))[1] == 2
    with pytest.raises(OverflowError):
        B._arr([2**31])


def test_ancestor_masks_may_be_negative(monkeypatch):
    seen = []

    class Lib:
        @staticmethod
        def apar_tree_verify_attention(ctx, n, tids, cands, masks, q, out, scale, stream):
            seen.append(list(masks))
            return 0
    monkeypatch.setattr(B, "lib", Lib)
    B.apar_tree_verify_attention(None, [0], [2], [1, 2**64 - 1], 0, 0, 1.0)
    B.apar_tree_verify_attention(None, [0], [2], [1, -1], 0, 0, 1.0)
    assert seen == [[1, 2**64 - 1]] * 2


def test_rows_of_an_expanded_tensor():
    """Rope hands apar_rope rows that exist: a stride of 0 between tokens would mean contiguous rows."""
    import torch
    from paper_2401_06761_b200.session import Rope
    one = torch.arange(256).reshape(1, 2, 128).to(torch.bfloat16)
    many = one.expand(5, 2, 128)
    rows = Rope._rows(many, False)
    assert rows.stride(0) == 256 and torch.equal(rows, many)
    with pytest.raises(ValueError):
        Rope._rows(many, True)
    fused = torch.zeros(5, 6, 128, dtype=torch.bfloat16)[:, 1:3]
    for x in (fused, one, many[:1], many[:0]):                 # as they are
        assert Rope._rows(x, False) is x and Rope._rows(x, True) is x


def test_read_kv_takes_lists_of_one_length():
    ctx = B.apar_create_host_only(B.make_config(100, 8, 2, 4, 10))
    t, u = B.apar_new_threads(ctx, 2)
    B.apar_append_kv(ctx, [t, u], [5, 5], 0, 0)
    for tids, begin, count in (([t, u], [0], [5, 5]), ([t, u], [0, 0], [5]), ([t], [0, 0], [5]),
                               ([t], [0], [5, 5]), ([t], [], [])):
        with pytest.raises(B.AparError) as e:
            B.apar_read_kv(ctx, 0, tids, begin, count, 256, 256)
        assert e.value.code == "INVALID_ARG"
    B.apar_destroy(ctx)


def test_lists_shorter_than_the_threads_they_go_with(monkeypatch):
    """Refused before the library would read past them; what is as long or longer goes through."""
    calls = []

    class Lib:
        def __getattr__(self, name):
            if name == "apar_status_string":
                return lambda status: b""
            return lambda *args: calls.append(name) or 0
    monkeypatch.setattr(B, "lib", Lib())
    cfg = B.make_config(100, 8, 2, 4, 3)

    def refused(f, *args):
        before = len(calls)
        with pytest.raises(B.AparError) as e:
            f(*args)
        assert e.value.code == "INVALID_ARG" and len(calls) == before
    refused(B.apar_append_kv, None, [1, 2], [3], 0, 0)
    refused(B.apar_tree_prefix_attention, None, [1, 2], [3], 0, 0, 1.0)
    refused(B.apar_tree_verify_attention, None, [1, 2], [1], [1, 1], 0, 0, 1.0)
    refused(B.apar_tree_verify_attention, None, [1, 2], [1, 2], [1, 1], 0, 0, 1.0)
    refused(B.apar_accept_candidates, None, [1, 2], [1], [[0], [0]])
    refused(B.apar_accept_candidates, None, [1, 2], [1, 1], [[0]])
    refused(B.apar_tree_prefill_attention, None, 0, [1, 2], [0], [1, 1], 0, 0, 1.0)
    refused(B.apar_tree_prefill_attention, None, 0, [1, 2], [0, 0], [1], 0, 0, 1.0)
    refused(B.apar_tree_decode_attention_tables, cfg, [[0, 1, 2], [0, 1]], [16, 16], 0, 0, 1.0)
    B.apar_append_kv(None, [1, 2], None, 0, 0)
    B.apar_append_kv(None, [1, 2], [3, 4, 5], 0, 0)
    B.apar_tree_prefix_attention(None, [1, 2], [3, 4], 0, 0, 1.0)
    B.apar_tree_verify_attention(None, [1, 2], [1, 2], [1, 1, 3], 0, 0, 1.0)
    B.apar_accept_candidates(None, [1, 2], [1, 1], [[0], []])
    B.apar_tree_prefill_attention(None, 0, [1, 2], [0, 0], [1, 1], 0, 0, 1.0)
    B.apar_tree_decode_attention_tables(cfg, [[0, 1, 2], [0, 1, 2]], [16, 16], 0, 0, 1.0)
    assert len(calls) == 7


def test_ancestor_masks_in_arrays(monkeypatch):
    import torch
    seen = []

    class Lib:
        @staticmethod
        def apar_tree_verify_attention(ctx, n, tids, cands, masks, q, out, scale, stream):
            seen.append(list(masks))
            return 0
    monkeypatch.setattr(B, "lib", Lib)
    for masks in (np.array([1, 3], np.uint64), np.array([1, 3]), torch.tensor([1, 3]), (1, 3), [np.uint64(1), 3]):
        B.apar_tree_verify_attention(None, [0], [2], masks, 0, 0, 1.0)
    assert seen == [[1, 3]] * 5
    for masks in (np.array([1, -1]), torch.tensor([1, -1])):   # (negative: the 64 low bits)
        B.apar_tree_verify_attention(None, [0], [2], masks, 0, 0, 1.0)
    assert seen[5:] == [[1, 2**64 - 1]] * 2
    for masks in (np.array([], np.uint64), torch.tensor([], dtype=torch.int64), []):
        B.apar_tree_verify_attention(None, [], [], masks, 0, 0, 1.0)


def test_argument_lists_of_tensors():
    import torch
    for xs in ([torch.tensor(3.0), torch.tensor(-1)], [torch.tensor([3]), -1], torch.tensor([3, -1])):
        buf, n = B._arr(xs)
        assert n == 2 and list(buf) == [3, -1]


def test_argument_lists_that_are_pairs():
    """A tuple of two ints is a list of two; what int32_array made goes through as it is."""
    buf, n = B._arr((5, 7))
    assert n == 2 and list(buf) == [5, 7]
    made = B.int32_array([5, 7, 9])
    assert B._arr(made) is made


def test_a_failed_launch_without_a_context_leaves_its_code():
    """In a process that sees no device: every call fails before anything is launched, and the code
    can be read afterwards, once more after a second call too."""
    import os
    import subprocess
    import sys
    code = """
from paper_2401_06761_b200 import binding as B
assert B.apar_last_cuda_error(None) == 0
for call in (lambda: B.apar_rope(B.make_rope_config(), 1, 4096, 1, 4096, 0, 8192, 0, 0, 0, 0, 0, 0),
             lambda: B.apar_stream_read(4096, 16, 8192)) * 2:
    try:
        call()
        raise SystemExit(2)
    except B.AparError as e:
        assert e.code == "CUDA", e.code
    assert B.apar_last_cuda_error(None) != 0
"""
    env = dict(os.environ, CUDA_VISIBLE_DEVICES="")
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    done = subprocess.run([sys.executable, "-c", code], env=env, cwd=root, capture_output=True, text=True)
    assert done.returncode == 0, done.stderr
