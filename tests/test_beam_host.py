"""Refusals of beam selection: made before anything is launched, so no GPU is needed."""
import pytest

from paper_2401_06761_b200 import binding as B

GOOD = dict(vocab=100, num_beams=4, num_select=8, logits_type="bfloat16", eos=2)
ADDR = 1 << 20                    # an address that is aligned and never touched


def call(cfg, n=1, logits=ADDR, scores=ADDR, finished=0, out=ADDR, work=ADDR, nbytes=1 << 20):
    B.apar_beam_select(cfg, n, logits, 0, 0, scores, finished, out, out, out, work, nbytes)


@pytest.mark.parametrize("change", [
    dict(vocab=0), dict(vocab=1 << 28), dict(num_beams=0), dict(num_beams=65), dict(num_select=0),
    dict(num_select=65), dict(eos=100), dict(eos=-2)])
def test_bad_configurations(change):
    cfg = B.make_beam_config(**{**GOOD, **change})
    assert B.apar_beam_workspace_bytes(cfg, 1) == 0
    with pytest.raises(B.AparError) as e:
        call(cfg)
    assert e.value.code == "INVALID_ARG"


def test_unknown_logits_type():
    cfg = B.make_beam_config(**GOOD)
    for t in (-1, 3):
        cfg.logits_type = t
        with pytest.raises(B.AparError):
            call(cfg)


@pytest.mark.parametrize("args", [
    dict(n=-1), dict(n=1 << 30), dict(logits=0), dict(scores=0), dict(out=0), dict(work=0),
    dict(logits=ADDR + 1), dict(scores=ADDR + 2), dict(out=ADDR + 2), dict(work=ADDR + 128)])
def test_bad_arguments(args):
    with pytest.raises(B.AparError) as e:
        call(B.make_beam_config(**GOOD), **args)
    assert e.value.code == "INVALID_ARG"


def test_finished_beams_need_an_end_token():
    with pytest.raises(B.AparError) as e:
        call(B.make_beam_config(**{**GOOD, "eos": None}), finished=ADDR)
    assert e.value.code == "INVALID_ARG"


def test_scratch_too_small_and_no_sequences():
    cfg = B.make_beam_config(**GOOD)
    need = B.apar_beam_workspace_bytes(cfg, 3)
    assert need > 0
    with pytest.raises(B.AparError) as e:
        call(cfg, n=3, nbytes=need - 1)
    assert e.value.code == "WORKSPACE_TOO_SMALL"
    call(cfg, n=0, logits=0, scores=0, out=0, work=0)    # nothing to do
