"""Distillation with finite masks in key_bias, and with a teacher's numbers that are no log probabilities."""
import numpy as np
import pytest

from test_gpu_distill import TYPES, call, case, rn       # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("tail", [False, True])
@pytest.mark.parametrize("low", [float(np.finfo(np.float32).min), -2.1e38])
def test_the_lowest_float_leaves_a_key_out(rn, low, tail, dtype):       # noqa: F811
    """As -infinity does, on a list and off it; a query all of whose keys are masked does not count."""
    import torch
    c = case(70, 300, 40, 8, dtype, 31)
    out = np.arange(300) % 3 == 1
    c["teacher_ids"][5] = 1         # only masked ones
    for masked in (out, np.ones(300, bool)):
        want = call(rn, dict(c, key_bias=np.where(masked, np.float32(-np.inf), c["key_bias"])), 3.0, tail)
        got = call(rn, dict(c, key_bias=np.where(masked, np.float32(low), c["key_bias"])), 3.0, tail)
        for x, y in zip(got, want):
            assert torch.equal(x, y)
        assert got[0][5] == 0 and (got[1][5] == 0).all()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("add", [80.0, 700.0, 1000.0, 1e30])
def test_more_than_a_probability_with_the_rest(rn, add, dtype):       # noqa: F811
    """tail = 1: numbers that add up to more than 1 are divided by their sum, however large they are (exp(710) is beyond double precision)."""
    import torch
    c = case(40, 200, 24, 6, dtype, 32)
    c["teacher_logits"] = np.where(np.isfinite(c["teacher_logits"]), np.round(c["teacher_logits"] * 16) / 16 + np.float32(add), -np.inf).astype(np.float32)
    want = call(rn, c, 3.0, False)      # above 1 there is no rest
    got = call(rn, c, 3.0, True)
    for x, y in zip(got, want):
        assert torch.isfinite(x.float()).all()
        # p is formed in double precision both times, from differences of about 10 (rounded to steps of 2^-4, so all but 1e30 hold them); float32 from there on
        assert (x.double() - y.double()).abs().max() <= 2.0 ** -20 * (1 + y.double().abs().max())
