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


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("mask", [-1e9, -1e30])
def test_all_keys_off_the_lists_masked(rn, mask, dtype):       # noqa: F811
    """What the teacher left has only masked keys to go to.  Their logits are as good as equal (a step of float32 is 64 or more there), and however it is
    divided among them, g is R - r = -r in all; on the list it is P - p.  So a query's gradient is 2 scale w times differences that add up to 1 + 2 r
    in weight, and the loss is r times the mask but for 4 steps and terms that do not grow with it."""
    import torch
    B, M, d, n = 50, 3000, 48, 6
    c = case(B, M, d, n, dtype, 33, ids=False, mass=0.9)
    c["teacher_ids"] = np.tile(np.arange(n) * 400, (B, 1)).astype(np.int32)
    c["teacher_logits"] = np.log(np.tile(np.linspace(1, 2, n) / 10, (B, 1))).astype(np.float32)
    r = 1 - np.exp(c["teacher_logits"].astype(np.float64)).sum(1)
    c["key_bias"] = np.full(M, mask, np.float32)
    c["key_bias"][c["teacher_ids"][0]] = 0.0
    c["row_weight"] = np.ones(B, np.float32)
    loss, dq, dk = call(rn, c, 3.0, True)
    assert (abs(loss.double().cpu().numpy() + r * mask) <= 8 * 2.0 ** -24 * abs(mask) + 100).all()
    q, k = c["Q"].double(), c["K"].double()
    # (16-bit rows: a product's g is off by half a step of itself, 2^-9, and the result by as much)
    assert (dq.double().abs() <= 2 * 3.0 * (1 + 2 * r.max()) * (k.abs().max() + q.abs().max()) * (1 + 2.0 ** -7)).all()
    listed = torch.zeros(M, dtype=torch.bool, device="cuda")
    listed[torch.from_numpy(c["teacher_ids"][0]).long().cuda()] = True
    # the keys off the lists: -r of each query among them all
    assert dk[~listed].double().abs().sum(0).max() <= 2 * 3.0 * r.sum() * (k.abs().max() + q.abs().max()) * (1 + 2.0 ** -7)
