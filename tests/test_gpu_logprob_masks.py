"""Masks in key_bias that are finite: the lowest float leaves a key out as -infinity does.  What such keys do not change are the answers about the others."""
import numpy as np
import pytest

from test_gpu_logprob import TYPES, call, case, rn       # noqa: F401

pytestmark = pytest.mark.gpu

LOWEST = float(np.finfo(np.float32).min)
# few queries, few and many by tiles (the keys' norms along with the product or by themselves; keys in place or copied)
SIZES = [(3, 900, 40), (8, 900, 64), (40, 900, 64), (40, 900, 40), (1100, 900, 64)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("B,M,d", SIZES)
@pytest.mark.parametrize("low", [LOWEST, -2.5e38, -2.1e38])
def test_the_lowest_float_leaves_a_key_out(rn, B, M, d, low, dtype):       # noqa: F811
    """Nine keys are left, six of them side by side, so that groups of keys hold good ones and others; 20 alternatives are asked for."""
    import torch
    c = case(B, M, d, dtype, 21)
    masked = np.ones(M, bool)
    masked[[96, 97, 98, 99, 100, 101, 300, 555, 801]] = False
    c["key_ids"][~masked] = 5000 + np.arange(9)
    c["query_ids"][0] = 5000
    c["target"][-1] = 200        # a masked one
    for few in (False, True):       # nearly all, or nearly none
        out = masked if not few else np.arange(M) % 97 == 1
        ref = dict(c, key_bias=np.where(out, np.float32(-np.inf), np.float32(0.5)))
        got = call(rn, dict(c, key_bias=np.where(out, np.float32(low), np.float32(0.5))), 3.0, 20)
        for x, y in zip(got, call(rn, ref, 3.0, 20)):
            assert torch.equal(x, y)
        if not few:
            assert (got[2][:, 9:] == -1).all() and (got[3][:, 9:] == -float("inf")).all() and (got[2][0] >= 0).sum() == 8
            assert got[0][-1] == 0
    got = call(rn, dict(c, key_bias=np.full(M, low, np.float32)), 3.0, 20)
    assert (got[0] == 0).all() and (got[1] == 0).all() and (got[2] == -1).all() and (got[3] == -float("inf")).all()


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("B,M,d", SIZES)
def test_distances_that_float32_does_not_hold(rn, B, M, d, dtype):       # noqa: F811
    """Logits below about -2e38 count as -infinity, also where a distance made them so."""
    import torch
    c = case(B, M, d, dtype, 22, bias=False)
    c["K"][100:104, 0] = 1.2e19         # 3 |k|^2 = 4.3e38
    c["key_ids"][:] = -1
    c["key_ids"][98:106] = 5000 + np.arange(8)
    c["target"][-1] = 101
    lp, ent, ids, tops = call(rn, c, 3.0, 8)
    assert lp[-1] == -float("inf")
    near = torch.tensor([98, 99, 104, 105], dtype=torch.int32, device="cuda")
    assert torch.equal(ids[:, :4].sort(1)[0], near.expand(B, 4)) and (ids[:, 4:] == -1).all() and (tops[:, 4:] == -float("inf")).all()
    assert torch.isfinite(tops[:, :4]).all() and torch.isfinite(ent).all()
