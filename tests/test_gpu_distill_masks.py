"""Distillation with finite masks in key_bias."""
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
