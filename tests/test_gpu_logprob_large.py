"""Log probabilities where logits are so large that a step of float32 is more than the exponent's range: whatever the sums make of them, answers are
numbers, and the order of the alternatives is that of double precision."""
import numpy as np
import pytest

from test_gpu_logprob import U, call, error_of_a_logit, logits_of, rn       # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["float16", "bfloat16", "float32"])
@pytest.mark.parametrize("B,M,d,size", [(20, 3000, 64, 3000.0), (1100, 2000, 64, 3000.0), (200, 131_072, 192, 1300.0), (4, 3000, 64, 3000.0)])
def test_logits_of_many_millions(rn, B, M, d, size, dtype):       # noqa: F811
    """|k|^2 of some 3 to 6e8, logits in base 2 of 2^28 and more (tiles of 256 keep groups of 8 keys) or 2^29 (groups of 4).  A logit is off by e, so lse
    and a log probability are (both change by no more than the logits do), and by the joins of the sums."""
    import torch
    g = np.random.Generator(np.random.PCG64(B + M))
    K = torch.from_numpy(g.normal(size=(M, d)) * size).to(getattr(torch, dtype)).cuda()
    Q = torch.from_numpy(g.normal(size=(B, d)) * size).to(getattr(torch, dtype)).cuda()
    c = dict(Q=Q, K=K, target=g.integers(0, M, size=B).astype(np.int32))
    s, out, bias = logits_of(c, 1.0)
    top = s.max(1, keepdims=True)
    logp = s - top - np.log(np.exp(s - top).sum(1, keepdims=True))
    bound = error_of_a_logit(c, 1.0, bias, out) + (300 + M / 250) * U
    lp, ent, ids, tops = call(rn, c, 1.0, 12)
    assert torch.isfinite(lp).all() and torch.isfinite(ent).all() and (ent >= 0).all() and (ent <= np.log(M) + 1e-3).all()
    order = np.argsort(-s, axis=1, kind="stable")[:, :12]
    assert (ids.cpu().numpy() == order).all()
    for got, at in ((tops, order), (lp[:, None], c["target"][:, None].astype(np.int64))):
        want = np.take_along_axis(logp, at, 1)
        assert (abs(got.double().cpu().numpy() - want) <= bound[:, None] + 4 * U * abs(want)).all()
    assert torch.isfinite(call(rn, c, 1.0, 0)[1]).all()
