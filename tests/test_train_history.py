"""The training calls record no history for automatic differentiation, and say so instead of returning tensors that look as if they had none to
record.  (On the CPU what is not refused so is refused for lying in host memory.)"""
import pytest
import torch

import paper_2310_20419_amd as rn


def calls(x):
    ids = torch.zeros(3, dtype=torch.int32)
    plain = torch.zeros(3, 4)
    return (lambda: rn.rnnd_embed(x, ids), lambda: rn.rnnd_embed(plain, ids, out=x), lambda: rn.rnnd_embed_grad(x, ids, 3),
            lambda: rn.rnnd_embed_grad(plain, ids, 3, grad=x), lambda: rn.rnnd_contrast(x, plain, ids, 1.0),
            lambda: rn.rnnd_contrast(plain, x, ids, 1.0), lambda: rn.rnnd_contrast(plain, plain, ids, 1.0, key_bias=x[0]),
            lambda: rn.rnnd_contrast(plain, plain, ids, 1.0, row_weight=x[0]))


def test_tensors_that_require_gradients_are_refused():
    for call in calls(torch.zeros(3, 4, requires_grad=True)):
        with pytest.raises(ValueError, match="records no history"):
            call()


def test_others_and_calls_without_gradients_are_not():
    for call in calls(torch.zeros(3, 4)):
        with pytest.raises(ValueError, match="device memory"):
            call()
    with torch.no_grad():
        for call in calls(torch.zeros(3, 4, requires_grad=True)):
            with pytest.raises(ValueError, match="device memory"):
                call()


@pytest.mark.gpu
def test_under_no_grad_and_detached():
    table = torch.randn(5, 8, device="cuda", requires_grad=True)
    ids = torch.tensor([4, 0, -1], device="cuda", dtype=torch.int32)
    with torch.no_grad():
        a = rn.rnnd_embed(table, ids)
    b = rn.rnnd_embed(table.detach(), ids)
    assert torch.equal(a, b) and torch.equal(a[:2], table.detach()[[4, 0]]) and not a.requires_grad
    with pytest.raises(ValueError):
        rn.rnnd_embed(table, ids)
    with pytest.raises(ValueError):
        rn.rnnd_contrast(table, table.detach(), ids, 1.0)
