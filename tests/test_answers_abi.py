"""CPU-side checks of the log probabilities and of distillation: what they refuse, before any GPU call, and what their workspace queries say."""
import ctypes
import os

import pytest

import paper_2310_20419_amd as rn

ONE = ctypes.c_void_p(256)      # never dereferenced: validation comes first
ODD = ctypes.c_void_p(258)
BIG = 1 << 45


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(rn.lib_path()):
        from paper_2310_20419_amd import build
        build.build()
    return rn.load_library()


def test_distill_refusals(lib):
    def call(Q=ONE, B=4, K=ONE, M=6, d=8, dtype=3, metric=0, ti=ONE, tl=ONE, n=3, tail=1, qi=None, ki=None, bias=None, w=None, scale=1.0,
             loss=ONE, dQ=ONE, dK=ONE, ws=ONE, size=BIG):
        return lib.rnnd_distill(Q, B, K, M, d, dtype, metric, ti, tl, n, tail, qi, ki, bias, w, scale, loss, dQ, dK, ws, size, None)
    assert call(dtype=0) == -4 and call(dtype=4) == -4 and call(metric=1) == -4
    assert call(B=-1) == -2 and call(M=0) == -2 and call(M=2**20 + 1) == -2 and call(B=2**20 + 1) == -2 and call(d=0) == -2 and call(d=65537) == -2
    assert call(n=0) == -3 and call(n=129) == -3 and call(tail=2) == -3 and call(tail=-1) == -3
    for missing in ("Q", "K", "ti", "tl", "loss", "ws", "dQ", "dK"):
        assert call(**{missing: None}) == -1, missing
    assert call(qi=ONE) == -1       # query ids without key ids
    assert call(scale=float("nan")) == -3 and call(scale=float("inf")) == -3
    for bad in ("ti", "tl", "qi", "ki", "bias", "w", "loss"):
        assert call(**dict(dict(ki=ONE), **{bad: ODD})) == -3, bad
    assert call(Q=ctypes.c_void_p(257)) == -3 and call(dK=ODD, dtype=1) == -3 and call(ws=ctypes.c_void_p(264)) == -3
    for want in (True, False):
        need = rn.rnnd_distill_workspace(4, 6, 8, rn.RNND_BF16, 3, want)
        assert call(size=need - 1, **({} if want else dict(dQ=None, dK=None))) == -7
    assert rn.rnnd_distill_workspace(4, 6, 8, rn.RNND_BF16, 3, False) < rn.rnnd_distill_workspace(4, 6, 8, rn.RNND_BF16, 3, True)
    assert call(B=0, Q=None, ti=None, tl=None, loss=None, dQ=None, dK=None, ws=None, size=0) == 0
    assert rn.rnnd_distill_workspace(0, 6, 8, rn.RNND_BF16, 3) == 0
    assert lib.rnnd_distill_workspace(4, 6, 8, 3, 3, 1, None) == -1
    with pytest.raises(rn.RnndError):
        rn.rnnd_distill_workspace(4, 6, 8, rn.RNND_BF16, 129)


def test_logprob_refusals(lib):
    def call(Q=ONE, B=4, K=ONE, M=6, d=8, dtype=3, metric=0, t=ONE, qi=None, ki=None, bias=None, scale=1.0, k=2, lp=ONE, ent=ONE, ids=ONE,
             top=ONE, ws=ONE, size=BIG):
        return lib.rnnd_logprob(Q, B, K, M, d, dtype, metric, t, qi, ki, bias, scale, k, lp, ent, ids, top, ws, size, None)
    assert call(dtype=0) == -4 and call(metric=1) == -4
    assert call(B=-1) == -2 and call(M=0) == -2 and call(M=2**20 + 1) == -2 and call(B=2**20 + 1) == -2 and call(d=0) == -2
    assert call(k=-1) == -3 and call(k=129) == -3
    for missing in ("Q", "K", "t", "lp", "ids", "top", "ws"):
        assert call(**{missing: None}) == -1, missing
    assert call(qi=ONE) == -1
    assert call(scale=float("nan")) == -3 and call(scale=float("-inf")) == -3
    for bad in ("t", "qi", "ki", "bias", "lp", "ent", "ids", "top"):
        assert call(**dict(dict(ki=ONE), **{bad: ODD})) == -3, bad
    assert call(K=ctypes.c_void_p(257)) == -3 and call(ws=ctypes.c_void_p(264)) == -3
    for B in (4, 40):
        need = rn.rnnd_logprob_workspace(B, 6, 8, rn.RNND_BF16, 2)
        assert call(B=B, size=need - 1) == -7
    assert call(B=0, Q=None, t=None, lp=None, ent=None, ids=None, top=None, ws=None, size=0) == 0
    assert rn.rnnd_logprob_workspace(0, 6, 8, rn.RNND_BF16, 2) == 0
    assert lib.rnnd_logprob_workspace(4, 6, 8, 3, 2, None) == -1


def test_the_workspace_of_log_probabilities_does_not_grow_with_the_queries_for_ever():
    """Queries go through the keys in runs: a million queries against a million keys work in a few GB."""
    assert rn.rnnd_logprob_workspace(2**20, 2**20, 96, rn.RNND_F32, 10) < 4 << 30
    assert rn.rnnd_logprob_workspace(1, 2**20, 96, rn.RNND_F32, 10) < 4 << 20


def test_the_binding_refuses_what_it_cannot_pass_on():
    import torch
    with pytest.raises(ValueError):
        rn.rnnd_logprob(torch.zeros(3, 4), torch.zeros(3, 4), 1.0)
    with pytest.raises(ValueError):
        rn.rnnd_distill(torch.zeros(3, 4), torch.zeros(3, 4), torch.zeros(3, 2, dtype=torch.int32), torch.zeros(3, 2), 1.0)
    with pytest.raises(ValueError):
        rn.rnnd_logprob(torch.zeros(3, 4, requires_grad=True), torch.zeros(3, 4), 1.0)
