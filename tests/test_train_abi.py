"""CPU-side checks of the calls that train rows: what they refuse, before any GPU call, and what their workspace queries say."""
import ctypes
import os

import pytest

import paper_2310_20419_amd as rn
from paper_2310_20419_amd import _binding

ONE = ctypes.c_void_p(256)      # never dereferenced: validation comes first
BIG = 1 << 40


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(rn.lib_path()):
        from paper_2310_20419_amd import build
        build.build()
    return rn.load_library()


def test_embed_refusals(lib):
    def call(table=ONE, V=100, d=8, dtype=1, ids=ONE, n=5, out=ONE, out_dtype=1):
        return lib.rnnd_embed(table, V, d, dtype, ids, n, 1.0, out, out_dtype, None)
    assert call(dtype=0) == -4 and call(dtype=4) == -4 and call(out_dtype=0) == -4 and call(out_dtype=-1) == -4
    assert call(V=0) == -2 and call(V=2**31 - 1) == -2 and call(d=0) == -2 and call(d=65537) == -2 and call(n=-1) == -2
    assert call(table=None) == -1 and call(ids=None) == -1 and call(out=None) == -1
    assert call(table=ctypes.c_void_p(258)) == -3 and call(ids=ctypes.c_void_p(258)) == -3
    assert call(out=ctypes.c_void_p(257), out_dtype=2) == -3
    assert call(n=0, ids=None, out=None) == 0


def test_embed_grad_refusals(lib):
    def call(dout=ONE, dtype=1, ids=ONE, n=5, d=8, V=100, grad=ONE, grad_dtype=1, acc=0, ws=ONE, size=BIG):
        return lib.rnnd_embed_grad(dout, dtype, ids, n, d, 1.0, V, grad, grad_dtype, acc, ws, size, None)
    assert call(dtype=0) == -4 and call(grad_dtype=7) == -4 and call(V=0) == -2 and call(d=0) == -2 and call(n=-1) == -2
    assert call(dout=None) == -1 and call(ids=None) == -1 and call(grad=None) == -1 and call(ws=None) == -1
    assert call(acc=2) == -3 and call(ws=ctypes.c_void_p(264)) == -3 and call(grad=ctypes.c_void_p(257)) == -3
    need = rn.rnnd_embed_grad_workspace(5, 8, 100)
    assert call(size=need - 1) == -7 and "workspace" in rn.rnnd_strerror(-7)
    assert call(n=0, acc=1, dout=None, ids=None) == 0       # nothing to add
    assert rn.rnnd_embed_grad_workspace(1_000_000, 96, 1_000_000) < 64 << 20
    assert lib.rnnd_embed_grad_workspace(5, 8, 100, None) == -1
    with pytest.raises(rn.RnndError):
        rn.rnnd_embed_grad_workspace(-1, 8, 100)


def test_contrast_refusals(lib):
    def call(Q=ONE, B=4, K=ONE, M=6, d=8, dtype=3, metric=0, t=ONE, qi=None, ki=None, bias=None, w=None, scale=1.0, loss=ONE,
             dQ=ONE, dK=ONE, ws=ONE, size=BIG):
        return lib.rnnd_contrast(Q, B, K, M, d, dtype, metric, t, qi, ki, bias, w, scale, loss, dQ, dK, ws, size, None)
    assert call(dtype=0) == -4 and call(metric=1) == -4
    assert call(B=-1) == -2 and call(M=0) == -2 and call(M=2**20 + 1) == -2 and call(B=2**20 + 1) == -2 and call(d=0) == -2
    assert call(Q=None) == -1 and call(K=None) == -1 and call(t=None) == -1 and call(loss=None) == -1 and call(ws=None) == -1
    assert call(dQ=None) == -1 and call(dK=None) == -1 and call(qi=ONE) == -1       # query ids without key ids
    assert call(scale=float("nan")) == -3 and call(scale=float("inf")) == -3
    for bad in ("t", "qi", "ki", "bias", "w", "loss"):
        assert call(**dict(dict(ki=ONE), **{bad: ctypes.c_void_p(258)})) == -3, bad
    assert call(Q=ctypes.c_void_p(257)) == -3 and call(ws=ctypes.c_void_p(264)) == -3
    for want in (True, False):
        need = rn.rnnd_contrast_workspace(4, 6, 8, rn.RNND_BF16, want)
        assert call(size=need - 1, **({} if want else dict(dQ=None, dK=None))) == -7
    assert rn.rnnd_contrast_workspace(4, 6, 8, rn.RNND_BF16, False) < rn.rnnd_contrast_workspace(4, 6, 8, rn.RNND_BF16, True)
    assert call(B=0, Q=None, t=None, loss=None, dQ=None, dK=None, ws=None, size=0) == 0
    assert rn.rnnd_contrast_workspace(0, 6, 8, rn.RNND_BF16, True) == 0
    assert lib.rnnd_contrast_workspace(4, 6, 8, 3, 1, None) == -1


def test_adamw_refusals(lib):
    def tensor(**kw):
        t = _binding.AdamwTensor()
        for k, v in dict(dict(param=256, grad=256, m=256, v=256, n=10, grad_dtype=1, state_bits=32), **kw).items():
            setattr(t, k, v)
        return t

    def call(t=None, count=1, step=1, lr=1e-3, b1=0.9, b2=0.999, eps=1e-8, wd=0.0, gs=1.0):
        return lib.rnnd_adamw((_binding.AdamwTensor * 1)(t or tensor()), count, step, lr, b1, b2, eps, wd, gs, 0, None)
    assert call(count=-1) == -2 and lib.rnnd_adamw(None, 1, 1, 1e-3, 0.9, 0.999, 1e-8, 0.0, 1.0, 0, None) == -1
    assert call(step=0) == -3 and call(b1=1.0) == -3 and call(b2=-0.1) == -3 and call(eps=-1.0) == -3
    nan, inf = float("nan"), float("inf")
    assert call(lr=nan) == -3 and call(b1=nan) == -3 and call(eps=inf) == -3 and call(wd=inf) == -3 and call(gs=nan) == -3
    assert call(tensor(n=-1)) == -2 and call(tensor(n=2**40 + 1)) == -2
    assert call(tensor(state_bits=16)) == -4 and call(tensor(grad_dtype=0)) == -4 and call(tensor(copy=256, copy_dtype=1)) == -4
    for name in ("param", "grad", "m", "v"):
        assert call(tensor(**{name: None})) == -1, name
    eight = dict(state_bits=8, m_scale=256, v_scale=256)
    assert call(tensor(**dict(eight, m_scale=None))) == -1 and call(tensor(**dict(eight, v_scale=None))) == -1
    assert call(tensor(**dict(eight, counter=3))) == -3
    assert call(tensor(param=258)) == -3 and call(tensor(grad=257, grad_dtype=2)) == -3 and call(tensor(m=258)) == -3
    assert call(tensor(copy=257, copy_dtype=2)) == -3
    assert lib.rnnd_adamw(None, 0, 1, 1e-3, 0.9, 0.999, 1e-8, 0.0, 1.0, 0, None) == 0
    assert call(tensor(n=0, param=None)) == 0


def test_the_binding_refuses_what_is_not_rows_in_device_memory():
    import torch
    with pytest.raises(ValueError):
        rn.rnnd_embed(torch.zeros(3, 4), torch.zeros(2, dtype=torch.int32))
    with pytest.raises(ValueError):
        rn.rnnd_contrast(torch.zeros(3, 4), torch.zeros(3, 4), torch.zeros(3, dtype=torch.int32), 1.0)
    with pytest.raises(ValueError):
        rn.AdamwTensors([dict(param=torch.zeros(3), grad=torch.zeros(3), m=torch.zeros(3), v=torch.zeros(3))])
    with pytest.raises(ValueError):
        rn.AdamwTensors([dict(param=torch.zeros(3), grad=torch.zeros(3), m=torch.zeros(3), v=torch.zeros(3), what=1)])
