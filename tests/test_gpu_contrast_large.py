"""The loss and its gradients at sizes that take the wide tiles, against double precision."""
import math

import pytest

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def rn():
    import torch
    assert torch.cuda.is_available(), "these tests need the MI355X"
    import paper_2310_20419_amd as m
    m.load_library()
    return m


@pytest.mark.parametrize("dtype,B,M,d", [("bfloat16", 4101, 8195, 392), ("float16", 4101, 8195, 450), ("bfloat16", 2050, 17000, 777),
                                         ("float32", 1500, 4200, 392), ("bfloat16", 3000, 9000, 64)])
def test_wide_tiles(rn, dtype, B, M, d):
    """Bounds as those of the small cases (u = 2^-24, h half a step of the rows' type), with sum_j e_ij |k_j - q_i| <= sum_j e_ij
    (|k_j| + |q_i|), and the spread of a sum's rounding taken as its worst case."""
    import torch
    t = getattr(torch, dtype)
    g = torch.Generator(device="cuda").manual_seed(B + d)
    K = (torch.randn(M, d, device="cuda", generator=g) / math.sqrt(d))
    target = torch.randint(0, M, (B,), device="cuda", generator=g, dtype=torch.int32)
    Q = (0.8 * K[target.long()] + 0.6 * torch.randn(B, d, device="cuda", generator=g) / math.sqrt(d)).to(t)
    K = K.to(t)
    key_ids = torch.randint(0, 5 * M, (M,), device="cuda", generator=g, dtype=torch.int32)
    key_ids[torch.rand(M, device="cuda", generator=g) < 0.02] = -1
    query_ids = torch.randint(0, 5 * M, (B,), device="cuda", generator=g, dtype=torch.int32)
    bias = -torch.rand(M, device="cuda", generator=g)
    bias[5::97] = -math.inf
    target[::50] = -1
    weight = (torch.rand(B, device="cuda", generator=g) + 0.5) / B * (512.0 if dtype == "float16" else 1.0)
    scale = 4.0
    loss, dq, dk = rn.rnnd_contrast(Q, K, target, scale, query_ids=query_ids, key_ids=key_ids, key_bias=bias, row_weight=weight)

    gone = (key_ids < 0) | (bias == -math.inf)
    at = target.long().clamp(min=0)
    counts = (target >= 0) & ~gone[at]
    q, k = Q.double() * counts[:, None], torch.where(gone[:, None], 0.0, K.double())
    s = bias.double()[None, :] - scale * (q.square().sum(1)[:, None] + k.square().sum(1)[None, :] - 2 * q @ k.T)
    twin = (key_ids[None, :] == key_ids[at][:, None]) | (key_ids[None, :] == query_ids[:, None])
    twin.scatter_(1, at[:, None], False)
    s.masked_fill_(twin | gone[None, :], -math.inf)
    del twin
    own = s.gather(1, at[:, None])
    s.scatter_(1, at[:, None], -math.inf)
    x = torch.logsumexp(s, 1, keepdim=True) - own
    want = torch.where(counts, torch.nn.functional.softplus(x[:, 0]), 0.0)
    p = torch.exp(s - own - torch.nn.functional.softplus(x))
    del s
    p.scatter_(1, at[:, None], torch.expm1(-torch.nn.functional.softplus(x)))
    p = torch.where(counts[:, None], p * weight.double()[:, None], 0.0)
    want_q = 2 * scale * (p @ k - p.sum(1)[:, None] * q)
    want_k = 2 * scale * (p.T @ q - p.sum(0)[:, None] * k)

    info, u = torch.finfo(t), 2.0 ** -24
    h = u if dtype == "float32" else info.eps / 2
    planes = 6 if dtype == "float32" else 1
    nq, nk = q.norm(dim=1).max().item(), k.norm(dim=1).max().item()
    e = u * ((planes * d + 4) * 2 * scale * nq * nk + (d + 4) * scale * nk * nk + 4)
    assert ((loss.double() - want).abs() <= torch.where(counts, 2 * e + 20 * u * (1 + want), 0.0)).all()
    each = 2 * e + 24 * u + h * 1.01
    a = p.abs()
    floor = weight.max().item() * 2.0 ** -38 if dtype == "float16" else 0.0
    for got, exact, m, mine, theirs in ((dq, want_q, a, q, k), (dk, want_k, a.T, k, q)):
        error = m * (each + (m.shape[1] * planes + 8) * u) + floor
        bound = 2 * scale * (error @ theirs.abs() + error.sum(1)[:, None] * mine.abs())
        bound += exact.abs() * (info.eps / 2 + 4 * u) * 1.01 + info.smallest_normal * info.eps / 2
        off = (got.double() - exact).abs()
        assert (off <= bound).all(), ((off - bound).max().item(), off.max().item())
        # and as a whole: roundings do not all point the same way
        assert off.norm() <= 1.5 * max(h, 1e-6) * exact.norm() + floor
    assert (loss[~counts] == 0).all() and (dq[~counts] == 0).all() and (dk[gone] == 0).all()


@pytest.mark.parametrize("B,M,d", [(2050, 4200, 72), (1100, 8300, 320), (2050, 4200, 321), (4300, 2100, 5)])
def test_float32_rows_by_either_product(rn, B, M, d):
    """More than 256 tiles of 128: rows of up to 320 coordinates take two workgroups a CU, longer ones all terms of a step at once."""
    test_wide_tiles(rn, "float32", B, M, d)
