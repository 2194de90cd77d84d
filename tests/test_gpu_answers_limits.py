"""Log probabilities and distillation at their limits: the largest counts, element offsets above 2^31, workspaces that hold NaN beforehand."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

U = 2.0 ** -24      # half a float32 step


@pytest.fixture(scope="module")
def rn():
    import torch
    assert torch.cuda.is_available(), "these tests need the MI355X"
    import paper_2310_20419_amd as m
    m.load_library()
    return m


def logits64(Q, K, scale, bias=None, chunk=65536):
    import torch
    q = Q.double()
    s = torch.empty(len(q), len(K), dtype=torch.float64, device="cuda")
    for j in range(0, len(K), chunk):
        k = K[j:j + chunk].double()
        s[:, j:j + chunk] = -scale * (q.square().sum(1)[:, None] + k.square().sum(1)[None, :] - 2 * (q @ k.T))
    return s if bias is None else s + bias.double()[None, :]


def error_of(Q, K, scale, terms=1):
    """The bound of test_gpu_logprob.py, with the largest norms."""
    d = Q.shape[1]
    nq, nk = Q.float().norm(dim=1).max().item(), K.float().norm(dim=1).max().item()
    return U * scale * ((terms * d + 4) * 2 * nq * nk + (d + 4) * (nk * nk + nq * nq))


@pytest.mark.parametrize("B", [2, 20])
def test_offsets_above_2_to_the_31(rn, B):
    """1,048,576 keys of 2,112 bfloat16 coordinates (4.4 GB): the last rows are the queries themselves."""
    import torch
    M, d = 1 << 20, 2112
    g = torch.Generator(device="cuda").manual_seed(1)
    K = torch.empty(M, d, dtype=torch.bfloat16, device="cuda")
    for j in range(0, M, 1 << 17):
        K[j:j + (1 << 17)] = torch.randn(1 << 17, d, device="cuda", generator=g).mul_(d ** -0.5)
    Q = K[M - B:].clone()
    target = torch.arange(M - B, M, device="cuda", dtype=torch.int32)
    lp, ent, ids, tops = rn.rnnd_logprob(Q, K, 4.0, target=target, alternatives=7)
    assert torch.equal(ids[:, 0], target) and torch.equal(tops[:, 0], lp)
    s = logits64(Q, K, 4.0)
    lse = torch.logsumexp(s, 1)
    best, at = s.sort(dim=1, descending=True, stable=True)
    assert torch.equal(ids.long(), at[:, :7])
    # (joins of the sums: 260 + M / 250 steps)
    assert (tops.double() - (best[:, :7] - lse[:, None])).abs().max() <= error_of(Q, K, 4.0) + (260 + M / 250) * U + 40 * U


def test_as_many_queries_as_there_may_be(rn):
    import torch
    B, M = 1 << 20, 64
    g = torch.Generator(device="cuda").manual_seed(2)
    Q, K = torch.randn(B, 16, device="cuda", generator=g) / 4, torch.randn(M, 16, device="cuda", generator=g) / 4
    target = torch.randint(-1, M, (B,), device="cuda", generator=g, dtype=torch.int32)
    lp, ent, ids, tops = rn.rnnd_logprob(Q, K, 2.0, target=target, alternatives=2)
    s = logits64(Q, K, 2.0)
    logs = torch.log_softmax(s, 1)
    bound = error_of(Q, K, 2.0, 6) + 300 * U
    want = torch.where(target >= 0, logs.gather(1, target.clamp(min=0).long()[:, None])[:, 0], 0.0)
    assert (lp.double() - want).abs().max() <= bound + 4 * U * want.abs().max()
    best, at = logs.sort(dim=1, descending=True, stable=True)
    assert torch.equal(ids.long(), at[:, :2])


@pytest.mark.parametrize("B,M", [(3, 1 << 20), (30_000, 70)])
def test_distillation_with_very_many_keys_or_queries(rn, B, M):
    import torch
    g = torch.Generator(device="cuda").manual_seed(3)
    d, n, scale = 16, 5, 2.0
    Q, K = torch.randn(B, d, device="cuda", generator=g) / 4, torch.randn(M, d, device="cuda", generator=g) / 4
    ids = torch.stack([torch.randperm(M, device="cuda", generator=g)[:n] if B < 10 else (torch.arange(n, device="cuda") * 13 + i) % M for i in range(B)]) \
        if B < 10 else (torch.arange(n, device="cuda")[None, :] * 13 + torch.randint(0, M, (B, 1), device="cuda", generator=g)) % M
    logp = torch.log_softmax(torch.randn(B, n, device="cuda", generator=g), 1) + np.log(0.7)
    w = torch.rand(B, device="cuda", generator=g)
    loss, dq, dk = rn.rnnd_distill(Q, K, ids.int(), logp, scale, tail=True, row_weight=w)
    q, k = Q.double().requires_grad_(), K.double().requires_grad_()
    s = -scale * (q.square().sum(1)[:, None] + k.square().sum(1)[None, :] - 2 * (q @ k.T))
    logs = torch.log_softmax(s, 1)
    p = logp.double().exp()
    r = 1 - p.sum(1)
    off = torch.logsumexp(logs.scatter(1, ids, -float("inf")), 1)
    want = (p * (logp.double() - logs.gather(1, ids))).sum(1) + r * (r.log() - off)
    wq, wk = torch.autograd.grad((w.double() * want).sum(), (q, k))
    e = error_of(Q, K, scale, 6)
    size = 4 + 2 * logs.gather(1, ids).abs().max().item()
    assert (loss.double() - want).abs().max() <= 2 * e + 40 * U * (1 + size) + M / 250 * U
    # g: 2 e + 60 u of P + p each; a gradient sums to at most 2 scale w (2 of them) |k - q|, |k - q| < 4; a key's over the queries
    each = 2 * scale * 2 * (2 * e + (60 + M / 250) * U + 40 * U) * 4 * 2
    assert (dq.double() - wq).abs().max() <= each
    share = torch.zeros(M, device="cuda").index_add_(0, ids.flatten(), w[:, None].expand(B, n).flatten()) + w.sum() / M * 50
    assert ((dk.double() - wk).abs() <= (each + 2.0 ** -20) * (1 + share)[:, None]).all()


@pytest.mark.parametrize("B,M,d,dtype", [(1, 900, 40, "float32"), (7, 3000, 64, "bfloat16"), (40, 900, 40, "float32"), (300, 1000, 64, "float16"), (1100, 3000, 64, "bfloat16"),
                                         (50, 700, 33, "float16")])
def test_workspaces_that_hold_nan(rn, B, M, d, dtype):
    """What the calls leave and find there does not matter, and the sizes that the queries give are enough."""
    import torch
    g = torch.Generator(device="cuda").manual_seed(4)
    t = getattr(torch, dtype)
    Q, K = (torch.randn(x, d, device="cuda", generator=g).div(d ** 0.5).to(t) for x in (B, M))
    code = {"float32": rn.RNND_F32, "float16": rn.RNND_F16, "bfloat16": rn.RNND_BF16}[dtype]
    names = torch.arange(M, device="cuda", dtype=torch.int32)
    names[::9] = -1
    K[::9] = float("nan")
    query = torch.arange(B, device="cuda", dtype=torch.int32)
    bias = torch.randn(M, device="cuda", generator=g)
    kw = dict(query_ids=query, key_ids=names, key_bias=bias)
    _, _, ids, logp = want = rn.rnnd_logprob(Q, K, 3.0, target=query.remainder(M), alternatives=9, **kw)
    learnt = rn.rnnd_distill(Q, K, ids, logp, 3.0, tail=True, **kw)
    assert all(torch.isfinite(x.float()).all() for x in want + learnt)
    guard = 4096
    for size, run in ((rn.rnnd_logprob_workspace(B, M, d, code, 9), lambda w: rn.rnnd_logprob(Q, K, 3.0, target=query.remainder(M), alternatives=9, workspace=w, **kw)),
                      (rn.rnnd_distill_workspace(B, M, d, code, 9), lambda w: rn.rnnd_distill(Q, K, ids, logp, 3.0, tail=True, workspace=w, **kw))):
        for fill in (0xFF, 0x7F, 0x00):
            room = torch.full((size + guard,), fill, dtype=torch.uint8, device="cuda")
            got = run(room[:size])
            for x, y in zip(got, want if len(got) == 4 else learnt):
                assert torch.equal(x, y), fill
            assert (room[size:] == fill).all()


def test_many_queries_of_16_bit_rows_that_hold_nan_or_are_not_aligned(rn):
    """More than 1,024 queries: the keys' norms are formed by themselves."""
    import torch
    g = torch.Generator(device="cuda").manual_seed(5)
    Q, K = (torch.randn(x, 128, device="cuda", generator=g).div(11).half() for x in (1500, 20_000))
    names = torch.arange(20_000, device="cuda", dtype=torch.int32)
    names[5::7] = -1
    want = rn.rnnd_logprob(Q, K, 3.0, alternatives=5, key_ids=names)
    s = logits64(Q, K, 3.0).masked_fill_((names < 0)[None, :], -float("inf"))
    assert torch.equal(want[2].long(), s.sort(dim=1, descending=True, stable=True)[1][:, :5])
    lse = torch.logsumexp(s, 1)
    assert (want[3].double() - (s.gather(1, want[2].long()) - lse[:, None])).abs().max() <= error_of(Q, K, 3.0) + 400 * U
    K[5::7] = float("nan")
    room = torch.empty(K.numel() + 3, dtype=torch.half, device="cuda")
    room[3:] = K.flatten()
    for k in (K, room[3:].view(K.shape)):
        for x, y in zip(want[1:], rn.rnnd_logprob(Q, k, 3.0, alternatives=5, key_ids=names)[1:]):
            assert torch.equal(x, y)
