"""The forms that large calls take, each against double precision: tiles of 256 with the keys read where they are (their norms along with the product or by
themselves) or copied in parts, rows of several passes with keys that many queries list."""
import numpy as np
import pytest

import test_gpu_distill as distill
import test_gpu_logprob as logprob
from test_gpu_logprob import rn       # noqa: F401

pytestmark = pytest.mark.gpu

U = 2.0 ** -24      # half a float32 step


@pytest.mark.parametrize("B,M,d,dtype", [(200, 131_100, 192, "bfloat16"), (200, 131_100, 192, "float16"), (1100, 33_000, 384, "float16"),
                                         (1100, 33_000, 384, "bfloat16")])
def test_logprob_with_tiles_of_256(rn, B, M, d, dtype):       # noqa: F811
    """Up to 1,024 queries take the keys' norms from the product, more from a pass of their own.  Keys that do not lie at a multiple of 16 bytes
    are copied 16,384 at a time, and the answers are the same bits."""
    import torch
    c = logprob.case(B, M, d, dtype, 41)
    logprob.check(rn, c, 3.0, 9)
    want = logprob.call(rn, c, 3.0, 9)
    room = torch.empty(c["K"].numel() + 1, dtype=c["K"].dtype, device="cuda")
    room[1:] = c["K"].flatten()
    for x, y in zip(want, logprob.call(rn, dict(c, K=room[1:].view(M, d)), 3.0, 9)):
        assert torch.equal(x, y)


@pytest.mark.parametrize("dtype", distill.TYPES)
@pytest.mark.parametrize("d", [600, 1100])
def test_distill_rows_of_several_passes(rn, d, dtype):       # noqa: F811
    """768 coordinates a pass; two keys that more than 128 queries list, which a whole block sums."""
    B = 300
    c = distill.case(B, 90, d, 6, dtype, 42 + d)
    g = np.random.Generator(np.random.PCG64(d))
    c["teacher_ids"][:, 1], c["teacher_ids"][g.random(B) < 0.7, 2] = 17, 18
    for j in (17, 18):
        c["key_ids"][j], c["key_bias"][j] = 1000 + j, 0.0
    distill.check(rn, c, 3.0, True)
    distill.check(rn, c, 3.0, False)


@pytest.mark.parametrize("tail", [False, True])
@pytest.mark.parametrize("B,M,d,dtype", [(256, 131_072, 392, "bfloat16"), (1100, 28_000, 448, "float16")])
def test_distill_with_tiles_of_256(rn, B, M, d, dtype, tail):       # noqa: F811
    """Loss, dQ and dK, all rows, with the bounds of test_gpu_distill.py; a gradient's with |k_j - q_i| <= |k_j| + |q_i| and M or B terms."""
    import torch
    n, scale = 40, 3.0
    c = distill.case(B, M, d, n, dtype, 43)
    c["teacher_ids"][::2, 5], c["key_ids"][77], c["key_bias"][77] = 77, 5 * M, 0.0       # in the lists of half the queries
    x = {k: torch.from_numpy(v).cuda() if isinstance(v, np.ndarray) else v for k, v in c.items()}
    loss, dq, dk = distill.call(rn, c, scale, tail)
    q, k, w, bias = x["Q"].double(), x["K"].double(), x["row_weight"].double(), x["key_bias"].double()
    inf = float("inf")
    gone = (x["key_ids"] < 0) | (bias == -inf)
    out = gone[None, :] | (x["key_ids"][None, :] == x["query_ids"][:, None])
    p = torch.zeros(B, M, dtype=torch.float64, device="cuda")
    on = torch.zeros(B, M, dtype=torch.bool, device="cuda")
    logits = x["teacher_logits"].double()
    for e in reversed(range(n)):        # (of two entries for a key the first counts)
        j = x["teacher_ids"][:, e].long()
        at = j.clamp(0, M - 1)[:, None]
        fine = ((j >= 0) & (j < M) & (logits[:, e] > -inf))[:, None] & ~out.gather(1, at)
        p.scatter_(1, at, torch.where(fine, logits[:, e:e + 1].exp(), p.gather(1, at)))
        on.scatter_(1, at, fine | on.gather(1, at))
    counts = on.any(1)
    q = torch.where(counts[:, None], q, 0.0)
    k = torch.where(gone[:, None], 0.0, k)
    s = bias.clamp(min=-1e30)[None, :] - scale * (q.square().sum(1)[:, None] + k.square().sum(1)[None, :] - 2 * q @ k.T)
    s = torch.where(out, -inf, s)
    lse = torch.logsumexp(s, 1)
    P = torch.exp(s - lse[:, None])
    log_off = torch.logsumexp(s.masked_fill(on, -inf), 1) - lse
    R = log_off.exp()
    total = p.sum(1)
    rest = (1 - total).clamp(min=0) if tail else torch.zeros_like(total)
    mass = torch.where(counts, total + rest, 1.0)
    p, rest = p / mass[:, None], rest / mass
    log_p, logP = torch.where(p > 0, p.log(), 0.0), torch.where(on, s - lse[:, None], 0.0)
    tail_loss = torch.where(rest > 0, rest * (rest.log() - log_off), 0.0)
    want = torch.where(counts, (p * (log_p - logP)).sum(1) + tail_loss, 0.0)
    g = torch.where(on, P - p, P * (1 - rest / R)[:, None])
    g = torch.where(counts[:, None], g * w[:, None], 0.0)
    wq, wk = 2 * scale * (g @ k - g.sum(1)[:, None] * q), 2 * scale * (g.T @ q - g.sum(0)[:, None] * k)
    nq, nk = q.norm(dim=1), k.norm(dim=1)
    e = (U * ((d + 4) * 2 * scale * nq[:, None] * nk.max() + (d + 4) * scale * nk.max() ** 2 + 4 * bias[~gone].abs().max()))[:, 0]
    size = (p * (log_p.abs() + logP.abs())).sum(1) + tail_loss.abs() + torch.where(rest > 0, 2 * rest * rest.log().abs(), 0.0)
    off = (loss.double() - want).abs()
    assert (off <= torch.where(counts, 2 * e + 40 * U * (1 + size), 0.0)).all(), off.max()
    h = torch.finfo(x["K"].dtype).eps / 2
    terms = torch.where(on, P + p, (P / R[:, None]) * (R + rest)[:, None]) * torch.where(counts, w.abs(), 0.0)[:, None]
    ge = terms * (2 * e[:, None] + 60 * U) + g.abs() * h * 1.01
    if dtype == "float16":
        ge = ge + torch.where(counts, w.abs().max() * 2.0 ** -14 * 2.0 ** -24, 0.0)[:, None]
    del terms, P, p, s, logP, log_p
    for name, got, true, rows, other, gg, err in (("dQ", dq, wq, q, k, g, ge), ("dK", dk, wk, k, q, g.T, ge.T)):
        each = err + (gg.shape[1] + 8) * U * (gg.abs() + err)
        bound = 2 * scale * (each @ other.abs() + each.sum(1)[:, None] * rows.abs())
        bound += true.abs() * (h + 4 * U) * 1.01 + torch.finfo(x["K"].dtype).smallest_normal * h + 1e-44
        off = (got.double() - true).abs()
        assert (off <= bound).all(), (name, (off - bound).max())
        # bounds of single terms do not show an error that is the same for all: most of the gradient's size has to be there
        assert off.norm() <= 0.01 * true.norm(), (name, off.norm() / true.norm())
    assert (dk[gone] == 0).all() and (dq[~counts] == 0).all()
