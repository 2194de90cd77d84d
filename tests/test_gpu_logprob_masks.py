"""Masks in key_bias that are finite: the lowest float, which leaves a key out as -infinity does, large ones that count, and the usual -1e9; and rows
far away from all others.  What such keys do not change are the answers about the others, nor (by much) the time that these take."""
import numpy as np
import pytest

from test_gpu_logprob import TYPES, U, call, case, check, error_of_a_logit, rn       # noqa: F401

pytestmark = pytest.mark.gpu

LOWEST = float(np.finfo(np.float32).min)
# few queries, few and many by tiles (the keys' norms along with the product or by themselves; keys in place or copied)
SIZES = [(3, 900, 40), (8, 900, 64), (40, 900, 64), (40, 900, 40), (1100, 900, 64)]


class Biased:
    """Calls with other biases than the case that the answers are compared with."""

    def __init__(self, rn, bias):       # noqa: F811
        self.rn, self.bias = rn, bias

    def rnnd_logprob(self, *a, key_bias, **kw):
        import torch
        return self.rn.rnnd_logprob(*a, key_bias=torch.from_numpy(self.bias).cuda(), **kw)


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


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("B,M,d", SIZES)
@pytest.mark.parametrize("mask", [-1e9, -1e30, -1e37, -1e38, -1.9e38])
def test_masks_that_count(rn, B, M, d, mask, dtype):       # noqa: F811
    """Probabilities of nothing, wherever they stand, whole parts of the keys among them."""
    c = case(B, M, d, dtype, 23)
    out = (np.arange(M) >= 300) | (np.arange(M) % 7 == 3)
    ref = np.where(out, np.float32(-np.inf), c["key_bias"])
    c["target"] = np.where(out[np.clip(c["target"], 0, M - 1)], 0, c["target"]).astype(np.int32)      # (that of a masked key is the mask)
    for k in (0, 12):
        check(Biased(rn, np.where(out & (c["key_bias"] > -np.inf), np.float32(mask), c["key_bias"])), dict(c, key_bias=ref), 3.0, k)


@pytest.mark.parametrize("B,d", [(3, 40), (40, 64), (40, 40), (1100, 64)])
@pytest.mark.parametrize("dtype", TYPES)
def test_two_biases_above_all(rn, B, d, dtype):       # noqa: F811
    """1e38 beside biases from 0 to -1.9e38: the two have the same logit (their distances are lost in a step of 1e31), so the entropy is log 2.  (A sum of
    two ones, its logarithm and a quotient of zeros: a few steps.)  A log probability is a logit of double precision less the log of the sum, which
    has the error of a float32 logit: bias times 1.44269504f, whose constant is off by less than U of itself and whose product is rounded, 2 U, and as much
    again where the bias and the distance are two terms: 4 U 1e38, about 2.4e31.  It is not above 0."""
    import torch
    c = case(B, 900, d, dtype, 24, ids=False)
    for other in (0.0, -1e30, -1.9e38, -np.inf):
        c["key_bias"] = np.full(900, other, np.float32)
        c["key_bias"][[100, 511]] = 1e38
        c["target"][:] = 511
        lp, ent, ids, tops = call(rn, c, 3.0, 2)
        assert (ent.double() - np.log(2.0)).abs().max() <= 16 * 2.0 ** -24
        for x in (lp, tops[:, 0], tops[:, 1]):
            assert (x.double() + np.log(2.0)).abs().max() <= 4 * 2.0 ** -24 * 1e38 and (x <= 0).all()
        assert torch.equal(ids.sort(1)[0], torch.tensor([[100, 511]], dtype=torch.int32, device="cuda").expand(B, 2))


def microseconds(run):
    import torch
    times = []
    for i in range(8):
        a, b = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
        a.record()
        run()
        b.record()
        torch.cuda.synchronize()
        if i:
            times.append(a.elapsed_time(b) * 1e3)
    return min(times)


@pytest.mark.parametrize("dtype,B,M,d", [("float32", 1, 200_000, 96), ("float32", 5, 100_000, 33), ("bfloat16", 2, 100_000, 64), ("float32", 300, 20_000, 40),
                                         ("bfloat16", 64, 100_000, 64), ("float16", 1100, 20_000, 64), ("float16", 40, 50_000, 40)])
@pytest.mark.parametrize("what", ["-1e9", "-1e30", "far", "farther", "infinite"])
def test_keys_that_cannot_be_probable_cost_no_time(rn, dtype, B, M, d, what):       # noqa: F811
    """One key in 100 masked, or one a long way off: the alternatives are those of double precision, and take no longer than without (1,000 times
    as long where all keys are gone through; 4 times is far from either)."""
    import torch
    c = case(B, M, d, dtype, 25, ids=False, bias=False)
    c["key_bias"] = np.zeros(M, np.float32)
    x = {n: torch.from_numpy(v).cuda() if isinstance(v, np.ndarray) else v for n, v in c.items()}

    def run():
        return rn.rnnd_logprob(x["Q"], x["K"], 3.0, target=x["target"], alternatives=10, key_bias=x["key_bias"])
    before = microseconds(run)
    want = run()
    keep = torch.ones(M, dtype=torch.bool, device="cuda")
    if what[0] == "-":
        x["key_bias"][7::100] = float(what)
        keep[7::100] = False
    else:
        # (float16 has nothing beyond 65504, whose square times 64 is as far as it goes)
        x["K"][M // 2] = 100.0 * x["K"][M // 2] if what == "far" else 6e4 if what == "farther" else 6e4 if dtype == "float16" else 1e25
        keep[M // 2] = False
    got = run()
    assert microseconds(run) <= 4 * before
    # what has gone was among the alternatives of some queries only: all others have theirs, in that order
    same = keep[want[2].long()].all(1)
    assert torch.equal(got[2][same], want[2][same]) and same.any()
    # and as if these keys were left out (their probabilities are nothing: exp(-20,000) and less); two sums of logits that are each off by e,
    # joined from at most M / 1000 + 40 parts with 4 u a time (float32 rows are taken from another point where a key that gives it has gone)
    plain = dict(c, Q=x["Q"], K=torch.where(keep[:, None], x["K"], torch.zeros_like(x["K"])), key_bias=np.zeros(M, np.float32))
    e = torch.from_numpy(error_of_a_logit(plain, 3.0, plain["key_bias"], np.zeros((B, M), bool))).cuda()
    x["key_bias"] = torch.where(keep, 0.0, -float("inf"))
    gone = run()
    assert torch.equal(got[2], gone[2])
    assert ((got[3].double() - gone[3].double()).abs() <= (2 * e + 2 * (260 + M / 250) * U)[:, None]).all()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("B,d", [(8, 64), (64, 64), (64, 40), (1100, 64)])
def test_biases_that_make_up_for_distances(rn, B, d, dtype):       # noqa: F811
    """Long keys with biases as large as their squares, so that logits are small differences, beside biases of zero with a sign: the first pass's error is
    that of the long keys, and the order that of double precision."""
    import torch
    g = torch.Generator(device="cuda").manual_seed(26)
    M, scale, k = 20_000, 1.0, 10
    K = (30.0 * torch.randn(M, d, device="cuda", generator=g)).to(getattr(torch, dtype))
    Q = (0.003 * torch.randn(B, d, device="cuda", generator=g)).to(K.dtype)
    K[::8] = 0
    bias = K.double().square().sum(1).float()
    bias[::8] = -0.0
    ids = rn.rnnd_logprob(Q, K, scale, alternatives=k, key_bias=bias)[2]
    s = torch.stack([bias.double() - (K.double() - q.double()).square().sum(1) for q in Q])
    assert torch.equal(ids.long(), s.sort(dim=1, descending=True, stable=True)[1][:, :k])
