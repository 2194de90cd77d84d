"""Log probabilities, entropies and most probable keys, against the formulas in double precision: small and large calls (few queries go another
way than many), ties, keys that are left out, rows far from the origin, queries that no key answers."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

U = 2.0 ** -24      # half a float32 step
TYPES = ["float32", "float16", "bfloat16"]


@pytest.fixture(scope="module")
def rn():
    import torch
    assert torch.cuda.is_available(), "these tests need the MI355X"
    import paper_2310_20419_amd as m
    m.load_library()
    return m


def case(B, M, d, dtype, seed, far=0.0, ids=True, bias=True):
    import torch
    g = np.random.Generator(np.random.PCG64(seed))
    centre = far * g.normal(size=d) / np.sqrt(d)
    K = g.normal(size=(M, d)) / np.sqrt(d)
    t = g.integers(0, M, size=B)
    Q = 0.7 * K[t] + 0.7 * g.normal(size=(B, d)) / np.sqrt(d)
    c = dict(Q=torch.from_numpy(Q + centre).to(getattr(torch, dtype)).cuda(), K=torch.from_numpy(K + centre).to(getattr(torch, dtype)).cuda(),
             target=t.astype(np.int32))
    if ids:
        c["key_ids"] = g.integers(0, max(2, 3 * M), size=M).astype(np.int32)
        c["key_ids"][g.random(M) < 0.05] = -1
        c["query_ids"] = g.integers(-1, max(2, 3 * M), size=B).astype(np.int32)
        c["query_ids"][::3] = c["key_ids"][t[::3]]
    if bias:
        c["key_bias"] = g.normal(size=M).astype(np.float32)
        c["key_bias"][g.random(M) < 0.03] = -np.inf
    if B > 3:
        c["target"][1], c["target"][2] = -1, M
    return c


def call(rn, c, scale, k, **kw):
    import torch
    x = {n: torch.from_numpy(v).cuda() if isinstance(v, np.ndarray) else v for n, v in c.items()}
    return rn.rnnd_logprob(x.pop("Q"), x.pop("K"), scale, alternatives=k, **x, **kw)


def left_out(c, B, M):
    out = np.zeros((B, M), bool)
    if "key_bias" in c:
        out |= (c["key_bias"] == -np.inf)[None, :]
    if "key_ids" in c:
        out |= (c["key_ids"] < 0)[None, :]
        if "query_ids" in c:
            out |= c["key_ids"][None, :] == c["query_ids"][:, None]
    return out


def logits_of(c, scale):
    """float64, from differences, a row at a time: equal rows have equal logits."""
    import torch
    q, k = c["Q"].double(), c["K"].double()
    B, M = len(q), len(k)
    out = left_out(c, B, M)
    bias = np.where(np.isfinite(c["key_bias"]), c["key_bias"], 0.0).astype(np.float64) if "key_bias" in c else np.zeros(M)
    gone = torch.from_numpy(out.all(0)).cuda() if B else None
    k = torch.where(gone[:, None], torch.zeros_like(k), k)
    dist = torch.stack([(k - row).square().sum(1) for row in q]).cpu().numpy()
    return np.where(out, -np.inf, bias[None, :] - scale * dist), out, bias


def error_of_a_logit(c, scale, bias, out):
    """u * ((n + 4) 2 |scale| |q||k| + (d + 4) |scale| |k|^2 + 4 |bias|), n = d or, of float32 rows in three terms, 6 d: the bound of the
    sums of products; sums of squared differences stay below it but for what a square of the difference takes, (|q| + |k|)^2."""
    q, k = c["Q"].double().cpu().numpy(), c["K"].double().cpu().numpy()
    on = ~out.all(0)
    d = q.shape[1]
    n = 6 * d if str(c["Q"].dtype) == "torch.float32" else d
    nq, nk = np.sqrt(np.square(q).sum(1)), np.sqrt(np.square(k[on]).sum(1))
    if not on.any():
        return np.zeros(len(q))
    e = U * ((n + 4) * 2 * abs(scale) * nq[:, None] * nk[None, :] + (d + 4) * abs(scale) * (np.square(nk)[None, :] + np.square(nq)[:, None])
             + 4 * abs(bias[on])[None, :])
    return e.max(1)


def check(rn, c, scale, k, **kw):
    """A logit is off by e (above).  The sum of the exponentials: each is off by 2 u of itself and of |x| u for its argument x, and it is joined with a
    part's about M / 1000 + 40 times, each for some 4 u; so lse is off by e + (260 + M / 250) u, and a log probability by as much and the
    roundings of its own steps (the key's own logit is from double precision).  The entropy's derivative with respect to logit j is
    -P_j (log P_j + H), so logits off by e each move it by e sum P |log P + H| at most; its sums as above, of size 1 + H."""
    import torch
    B, M = len(c["Q"]), len(c["K"])
    s, out, bias = logits_of(c, scale)
    lp, ent, ids, tops = call(rn, c, scale, k, **kw)
    e = error_of_a_logit(c, scale, bias, out)
    none = out.all(1)
    own = np.where(none[:, None], 0.0, s)
    top = own.max(1)
    lse = top + np.log(np.exp(own - top[:, None]).sum(1))
    logp = s - lse[:, None]
    p = np.exp(np.where(none[:, None], -np.inf, logp))
    fine = np.where(p > 0, logp, 0.0)
    h = -(p * fine).sum(1)
    joins = (260 + M / 250) * U
    bound = e + joins + 4 * U
    t = c["target"].astype(np.int64)
    at = np.clip(t, 0, M - 1)
    asked = (t >= 0) & (t < M) & ~out[np.arange(B), at]
    want = np.where(asked, logp[np.arange(B), at], 0.0)
    off = abs(lp.double().cpu().numpy() - want)
    assert (off <= np.where(asked, bound + 4 * U * abs(want), 0.0)).all(), ("logprob", off.max())
    off = abs(ent.double().cpu().numpy() - h)
    assert (off <= np.where(none, 0.0, e * (p * abs(fine + h[:, None])).sum(1) + 2 * joins * (1 + h))).all(), ("entropy", off.max())
    if not k:
        assert ids is None and tops is None
        return
    order = np.argsort(-s, axis=1, kind="stable")[:, :k]
    best = np.take_along_axis(s, order, 1)
    order = np.where(best > -np.inf, order, -1)
    if order.shape[1] < k:
        pad = k - order.shape[1]
        order, best = np.pad(order, ((0, 0), (0, pad)), constant_values=-1), np.pad(best, ((0, 0), (0, pad)), constant_values=-np.inf)
    assert (ids.cpu().numpy() == order).all(), ("ids", np.nonzero((ids.cpu().numpy() != order).any(1))[0][:5])
    got = tops.double().cpu().numpy()
    assert (got[order < 0] == -np.inf).all()
    on = order >= 0
    want = best - lse[:, None]
    off = np.where(on, abs(np.where(on, got, 0.0) - np.where(on, want, 0.0)), 0.0)
    assert (off <= bound[:, None] + 4 * U * abs(np.where(on, want, 0.0))).all(), ("top_logprob", off.max())
    assert (np.where(on, got, 0.0) <= 0).all()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("B,M,d,k", [(1, 1, 1, 1), (1, 70, 33, 10), (2, 1000, 96, 10), (3, 65, 7, 128), (5, 3001, 100, 20), (8, 700, 768, 3), (7, 5000, 1100, 40),
                                     (9, 1, 5, 2), (9, 130, 33, 10), (64, 255, 32, 64), (130, 1025, 100, 128), (300, 3000, 48, 10), (40, 2000, 768, 1),
                                     (1, 900, 40, 0), (20, 900, 40, 0)])
def test_against_double_precision(rn, B, M, d, k, dtype):
    check(rn, case(B, M, d, dtype, seed=B * 7 + M + d), 3.0, k)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("B", [3, 50])
def test_without_ids_and_biases(rn, B, dtype):
    check(rn, case(B, 800, 64, dtype, 5, ids=False, bias=False), 4.0, 12)


@pytest.mark.parametrize("B", [2, 30])
@pytest.mark.parametrize("scale", [0.0, -1.5, 60.0])
def test_scales(rn, B, scale):
    """0: all logits are the biases; a negative one prefers what is far."""
    check(rn, case(B, 600, 24, "float32", 6), scale, 9)


@pytest.mark.parametrize("B", [4, 60])
def test_equal_keys_come_in_the_order_of_their_positions(rn, B):
    import torch
    c = case(B, 900, 40, "float32", 8, bias=False)
    c["K"] = c["K"][torch.arange(900, device="cuda") // 3].contiguous()
    check(rn, c, 3.0, 10)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("B", [2, 20])
def test_more_equal_keys_than_there_is_room_for(rn, B, dtype):
    """6,000 copies of one row, and some others; most of the alternatives are the first copies that are not left out."""
    import torch
    c = case(B, 6500, 24, dtype, 9, bias=False)
    c["K"][250:6250] = c["K"][250].clone()
    c["Q"][0] = c["K"][250]
    check(rn, c, 3.0, 100)


@pytest.mark.parametrize("B", [1, 12])
@pytest.mark.parametrize("run", [16, 32, 64, 128, 256])
def test_crowds_of_probable_keys(rn, B, run):
    """One run of keys in 64 holds those that count, far above all others: a few large values say little about the k-th largest, and more groups of keys lie
    above the first bound than there is room for at once."""
    c = case(B, 200_000, 8, "float32", 18, ids=False)
    c["key_bias"][np.arange(200_000) // run % 64 == 5] += 30.0
    check(rn, c, 1.0, 50)


@pytest.mark.parametrize("B", [4, 64])
def test_logits_closer_together_than_the_first_pass_sees(rn, B):
    """Keys that differ in a last bit: float32 sums do not tell them apart, the order is still that of double precision."""
    import torch
    c = case(B, 700, 50, "float32", 10, ids=False, bias=False)
    one = c["K"][0].clone()
    c["K"][100:200] = one
    c["K"][100:200, 0] = one[0] * (1 + torch.randperm(100, device="cuda") * 2.0 ** -23)
    c["Q"][:] = one + 0.3 * c["Q"]
    check(rn, c, 2.0, 50)


@pytest.mark.parametrize("far", [30.0, 1000.0])
def test_float32_rows_far_from_the_origin(rn, far):
    """The error goes with the distances from a point among the keys: the bound is that of rows moved there."""
    for B in (3, 40):
        c = case(B, 900, 64, "float32", 11, far=far)
        check(rn, c, 3.0, 10)
        moved = dict(c, Q=c["Q"].double() - c["K"].double()[0], K=c["K"].double() - c["K"].double()[0])
        s, out, bias = logits_of(moved, 3.0)
        lse = np.log(np.exp(s).sum(1))
        e = error_of_a_logit(dict(moved, Q=moved["Q"].float(), K=moved["K"].float()), 3.0, bias, out)
        tops = call(rn, c, 3.0, 10)[3].double().cpu().numpy()
        want = np.sort(s, 1)[:, ::-1][:, :10] - lse[:, None]
        # (a row and the point are float32 numbers; their difference, rounded, is off by U of itself)
        assert (abs(tops - want) <= 4 * e[:, None] + 400 * U * (1 + abs(want))).all()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("B,d", [(3, 40), (33, 40), (33, 64), (3, 64)])
def test_what_is_left_out_is_never_read_as_a_number(rn, B, d, dtype):
    import torch
    c = case(B, 500, d, dtype, 12)
    want = call(rn, c, 3.0, 8)
    gone = torch.from_numpy((c["key_ids"] < 0) | (c["key_bias"] == -np.inf)).cuda()
    c["K"][gone] = float("nan")
    c["K"][gone.nonzero()[0, 0]] = float("inf")
    for x, y in zip(want, call(rn, c, 3.0, 8)):
        assert torch.equal(x, y)


@pytest.mark.parametrize("B", [2, 12])
def test_no_key_at_all(rn, B):
    c = case(B, 300, 16, "bfloat16", 13)
    c["key_ids"][:] = -1
    lp, ent, ids, tops = call(rn, c, 3.0, 5)
    assert (lp == 0).all() and (ent == 0).all() and (ids == -1).all() and (tops == -float("inf")).all()
    c["key_ids"][7], c["query_ids"][:], c["key_bias"][7] = 4, 4, 0.0       # one key, which is every query's own
    lp, ent, ids, tops = call(rn, c, 3.0, 5)
    assert (lp == 0).all() and (ent == 0).all() and (ids == -1).all()
    c["query_ids"][1] = 5
    c["target"][1] = 7
    lp, ent, ids, tops = call(rn, c, 3.0, 5)
    # its probability is 1; the first pass has its logit with an error of u ((16 + 4) 2 scale |q||k| + (16 + 4) scale (|q|^2 + |k|^2)), and |q|, |k| < 2
    one = U * (20 * 6 * 4 + 20 * 3 * 8)
    # its entropy is log2(sum) - w / sum in base 2, with sum = 2^x and w = x sum for some x near zero: the sum is off by 2 u, its logarithm by 3 u for that
    # and 2 u for itself, the quotient by 3 u of |x| < 1
    assert abs(lp[1]) <= one and abs(tops[1, 0]) <= one and 0 <= ent[1] <= 8 * U and ids[1].tolist() == [7, -1, -1, -1, -1] and (ids[0] == -1).all()


@pytest.mark.parametrize("B", [2, 12])
def test_a_logit_that_is_no_number(rn, B):
    import torch
    for bad in ("row", "bias"):
        c = case(B, 300, 16, "float32", 14, bias=True)
        c["key_ids"][9], c["query_ids"][:], c["query_ids"][0], c["key_bias"][9] = 11, 12, 11, 0.0
        if bad == "row":
            c["K"][9, 3] = float("nan")
        else:
            c["key_bias"][9] = np.inf
        c["target"][:] = 20
        c["key_ids"][20], c["key_bias"][20] = 400, 0.0
        lp, ent, ids, tops = call(rn, c, 3.0, 5)
        assert torch.isnan(lp[1:]).all() and torch.isnan(ent[1:]).all() and (ids[1:] == -1).all() and torch.isnan(tops[1:]).all()
        assert torch.isfinite(lp[0]) and torch.isfinite(ent[0]) and (ids[0] >= 0).all()        # the query that leaves that key out


def test_queries_in_several_runs_through_the_keys(rn):
    """1,100 queries against 131,000 keys work in runs of fewer; the answers are those of runs of one."""
    import torch
    c = case(1100, 131_000, 16, "bfloat16", 15)
    got = call(rn, c, 3.0, 6)
    for at in (0, 500, 767, 768, 1023, 1024, 1099):
        part = dict(c, Q=c["Q"][at:at + 1].contiguous(), target=c["target"][at:at + 1], query_ids=c["query_ids"][at:at + 1])
        one = call(rn, part, 3.0, 6)
        assert torch.equal(one[2][0], got[2][at])
        assert torch.allclose(one[3][0], got[3][at], rtol=0, atol=1e-4) and torch.allclose(one[1][0], got[1][at], rtol=0, atol=1e-4)


def test_tiles_of_256(rn):
    """Long 16-bit rows and enough of them: the other tile."""
    check(rn, case(300, 70_000, 392, "float16", 16), 3.0, 33)


@pytest.mark.parametrize("B,M,d", [(1, 400, 64), (40, 400, 64), (300, 33_000, 64), (40, 400, 62)])
def test_rows_that_are_not_aligned(rn, B, M, d):
    """(Of 33,000 keys not all fit the room for copies at once.)"""
    import torch
    c = case(B, M, d, "bfloat16", 17)
    want = call(rn, c, 3.0, 7)
    for name in ("Q", "K"):
        room = torch.empty(c[name].numel() + 1, dtype=torch.bfloat16, device="cuda")
        room[1:] = c[name].flatten()
        c[name] = room[1:].view(c[name].shape)
    for x, y in zip(want, call(rn, c, 3.0, 7)):
        assert torch.equal(x, y)
