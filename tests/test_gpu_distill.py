"""Distillation and its gradients, against the formulas in double precision and against differences, and with the teacher's
log probabilities as they come from rnnd_logprob."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

TYPES = ["float32", "float16", "bfloat16"]


@pytest.fixture(scope="module")
def rn():
    import torch
    assert torch.cuda.is_available(), "these tests need the MI355X"
    import paper_2310_20419_amd as m
    m.load_library()
    return m


def case(B, M, d, n, dtype, seed, mass=0.9, ids=True, bias=True, weight=True, far=0.0):
    """mass: what the teacher's log probabilities add up to, about."""
    import torch
    g = np.random.Generator(np.random.PCG64(seed))
    centre = far * g.normal(size=d) / np.sqrt(d)
    K = g.normal(size=(M, d)) / np.sqrt(d)
    t = g.integers(0, M, size=B)
    Q = 0.7 * K[t] + 0.7 * g.normal(size=(B, d)) / np.sqrt(d)
    c = dict(Q=torch.from_numpy(Q + centre).to(getattr(torch, dtype)).cuda(), K=torch.from_numpy(K + centre).to(getattr(torch, dtype)).cuda())
    if ids:
        c["key_ids"] = g.integers(0, max(2, 3 * M), size=M).astype(np.int32)
        c["key_ids"][g.random(M) < 0.05] = -1
        c["query_ids"] = g.integers(-1, max(2, 3 * M), size=B).astype(np.int32)
        c["query_ids"][::3] = c["key_ids"][t[::3]]
    if bias:
        c["key_bias"] = g.normal(size=M).astype(np.float32)
        c["key_bias"][g.random(M) < 0.03] = -np.inf
    if weight:
        c["row_weight"] = (g.normal(size=B) / B).astype(np.float32)
    c["teacher_ids"] = g.integers(0, M, size=(B, n)).astype(np.int32)      # some twice
    c["teacher_ids"][:, 0] = t
    raw = g.normal(size=(B, n)) * 2
    c["teacher_logits"] = (raw - np.log(np.exp(raw).sum(1, keepdims=True)) + np.log(mass)).astype(np.float32)
    c["teacher_logits"][g.random((B, n)) < 0.05] = -np.inf
    c["teacher_ids"][g.random((B, n)) < 0.05] = -1
    if B > 3:
        c["teacher_ids"][1], c["teacher_ids"][2, 0] = -1, M
    return c


def call(rn, c, scale, tail, **kw):
    import torch
    x = {k: torch.from_numpy(v).cuda() if isinstance(v, np.ndarray) else v for k, v in c.items()}
    return rn.rnnd_distill(x.pop("Q"), x.pop("K"), x.pop("teacher_ids"), x.pop("teacher_logits"), scale, tail=tail, **x, **kw)


def reference(c, scale, tail):
    """loss, dq, dk in float64, and what their errors go with."""
    q, k = c["Q"].double().cpu().numpy(), c["K"].double().cpu().numpy()
    B, M = len(q), len(k)
    bias = c["key_bias"].astype(np.float64) if "key_bias" in c else np.zeros(M)
    w = c["row_weight"].astype(np.float64) if "row_weight" in c else np.ones(B)
    gone = bias == -np.inf
    if "key_ids" in c:
        gone = gone | (c["key_ids"] < 0)
    out = np.repeat(gone[None, :], B, 0)
    if "query_ids" in c:
        out |= c["key_ids"][None, :] == c["query_ids"][:, None]
    p = np.zeros((B, M))
    on = np.zeros((B, M), bool)
    for i in range(B):
        entries = {}
        for j, l in zip(c["teacher_ids"][i].tolist(), c["teacher_logits"][i].astype(np.float64)):
            if 0 <= j < M and l > -np.inf and not out[i, j] and j not in entries:
                entries[j] = l
        if not entries:
            continue
        at, l = list(entries), np.array(list(entries.values()))
        on[i, at] = True
        p[i, at] = np.exp(l if tail else l - l.max())
    counts = on.any(1)
    q, k = np.where(counts[:, None], q, 0.0), np.where(gone[:, None], 0.0, k)
    dist = np.square(q).sum(1)[:, None] + np.square(k).sum(1)[None, :] - 2 * q @ k.T
    s = np.where(out, -np.inf, np.where(gone, 0.0, bias)[None, :] - scale * dist)
    top = np.where(out.all(1), 0.0, np.where(out, -1e300, s).max(1))
    rest = np.clip(1 - p.sum(1), 0, None) if tail else np.zeros(B)
    rest = np.where((~out & ~on).any(1) & counts, rest, 0.0)
    mass = np.where(counts, p.sum(1) + rest, 1.0)
    p, rest = p / mass[:, None], rest / mass
    with np.errstate(divide="ignore", invalid="ignore"):
        e = np.exp(s - top[:, None])
        lse = top + np.log(e.sum(1))
        logp = np.where(on, s - lse[:, None], 0.0)
        off = np.where(on, 0.0, e)
        log_off = top + np.log(off.sum(1)) - lse
        each = np.where(p > 0, p * (np.log(p) - logp), 0.0)
        log_p = np.where(p > 0, np.log(p), 0.0)
        tail_loss = np.where(rest > 0, rest * (np.log(rest) - log_off), 0.0)
        loss = np.where(counts, each.sum(1) + tail_loss, 0.0)
        prob = np.where(counts[:, None], e / e.sum(1)[:, None], 0.0)
        R = np.where(counts, off.sum(1) / e.sum(1), 0.0)
        ratio = np.where(rest > 0, rest / R, 0.0)
    g = np.where(on, prob - p, prob * (1 - ratio[:, None])) * np.where(counts, w, 0.0)[:, None]
    dq = 2 * scale * (g @ k - g.sum(1)[:, None] * q)
    dk = 2 * scale * (g.T @ q - g.sum(0)[:, None] * k)
    size = (p * (abs(log_p) + abs(logp))).sum(1) + np.where(rest > 0, rest * (abs(np.log(np.where(rest > 0, rest, 1))) + abs(np.where(rest > 0, log_off, 0))), 0.0)
    # of |g|: each of its two terms by itself
    with np.errstate(divide="ignore", invalid="ignore"):
        share = np.where(off.sum(1)[:, None] > 0, off / off.sum(1)[:, None], 0.0)
    terms = np.where(on, prob + p, share * (R + rest)[:, None]) * np.where(counts, abs(w), 0.0)[:, None]
    return loss, dq, dk, g, q, k, counts, size, terms, w


def check(rn, c, scale, tail):
    """Bounds, with u = 2^-24 (half a float32 step) and h = half a step of the rows' type:
      - a logit: e = u ((n + 4) 2 |scale| |q||k| + (d + 4) |scale| |k|^2 + 4 |bias|), n = d, or 6 d of float32 rows in three terms
      - log P: e of the key and e of lse; so the loss, whose weights add up to 1: 2 e, and 40 u of the sizes of its terms for the
        exponentials, logarithms, the roundings of p and r, and sums
      - g: its terms w P and w p (off the list w R and w r times a share of the sum there) 2 e + 60 u of themselves each; then h of g
      - a gradient: every g_ij (k_j - q_i) with the error of g and that of a sum of as many products as there are, where the
        sum is formed as sum g k - q sum g; then the rounding."""
    import torch
    loss, dq, dk, g, q, k, counts, size, terms, w = reference(c, scale, tail)
    got_loss, got_q, got_k = call(rn, c, scale, tail)
    dtype = c["Q"].dtype
    u, info = 2.0 ** -24, torch.finfo(dtype)
    h = u if dtype == torch.float32 else info.eps / 2
    d, (B, M) = q.shape[1], g.shape
    n = 6 * d if dtype == torch.float32 else d
    nq, nk = np.sqrt(np.square(q).sum(1)), np.sqrt(np.square(k).sum(1))
    bias = c.get("key_bias", np.zeros(M, np.float32))
    bias = np.where(np.isfinite(bias), bias, 0.0)
    e = (u * ((n + 4) * 2 * abs(scale) * nq[:, None] * nk[None, :] + (d + 4) * abs(scale) * np.square(nk)[None, :] + 4 * abs(bias)[None, :])).max(1)
    off = abs(got_loss.double().cpu().numpy() - loss)
    bound = np.where(counts, 2 * e + 40 * u * (1 + size), 0.0)
    assert (off <= bound).all(), ("loss", (off - bound).max(), off.max())
    ge = terms * (2 * e[:, None] + 60 * u) + abs(g) * h * 1.01
    if dtype == torch.float16:      # g below the normal numbers of its scaled form
        ge = ge + np.where(counts, abs(w).max() * 2.0 ** -14 * 2.0 ** -24, 0.0)[:, None]
    for name, got, want, rows, other, gg, err in (("dQ", got_q, dq, q, k, g, ge), ("dK", got_k, dk, k, q, g.T, ge.T)):
        m = gg.shape[1] * (6 if dtype == torch.float32 else 1)
        bound = np.zeros_like(want)
        for i in range(len(want)):
            bound[i] = 2 * abs(scale) * ((err[i][:, None] * abs(other - rows[i])).sum(0) + (m + 8) * u * ((abs(gg[i]) + err[i])[:, None] * (abs(other) + abs(rows[i]))).sum(0))
        bound += abs(want) * (info.eps / 2 + 4 * u) * 1.01 + info.smallest_normal * info.eps / 2 + 1e-44
        off = abs(got.double().cpu().numpy() - want)
        assert (off <= bound).all(), (name, (off - bound).max(), off.max(), abs(want).max())
    none = torch.from_numpy(~counts).cuda()
    assert (got_loss[none] == 0).all() and (got_q[none] == 0).all()
    only, nothing_q, nothing_k = call(rn, c, scale, tail, want_grad=False)
    assert nothing_q is None and nothing_k is None and torch.equal(only, got_loss)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("tail", [False, True])
@pytest.mark.parametrize("B,M,d,n", [(1, 1, 1, 1), (1, 300, 33, 10), (5, 7, 3, 6), (65, 130, 32, 1), (100, 1100, 32, 128), (40, 129, 100, 20), (130, 260, 257, 30),
                                     (300, 50, 16, 65)])
def test_against_double_precision(rn, B, M, d, n, tail, dtype):
    check(rn, case(B, M, d, n, dtype, seed=B + M + d + n), 3.0, tail)


@pytest.mark.parametrize("dtype", TYPES)
def test_without_ids_biases_and_weights(rn, dtype):
    check(rn, case(60, 200, 48, 12, dtype, 3, ids=False, bias=False, weight=False), 3.0, True)


@pytest.mark.parametrize("mass", [1.5, 1.0, 0.001])
def test_what_the_teacher_leaves_to_the_others(rn, mass):
    """More than everything (rounded sums), nothing, nearly everything."""
    check(rn, case(70, 300, 40, 9, "float32", 4, mass=mass), 3.0, True)


def test_large_logits_of_the_teacher_are_scores(rn):
    c = case(30, 200, 40, 9, "float32", 5)
    c["teacher_logits"] = (c["teacher_logits"] * 30 + 500).astype(np.float32)
    check(rn, c, 3.0, False)


@pytest.mark.parametrize("tail", [False, True])
@pytest.mark.parametrize("dtype", TYPES)
def test_all_keys_listed(rn, tail, dtype):
    """No key is off the list: what the teacher left has nobody to go to.  More entries in a tile than have room in LDS."""
    c = case(140, 100, 24, 128, dtype, 6, ids=False, bias=False)
    g = np.random.Generator(np.random.PCG64(7))
    c["teacher_ids"] = np.stack([np.concatenate([g.permutation(100), np.full(28, -1)]) for _ in range(140)]).astype(np.int32)
    c["teacher_logits"] = np.where(np.isfinite(c["teacher_logits"]), c["teacher_logits"], -3.0).astype(np.float32)
    check(rn, c, 3.0, tail)


def test_tiles_of_256(rn):
    """16-bit rows long and many enough: the other tile, for the logits and for the gradients."""
    import torch
    c = case(256, 131_072, 392, 40, "bfloat16", 8)
    loss, dq, dk = call(rn, c, 3.0, True)
    assert torch.isfinite(dk).all()
    # one query at a time works with the small tiles
    for i in (0, 1, 2, 100, 255):
        part = dict(c, Q=c["Q"][i:i + 1].contiguous(), **{n: c[n][i:i + 1] for n in ("query_ids", "teacher_ids", "teacher_logits", "row_weight")})
        l, q, _ = call(rn, part, 3.0, True)
        # sums of the same logits, parted differently: 40 u of 1 + the loss; a gradient's terms are rounded alike, its sum in another order and its result once more
        assert abs(l[0] - loss[i]) <= 2.0 ** -24 * 100 * (1 + abs(loss[i]))
        assert (q[0].double() - dq[i].double()).norm() <= 2.0 ** -7 * dq[i].double().norm()


def test_a_student_that_agrees_has_no_gradient(rn):
    """The list is what the student says itself: loss and gradients are their errors.  (2 e + 60 u of P + p, with |q| = |k| = 1 or so.)"""
    import torch
    g = torch.Generator(device="cuda").manual_seed(9)
    K = torch.randn(900, 64, device="cuda", generator=g) / 8
    Q = K[:120] + 0.5 * torch.randn(120, 64, device="cuda", generator=g) / 8
    _, _, ids, logp = rn.rnnd_logprob(Q, K, 4.0, alternatives=32)
    loss, dq, dk = rn.rnnd_distill(Q, K, ids, logp, 4.0, tail=True)
    assert loss.abs().max() < 1e-3 and dq.abs().max() < 1e-3 and dk.abs().max() < 1e-3
    other, dq, _ = rn.rnnd_distill(Q, K, ids, logp - 0.5, 4.0, tail=True)
    assert (other > 1e-3).all() and dq.abs().max() > 1e-3


def test_gradients_against_differences(rn):
    """float32, steps along random directions: the loss's second differences bound the error of a first one."""
    import torch
    c = case(24, 150, 20, 8, "float32", 10)
    for tail in (False, True):
        _, dq, dk = call(rn, c, 2.0, tail)
        w = c["row_weight"].astype(np.float64)

        def total(x):
            return (reference(x, 2.0, tail)[0] * w).sum()
        g = torch.Generator(device="cuda").manual_seed(3)
        for name, grad in (("Q", dq), ("K", dk)):
            step = torch.randn(c[name].shape, device="cuda", generator=g)
            step = (step / step.norm()).double()
            h = 1e-4
            up, down = total(dict(c, **{name: c[name].double() + h * step})), total(dict(c, **{name: c[name].double() - h * step}))
            slope = (grad.double() * step).sum().item()
            # the central difference is off by h^2 / 6 of a third derivative of order (2 scale)^3; the gradient by float32 errors (see above)
            assert abs((up - down) / (2 * h) - slope) <= 1e-5 * (1 + abs(slope)), (name, tail)


@pytest.mark.parametrize("dtype", TYPES)
def test_what_is_left_out_is_never_read_as_a_number(rn, dtype):
    import torch
    c = case(60, 300, 40, 8, dtype, 11)
    want = call(rn, c, 3.0, True)
    gone = torch.from_numpy((c["key_ids"] < 0) | (c["key_bias"] == -np.inf)).cuda()
    c["K"][gone] = float("nan")
    c["Q"][1] = float("inf")         # no entry
    for x, y in zip(want, call(rn, c, 3.0, True)):
        assert torch.equal(x, y)


def test_float32_rows_far_from_the_origin(rn):
    """Logits go with the distances: rows moved by a vector that float32 holds exactly have the same loss."""
    import torch
    c = case(50, 300, 64, 8, "float32", 12)
    c["Q"], c["K"] = (x.mul(2 ** 12).round().div(2 ** 12) for x in (c["Q"], c["K"]))
    want = call(rn, c, 3.0, True)
    got = call(rn, dict(c, Q=c["Q"] + 64, K=c["K"] + 64), 3.0, True)
    for x, y in zip(want, got):
        assert (x - y).abs().max() <= 2.0 ** -24 * 6 * 70 * 3 * 16 * max(1.0, x.abs().max().item())


def test_no_query(rn):
    import torch
    K = torch.randn(30, 8, device="cuda")
    i, l = torch.zeros(0, 4, dtype=torch.int32, device="cuda"), torch.zeros(0, 4, device="cuda")
    loss, dq, dk = rn.rnnd_distill(K[:0], K, i, l, 1.0)
    assert loss.shape == (0,) and dq.shape == (0, 8) and (dk == 0).all()
    lp, ent, ids, top = rn.rnnd_logprob(K[:0], K, 1.0, alternatives=3)
    assert lp is None and ent.shape == (0,) and ids.shape == (0, 3) and top.shape == (0, 3)


def test_a_captured_round_of_answers_and_distillation_replays_as_the_eager_one(rn):
    """The teacher answers, the student learns from it; several replays, with eager work and synchronizations in between."""
    import torch
    g = torch.Generator(device="cuda").manual_seed(13)
    T, S = torch.randn(700, 96, device="cuda", generator=g) / 10, (torch.randn(700, 32, device="cuda", generator=g) / 6).bfloat16()
    names = torch.arange(700, device="cuda", dtype=torch.int32)
    query = torch.randint(0, 700, (100,), device="cuda", generator=g, dtype=torch.int32)

    def together():
        tq, sq = rn.rnnd_embed(T, query), rn.rnnd_embed(S, query)
        _, ent, ids, logp = rn.rnnd_logprob(tq, T, 5.0, alternatives=16, query_ids=query, key_ids=names)
        one = rn.rnnd_logprob(tq[:2], T, 5.0, alternatives=16, query_ids=query[:2], key_ids=names)
        loss, dq, dk = rn.rnnd_distill(sq, S, ids, logp, 5.0, tail=True, query_ids=query, key_ids=names)
        return [ent, ids, logp, loss, dq, dk, rn.rnnd_embed_grad(dq, query, 700)] + list(one[1:])
    together()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        captured = together()
    for i in range(4):
        want = together()
        graph.replay()
        torch.cuda.synchronize()
        for x, y in zip(captured, want):
            assert torch.equal(x, y), i
        assert torch.equal(want[1][:2], want[8])
        query.copy_(torch.randint(0, 700, (100,), device="cuda", dtype=torch.int32))
        S.add_(0.01 * torch.randn(700, 32, device="cuda"))


def test_streams_of_their_own_give_the_same_bits(rn):
    """Two calls at once, each on its stream, and memory that the current stream takes meanwhile."""
    import torch
    c = case(200, 3000, 64, 20, "bfloat16", 14)
    x = {k: torch.from_numpy(v).cuda() if isinstance(v, np.ndarray) else v for k, v in c.items()}
    answer = {k: x[k] for k in ("query_ids", "key_ids", "key_bias")}

    def both(a, b):
        return (rn.rnnd_distill(x["Q"], x["K"], x["teacher_ids"], x["teacher_logits"], 3.0, tail=True, row_weight=x["row_weight"], stream=a, **answer)
                + rn.rnnd_logprob(x["Q"], x["K"], 3.0, alternatives=20, stream=b, **answer)[1:])
    want = both(None, None)
    torch.cuda.synchronize()
    a, b = torch.cuda.Stream(), torch.cuda.Stream()
    for _ in range(3):
        got = both(a, b)
        junk = [torch.full((1 << 20,), float("nan"), device="cuda") for _ in range(4)]
        a.synchronize()
        b.synchronize()
        for u, v in zip(got, want):
            assert torch.equal(u, v)
        del junk


@pytest.mark.parametrize("dtype", TYPES)
def test_keys_that_many_queries_list(rn, dtype):
    """One key in every list, one in a fifth of them: a whole block sums these; row for row against float64."""
    c = case(1300, 90, 24, 5, dtype, 15)
    g = np.random.Generator(np.random.PCG64(16))
    c["teacher_ids"][:, 1], c["teacher_ids"][g.random(1300) < 0.2, 2] = 17, 18
    for j in (17, 18):
        c["key_ids"][j], c["key_bias"][j] = 1000 + j, 0.0
    check(rn, c, 3.0, True)


def test_a_gradient_that_is_a_small_difference(rn):
    """Teacher and student differ only in how they divide the probability between two keys that lie close together: g of the two is large and
    of both signs, the gradient small.  Its terms are float32, so the gradient is off by little more than the rounding of its own values."""
    import torch
    c = case(40, 200, 64, 2, "float16", 17, ids=False, bias=False, weight=False)
    K = c["K"].float()
    K[1::2] = K[0::2] + 0.01 * K[1::2]
    c["K"], c["Q"] = K.half(), (K[0:80:2] + 0.05 * c["Q"].float()).half()
    c["teacher_ids"] = np.arange(80).reshape(40, 2).astype(np.int32)
    c["teacher_logits"] = np.tile(np.log(np.array([[0.8, 0.2]])), (40, 1)).astype(np.float32)
    _, dq, _, *_ = reference(c, 20.0, True)
    got = call(rn, c, 20.0, True)[1].double().cpu().numpy()
    # half a step for the rounding of the result, as much again for all else: g off the list is below 2^-8 here, rounded with 2^-11 of itself
    assert np.sqrt(np.square(got - dq).sum()) <= 2 * 2.0 ** -11 * np.sqrt(np.square(dq).sum())
