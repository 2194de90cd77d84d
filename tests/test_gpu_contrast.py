"""The softmax loss over squared distances and its gradients, against the formulas in double precision and against differences."""
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


def case(B, M, d, dtype, seed, ids=True, bias=True, weight=True, spread=1.0, far=0.0):
    """Inputs of a batch whose queries lie near their positives; far: how far the rows lie from the origin."""
    import torch
    g = np.random.Generator(np.random.PCG64(seed))
    centre = far * g.normal(size=d) / np.sqrt(d)
    K = g.normal(size=(M, d)) / np.sqrt(d)
    t = g.integers(0, M, size=B)
    Q = 0.7 * K[t] + spread * 0.7 * g.normal(size=(B, d)) / np.sqrt(d)
    c = dict(Q=torch.from_numpy(Q + centre).to(getattr(torch, dtype)).cuda(), K=torch.from_numpy(K + centre).to(getattr(torch, dtype)).cuda(),
             target=t.astype(np.int32))
    if ids:
        c["key_ids"] = g.integers(0, max(2, 3 * M), size=M).astype(np.int32)
        c["key_ids"][g.random(M) < 0.05] = -1
        c["query_ids"] = g.integers(-1, max(2, 3 * M), size=B).astype(np.int32)
    if bias:
        c["key_bias"] = g.normal(size=M).astype(np.float32)
        c["key_bias"][g.random(M) < 0.03] = -np.inf
    if weight:
        c["row_weight"] = (g.normal(size=B) / B).astype(np.float32)
    if B > 3:
        c["target"][1], c["target"][2] = -1, M
    return c


def call(rn, c, scale, **kw):
    import torch
    x = {k: torch.from_numpy(v).cuda() if isinstance(v, np.ndarray) else v for k, v in c.items()}
    return rn.rnnd_contrast(x.pop("Q"), x.pop("K"), x.pop("target"), scale, **x, **kw)


def reference(c, scale):
    """loss, dq, dk in float64; and g, to bound the errors with."""
    q, k = c["Q"].double().cpu().numpy(), c["K"].double().cpu().numpy()
    B, M = len(q), len(k)
    t = c["target"].astype(np.int64)
    bias = c["key_bias"].astype(np.float64) if "key_bias" in c else np.zeros(M)
    w = c["row_weight"].astype(np.float64) if "row_weight" in c else np.ones(B)
    gone = bias == -np.inf
    if "key_ids" in c:
        gone = gone | (c["key_ids"] < 0)
    at = np.clip(t, 0, M - 1)
    counts = (t >= 0) & (t < M) & ~gone[at]
    q, k = np.where(counts[:, None], q, 0.0), np.where(gone[:, None], 0.0, k)
    out = np.repeat(gone[None, :], B, 0)
    if "key_ids" in c:
        twin = c["key_ids"][None, :] == c["key_ids"][at][:, None]
        if "query_ids" in c:
            twin |= c["key_ids"][None, :] == c["query_ids"][:, None]
        twin[np.arange(B), at] = False
        out = out | twin
    dist = np.square(q).sum(1)[:, None] + np.square(k).sum(1)[None, :] - 2 * q @ k.T
    s = np.where(out, -np.inf, np.where(gone, 0.0, bias)[None, :] - scale * dist)
    with np.errstate(invalid="ignore", divide="ignore"):
        own = s[np.arange(B), at]
        others = s.copy()
        others[np.arange(B), at] = -np.inf
        top = others.max(1)
        x = np.where(top == -np.inf, -np.inf, top + np.log(np.exp(others - np.where(top == -np.inf, 0, top)[:, None]).sum(1))) - own
        loss = np.where(counts, np.logaddexp(0.0, x), 0.0)
        p = np.exp(s - (own + loss)[:, None])
    p[np.arange(B), at] = np.expm1(-loss)
    g = np.where(counts[:, None], p * w[:, None], 0.0)
    dq = 2 * scale * (g @ k - g.sum(1)[:, None] * q)
    dk = 2 * scale * (g.T @ q - g.sum(0)[:, None] * k)
    return loss, dq, dk, g, q, k, w, counts


def check(rn, c, scale):
    """Bounds, with u = 2^-24 (half a float32 step) and h = half a step of the rows' type:
      - a logit: a sum of d products (and float32 rows' terms: 6 d of them), its scaling, the key's own sum and the rounding of
        their sum: e = u * ((n + 4) * 2 |scale| |q||k| + (d + 4) * |scale| |k|^2 + 4 |bias|), n = d or 6 d
      - the loss: both lse and the target's logit carry e; the exponentials and logarithms some 20 u of themselves
      - g: 2 e + 24 u of itself, then h (float32 rows: 2^-24 again)
      - a gradient: every g_ij (k_j - q_i) with the error of g and that of a sum of as many products as there are, where
        the sum is formed as sum g k - q sum g; then the rounding."""
    import torch
    loss, dq, dk, g, q, k, w, counts = reference(c, scale)
    got_loss, got_q, got_k = call(rn, c, scale)
    dtype = c["Q"].dtype
    u, info = 2.0 ** -24, torch.finfo(dtype)
    h = u if dtype == torch.float32 else info.eps / 2
    d, (B, M) = q.shape[1], g.shape
    n = 6 * d if dtype == torch.float32 else d
    nq, nk = np.sqrt(np.square(q).sum(1)), np.sqrt(np.square(k).sum(1))
    bias = np.where(np.isfinite(c.get("key_bias", np.zeros(M, np.float32))), c.get("key_bias", np.zeros(M, np.float32)), 0.0)
    e = u * ((n + 4) * 2 * abs(scale) * nq[:, None] * nk[None, :] + (d + 4) * abs(scale) * np.square(nk)[None, :] + 4 * abs(bias)[None, :])
    e_row = e.max(1) if M else 0.0
    off = abs(got_loss.double().cpu().numpy() - loss)
    bound = np.where(counts, 2 * e_row + 20 * u * (1 + loss), 0.0)
    assert (off <= bound).all(), ("loss", (off - bound).max())
    ge = abs(g) * (2 * e_row[:, None] + 24 * u + h * 1.01)
    if dtype == torch.float16:      # g below the normal numbers of its scaled form
        ge = ge + np.where(counts, abs(w).max() * 2.0 ** -14 * 2.0 ** -24, 0.0)[:, None]
    for name, got, want, rows, other, gg, err in (("dQ", got_q, dq, q, k, g, ge), ("dK", got_k, dk, k, q, g.T, ge.T)):
        m = gg.shape[1] * (6 if dtype == torch.float32 else 1)
        bound = np.zeros_like(want)
        for i in range(len(want)):
            bound[i] = 2 * abs(scale) * ((err[i][:, None] * abs(other - rows[i])).sum(0) + (m + 8) * u * (abs(gg[i])[:, None] * (abs(other) + abs(rows[i]))).sum(0))
        bound += abs(want) * (info.eps / 2 + 4 * u) * 1.01 + info.smallest_normal * info.eps / 2 + 1e-44
        off = abs(got.double().cpu().numpy() - want)
        assert (off <= bound).all(), (name, (off - bound).max(), off.max(), abs(want).max())
    none = torch.from_numpy(~counts).cuda()
    assert (got_loss[none] == 0).all() and (got_q[none] == 0).all()
    gone = c["key_ids"] < 0 if "key_ids" in c else np.zeros(M, bool)
    if "key_bias" in c:
        gone = gone | (c["key_bias"] == -np.inf)
    assert (got_k[torch.from_numpy(gone).cuda()] == 0).all()
    only, no_q, no_k = call(rn, c, scale, want_grad=False)
    assert no_q is None and no_k is None and torch.equal(only, got_loss)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("B,M,d", [(1, 1, 1), (1, 2, 3), (2, 1, 8), (1, 300, 96), (5, 129, 7), (64, 64, 64), (127, 130, 65), (128, 128, 128),
                                   (129, 257, 100), (100, 1100, 32), (300, 400, 200), (70, 515, 768)])
def test_loss_and_gradients(rn, dtype, B, M, d):
    check(rn, case(B, M, d, dtype, B * 7 + M), 4.0)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("ids,bias,weight", [(False, False, False), (True, False, False), (False, True, True), (True, True, False)])
def test_without_some_of_the_arguments(rn, dtype, ids, bias, weight):
    c = case(90, 200, 48, dtype, 3, ids, bias, weight)
    check(rn, c, 2.5)
    if ids:
        del c["query_ids"]
        check(rn, c, 2.5)


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("B,M,d", [(1500, 300, 40), (40, 6000, 24), (900, 2100, 130)])
def test_sums_that_are_split(rn, dtype, B, M, d):
    check(rn, case(B, M, d, dtype, 11), 3.0)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("scale", [0.0, 1e-3, 30.0, -1.0])
def test_scales(rn, dtype, scale):
    check(rn, case(60, 90, 32, dtype, 5), scale)


@pytest.mark.parametrize("dtype", TYPES)
def test_small_losses_and_rows_far_from_the_origin(rn, dtype):
    check(rn, case(50, 80, 64, dtype, 6, ids=False, bias=False, spread=0.02), 20.0)
    check(rn, case(50, 80, 64, dtype, 7, far=4.0), 4.0)


@pytest.mark.parametrize("dtype", TYPES)
def test_masks_that_leave_only_the_target_or_nothing(rn, dtype):
    import torch
    c = case(40, 70, 32, dtype, 8, bias=False)
    c["key_ids"][:] = 4                 # every key is the positive again
    c["target"][:] = np.arange(40) % 7
    check(rn, c, 4.0)
    loss, dq, dk = call(rn, c, 4.0)
    assert (loss == 0).all() and (dq == 0).all() and (dk == 0).all()
    c["key_ids"][:] = -1                # no key at all
    loss, dq, dk = call(rn, c, 4.0)
    assert (loss == 0).all() and (dq == 0).all() and (dk == 0).all()
    c = case(40, 70, 32, dtype, 8)
    c["target"][:] = [-1, 70, -2**31, 2**31 - 1] * 10
    loss, dq, dk = call(rn, c, 4.0)
    assert (loss == 0).all() and (dq == 0).all() and (dk == 0).all()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), float("-inf")])
def test_what_rows_that_are_left_out_hold_does_not_matter(rn, dtype, bad):
    import torch
    c = case(150, 170, 40, dtype, 9)
    c["key_ids"][5], c["key_bias"][140] = -1, -np.inf
    c["target"][7] = 5
    clean = dict(c)
    want = call(rn, c, 4.0)
    _, _, _, _, _, _, _, counts = reference(c, 4.0)
    gone = (c["key_ids"] < 0) | (c["key_bias"] == -np.inf)
    clean["Q"], clean["K"] = c["Q"].clone(), c["K"].clone()
    clean["Q"][torch.from_numpy(~counts).cuda()] = bad
    clean["K"][torch.from_numpy(gone).cuda()] = bad
    if "row_weight" in clean:
        clean["row_weight"] = np.where(counts, c["row_weight"], bad).astype(np.float32)
    clean["key_bias"] = np.where(gone & (c["key_ids"] < 0), np.float32(np.nan), c["key_bias"])
    check(rn, c, 4.0)
    for a, b in zip(call(rn, clean, 4.0), want):
        assert torch.equal(a, b)


def test_biases_of_the_types_lowest_value(rn):
    c = case(30, 60, 16, "float32", 10, ids=False)
    c["key_bias"][::3] = np.finfo(np.float32).min
    c["target"][:] = 1
    c["key_bias"][1] = 0.0
    loss, dq, dk, *_ = reference(c, 1.0)
    got = call(rn, c, 1.0)
    assert np.allclose(got[0].cpu().numpy(), loss, rtol=1e-5) and np.isfinite(got[1].cpu().numpy()).all()
    assert (got[2][::3] == 0).all()


def test_a_row_that_is_not_finite_shows(rn):
    c = case(30, 60, 16, "bfloat16", 10, ids=False, bias=False)
    c["Q"][4, 3] = float("nan")
    loss, dq, dk = call(rn, c, 1.0)
    assert loss[4].isnan() and dq[4].isnan().all()
    assert int(loss.isnan().sum()) == 1


@pytest.mark.parametrize("exponent", [-60, 0, 60])
def test_weights_of_any_size(rn, exponent):
    """float16 gradients hold what their type can; the weights' size does not change g's precision on the way."""
    import torch
    c = case(50, 400, 32, "float16", 12)
    _, q0, k0 = call(rn, c, 4.0)
    for dtype in ("float32", "bfloat16"):
        x = dict(case(50, 400, 32, dtype, 12))
        x["row_weight"] = x["row_weight"] * np.float32(2.0 ** exponent)
        check(rn, x, 4.0)
    c["row_weight"] = c["row_weight"] * np.float32(2.0 ** 10)
    _, q1, k1 = call(rn, c, 4.0)
    for a, b in ((q0, q1), (k0, k1)):
        big = a.float().abs() > 1e-3       # normal numbers before and after
        assert torch.equal((a.float() * 1024)[big], b.float()[big])


@pytest.mark.parametrize("metric", ["query", "key"])
def test_against_differences(rn, metric):
    """Central differences of the library's own loss: an error of h^2 times a third derivative, below (2 scale |k - q|)^3 h^2 / 6
    of a loss of order 1, and 2e-7 * scale / h of its float32 values."""
    import torch
    c = case(12, 30, 8, "float32", 13)
    w = torch.from_numpy(c["row_weight"]).cuda().double()
    c["row_weight"] = c["row_weight"] * 12
    w = w * 12
    _, dq, dk = call(rn, c, 2.0)
    name, grad = ("Q", dq) if metric == "query" else ("K", dk)
    h = 1e-2
    x = c[name]
    for i in range(0, x.shape[0], 3):
        for e in range(0, 8, 3):
            sides = []
            for sign in (1, -1):
                y = dict(c)
                y[name] = x.clone()
                y[name][i, e] += sign * h
                step = (y[name][i, e] - x[i, e]).double().item()
                sides.append(((call(rn, y, 2.0, want_grad=False)[0].double() * w).sum().item(), step))
            diff = (sides[0][0] - sides[1][0]) / (sides[0][1] - sides[1][1])
            assert abs(diff - grad[i, e].item()) < 12 * (4 * h * h * 2 + 2e-6 / h * 0.1), (i, e, diff, grad[i, e].item())


@pytest.mark.parametrize("dtype", TYPES)
def test_the_same_call_gives_the_same_bits_on_any_workspace(rn, dtype):
    import torch
    B, M, d = 200, 333, 72
    c = case(B, M, d, dtype, 14)
    first = call(rn, c, 4.0)
    need = rn.rnnd_contrast_workspace(B, M, d, {"float32": 1, "float16": 2, "bfloat16": 3}[dtype])
    for fill in (0x00, 0xA5, 0xFF, 0x7F):
        block = torch.full((need + 256,), fill, dtype=torch.uint8, device="cuda")
        for a, b in zip(call(rn, c, 4.0, workspace=block[:need]), first):
            assert torch.equal(a, b)
        assert (block[need:] == fill).all()


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
def test_rows_at_any_alignment(rn, dtype):
    import torch
    c = case(50, 70, 24, dtype, 15)
    want = call(rn, c, 4.0)
    for k in ("Q", "K"):
        flat = torch.empty(c[k].numel() + 1, dtype=c[k].dtype, device="cuda")
        flat[1:] = c[k].reshape(-1)
        c[k] = flat[1:].view(c[k].shape)
    for a, b in zip(call(rn, c, 4.0), want):
        assert torch.equal(a, b)


def test_no_query(rn):
    import torch
    K = torch.ones(9, 5, device="cuda", dtype=torch.bfloat16)
    loss, dq, dk = rn.rnnd_contrast(K[:0], K, torch.empty(0, dtype=torch.int32, device="cuda"), 1.0)
    assert loss.shape == (0,) and dq.shape == (0, 5) and dk.shape == (9, 5) and (dk == 0).all()


def test_refusals_of_the_binding(rn):
    import torch
    q = torch.zeros(4, 8, device="cuda")
    t = torch.zeros(4, dtype=torch.int32, device="cuda")
    for args, kw in (((q, q.half(), t), {}), ((q, q[:, :4].contiguous(), t), {}), ((q, q.t(), t), {}), ((q, q, t.long()), {}), ((q, q, t[:3]), {}),
                     ((q.double(), q.double(), t), {}), ((q, q, t), dict(key_ids=t[:2])), ((q, q, t), dict(key_bias=q[0])),
                     ((q, q, t), dict(row_weight=t)), ((q, q, t), dict(query_ids=t.cpu()))):
        with pytest.raises(ValueError):
            rn.rnnd_contrast(*args, 1.0, **kw)
    with pytest.raises(rn.RnndError):
        rn.rnnd_contrast(q, q, t, 1.0, query_ids=t)
