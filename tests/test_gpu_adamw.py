"""The AdamW step against its formula in double precision, and the 8-bit states against their definition."""
import math

import numpy as np
import pytest

pytestmark = pytest.mark.gpu

G64 = 0x9E3779B97F4A7C15
MASK = (1 << 64) - 1
HYPER = dict(lr=2e-3, beta1=0.9, beta2=0.995, eps=1e-7, weight_decay=0.05, grad_scale=0.5)


@pytest.fixture(scope="module")
def rn():
    import torch
    assert torch.cuda.is_available(), "these tests need the MI355X"
    import paper_2310_20419_amd as m
    m.load_library()
    return m


def normal(n, seed, std=1.0):
    import torch
    g = torch.Generator(device="cuda").manual_seed(seed)
    return torch.randn(n, device="cuda", generator=g) * std


def at_offset(x, offset):
    """The same values at an address `offset` elements behind an aligned one."""
    import torch
    flat = torch.empty(x.numel() + offset, dtype=x.dtype, device="cuda")
    flat[offset:] = x
    return flat[offset:]


def formula(p, g, m, v, step, h):
    """(p, m, v) in float64, and bounds of a float32 evaluation's error.  u = 2^-24 is half a float32 step."""
    u = 2.0 ** -24
    b1, b2 = h["beta1"], h["beta2"]
    g = g * np.float64(np.float32(h["grad_scale"]))
    m1, v1 = b1 * m + (1 - b1) * g, b2 * v + (1 - b2) * g * g
    # two rounded constants, a rounded gradient, a product and a sum: at most 5 half steps of the summands
    em = 5 * u * (abs(b1 * m) + abs((1 - b1) * g)) + 1e-44
    ev = 6 * u * v1 + 1e-44
    c1, c2 = 1 - b1 ** step, 1 - b2 ** step
    den = np.sqrt(v1 / c2) + h["eps"]
    upd = h["lr"] / c1 * m1 / den
    p1 = p * (1 - h["lr"] * h["weight_decay"]) - upd
    # the root halves v's relative error; root, scale, eps, division, rate and their products: 8 half steps more
    ep = 3 * u * (abs(p) + abs(upd)) + abs(h["lr"] / c1) * (em / den) + abs(upd) * (3 * u + 8 * u) + 1e-44
    return p1, m1, v1, ep, em, ev


def np64(x):
    return x.double().cpu().numpy()


@pytest.mark.parametrize("grad_dtype", ["float32", "float16", "bfloat16"])
@pytest.mark.parametrize("copy", [None, "float16", "bfloat16"])
def test_states_in_32_bits(rn, grad_dtype, copy):
    import torch
    sizes = [1, 7, 8, 9, 127, 2048, 2049, 4096, 100_003] + [k * 37 + 1 for k in range(90)]     # several launches
    tensors, before = [], []
    for i, n in enumerate(sizes):
        t = dict(param=normal(n, i), grad=normal(n, 1000 + i, 0.1).to(getattr(torch, grad_dtype)), m=normal(n, 2000 + i, 0.05),
                 v=normal(n, 3000 + i, 0.1).square())
        if i % 3 == 1:      # addresses that allow no wide accesses
            t = {k: at_offset(x, 1 + i % 3) for k, x in t.items()}
        if copy:
            t["copy"] = torch.full((n,), -7.0, device="cuda", dtype=getattr(torch, copy))
        tensors.append(t)
        before.append([np64(t[k]) for k in ("param", "grad", "m", "v")])
    rn.rnnd_adamw(rn.AdamwTensors(tensors), 3, **HYPER)
    for t, (p, g, m, v) in zip(tensors, before):
        p1, m1, v1, ep, em, ev = formula(p, g, m, v, 3, HYPER)
        for name, want, bound in (("param", p1, ep), ("m", m1, em), ("v", v1, ev)):
            off = abs(np64(t[name]) - want)
            assert (off <= bound).all(), (name, len(p), (off / bound).max())
        if copy:
            assert torch.equal(t["copy"], t["param"].to(t["copy"].dtype))


def test_many_steps_from_nothing_follow_the_formula(rn):
    """Zero moments, 20 steps: against the same steps in float64, with the first steps' large corrections."""
    import torch
    n, h = 5_000, dict(HYPER, weight_decay=0.0)
    p = normal(n, 1)
    t = dict(param=p.clone(), grad=torch.zeros(n, device="cuda"), m=torch.zeros(n, device="cuda"), v=torch.zeros(n, device="cuda"))
    plan = rn.AdamwTensors([t])
    wp, wm, wv = np64(p), np.zeros(n), np.zeros(n)
    for step in range(1, 21):
        t["grad"].copy_(normal(n, 100 + step, 10.0 ** (step % 5 - 2)))
        rn.rnnd_adamw(plan, step, **h)
        wp, wm, wv, _, _, _ = formula(wp, np64(t["grad"]), wm, wv, step, h)
    # a step moves a parameter by about lr; 20 of them, each with an error of some 30 half steps of its update
    assert abs(np64(t["param"]) - wp).max() <= 20 * (2.0 ** -24 * 3 * 6 + 30 * 2.0 ** -24 * 10 * h["lr"])


# ---------------------------------------------------------------- 8 bits
def mix64(z):
    z = ((z ^ (z >> np.uint64(30))) * np.uint64(0xBF58476D1CE4E5B9))
    z = ((z ^ (z >> np.uint64(27))) * np.uint64(0x94D049BB133111EB))
    return z ^ (z >> np.uint64(31))


def random_bits(n, counter, seed, step):
    with np.errstate(over="ignore"):
        key = mix64(np.array([(seed + G64 * (step + 1)) & MASK], np.uint64))
        i = np.arange(n, dtype=np.uint64) + np.uint64(counter)
        w = mix64(key + np.uint64(G64) * (i // np.uint64(2) + np.uint64(1)))
    half = np.where(i % np.uint64(2) == 1, w >> np.uint64(32), w & np.uint64(0xFFFFFFFF)).astype(np.int64)
    return half & 0xFFFF, half >> 16


def decode(codes, scale):
    import torch
    byte = scale.cpu().numpy().astype(np.float64)
    c = codes.view(torch.float8_e4m3fn).float().cpu().numpy().astype(np.float64)
    s = np.where(byte == 255, np.nan, np.exp2(byte - 127))
    return c * np.repeat(s, 128)[:len(c)]


def lattice(y, byte):
    """Distance of two codes around magnitudes y under the scale bytes."""
    s = np.repeat(np.exp2(byte.astype(np.float64) - 127), 128)[:len(y)]
    z = y / s
    e = np.floor(np.log2(np.maximum(z, 2.0 ** -6)))
    return s, np.exp2(e - 3)


def eight(rn, n, seed, grad_dtype, offset=0, zero=False):
    import torch
    t = dict(param=normal(n, seed), grad=normal(n, seed + 1, 0.1).to(grad_dtype),
             m=torch.zeros(n, dtype=torch.uint8, device="cuda"), v=torch.zeros(n, dtype=torch.uint8, device="cuda"))
    blocks = -(-n // 128)
    t["m_scale"] = torch.zeros(blocks, dtype=torch.uint8, device="cuda")
    t["v_scale"] = torch.zeros(blocks, dtype=torch.uint8, device="cuda")
    if not zero:        # any codes that are numbers, any sensible scales
        g = torch.Generator(device="cuda").manual_seed(seed)
        t["m"] = (torch.randint(0, 0x79, (n,), device="cuda", generator=g) + 128 * torch.randint(0, 2, (n,), device="cuda", generator=g)).to(torch.uint8)
        t["v"] = torch.randint(0, 0x79, (n,), device="cuda", generator=g).to(torch.uint8)
        t["m_scale"] = torch.randint(110, 120, (blocks,), device="cuda", generator=g).to(torch.uint8)
        t["v_scale"] = torch.randint(110, 120, (blocks,), device="cuda", generator=g).to(torch.uint8)
    return {k: at_offset(x, offset) for k, x in t.items()} if offset else t


@pytest.mark.parametrize("n,offset", [(1, 0), (8, 0), (127, 0), (128, 0), (129, 0), (2048, 0), (2047, 3), (50_001, 0), (50_001, 1), (131_072, 0)])
@pytest.mark.parametrize("grad_dtype", ["float32", "bfloat16"])
def test_states_in_8_bits(rn, n, offset, grad_dtype):
    import torch
    t = eight(rn, n, n, getattr(torch, grad_dtype), offset)
    p, g = np64(t["param"]), np64(t["grad"])
    m, r = decode(t["m"], t["m_scale"]), decode(t["v"], t["v_scale"])
    seed, step, counter = 77, 5, 2 * n + 6
    rn.rnnd_adamw(rn.AdamwTensors([dict(t, counter=counter)]), step, seed=seed, **HYPER)
    p1, m1, v1, ep, em, ev = formula(p, g, m, r * r, step, HYPER)
    ep += abs(p1 - p) * 2.0 ** -24 * 2        # the stored root is squared first
    assert (abs(np64(t["param"]) - p1) <= ep).all()
    for_m, for_v = random_bits(n, counter, seed, step)
    for name, want, bits, err in (("m", m1, for_m, em), ("v", np.sqrt(v1), for_v, 6 * 2.0 ** -24 * np.sqrt(v1) + 1e-44)):
        byte = t[name + "_scale"].cpu().numpy()
        top = np.array([abs(want[i:i + 128]).max() for i in range(0, n, 128)])
        z_top = top / np.exp2(byte.astype(np.float64) - 127)
        assert (z_top * 1.01 < 256 * (1 + 1e-6)).all() and ((z_top * 1.01 >= 128 * (1 - 1e-6)) | (byte == 0)).all()
        s, gap = lattice(abs(want), byte)
        z = abs(want) / s
        code = np.floor(z / gap + bits / 65536.0) * gap
        if name == "v":
            code = np.where((z > 0) & (code == 0), 2.0 ** -9, code)
        got = decode(t[name], t[name + "_scale"])
        exp = np.copysign(code * s, want)
        wrong = got != exp
        # where the last bits of the float32 value decide, one code up or down; as often as such bits do
        assert (abs(got - exp)[wrong] <= (1.0001 * gap * s)[wrong]).all()
        near = abs((z / gap + bits / 65536.0) % 1.0 + 0.5) % 1.0 - 0.5        # distance from the border, in codes
        assert (abs(near[wrong]) <= (err / s / gap)[wrong] * 1.01 + 2.0 ** -18).all()


@pytest.mark.parametrize("grad_dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("bits", [8, 32])
def test_moments_are_bit_for_bit_those_of_separate_float32_operations(rn, bits, grad_dtype):
    """Five steps: every product and sum of the moments rounded on its own, so that 8-bit codes, which a last bit can decide,
    are the ones that a program of plain float32 operations finds."""
    import torch
    n, seed, h = 300_007, 5, dict(HYPER, grad_scale=0.75)
    f = np.float32
    if bits == 8:
        t = eight(rn, n, 9, getattr(torch, grad_dtype))
    else:
        t = dict(param=normal(n, 1), grad=normal(n, 2, 0.1).to(getattr(torch, grad_dtype)), m=normal(n, 3, 0.05), v=normal(n, 4, 0.1).square())
    plan = rn.AdamwTensors([t])
    for step in range(7, 12):
        g = t["grad"].float().cpu().numpy() * f(h["grad_scale"])
        if bits == 8:
            m, v = decode(t["m"], t["m_scale"]).astype(f), np.square(decode(t["v"], t["v_scale"]).astype(f))
        else:
            m, v = t["m"].cpu().numpy(), t["v"].cpu().numpy()
        rn.rnnd_adamw(plan, step, seed=seed, **h)
        m = f(h["beta1"]) * m + f(1 - h["beta1"]) * g
        v = f(h["beta2"]) * v + f(1 - h["beta2"]) * g * g
        assert m.dtype == f and v.dtype == f
        if bits == 32:
            assert np.array_equal(t["m"].cpu().numpy(), m) and np.array_equal(t["v"].cpu().numpy(), v)
            continue
        for name, y, random16 in zip(("m", "v"), (m, np.sqrt(v)), random_bits(n, 0, seed, step)):
            top = np.maximum.reduceat(abs(y), np.arange(0, n, 128)) * f(1.01)
            byte = np.clip(np.frexp(top)[1] + 126 - 7, 0, 254)      # (no block of zeros here)
            assert np.array_equal(t[name + "_scale"].cpu().numpy(), byte.astype(np.uint8))
            s, gap = lattice(abs(y.astype(np.float64)), byte)
            z = abs(y.astype(np.float64)) / s / gap
            steps = np.where(z < 8, np.floor((z.astype(f) + (random16 / 65536.0).astype(f)).astype(np.float64)), np.floor(z + random16 / 65536.0))
            code = steps * gap
            if name == "v":
                code = np.where((y > 0) & (code == 0), 2.0 ** -9, code)
            assert np.array_equal(decode(t[name], t[name + "_scale"]), np.copysign(code * s, y.astype(np.float64)))


def test_rounding_of_8_bit_states_has_no_bias(rn):
    """The mean over many steps of what a value is stored as is the value: standard error of N draws of at most a code's distance."""
    import torch
    n, reps = 128 * 64, 64
    t = eight(rn, n, 5, torch.float32)
    start = {k: x.clone() for k, x in t.items()}
    sums, want = {"m": np.zeros(n), "v": np.zeros(n)}, None
    plan = rn.AdamwTensors([t])
    for seed in range(reps):
        for k in t:
            t[k].copy_(start[k])
        rn.rnnd_adamw(plan, 9, seed=seed, **HYPER)
        for k in sums:
            sums[k] += decode(t[k], t[k + "_scale"])
        if want is None:
            r = decode(start["v"], start["v_scale"])
            _, m1, v1, _, _, _ = formula(np64(start["param"]), np64(start["grad"]), decode(start["m"], start["m_scale"]), r * r, 9, HYPER)
            want = {"m": m1, "v": np.sqrt(v1)}
    for k in sums:
        s, gap = lattice(abs(want[k]), t[k + "_scale"].cpu().numpy())
        off = (sums[k] / reps - want[k]) / (s * gap)       # in codes: deviation of one draw at most 1/2
        small = abs(want[k]) / s < 2.0 ** -9               # (roots that may not become zero)
        assert abs(off[~small].mean()) <= 5 * 0.5 / math.sqrt(reps * (~small).sum())


def test_a_second_moment_follows_a_vanishing_gradient(rn):
    """beta2 = 0.999 moves a root by 0.05 % a step: 3,000 steps without a gradient take it down by e^-1.5, not by nothing."""
    import torch
    n = 128 * 8
    t = eight(rn, n, 3, torch.float32, zero=True)
    t["grad"].fill_(1.0)
    plan = rn.AdamwTensors([t])
    h = dict(lr=1e-3, beta2=0.999)
    for step in range(1, 200):
        rn.rnnd_adamw(plan, step, seed=1, **h)
    start = decode(t["v"], t["v_scale"]).mean()
    # (rounding a root adds its variance to v: a code's distance, 0.09 of the root, times the 1 / 2t that step t moves it)
    assert abs(start - math.sqrt(1 - 0.999 ** 199)) < 0.25 * start
    t["grad"].zero_()
    for step in range(200, 3200):
        rn.rnnd_adamw(plan, step, seed=1, **h)
    assert abs(decode(t["v"], t["v_scale"]).mean() / start - 0.999 ** 1500) < 0.05


def test_zero_blocks_and_blocks_that_are_not_finite(rn):
    import torch
    n = 128 * 5
    t = eight(rn, n, 3, torch.float32, zero=True)
    t["grad"].zero_()
    t["grad"][200] = float("inf")
    t["grad"][300] = float("nan")
    t["grad"][400] = 1e-15
    p = t["param"].clone()
    plan = rn.AdamwTensors([t])
    rn.rnnd_adamw(plan, 1, lr=1e-3)
    assert torch.equal(t["param"][:128], p[:128]) and (t["m"][:128] == 0).all() and (t["v"][:128] == 0).all()
    assert t["m_scale"].tolist()[1:3] == [255, 255] and t["v_scale"].tolist()[1:3] == [255, 255]
    assert t["m_scale"][0] == 0 and t["m_scale"][3] < 255 and t["v"][400] > 0 and t["m"][400] > 0
    assert int((~t["param"].isfinite()).sum()) == 2
    rn.rnnd_adamw(plan, 2, lr=1e-3)         # what a lost block holds is not a number from then on
    assert t["param"][128:384].isnan().all() and t["param"][:128].isfinite().all() and t["param"][384:].isfinite().all()


def test_nothing_around_the_tensors_is_written(rn):
    import torch
    for bits in (8, 32):
        for n in (1, 5, 8, 130, 2049):
            flat = {k: torch.full((n + 64,), 3, dtype=d, device="cuda") for k, d in
                    dict(param=torch.float32, grad=torch.float32, m=torch.uint8 if bits == 8 else torch.float32,
                         v=torch.uint8 if bits == 8 else torch.float32, copy=torch.bfloat16).items()}
            t = {k: x[32:32 + n] for k, x in flat.items()}
            if bits == 8:
                blocks = -(-n // 128)
                for k in ("m_scale", "v_scale"):
                    flat[k] = torch.full((blocks + 64,), 100, dtype=torch.uint8, device="cuda")
                    t[k] = flat[k][32:32 + blocks]
            before = {k: x.clone() for k, x in flat.items()}
            rn.rnnd_adamw(rn.AdamwTensors([t]), 1, lr=1e-3)
            for k, x in flat.items():
                m = t[k].numel()
                assert torch.equal(x[:32], before[k][:32]) and torch.equal(x[32 + m:], before[k][32 + m:]), (k, n)
            assert not torch.equal(flat["param"], before["param"])


def test_states_of_both_kinds_in_one_call_and_empty_tensors(rn):
    import torch
    a = eight(rn, 1000, 1, torch.float32)
    b = dict(param=normal(300, 2), grad=normal(300, 3), m=normal(300, 4), v=normal(300, 5).square())
    c = {k: torch.empty(0, device="cuda") for k in ("param", "grad", "m", "v")}
    alone_a, alone_b = ({k: x.clone() for k, x in t.items()} for t in (a, b))
    rn.rnnd_adamw(rn.AdamwTensors([c, dict(a, counter=0), b, c]), 4, lr=1e-2, seed=9)
    rn.rnnd_adamw(rn.AdamwTensors([dict(alone_a, counter=0)]), 4, lr=1e-2, seed=9)
    rn.rnnd_adamw(rn.AdamwTensors([alone_b]), 4, lr=1e-2, seed=9)
    for t, s in ((a, alone_a), (b, alone_b)):
        for k in t:
            assert torch.equal(t[k], s[k]), k


def test_refusals_of_the_binding(rn):
    import torch
    x = torch.zeros(256, device="cuda")
    b = torch.zeros(256, dtype=torch.uint8, device="cuda")
    s = torch.zeros(2, dtype=torch.uint8, device="cuda")
    ok = dict(param=x, grad=x.clone(), m=x.clone(), v=x.clone())
    bad = [dict(ok, param=x.half()), dict(ok, grad=x[:255]), dict(ok, m=x[::2]), dict(ok, v=x.double()), dict(ok, m=b), dict(ok, m_scale=s, v_scale=s),
           dict(ok, m=b, v=b.clone()), dict(ok, m=b, v=b.clone(), m_scale=s), dict(ok, m=b, v=b.clone(), m_scale=s, v_scale=s[:1]),
           dict(ok, copy=x), dict(ok, copy=x.half()[:10]), dict(ok, grad=x.cpu())]
    for t in bad:
        with pytest.raises(ValueError):
            rn.AdamwTensors([t])
    rn.AdamwTensors([ok])
    with pytest.raises(rn.RnndError) as e:
        rn.rnnd_adamw(rn.AdamwTensors([ok]), 0, lr=1e-3)
    assert e.value.status == -3
    rn.rnnd_adamw(rn.AdamwTensors([]), 1, lr=1e-3)
