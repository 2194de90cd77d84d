"""Lookups and their gradient against the definitions in double precision."""
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


def half_step(dtype):
    """Largest relative rounding error, and the absolute one below the normal numbers."""
    import torch
    info = torch.finfo(dtype)
    return info.eps / 2, info.smallest_normal * info.eps / 2


def rows(n, d, dtype, seed, offset=0):
    """n x d normal values in device memory; offset: elements by which the address misses its alignment."""
    import torch
    g = torch.Generator(device="cuda").manual_seed(seed)
    flat = torch.randn(n * d + offset, device="cuda", generator=g).to(dtype)
    return flat[offset:].view(n, d)


def check_lookup(rn, table, ids, scale, out_dtype, out=None):
    import torch
    V = table.shape[0]
    got = rn.rnnd_embed(table, torch.from_numpy(ids).cuda(), scale=scale, out_dtype=None if out is not None else out_dtype, out=out)
    assert got.dtype == out_dtype and got.shape == (len(ids), table.shape[1])
    t = table.double().cpu().numpy()
    inside = (ids >= 0) & (ids < V)
    want = np.where(inside[:, None], t[np.where(inside, ids, 0)] * np.float64(np.float32(scale)), 0.0)
    rel, tiny = half_step(out_dtype)
    off = np.abs(got.double().cpu().numpy() - want)
    assert (off <= np.abs(want) * (rel + 2.0 ** -24) * 1.001 + tiny + 2.0 ** -149).all(), off.max()
    assert (got[torch.from_numpy(~inside).cuda()] == 0).all()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("out_dtype", TYPES)
@pytest.mark.parametrize("n,d,V", [(1, 96, 100), (3, 1, 1), (257, 7, 1000), (64, 100, 5000), (1000, 768, 3000), (5, 4099, 20), (2500, 34, 60)])
def test_lookup(rn, dtype, out_dtype, n, d, V):
    import torch
    g = np.random.Generator(np.random.PCG64(n * 1000 + d))
    ids = g.integers(-2, V + 2, size=n).astype(np.int32)
    check_lookup(rn, rows(V, d, getattr(torch, dtype), d), ids, float(np.sqrt(d)), getattr(torch, out_dtype))


@pytest.mark.parametrize("offset", [0, 1, 2, 3, 4])
@pytest.mark.parametrize("d", [8, 16, 20, 24])
def test_lookup_at_any_alignment(rn, offset, d):
    import torch
    ids = np.array([5, 0, -1, 49, 50, 2**31 - 1, -2**31, 7, 7], np.int32)
    for dtype in (torch.float32, torch.bfloat16):
        out = rows(len(ids), d, torch.float16, 9, offset=5 - offset)
        check_lookup(rn, rows(50, d, dtype, 3, offset=offset), ids, 0.37, torch.float16, out=out)


def test_lookup_without_a_scale_moves_the_bits(rn):
    import torch
    table = rows(1000, 96, torch.bfloat16, 4)
    table[3, 5], table[4, 0], table[5, 1] = float("inf"), float("nan"), -0.0
    ids = torch.randint(0, 1000, (5000,), device="cuda", dtype=torch.int32)
    ids[:3] = torch.tensor([3, 4, 5])
    got = rn.rnnd_embed(table, ids)
    want = table[ids.long()]
    same = (got.view(torch.int16) == want.view(torch.int16)) | (got.isnan() & want.isnan())
    assert same.all()


def test_lookup_of_nothing(rn):
    import torch
    table = rows(10, 8, torch.float32, 1)
    assert rn.rnnd_embed(table, torch.empty(0, dtype=torch.int32, device="cuda")).shape == (0, 8)


def test_rows_beyond_four_billion_elements(rn):
    import torch
    V, d = 9_000_000, 512          # 4.6e9 elements of 2 bytes
    table = torch.zeros(V, d, device="cuda", dtype=torch.bfloat16)
    ids = np.array([V - 1, 0, 8_388_609, V, 8_388_607], np.int32)
    for i in ids:
        if i < V:
            table[int(i)] = float(int(i) % 251)
    got = rn.rnnd_embed(table, torch.from_numpy(ids).cuda(), out_dtype=torch.float32)
    want = [float(int(i) % 251) if i < V else 0.0 for i in ids]
    assert got[:, 0].tolist() == want and got[:, -1].tolist() == want
    # and the gradient of such a table, added to in place
    dout = torch.ones(len(ids), d, device="cuda", dtype=torch.bfloat16)
    before = table[ids[0]].float()
    rn.rnnd_embed_grad(dout, torch.from_numpy(ids).cuda(), V, grad=table, accumulate=True)
    assert (table[int(ids[0])].float() == before + 1).all() and (table[int(ids[2])].float() == float(8_388_609 % 251) + 1).all()


def check_gradient(rn, dout, ids, V, scale, grad_dtype, accumulate, grad=None):
    import torch
    n, d = dout.shape
    start = None
    if accumulate:
        start = grad.double().cpu().numpy()
    got = rn.rnnd_embed_grad(dout, torch.from_numpy(ids).cuda(), V, scale=scale, grad_dtype=None if grad is not None else grad_dtype,
                             grad=grad, accumulate=accumulate)
    x = dout.double().cpu().numpy()
    inside = (ids >= 0) & (ids < V)
    want, size = np.zeros((V, d)), np.zeros((V, d))
    np.add.at(want, ids[inside], x[inside])
    np.add.at(size, ids[inside], np.abs(x[inside]))
    count = np.bincount(ids[inside], minlength=V)[:, None]
    want, size = want * np.float64(np.float32(scale)), size * abs(scale)
    if accumulate:
        want, size = want + start, size + np.abs(start)
    rel, tiny = half_step(grad_dtype)
    # count additions, one product and one more addition in float32, then the rounding
    bound = size * (count + 3) * 2.0 ** -24 + np.abs(want) * rel * 1.001 + tiny + 2.0 ** -149
    off = np.abs(got.double().cpu().numpy() - want)
    assert (off <= bound).all(), (off - bound).max()
    untouched = (count == 0)[:, 0]
    now = got.double().cpu().numpy()
    assert (now[untouched] == (start[untouched] if accumulate else 0.0)).all()
    return got


def zipf(n, V, seed):
    g = np.random.Generator(np.random.PCG64(seed))
    ids = (np.exp(g.random(n) * np.log(V + 1)) - 1).astype(np.int32)
    ids[g.random(n) < 0.03] = -1
    ids[g.random(n) < 0.01] = V
    return ids


@pytest.mark.parametrize("dtype,grad_dtype", [("float32", "float32"), ("bfloat16", "float32"), ("float16", "float16"),
                                              ("bfloat16", "bfloat16"), ("float32", "bfloat16"), ("float16", "bfloat16")])
@pytest.mark.parametrize("n,d,V", [(1, 96, 50), (2, 1, 1), (63, 3, 5), (1000, 32, 5000), (4096, 100, 900), (4097, 8, 1023),
                                   (20_000, 129, 1024), (9_000, 768, 70_000), (70_001, 20, 3)])
@pytest.mark.parametrize("accumulate", [False, True])
def test_gradient(rn, dtype, grad_dtype, n, d, V, accumulate):
    import torch
    dout = rows(n, d, getattr(torch, dtype), n + d)
    grad = rows(V, d, getattr(torch, grad_dtype), 7) if accumulate else None
    check_gradient(rn, dout, zipf(n, V, n), V, 1.25, getattr(torch, grad_dtype), accumulate, grad)


def runs(lengths, V, seed):
    """ids whose sorted order holds runs of the given lengths, in a random order of the tokens."""
    g = np.random.Generator(np.random.PCG64(seed))
    names = np.sort(g.permutation(V)[:len(lengths)])
    return g.permutation(np.repeat(names, lengths)).astype(np.int32)


@pytest.mark.parametrize("first", range(0, 17, 4))
@pytest.mark.parametrize("d", [5, 96, 600])
def test_gradient_of_ids_that_end_around_the_pieces_of_the_sum(rn, first, d):
    """Runs of one id that end just before, at and behind one and two chunks of 16, at every kind of offset."""
    import torch
    lengths = [first + 1] + [k for c in (16, 32, 48) for k in (c - 1, c, c + 1)] + [1, 2, 3, 16, 16, 32, 17, 15, 33, 100, 64, 5, 400]
    ids = runs(lengths, 200, first)
    check_gradient(rn, rows(len(ids), d, torch.float32, d), ids, 200, 1.0, torch.float32, False)
    check_gradient(rn, rows(len(ids), d, torch.bfloat16, d), ids, 200, 1.0, torch.float32, True, rows(200, d, torch.float32, 1))


@pytest.mark.parametrize("dtype,grad_dtype", [("float32", "float32"), ("bfloat16", "float16")])
@pytest.mark.parametrize("n,d,V", [(4096, 2050, 7), (4096, 33, 1), (3001, 1100, 3), (4095, 8, 20_000), (9, 768, 9_001), (300, 5, 70_000), (4096, 24, 4096)])
@pytest.mark.parametrize("accumulate", [False, True])
def test_gradient_of_few_tokens(rn, dtype, grad_dtype, n, d, V, accumulate):
    """Ids that many tokens share, rows of more pieces than blocks take at once, and borders of the blocks that clear."""
    import torch
    dout = rows(n, d, getattr(torch, dtype), 5)
    grad = rows(V, d, getattr(torch, grad_dtype), 6) if accumulate else None
    for ids in (zipf(n, V, 3), np.full(n, V - 1, np.int32), np.arange(n, dtype=np.int32)[::-1].copy() * 5 - 3):
        check_gradient(rn, dout, ids.astype(np.int32), V, 1.5, getattr(torch, grad_dtype), accumulate, None if grad is None else grad.clone())


@pytest.mark.parametrize("first", range(0, 9, 2))
@pytest.mark.parametrize("d", [5, 96, 600])
def test_gradient_of_sorted_ids_that_end_around_the_pieces_of_the_sum(rn, first, d):
    """The same runs among enough other ids that the tokens are sorted: just before, at and behind chunks of 8 and 16."""
    import torch
    lengths = [first + 1] + [k for c in (8, 16, 24, 32, 48) for k in (c - 1, c, c + 1)] + [1, 2, 3, 8, 8, 16, 32, 17, 33, 100, 64, 5, 400] + [1] * 4_200
    ids = runs(lengths, 5_000, first)
    check_gradient(rn, rows(len(ids), d, torch.float32, d), ids, 5_000, 1.0, torch.float32, False)
    check_gradient(rn, rows(len(ids), d, torch.bfloat16, d), ids, 5_000, 1.0, torch.float32, True, rows(5_000, d, torch.float32, 1))


def test_gradient_of_long_calls(rn):
    """More tokens than the chunks of 128 need; a few ids hold most of them."""
    import torch
    n, V, d = 700_001, 2_000, 8
    lengths = [250_000, 127, 128, 129, 255, 256, 257, 385, 1, 100_000]
    ids = np.concatenate([runs(lengths, V, 3), zipf(n - sum(lengths), V, 4)])
    check_gradient(rn, rows(n, d, torch.float32, 5), ids, V, 0.5, torch.float32, False)


@pytest.mark.parametrize("V", [1, 255, 256, 1023, 1024, 5000, 1_048_575, 1_048_576, 3_000_000])
def test_every_number_of_sorting_passes(rn, V):
    import torch
    n = 6_000
    g = np.random.Generator(np.random.PCG64(V))
    ids = g.integers(0, V, size=n).astype(np.int32)
    ids[:50] = V - 1
    ids[50:60] = -5
    check_gradient(rn, rows(n, 4, torch.float32, 2), g.permutation(ids), V, 1.0, torch.float32, False)


def test_gradient_where_no_id_is_a_row_and_of_nothing(rn):
    import torch
    for n in (0, 1, 5000):
        ids = torch.full((n,), -1, dtype=torch.int32, device="cuda")
        dout = torch.full((n, 12), float("nan"), device="cuda")
        assert (rn.rnnd_embed_grad(dout, ids, 40) == 0).all()
        grad = rows(40, 12, torch.float32, 3)
        before = grad.clone()
        rn.rnnd_embed_grad(dout, ids, 40, grad=grad, accumulate=True)
        assert torch.equal(grad, before)


@pytest.mark.parametrize("offset", [0, 1, 2, 3])
def test_gradient_at_any_alignment(rn, offset):
    import torch
    for d in (8, 12, 33):
        check_gradient(rn, rows(300, d, torch.float32, 1, offset), zipf(300, 40, d), 40, 1.0, torch.float32, False,
                       rows(40, d, torch.float32, 2, 3 - offset))
        check_gradient(rn, rows(300, d, torch.bfloat16, 1, offset), zipf(300, 40, d), 40, 1.0, torch.bfloat16, True,
                       rows(40, d, torch.bfloat16, 2, 3 - offset))


def test_the_same_call_gives_the_same_bits(rn):
    import torch
    ids = torch.from_numpy(zipf(50_000, 3_000, 8)).cuda()
    dout = rows(50_000, 96, torch.float32, 8)
    first = rn.rnnd_embed_grad(dout, ids, 3_000)
    for _ in range(3):
        assert torch.equal(rn.rnnd_embed_grad(dout, ids, 3_000), first)


def test_a_workspace_of_the_callers(rn):
    import torch
    ids = torch.from_numpy(zipf(5_000, 300, 8)).cuda()
    dout = rows(5_000, 16, torch.float32, 8)
    want = rn.rnnd_embed_grad(dout, ids, 300)
    need = rn.rnnd_embed_grad_workspace(5_000, 16, 300)
    block = torch.full((need + 64,), 0xA5, dtype=torch.uint8, device="cuda")
    assert torch.equal(rn.rnnd_embed_grad(dout, ids, 300, workspace=block[:need]), want)
    assert (block[need:] == 0xA5).all()
    with pytest.raises(rn.RnndError) as e:
        rn.rnnd_embed_grad(dout, ids, 300, workspace=block[:need - 1])
    assert e.value.status == -7


def test_a_row_that_is_not_finite_stays_in_its_row(rn):
    import torch
    ids = torch.tensor([1, 2, 1, 3, 2], dtype=torch.int32, device="cuda")
    dout = torch.ones(5, 8, device="cuda")
    dout[3, 2] = float("inf")
    dout[1, 4] = float("nan")
    g = rn.rnnd_embed_grad(dout, ids, 5)
    assert g[3, 2] == float("inf") and g[2, 4].isnan() and g[1].tolist() == [2.0] * 8
    assert int((~g.isfinite()).sum()) == 2


def test_refusals_of_the_binding(rn):
    import torch
    table = rows(10, 8, torch.float32, 1)
    ids = torch.zeros(3, dtype=torch.int32, device="cuda")
    for call in (lambda: rn.rnnd_embed(table.t(), ids), lambda: rn.rnnd_embed(table, ids.long()), lambda: rn.rnnd_embed(table.to(torch.uint8), ids),
                 lambda: rn.rnnd_embed(table, ids, out=torch.empty(3, 9, device="cuda")), lambda: rn.rnnd_embed(table, ids.cpu()),
                 lambda: rn.rnnd_embed_grad(table[:3], ids, 5, accumulate=True), lambda: rn.rnnd_embed_grad(table, ids, 5),
                 lambda: rn.rnnd_embed_grad(table[:3], ids, 5, grad=torch.empty(4, 8, device="cuda")),
                 lambda: rn.rnnd_embed(table, torch.zeros(6, dtype=torch.int32, device="cuda")[::2])):
        with pytest.raises(ValueError):
            call()
