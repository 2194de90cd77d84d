"""Keys that are the target of many queries: their terms in float32, segment by segment, and without a chain as long as the queries are many."""
import numpy as np
import pytest

from test_gpu_contrast import call, case, check

pytestmark = pytest.mark.gpu

TYPES = ["float32", "float16", "bfloat16"]


@pytest.fixture(scope="module")
def rn():
    import torch
    assert torch.cuda.is_available(), "these tests need the MI355X"
    import paper_2310_20419_amd as m
    m.load_library()
    return m


def targets(kind, B, M, g):
    if kind == "one":
        return np.full(B, M // 2)
    if kind == "a tenth on one":
        return np.where(g.random(B) < 0.1, M // 2, g.integers(0, M, size=B))
    if kind == "eights and nines":          # on both sides of how many are taken one after the other
        return np.minimum(np.arange(B) * 2 // 17, M - 1)
    if kind == "64s and 65s":               # on both sides of what one wavefront takes of a segment
        return np.minimum(np.arange(B) * 2 // 129, M - 1)
    return g.integers(0, min(M, 16), size=B)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("kind", ["one", "a tenth on one", "eights and nines", "64s and 65s", "sixteen"])
@pytest.mark.parametrize("B,M,d", [(1_023, 200, 24), (1_025, 140, 7), (2_300, 300, 300), (3_000, 20, 33)])
def test_targets_of_many_queries(rn, dtype, kind, B, M, d):
    import torch
    g = np.random.Generator(np.random.PCG64(B + d))
    c = case(B, M, d, dtype, B + M)
    c["target"] = targets(kind, B, M, g).astype(np.int32)
    c["target"][g.random(B) < 0.05] = -1
    c["target"][g.random(B) < 0.02] = M
    c["key_ids"][M // 2] = 3 * M
    c["key_bias"][M // 2] = 0.5
    check(rn, c, 4.0)
    first = call(rn, c, 4.0)
    need = rn.rnnd_contrast_workspace(B, M, d, {"float32": 1, "float16": 2, "bfloat16": 3}[dtype])
    for fill in (0xFF, 0x7F):
        block = torch.full((need + 256,), fill, dtype=torch.uint8, device="cuda")
        for a, b in zip(call(rn, c, 4.0, workspace=block[:need]), first):
            assert torch.equal(a, b)
        assert (block[need:] == fill).all()
    for k in ("Q", "K"):        # rows that are not aligned
        flat = torch.empty(c[k].numel() + 1, dtype=c[k].dtype, device="cuda")
        flat[1:] = c[k].reshape(-1)
        c[k] = flat[1:].view(c[k].shape)
    for a, b in zip(call(rn, c, 4.0), first):
        assert torch.equal(a, b)


def test_queries_on_one_key_are_no_chain(rn):
    """A wavefront that looked for every query of a key and waited for it made a call with one target for all 15 times as long as with one for each
    (8,192 queries, 16,384 keys of 768 coordinates)."""
    import torch
    B, M, d = 4_096, 8_192, 768
    g = torch.Generator(device="cuda").manual_seed(3)
    Q, K = ((torch.randn(n, d, device="cuda", generator=g) / d ** 0.5).bfloat16() for n in (B, M))

    def us(target):
        work = torch.empty(rn.rnnd_contrast_workspace(B, M, d, rn.RNND_BF16), dtype=torch.uint8, device="cuda")
        best = float("inf")
        for _ in range(4):
            a, b = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
            a.record()
            for _ in range(5):
                rn.rnnd_contrast(Q, K, target, 5.0, workspace=work)
            b.record()
            b.synchronize()
            best = min(best, a.elapsed_time(b) / 5 * 1000)
        return best
    each = us(torch.arange(B, device="cuda", dtype=torch.int32))
    assert us(torch.full((B,), 7, device="cuda", dtype=torch.int32)) < 4 * each
    assert us(torch.arange(B, device="cuda", dtype=torch.int32) % 16) < 2 * each
