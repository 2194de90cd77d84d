"""A gradient's sums are taken in an order that types, sizes and ids decide: where the rows lie in memory changes no bit."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def rn():
    import torch
    assert torch.cuda.is_available(), "these tests need the MI355X"
    import paper_2310_20419_amd as m
    m.load_library()
    return m


@pytest.mark.parametrize("dtype,grad_dtype", [("float32", "float32"), ("bfloat16", "float32"), ("float16", "float16")])
@pytest.mark.parametrize("n,V,d", [(1_000, 1, 32), (1_000, 40, 96), (4_096, 3, 768), (6_000, 2, 32), (20_000, 50, 24), (9_000, 3, 520)])
def test_rows_anywhere_in_memory_give_the_same_bits(rn, dtype, grad_dtype, n, V, d):
    """Few tokens and sorted ones, ids that hold most of them."""
    import torch
    g = torch.Generator(device="cuda").manual_seed(n + d)
    dout = torch.randn(n, d, device="cuda", generator=g).to(getattr(torch, dtype))
    ids = torch.randint(0, 2 * V, (n,), device="cuda", generator=g, dtype=torch.int32) % (V + 1) - 1 + (V == 1)
    start = torch.randn(V, d, device="cuda", generator=g).to(getattr(torch, grad_dtype))

    def at(x, offset):
        flat = torch.empty(x.numel() + 8, dtype=x.dtype, device="cuda")
        y = flat[offset:offset + x.numel()].view(x.shape)
        return y.copy_(x)

    want = rn.rnnd_embed_grad(dout, ids, V, grad=at(start, 0))
    added = rn.rnnd_embed_grad(dout, ids, V, grad=at(start, 0), accumulate=True)
    for a, b in ((1, 0), (0, 1), (2, 2), (3, 1), (4, 6)):
        assert torch.equal(rn.rnnd_embed_grad(at(dout, a), ids, V, grad=at(start, b)), want), (a, b)
        assert torch.equal(rn.rnnd_embed_grad(at(dout, a), ids, V, grad=at(start, b), accumulate=True), added), (a, b)
