"""Gradients of few tokens where one id has many of them: what the blocks of its tokens share, and that it takes no longer than sorting them."""
import numpy as np
import pytest

from test_gpu_embed import check_gradient, rows

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def rn():
    import torch
    assert torch.cuda.is_available(), "these tests need the MI355X"
    import paper_2310_20419_amd as m
    m.load_library()
    return m


@pytest.mark.parametrize("dtype,grad_dtype", [("float32", "float32"), ("bfloat16", "float32"), ("float16", "bfloat16")])
@pytest.mark.parametrize("lengths", [[1, 2, 3, 5, 40], [255, 256, 257, 1], [1025], [1024, 3], [4096], [2000, 2000, 90, 6]])
@pytest.mark.parametrize("d", [1, 33, 96, 768, 2200])
def test_blocks_of_one_id_share_its_row(rn, dtype, grad_dtype, lengths, d):
    """Fewer tokens than slabs, as many, and more; lists on both sides of where the groups of lanes become smaller."""
    import torch
    g = np.random.Generator(np.random.PCG64(sum(lengths) + d))
    V = 50
    ids = np.repeat(np.sort(g.permutation(V)[:len(lengths)]), lengths).astype(np.int32)
    ids = g.permutation(np.concatenate([ids, np.full(min(7, 4096 - len(ids)), -1, np.int32)]))
    dout = rows(len(ids), d, getattr(torch, dtype), d)
    first = check_gradient(rn, dout, ids, V, 1.25, getattr(torch, grad_dtype), False)
    grad = rows(V, d, getattr(torch, grad_dtype), 7)
    check_gradient(rn, dout, ids, V, 1.25, getattr(torch, grad_dtype), True, grad.clone())
    assert torch.equal(rn.rnnd_embed_grad(dout, torch.from_numpy(ids).cuda(), V, scale=1.25, grad_dtype=getattr(torch, grad_dtype)), first)


@pytest.mark.parametrize("d,V", [(768, 2), (4096, 4)])
def test_no_cliff_before_the_tokens_are_sorted(rn, d, V):
    """4,096 tokens are summed without a sort, 4,097 with one, which shares a popular id among chunks.  One block for an id took 13 to 90
    times as long as that; several blocks take less."""
    import torch

    def us(n):
        dout = torch.ones(n, d, device="cuda")
        ids = torch.zeros(n, dtype=torch.int32, device="cuda")
        grad = torch.empty(V, d, device="cuda")
        work = torch.empty(max(256, rn.rnnd_embed_grad_workspace(n, d, V)), dtype=torch.uint8, device="cuda")
        best = float("inf")
        for _ in range(5):
            a, b = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
            a.record()
            for _ in range(20):
                rn.rnnd_embed_grad(dout, ids, V, grad=grad, workspace=work)
            b.record()
            b.synchronize()
            best = min(best, a.elapsed_time(b) / 20 * 1000)
        assert (grad[0] == n).all() and (grad[1:] == 0).all()
        return best
    assert us(4_096) < 3 * us(4_097)
