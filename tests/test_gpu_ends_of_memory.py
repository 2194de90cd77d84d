"""Inputs that end where their memory ends: nothing behind the last row, id or bias is read, however far the work is padded."""
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


def at_the_end(x):
    """A copy in the last bytes of an allocation of its own (16 MB: whole 2 MB pieces, which are not shared with smaller tensors)."""
    import torch
    room = torch.zeros(16 << 20, dtype=torch.uint8, device="cuda")
    n = x.numel() * x.element_size()
    room[room.numel() - n:] = x.contiguous().flatten().view(torch.uint8)
    return room[room.numel() - n:].view(x.dtype).view(x.shape)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("B,M,d", [(130, 260, 257), (3, 50, 33), (40, 400, 64), (8, 1, 4), (1100, 257, 64)])
def test_training_and_answers(rn, B, M, d, dtype):
    import torch
    g = torch.Generator(device="cuda").manual_seed(B + M)
    t = getattr(torch, dtype)

    def some(*shape):
        return torch.randn(*shape, device="cuda", generator=g)

    def ids(high, *shape):
        return torch.randint(0, high, shape, device="cuda", generator=g, dtype=torch.int32)
    x = dict(Q=(some(B, d) / d ** 0.5).to(t), K=(some(M, d) / d ** 0.5).to(t), target=ids(M, B), query_ids=ids(2 * M, B), key_ids=ids(2 * M, M),
             key_bias=some(M), row_weight=some(B), teacher_ids=ids(M, B, 7), teacher_logits=some(B, 7) - 3)

    def calls(x):
        names = {n: x[n] for n in ("query_ids", "key_ids", "key_bias")}
        return (rn.rnnd_contrast(x["Q"], x["K"], x["target"], 3.0, row_weight=x["row_weight"], **names)
                + rn.rnnd_distill(x["Q"], x["K"], x["teacher_ids"], x["teacher_logits"], 3.0, tail=True, row_weight=x["row_weight"], **names)
                + rn.rnnd_logprob(x["Q"], x["K"], 3.0, target=x["target"], alternatives=9, **names)
                + rn.rnnd_logprob(x["Q"][-2:], x["K"], 3.0, target=x["target"][-2:], alternatives=9, query_ids=x["query_ids"][-2:],
                                  key_ids=x["key_ids"], key_bias=x["key_bias"]))
    want = calls(x)
    torch.cuda.synchronize()
    torch.cuda.empty_cache()
    got = calls({n: at_the_end(v) for n, v in x.items()})
    torch.cuda.synchronize()
    for a, b in zip(got, want):
        assert torch.equal(a, b)
