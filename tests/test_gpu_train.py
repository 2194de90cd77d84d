"""The training calls together: on streams of their own, in a captured graph, and as one training step."""
import pytest

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def rn():
    import torch
    assert torch.cuda.is_available(), "these tests need the MI355X"
    import paper_2310_20419_amd as m
    m.load_library()
    return m


def setup(seed, V=3000, d=48, B=200, negatives=400, bits=8):
    import torch
    g = torch.Generator(device="cuda").manual_seed(seed)
    table = torch.randn(V, d, device="cuda", generator=g) / d ** 0.5
    s = dict(V=V, d=d, table=table, rows=table.bfloat16(), grad=torch.zeros(V, d, device="cuda"))
    byte = dict(dtype=torch.uint8, device="cuda")
    if bits == 8:
        state = dict(m=torch.zeros(V * d, **byte), v=torch.zeros(V * d, **byte), m_scale=torch.zeros(-(-V * d // 128), **byte),
                     v_scale=torch.zeros(-(-V * d // 128), **byte))
    else:
        state = dict(m=torch.zeros(V * d, device="cuda"), v=torch.zeros(V * d, device="cuda"))
    s["state"] = state
    s["query"] = torch.randint(0, V, (B,), device="cuda", generator=g, dtype=torch.int32)
    s["keys"] = torch.randint(-1, V, (B + negatives,), device="cuda", generator=g, dtype=torch.int32)
    s["target"] = torch.arange(B, device="cuda", dtype=torch.int32)
    s["weight"] = torch.full((B,), 1.0 / B, device="cuda")
    return s


def step(rn, s, plan, number, stream=None):
    import torch
    q = rn.rnnd_embed(s["rows"], s["query"], stream=stream)
    k = rn.rnnd_embed(s["rows"], s["keys"], stream=stream)
    loss, dq, dk = rn.rnnd_contrast(q, k, s["target"], 5.0, query_ids=s["query"], key_ids=s["keys"], row_weight=s["weight"], stream=stream)
    rn.rnnd_embed_grad(dq, s["query"], s["V"], grad=s["grad"], stream=stream)
    rn.rnnd_embed_grad(dk, s["keys"], s["V"], grad=s["grad"], accumulate=True, stream=stream)
    rn.rnnd_adamw(plan, number, lr=1e-2, seed=5, stream=stream)
    return loss


def plan_of(rn, s):
    return rn.AdamwTensors([dict(param=s["table"], grad=s["grad"], copy=s["rows"], **s["state"])])


@pytest.mark.parametrize("bits", [8, 32])
def test_a_step_lowers_the_loss_of_its_batch(rn, bits):
    s = setup(1, bits=bits)
    plan = plan_of(rn, s)
    losses = [step(rn, s, plan, i + 1).mean().item() for i in range(30)]
    assert losses[-1] < 0.2 * losses[0] and all(b < a + 0.05 for a, b in zip(losses, losses[1:]))


def test_a_stream_of_the_callers_gives_the_same_bits(rn):
    import torch
    a, b = setup(2), setup(2)
    pa, pb = plan_of(rn, a), plan_of(rn, b)
    la = [step(rn, a, pa, i + 1) for i in range(5)]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    lb = [step(rn, b, pb, i + 1, stream=side) for i in range(5)]
    # memory that the current stream frees and takes meanwhile must not be what the other stream still works in
    junk = [torch.full((1 << 20,), float("nan"), device="cuda") for _ in range(8)]
    side.synchronize()
    for x, y in zip(la, lb):
        assert torch.equal(x, y)
    assert torch.equal(a["table"], b["table"]) and torch.equal(a["rows"], b["rows"]) and len(junk) == 8


def test_a_captured_step_replays_as_the_eager_one(rn):
    """Several replays, with eager work and synchronizations in between; the graph and the eager steps start from the same state."""
    import torch
    a, b = setup(3), setup(3)
    pa, pb = plan_of(rn, a), plan_of(rn, b)
    step(rn, a, pa, 7)
    step(rn, b, pb, 7)          # warms the allocator up, and gives both the same state
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        captured = step(rn, b, pb, 7)
    for i in range(5):
        want = step(rn, a, pa, 7)
        for x in (b["query"], a["query"]):
            assert x.numel() == 200
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(captured, want), i
        assert torch.equal(a["table"], b["table"]) and torch.equal(a["rows"], b["rows"]) and torch.equal(a["grad"], b["grad"]), i
        new = torch.randint(0, 3000, (200,), device="cuda", dtype=torch.int32)
        a["query"].copy_(new)
        b["query"].copy_(new)
