"""Calls of more than 2^24 workgroups: a launch holds fewer than 2^32 threads."""
import pytest

pytestmark = pytest.mark.gpu


@pytest.fixture
def rn():
    import torch
    assert torch.cuda.is_available(), "these tests need the MI355X"
    import paper_2310_20419_amd as m
    m.load_library()
    torch.cuda.empty_cache()
    yield m
    torch.cuda.empty_cache()        # tens of GB


def test_a_lookup_of_18_billion_coordinates(rn):
    """186 million rows of 97 coordinates, one coordinate an access: 36 GB."""
    import torch
    n, d, V = 186_000_000, 97, 1_000
    table = torch.randn(V, d, device="cuda").bfloat16()
    ids = torch.randint(-1, V, (n,), device="cuda", dtype=torch.int32)
    out = torch.full((n, d), float("nan"), device="cuda", dtype=torch.bfloat16)
    rn.rnnd_embed(table, ids, out=out)
    step = 3_000_017
    for first in list(range(0, n, 31 * step)) + [n - 40_000]:
        some = ids[first:first + 40_000].long()
        want = torch.where((some >= 0)[:, None], table[some.clamp(min=0)], 0.0)
        assert torch.equal(out[first:first + 40_000], want), first
    assert not out[::1_009].isnan().any()


def test_the_loss_of_half_a_million_queries_and_keys(rn):
    """4,096 x 4,096 tiles of the logits; 50 queries against double precision.  Bound: as in the tests of small calls, u = 2^-24 times
    (d + 4) products for each of the two norms' worth of a logit, twice, and the exponentials."""
    import torch
    n, d, scale = 524_288, 64, 2.0
    g = torch.Generator(device="cuda").manual_seed(5)
    K = (torch.randn(n, d, device="cuda", generator=g) / 8).bfloat16()
    Q = (K.float() + torch.randn(n, d, device="cuda", generator=g) / 8).bfloat16()
    target = torch.arange(n, device="cuda", dtype=torch.int32)
    target[3] = -1
    loss, dq, dk = rn.rnnd_contrast(Q, K, target, scale, want_grad=False)
    assert dq is None and dk is None
    some = torch.randint(0, n, (50,), device="cuda", generator=g)
    some[0], some[1], some[2] = 0, n - 1, 3
    q, k = Q[some].double(), K.double()
    s = -scale * (q.square().sum(1)[:, None] + k.square().sum(1)[None, :] - 2 * q @ k.T)
    want = torch.logsumexp(s, 1) - s.gather(1, some[:, None])[:, 0]
    want[2] = 0.0
    u = 2.0 ** -24
    nq, nk = q.norm(dim=1).max().item(), k.norm(dim=1).max().item()
    e = u * ((d + 4) * 2 * scale * nq * nk + (d + 4) * scale * nk * nk)
    assert ((loss[some].double() - want).abs() <= 2 * e + 40 * u * (1 + want)).all()
    assert loss[3] == 0 and loss.isfinite().all() and (loss > 0).sum() == n - 1
