"""The gradient of long calls: every row against sums in double precision, on an output and a workspace that hold NaN beforehand."""
import math

import pytest

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def rn():
    import torch
    assert torch.cuda.is_available(), "these tests need the MI355X"
    import paper_2310_20419_amd as m
    m.load_library()
    return m


def check_every_row(rn, dout, ids, V, scale, passes=1):
    """Bound of a row that `count` tokens name, with u = 2^-24: count additions and one product in float32 and the rounding of the result,
    (count + 3) u of the sum of the magnitudes.  A row that no token names is zero."""
    import torch
    n, d = dout.shape
    inside = (ids >= 0) & (ids < V)
    at = ids[inside].long()
    count = torch.bincount(at, minlength=V)
    want = torch.zeros(V, d, device="cuda", dtype=torch.float64)
    size = torch.zeros(V, d, device="cuda", dtype=torch.float64)
    for first in range(0, d, 16):       # a few columns at a time: doubles of the rows are large
        x = dout[:, first:first + 16][inside].double()
        want[:, first:first + 16].index_add_(0, at, x)
        size[:, first:first + 16].index_add_(0, at, x.abs())
    want *= scale
    size *= abs(scale)
    bound = size * (count[:, None] + 3) * 2.0 ** -24 + 2.0 ** -149
    need = rn.rnnd_embed_grad_workspace(n, d, V)
    got = [rn.rnnd_embed_grad(dout, ids, V, scale=scale, grad=torch.full((V, d), float("nan"), device="cuda"),
                              workspace=torch.full((need,), 0xFF, dtype=torch.uint8, device="cuda")) for _ in range(passes)]
    for g in got:
        off = (g.double() - want).abs()
        wrong = (~(off <= bound)).any(1).nonzero()[:, 0]        # (a NaN is no smaller than the bound)
        assert len(wrong) == 0, (len(wrong), wrong[:5].tolist(), count[wrong[:5]].tolist())
        assert (g[count == 0] == 0).all()
        assert torch.equal(g, got[0])


def popular(n, V, generator):
    """The k-th most frequent id about 1/k as often as the first; one in fifty is padding."""
    import torch
    u = torch.rand(n, device="cuda", generator=generator, dtype=torch.float64)
    ids = (torch.exp(u * math.log(V + 1)) - 1).to(torch.int32).clamp_(0, V - 1)
    return torch.where(torch.rand(n, device="cuda", generator=generator) < 0.02, -1, ids)


def test_a_million_tokens_into_a_million_rows(rn):
    import torch
    n, V, d = 1_000_000, 1_000_000, 96
    g = torch.Generator(device="cuda").manual_seed(12)
    dout = torch.randn(n, d, device="cuda", generator=g) * 0.01
    check_every_row(rn, dout, popular(n, V, g), V, 9.5, passes=3)


@pytest.mark.parametrize("n", [131_072, 131_073, 200_003, 1_000_000])
@pytest.mark.parametrize("V,names", [(1_048_575, 700), (1_048_575, 300_000), (1_023, 400), (3_000_000, 5_000)])
def test_digits_of_ten_bits_on_both_sides_of_the_offsets_launch(rn, n, V, names):
    """Up to 131,072 tokens every block of a sort sums the counts of the blocks before it, beyond that a launch does: 16 workgroups of
    64 digits where a pass takes ten bits.  Named rows are few, or many, and spread over all digits."""
    import torch
    g = torch.Generator(device="cuda").manual_seed(n + names)
    rows = torch.randperm(V, device="cuda", generator=g)[:names].to(torch.int32)
    rows[0] = V - 1
    ids = rows[torch.randint(0, names, (n,), device="cuda", generator=g)]
    ids[::101] = -1
    ids[7::1009] = V
    check_every_row(rn, torch.randn(n, 8, device="cuda", generator=g), ids, V, 1.0)
