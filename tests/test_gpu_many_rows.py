"""More than 2^26 rows: a wavefront for each is more than 2^32 threads, which one launch does not hold."""
import numpy as np
import pytest

from test_gpu_scale import compact_round_check, reverse_union_check

pytestmark = pytest.mark.gpu


@pytest.fixture
def rn():
    import torch
    assert torch.cuda.is_available(), "these tests need the MI355X"
    import paper_2310_20419_amd as m
    m.load_library()
    m.rnnd_release_workspace()
    torch.cuda.empty_cache()
    yield m
    m.rnnd_release_workspace()          # tens of GB
    torch.cuda.empty_cache()


def test_67_million_rows(rn, oracle_mod):
    """RandomGraph of every row, one round of UpdateNeighbors and AddReverseEdges of sampled ones, rows of the last blocks among them."""
    import torch
    n, d, S, R, seed = 2**26 + 1_000, 8, 3, 8, 2310
    g = np.random.default_rng(3)
    X = g.integers(0, 256, size=(n, d), dtype=np.uint8)
    Xd = torch.from_numpy(X).cuda()
    keys, deg = rn.rnnd_random_graph(Xd, S, R, seed)
    assert (deg == S).all()
    ids = (keys[:, :S] >> 1) & 0x7FFFFFFF
    assert ((ids >= 0) & (ids < n)).all()
    for first in range(0, n, 1 << 24):          # the distances of all edges
        a = Xd[first:first + (1 << 24)].float()
        for s in range(S):
            b = Xd[ids[first:first + (1 << 24), s]].float()
            assert torch.equal((a - b).square().sum(1).long(), keys[first:first + (1 << 24), s] >> 32)
    del a, b, ids
    sample = np.unique(np.concatenate([g.choice(n, 80, replace=False), [0, 999, 1_000, 2**26 - 1, 2**26, n - 1]]))
    rows = keys[torch.from_numpy(sample).cuda()].cpu().numpy().view(np.uint64)
    for i, u in enumerate(sample):
        assert sorted(((rows[i, :S] >> np.uint64(1)) & np.uint64(0x7FFFFFFF)).tolist()) == sorted(oracle_mod.random_ids(n, int(u), S, seed).tolist())
    compact_round_check(rn, oracle_mod, X, Xd, keys, deg, R, sample, False, "N %d round 1" % n)
    reverse_union_check(rn, keys, deg, R, sample, "N %d AddReverseEdges" % n)
    graph, degree = rn.rnnd_export_graph(keys, deg, R)
    assert torch.equal(degree, deg)
    pad = torch.arange(R, device="cuda")[None, :] >= deg[:, None]
    assert torch.equal(graph, torch.where(pad, -1, (keys >> 1) & 0x7FFFFFFF).int())
