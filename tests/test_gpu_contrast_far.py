"""float32 rows far from the origin: distances, and so the loss, do not change when all rows are moved, and its error goes with the
distances between the rows, not with how far away they lie."""
import numpy as np
import pytest

from test_gpu_contrast import call, reference

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def rn():
    import torch
    assert torch.cuda.is_available(), "these tests need the MI355X"
    import paper_2310_20419_amd as m
    m.load_library()
    return m


def moved(B, M, d, offset, seed):
    """Queries near their positives, all coordinates moved by `offset` (and by half of it, every other one)."""
    import torch
    g = np.random.Generator(np.random.PCG64(seed))
    centre = offset * np.where(np.arange(d) % 2, 1.0, 0.5)
    K = g.normal(size=(M, d)) / np.sqrt(d)
    t = g.integers(0, M, size=B)
    Q = 0.7 * K[t] + 0.7 * g.normal(size=(B, d)) / np.sqrt(d)
    c = dict(Q=torch.from_numpy(Q + centre).float().cuda(), K=torch.from_numpy(K + centre).float().cuda(), target=t.astype(np.int32))
    c["key_ids"] = g.integers(0, 3 * M + 2, size=M).astype(np.int32)
    c["key_ids"][g.random(M) < 0.1] = -1
    c["key_bias"] = g.normal(size=M).astype(np.float32)
    c["row_weight"] = (g.normal(size=B) / B).astype(np.float32)
    return c


def check(rn, c, scale, counting=None):
    """The rows are taken from a point whose every coordinate is one that some key has there: with m the mean of the keys and r the norm of the
    largest deviations |k_e - m_e| of each coordinate, a row lies within |x - m| + r of it.  With u = 2^-24 and a sum of n roundings
    off by no more than 6 sqrt(n) u of the sum of the magnitudes (six times the spread of independent roundings):
      - a logit: 6 d products of terms, d squares, the subtraction of the point (u of each coordinate, twice), scaling and rounding of the whole:
        e = u ((6 sqrt(6 d) + 12) 2 scale |q||k| + (6 sqrt(d) + 12) scale |k|^2 + 4 |bias|)
      - the loss: 2 e + 20 u (1 + loss)
      - a gradient: g off by 2 e + 25 u of itself; sums of 6 M (or 6 B) products.
    counting: the keys that e is taken over (others have a probability of exactly zero)."""
    m = c["K"].double().mean(0) if counting is None else c["K"][counting].double().mean(0)
    at = dict(c, Q=c["Q"].double() - m, K=c["K"].double() - m)
    loss, dq, dk, g, q, k, w, counts = reference(at, scale)
    got = [x.double().cpu().numpy() for x in call(rn, c, scale)]
    u, (B, M), d = 2.0 ** -24, g.shape, q.shape[1]
    near = np.ones(M, bool) if counting is None else np.isin(np.arange(M), counting)
    r = np.sqrt(np.square(abs(k[near]).max(0)).sum())
    nq, nk = np.linalg.norm(q, axis=1) + r, np.linalg.norm(k, axis=1) + r
    e = u * ((6 * np.sqrt(6 * d) + 12) * 2 * scale * nq[:, None] * nk + (6 * np.sqrt(d) + 12) * scale * nk ** 2 + 4 * abs(c["key_bias"]))
    e = np.where(near, e, 0.0).max(1)
    off, bound = abs(got[0] - loss), np.where(counts, 2 * e + 20 * u * (1 + loss), 0.0)
    assert (off <= bound).all(), ("loss", off.max(), bound.max())
    for name, x, want, mine, theirs, gg, ee in (("dQ", got[1], dq, q, k, abs(g), e[:, None] + 0 * g), ("dK", got[2], dk, k, q, abs(g).T, (e[:, None] + 0 * g).T)):
        some = near if name == "dK" else np.ones(B, bool)
        n = 6 * np.sqrt(6 * gg.shape[1]) + 12
        bound = np.array([2 * scale * ((gg[i] * (2 * ee[i] + 25 * u))[:, None] * abs(theirs - mine[i]) +
                                       (n * u * gg[i])[:, None] * (abs(theirs) + abs(mine[i]) + 2 * r)).sum(0) for i in range(len(want))])
        off = abs(x - want)
        assert (off <= bound + abs(want) * 8 * u)[some].all(), (name, off.max(), bound.max())
        assert some.all() or (x[~some] == 0).all()


@pytest.mark.parametrize("offset", [0.0, 10.0, -100.0])
@pytest.mark.parametrize("B,M,d", [(60, 300, 768), (40, 90, 33), (3, 5, 100), (1, 1, 64), (200, 2_000, 96)])
def test_rows_moved_away_from_the_origin(rn, offset, B, M, d):
    check(rn, moved(B, M, d, offset, B + d), 5.0)


def test_more_than_256_tiles_of_rows_moved_away(rn):
    """Logits of more than 256 tiles of 128, two workgroups a CU."""
    check(rn, moved(2_200, 2_200, 40, 50.0, 3), 5.0)


@pytest.mark.parametrize("places", [[0], [0, 1, 2, 299], [7, 150]])
def test_a_few_keys_far_from_the_others(rn, places):
    """Keys 1,000 away have no probability, whatever the others' is; the others' error does not go with them."""
    c = moved(60, 300, 96, 0.0, 4)
    c["K"][places] += 1_000.0
    c["key_ids"][:] = np.arange(300)
    rest = np.setdiff1d(np.arange(300), places)
    c["target"][:] = rest[np.arange(60) % len(rest)]
    check(rn, c, 5.0, rest)
