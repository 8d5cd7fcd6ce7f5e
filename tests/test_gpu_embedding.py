"""Embedding lookup and the gradient of its table, against their definitions."""
import numpy as np
import pytest
import torch

from block_util import wide
from gpu_util import DEV, say
from paper_2511_00874_amd import lib as L

pytestmark = pytest.mark.gpu
U = 2.0**-24


def _x(shape, seed, dtype):
    return torch.from_numpy(np.random.default_rng(seed).standard_normal(shape)).to(DEV).to(dtype)


@pytest.mark.parametrize("M,V,D", [(1, 1, 8), (7, 100, 2048), (300, 50, 40), (4097, 1000, 768), (33000, 77, 16), (5, 9, 4104)])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("out", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("wide_ids", [True, False])
def test_lookup(M, V, D, dtype, out, wide_ids):
    say("embedding_fwd", M, V, D, dtype, out)
    table = _x((V, D), 0, dtype)
    ids = torch.from_numpy(np.random.default_rng(1).integers(0, V, M)).to(DEV).to(torch.int64 if wide_ids else torch.int32)
    for scale in (1.0, 45.25):
        y = L.sr_embedding_fwd(table, ids, scale=scale, dtype=out)
        assert torch.equal(y, (table[ids.long()].float() * scale).to(out))  # one multiplication, one rounding


def test_ids_outside_the_table():
    table = _x((10, 64), 0, torch.float32)
    ids = torch.tensor([3, -1, 10, 2**40, -2**40, 9], device=DEV)
    y = L.sr_embedding_fwd(table, ids)
    assert torch.equal(y[[0, 5]], table[[3, 9]]) and torch.isnan(y[1:5]).all()
    d = L.sr_embedding_bwd(torch.ones((6, 64), device=DEV), ids, 10)
    want = torch.zeros((10, 64), device=DEV)
    want[[3, 9]] = 1.0
    assert torch.equal(d, want)


def _ids(kind, M, V, rng):
    if kind == "same":
        return np.full(M, V - 1)
    if kind == "uniform":
        return rng.integers(0, V, M)
    if kind == "ascending":
        return np.arange(M) * V // M
    p = 1.0 / (np.arange(V) + 2.7)
    return rng.choice(V, M, p=p / p.sum())


# one place; pieces of the list that runs end in, fill, go through; one workgroup's sort and several's; one to three passes of it
@pytest.mark.parametrize("M,V,D", [(1, 1, 8), (9, 3, 64), (64, 2, 2056), (1000, 300, 768), (8192, 32000, 40), (8193, 1000, 16), (20000, 70000, 8), (70001, 600, 8),
                                   (9000, 300000, 8), (300000, 511, 8)])
@pytest.mark.parametrize("kind", ["words", "same", "uniform", "ascending"])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_gradient(M, V, D, kind, dtype):
    say("embedding_bwd", M, V, D, kind, dtype)
    rng = np.random.default_rng(M + V)
    ids = _ids(kind, M, V, rng)
    dy = _x((M, D), 2, dtype)
    t = torch.from_numpy(ids).to(DEV)
    scale = 3.0
    got = L.sr_embedding_bwd(dy, t, V, scale=scale)
    order = np.argsort(ids, kind="stable")
    d64 = wide(dy)
    begins = np.searchsorted(ids[order], np.arange(V + 1))
    sums, sizes = np.zeros((V + 1, D)), np.zeros((V + 1, D))
    np.add.at(sums, ids, d64)
    np.add.at(sizes, ids, np.abs(d64))
    # a sum's terms are added one after the other within pieces of at most 64, every fourth piece's sums, and those four: n of them in a row at most
    n = np.diff(begins)[:, None]
    depth = np.minimum(n, 64) + (n / (8 * 4) + 2) + 4
    err = scale * ((depth + 1) * U * sizes[:V] + U * np.abs(sums[:V])) + 1e-45
    assert np.all(np.abs(wide(got) - scale * sums[:V]) <= err)
    assert torch.equal(got, L.sr_embedding_bwd(dy, t.int(), V, scale=scale))
    more = torch.ones((V, D), device=DEV)
    L.sr_embedding_bwd(dy, t, V, scale=scale, beta=1.0, out=more)
    assert torch.equal(more, 1.0 + got)
    if M > 8:  # without one token
        pad = int(ids[M // 2])
        got2 = L.sr_embedding_bwd(dy, t, V, scale=scale, padding=pad)
        assert not got2[pad].any()
        got2[pad] = got[pad]
        assert V == 1 or kind == "same" or torch.allclose(got2, got, rtol=0, atol=float((2 * err).max()))


def test_long_sums():
    # a token with a large share of many places
    M, V, D = 200000, 20, 64
    ids = torch.from_numpy(np.random.default_rng(0).integers(0, V, M)).to(DEV)
    dy = _x((M, D), 1, torch.bfloat16)
    got = wide(L.sr_embedding_bwd(dy, ids, V))
    sums, sizes = np.zeros((V, D)), np.zeros((V, D))
    np.add.at(sums, ids.cpu().numpy(), wide(dy))
    np.add.at(sizes, ids.cpu().numpy(), np.abs(wide(dy)))
    assert np.all(np.abs(got - sums) <= (64 + M / V / 8 / 4 + 20) * U * sizes)


def test_gradient_against_differences():
    # the lookup is linear: differences of its definition are exact but for rounding
    M, V, D = 50, 11, 16
    rng = np.random.default_rng(3)
    ids, c, table, u = rng.integers(0, V, M), rng.standard_normal((M, D)), rng.standard_normal((V, D)), rng.standard_normal((V, D))
    got = wide(L.sr_embedding_bwd(torch.from_numpy(c).float().to(DEV), torch.from_numpy(ids).to(DEV), V, scale=2.5))
    num = ((2.5 * (table + u)[ids] * c).sum() - (2.5 * (table - u)[ids] * c).sum()) / 2
    assert abs(num - (got * u).sum()) <= 100 * U * (np.abs(got) * np.abs(u)).sum() + 1e-9


def test_infinities_stay_with_their_token():
    ids = torch.tensor([4, 2, 4, 0, 2, 2], device=DEV)
    dy = torch.ones((6, 24), device=DEV)
    dy[1, 3], dy[3, 5] = float("nan"), float("inf")
    d = L.sr_embedding_bwd(dy, ids, 6)
    want = torch.zeros((6, 24), device=DEV)
    want[4], want[2], want[0] = 2.0, 3.0, 1.0
    want[2, 3], want[0, 5] = float("nan"), float("inf")
    assert torch.equal(torch.nan_to_num(d, nan=-9.0), torch.nan_to_num(want, nan=-9.0))


def test_no_places():
    e, ids = torch.empty((0, 64), device=DEV), torch.empty(0, dtype=torch.int64, device=DEV)
    assert L.sr_embedding_fwd(_x((5, 64), 0, torch.float32), ids).shape == (0, 64)
    assert not L.sr_embedding_bwd(e, ids, 5).any()
    out = torch.ones((5, 64), device=DEV)
    L.sr_embedding_bwd(e, ids, 5, beta=1.0, out=out)
    assert (out == 1).all()
