"""Root-mean-square norm with the residual's addition, forward and backward, against its definition in 64 bits."""
import numpy as np
import pytest
import torch

import block_util as B
from gpu_util import DEV, say
from paper_2511_00874_amd import lib as L

pytestmark = pytest.mark.gpu

EPS = 1e-5
# one row, rows that end inside a group of threads, every number of threads a row
SHAPES = [(1, 16), (1, 2048), (5, 144), (3, 2064), (2049, 528), (2050, 2048), (7, 4112), (3, 8192), (2, 8208), (2, 16384), (4099, 1040)]
U = 2.0**-24


def _rows(shape, seed, dtype):
    rng = np.random.default_rng(seed)
    x = rng.standard_normal(shape) * np.exp2(rng.integers(-8, 8, (shape[0], 1)))
    if shape[0] > 2:
        x[shape[0] // 2] = 0.0  # a row of zeros: rstd is 1 / sqrt(eps)
    return torch.from_numpy(x).to(DEV).to(dtype)


def _gamma(D):
    return torch.from_numpy(1.0 + 0.1 * np.random.default_rng(9).standard_normal(D)).float().to(DEV)


@pytest.mark.parametrize("shape", SHAPES)
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("residual", [False, True])
def test_forward(shape, dtype, residual):
    say("rmsnorm_fwd", shape, dtype, residual)
    x, gamma = _rows(shape, 1, dtype), _gamma(shape[1])
    r = _rows(shape, 2, dtype).roll(1, 0) if residual else None
    y, h, rstd = L.sr_rmsnorm_fwd(x, gamma, EPS, residual=r)
    want_h = x if r is None else (x.float() + r.float()).to(dtype)
    assert torch.equal(h, want_h)
    v = B.wide(want_h)
    want_r = 1.0 / np.sqrt((v * v).mean(1) + EPS)
    # sum of D squares: at most D / 8 roundings in a row on a thread and log in the tree; three more for the root
    tol = (min(shape[1], 64) / 2 + 16) * U
    assert np.all(np.abs(B.wide(rstd) - want_r) <= tol * want_r)
    want = v * want_r[:, None] * B.wide(gamma)
    out_tol = tol + 3 * U + (2.0**-8 if dtype is torch.bfloat16 else 0.0)
    assert np.all(np.abs(B.wide(y) - want) <= out_tol * np.abs(want) + 1e-45)
    for q, sr in ((L.Quant(L.E4M3, 1.0, round_mode=L.RTN), False), (L.Quant(L.E5M2, 1.0, seed=3, counter_offset=7), True)):
        b, h2, rstd2 = L.sr_rmsnorm_fwd(x, gamma, EPS, residual=r, q=q)
        assert torch.equal(h2, h) and torch.equal(rstd2, rstd)
        B.check_blocks(b, want, (tol + 3 * U) * np.abs(want), "codes", sr)
        # the codes are the quantizer's own of the values in binary32
        if dtype is torch.float32:
            c = L.sr_block_quantize(y, q)
            assert B.same(c, b)


@pytest.mark.parametrize("shape", SHAPES)
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("with_dh", [False, True])
def test_backward(shape, dtype, with_dh):
    say("rmsnorm_bwd", shape, dtype, with_dh)
    h, gamma = _rows(shape, 3, dtype), _gamma(shape[1])
    dy = _rows(shape, 4, dtype).roll(1, 0)
    dh = _rows(shape, 5, dtype).roll(2, 0) if with_dh else None
    _, _, rstd = L.sr_rmsnorm_fwd(h, gamma, EPS)
    dx, dgamma = L.sr_rmsnorm_bwd(dy, h, rstd, gamma, dh=dh)
    g, v, r, w = B.wide(dy), B.wide(h), B.wide(rstd)[:, None], B.wide(gamma)
    xhat = v * r
    c = (g * w * xhat).mean(1, keepdims=True)
    own = r * (g * w - xhat * c)
    want = own + (B.wide(dh) if with_dh else 0.0)
    # the mean's error enters times xhat; each of the two terms is rounded a few times
    size = r * (np.abs(g * w) + np.abs(xhat) * np.abs(g * w * xhat).mean(1, keepdims=True))
    err = 64 * U * size + 2 * U * np.abs(want) + (2.0**-8 * np.abs(want) if dtype is torch.bfloat16 else 0.0)
    assert np.all(np.abs(B.wide(dx) - want) <= err + 1e-45)
    terms = np.abs(g * xhat).sum(0)
    assert np.all(np.abs(B.wide(dgamma) - (g * xhat).sum(0)) <= (3 + shape[0] / 8 + 32) * U * terms + 1e-45)
    more = torch.ones(shape[1], device=DEV)
    L.sr_rmsnorm_bwd(dy, h, rstd, gamma, dh=dh, out_dgamma=more, beta=1.0)
    assert torch.equal(more, 1.0 + dgamma)
    again = L.sr_rmsnorm_bwd(dy, h, rstd, gamma, dh=dh)
    assert torch.equal(again[0], dx) and torch.equal(again[1], dgamma)
    if with_dh:  # in place of what reaches h
        L.sr_rmsnorm_bwd(dy, h, rstd, gamma, dh=dh, out_dx=dh)
        assert torch.equal(dh, dx)


def test_backward_against_differences():
    # directional derivatives of sum(y * c) in binary64 differences of the definition
    rng = np.random.default_rng(0)
    M, D = 5, 272
    x, c, w = rng.standard_normal((M, D)), rng.standard_normal((M, D)), 1.0 + 0.1 * rng.standard_normal(D)

    def loss(v, g):
        return (v / np.sqrt((v * v).mean(1, keepdims=True) + EPS) * g * c).sum()

    h, gamma, dy = (torch.from_numpy(a).float().to(DEV) for a in (x, w, c))
    _, _, rstd = L.sr_rmsnorm_fwd(h, gamma, EPS)
    dx, dgamma = L.sr_rmsnorm_bwd(dy, h, rstd, gamma)
    for k in range(8):
        u, s, t = rng.standard_normal((M, D)), rng.standard_normal(D), 1e-5
        num = (loss(x + t * u, w) - loss(x - t * u, w)) / (2 * t)
        assert abs(num - (B.wide(dx) * u).sum()) <= 1e-5 * np.abs(B.wide(dx) * u).sum()
        num = (loss(x, w + t * s) - loss(x, w - t * s)) / (2 * t)
        assert abs(num - (B.wide(dgamma) * s).sum()) <= 1e-5 * np.abs(B.wide(dgamma) * s).sum()


def test_rows_with_nothing_finite_keep_to_themselves():
    x = torch.randn((2100, 528), generator=torch.Generator(device=DEV).manual_seed(0), device=DEV)
    gamma = _gamma(528)
    x[5, 3], x[9, 500], x[11] = float("inf"), float("nan"), 0.0
    y, _, rstd = L.sr_rmsnorm_fwd(x, gamma, EPS)
    b, _, _ = L.sr_rmsnorm_fwd(x, gamma, EPS, q=L.RTN_E4M3)
    fine = torch.isfinite(y).all(1).cpu().numpy()
    assert [i for i in range(2100) if not fine[i]] == [5, 9]
    assert torch.equal(y[11], torch.zeros_like(y[11])) and not b.codes[11, :528].any()
    assert (b.codes[9, :528] == 0x7F).all() and np.isfinite(B.values(b)[fine]).all()


def test_no_rows():
    e, gamma = torch.empty((0, 256), device=DEV), _gamma(256)
    y, h, rstd = L.sr_rmsnorm_fwd(e, gamma, EPS)
    dx, dgamma = L.sr_rmsnorm_bwd(e, e, rstd, gamma)
    assert y.shape == dx.shape == (0, 256) and not dgamma.any()
