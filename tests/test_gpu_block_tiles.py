"""Products and gated blocks on every size of tile, whole and in slices of the contraction: whole numbers, whose sums are exact in whatever
order, against 64-bit sums.  Sizes: for the exact and the fp8 pipeline each form is taken by some of them."""
import pytest
import torch

from gpu_util import DEV, say
from paper_2511_00874_amd import lib as L

pytestmark = pytest.mark.gpu
RTN = L.Quant(L.E4M3, 1.0, round_mode=L.RTN)
PRODUCTS = [(130, 130, 144), (130, 130, 1168), (1009, 2100, 144), (2000, 2100, 144), (2321, 3950, 144), (2000, 513, 4100), (130, 3950, 8200),
            (2321, 513, 8200), (200, 2100, 8200), (3000, 1000, 8200)]
GATED = [(20, 256, 400), (200, 256, 1040), (200, 5632, 144), (300, 1408, 2064), (600, 384, 2064), (700, 5632, 144), (2000, 1408, 144), (3000, 384, 2064),
         (3000, 1408, 144), (3000, 2816, 1040)]


def _numbers(rows, cols, most, unit, seed):
    """Whole numbers up to `most` times a unit, and the block-scaled matrix that holds just them."""
    g = torch.Generator(device=DEV).manual_seed(seed)
    x = torch.randint(-most, most + 1, (rows, cols), generator=g, device=DEV).double() * unit
    room = torch.zeros((rows, (cols + 15) // 16 * 16), device=DEV)
    room[:, :cols] = x
    b = L.sr_block_quantize(room, RTN)
    return x, L.Blocks(b.codes, b.exps, b.kind, cols) if room.shape[1] != cols else b


@pytest.mark.parametrize("dims", PRODUCTS)
@pytest.mark.parametrize("f8", [False, True])
def test_products(dims, f8):
    say("products", dims, f8)
    P, Q, R = dims
    x, X = _numbers(P, R, 8, 1.0, 1)
    z, Z = _numbers(Q, R, 8, 1.0, 2)
    got = L.sr_gemm_blocks(X, Z, f8_pipeline=f8)
    assert torch.equal(got.double(), x @ z.t().contiguous())


@pytest.mark.parametrize("size", GATED)
@pytest.mark.parametrize("act", [L.ACT_SILU, L.ACT_GELU])
@pytest.mark.parametrize("f8", [False, True])
def test_gated(size, act, f8):
    say("gated", size, act, f8)
    M, F, K = size
    x, X = _numbers(M, K, 8, 0.25, 3)
    w, W = _numbers(2 * F, K, 4, 1.0 / 32, 4)
    gu = x @ w.t().contiguous()
    g, u = gu[:, :F], gu[:, F:]
    a = g * torch.sigmoid(g) if act == L.ACT_SILU else g * 0.5 * (1.0 + torch.erf(g * 0.5**0.5))
    want = a * u
    # the activation in binary32: exponent and reciprocal, or 1 + erf, to a few units of 1, times |g|
    err = 1e-6 * (1 + g.abs()) * g.abs() * u.abs() + 1e-6 * want.abs()
    h, none = L.sr_gated_fwd(X, W, act=act, f8_pipeline=f8)
    assert none is None
    assert ((h.double() - want).abs() <= err + 2.0**-8 * want.abs() + 1e-38).all()
    hb, kept = L.sr_gated_fwd(X, W, act=act, qh=RTN, qgu=RTN, f8_pipeline=f8)
    sums = L.sr_block_quantize(gu.float(), RTN)  # (the sums are binary32 numbers)
    assert torch.equal(kept.codes, sums.codes)
    blocks = 2 * F // 128
    assert torch.equal(kept.exps[:, :blocks], sums.exps[:, :blocks])
    # H: a scale its block's largest value asks for, or one beside it; codes to half a step, of at least the smallest numbers of the scale
    s = torch.exp2(hb.exps[:, :F // 128].double() - 127)
    top, far = want.abs().view(M, -1, 128).amax(2), err.view(M, -1, 128).amax(2)
    assert ((top - far <= 448 * s) & ((top + far > 224 * s) | (top <= far))).all()
    step = torch.maximum(2.0**-4 * want.abs(), 2.0**-10 * s.repeat_interleave(128, 1))
    assert ((hb.values().double() - want).abs() <= step + 2 * err).all()
    only, _ = L.sr_gated_fwd(X, W, act=act, qh=RTN, f8_pipeline=f8)
    assert torch.equal(only.codes, hb.codes)
