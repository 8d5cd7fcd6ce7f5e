"""Every form of the tile kernel with every pair of formats and every kind of result, several tiles to a workgroup and slices beside whole tiles.

Operands are whole numbers up to 8 (times a power of two): both formats hold them exactly, sums are whole numbers below 2^24 in any order, and
products of one group differ by less than the fp8 pipeline's 14 bits.  So results are equal to the 64-bit ones, bit for bit."""
import pytest
import torch

import test_gpu_gated as gated_tests
from block_shapes import GATED, PRODUCTS
from gpu_util import DEV, say
from paper_2511_00874_amd import lib as L

pytestmark = pytest.mark.gpu
KINDS = [(L.E4M3, L.E4M3), (L.E5M2, L.E4M3), (L.E4M3, L.E5M2), (L.E5M2, L.E5M2)]
RTN = L.Quant(L.E4M3, 1.0, round_mode=L.RTN)


def _numbers(rows, cols, kind, seed, most=8, unit=1.0):
    g = torch.Generator(device=DEV).manual_seed(seed)
    x = torch.randint(-most, most + 1, (rows, cols), generator=g, device=DEV).double() * unit
    room = torch.zeros((rows, (cols + 15) // 16 * 16), device=DEV)
    room[:, :cols] = x
    b = L.sr_block_quantize(room, L.Quant(kind, 1.0, round_mode=L.RTN))
    return x, L.Blocks(b.codes, b.exps, b.kind, cols) if room.shape[1] != cols else b


@pytest.mark.parametrize("f8", [False, True])
@pytest.mark.parametrize("form", list(PRODUCTS[False]))
def test_products(form, f8):
    P, Q, R = PRODUCTS[f8][form]
    base = torch.randint(-100, 101, (P, Q), generator=torch.Generator(device=DEV).manual_seed(3), device=DEV).float()
    for kx, kz in KINDS:
        say("products", form, f8, (P, Q, R), kx, kz)
        x, X = _numbers(P, R, kx, 1)
        z, Z = _numbers(Q, R, kz, 2)
        want = x @ z.t().contiguous()
        got = L.sr_gemm_blocks(X, Z, f8_pipeline=f8)
        assert torch.equal(got.double(), want)
        for _ in range(2):
            assert torch.equal(L.sr_gemm_blocks(X, Z, f8_pipeline=f8), got)
        assert torch.equal(L.sr_gemm_blocks(X, Z, dtype=torch.bfloat16, f8_pipeline=f8), got.to(torch.bfloat16))
        out = base.clone()
        L.sr_gemm_blocks(X, Z, alpha=0.5, beta=1.0, out=out, f8_pipeline=f8)
        assert torch.equal(out.double(), 0.5 * want + base.double())


@pytest.mark.parametrize("f8,form", [(f8, form) for f8 in (False, True) for form in GATED[f8]])
@pytest.mark.parametrize("act", [L.ACT_SILU, L.ACT_GELU])
def test_gated_rounds_stochastically_as_the_quantizer(form, f8, act):
    M, F, K = GATED[f8][form]
    say("gated", form, f8, (M, F, K), act)
    x, X = _numbers(M, K, L.E4M3, 3, unit=0.25)
    w, W = _numbers(2 * F, K, L.E4M3, 4, most=4, unit=1.0 / 32)
    sums = (x @ w.t().contiguous()).float()  # (binary32 numbers)
    g, u = sums[:, :F].double(), sums[:, F:].double()
    a = g * torch.sigmoid(g) if act == L.ACT_SILU else 0.5 * g * torch.special.erfc(-g * 0.5**0.5)
    want = a * u
    # H in bfloat16, of either pipeline: the activation to a few units of 2^-24 of itself (GELU's tail: 4 g^2 + 64 of them)
    h, _ = L.sr_gated_fwd(X, W, act=act, f8_pipeline=f8)
    err = (4 * g * g + 64) * 2.0**-24 * want.abs()
    assert ((h.double() - want).abs() <= err + 2.0**-8 * want.abs() + 1e-30).all()
    # codes: the sums' are the quantizer's, bit for bit; H's where its binary32 value does not stand beside a threshold (its distance there is
    # uniform, a few 2^-24 of the value against steps of 2^-4 at least: 1e-5 of them, and a block's 128 where its largest is beside Qmax 2^e)
    qh, qgu = L.Quant(L.E4M3, 1.0, seed=7, counter_offset=100), L.Quant(L.E4M3, 1.0, seed=8, counter_offset=2**40)
    hb, kept = L.sr_gated_fwd(X, W, act=act, qh=qh, qgu=qgu, f8_pipeline=f8)
    asked = L.sr_block_quantize(sums, qgu)
    blocks = 2 * F // 128
    assert torch.equal(kept.codes, asked.codes) and torch.equal(kept.exps[:, :blocks], asked.exps[:, :blocks])
    differ = (L.sr_block_quantize(want.float(), qh).codes != hb.codes).double().mean().item()
    assert differ <= 1e-3
    again, _ = L.sr_gated_fwd(X, W, act=act, qh=qh, f8_pipeline=f8)
    assert torch.equal(again.codes, hb.codes)


@pytest.mark.parametrize("M,F", [(1, 128), (3, 256), (127, 384), (129, 128), (300, 640)])
@pytest.mark.parametrize("act", [L.ACT_SILU, L.ACT_GELU])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("kind,mode", [(L.E4M3, L.SR), (L.E5M2, L.RTN)])
def test_backward_in_the_other_formats(M, F, act, dtype, kind, mode):
    gated_tests.test_backward(M, F, act, dtype, kind, mode)
