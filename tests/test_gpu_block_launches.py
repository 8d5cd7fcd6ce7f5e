"""Calls whose launches would have 2^32 threads and more: rows and tiles of the documented range."""
import pytest
import torch

from gpu_util import DEV, say
from paper_2511_00874_amd import lib as L

pytestmark = pytest.mark.gpu


def _noise(rows, cols, dtype):
    x = torch.empty((rows, cols), dtype=dtype, device=DEV)
    for r in range(0, rows, 1 << 24):
        x[r:r + (1 << 24)].normal_(generator=torch.Generator(device=DEV).manual_seed(r))
    return x


@pytest.mark.parametrize("shape", [((1 << 26) + 3, 16), ((1 << 22) + 3, 8208)])  # four rows a workgroup of 256 threads, one of 1024
@pytest.mark.parametrize("coded", [False, True])
def test_norm_of_very_many_rows(shape, coded):
    say("norm of many rows", shape, coded)
    M, D = shape
    gamma = torch.linspace(0.5, 1.5, D, device=DEV)
    x = _noise(M, D, torch.bfloat16)
    if D == 16:
        q = L.Quant(L.E4M3, 1.0, seed=3, counter_offset=11) if coded else None
    else:
        q = L.RTN_E4M3 if coded else None
    y, h, rstd = L.sr_rmsnorm_fwd(x, gamma, 1e-5, q=q)
    assert h is x
    for at in (0, M // 2 // 4 * 4, (1 << 21) * (4 if D == 16 else 1) - 500, M - 1003):
        part = x[at:at + 1003].clone()
        if isinstance(q, L.Quant):  # the thresholds of these rows
            q = L.Quant(L.E4M3, 1.0, seed=3, counter_offset=11 + at * D // 8)
        want, _, r = L.sr_rmsnorm_fwd(part, gamma, 1e-5, q=q)
        n = part.shape[0]
        assert torch.equal(rstd[at:at + n], r)
        ref = torch.rsqrt(part.double().square().mean(1) + 1e-5)
        assert ((r.double() - ref).abs() <= 2.0**-18 * ref).all()  # sums of up to 8208 squares, in tens a thread and then pairs
        if coded:
            assert torch.equal(y.codes[at:at + n, :D], want.codes[:, :D])
            blocks = (D + 127) // 128
            assert torch.equal(y.exps[at:at + n, :blocks], want.exps[:, :blocks])
        else:
            assert torch.equal(y[at:at + n], want)


def test_turned_codes_of_very_many_rows():
    M, K = (1 << 30) - 64, 16
    say("turned codes", M, K)
    q = L.Quant(L.E5M2, 1.0, round_mode=L.RTN)
    x = _noise(M, K, torch.bfloat16)
    turned = L.sr_block_quantize(x, q, layout=L.TURNED)
    for at in (0, (1 << 28) - 256, M // 128 * 128 - 256):
        n = min(M - at, 1024)
        want = L.sr_block_quantize(x[at:at + n].contiguous(), q, layout=L.TURNED)
        assert torch.equal(turned.codes[:, at:at + n], want.codes[:, :n])
        assert torch.equal(turned.exps[:, at // 128:at // 128 + (n + 127) // 128], want.exps[:, :(n + 127) // 128])


def test_product_of_one_row_with_very_many():
    Q, R = (1 << 30) - 1, 16
    say("few rows", Q, R)
    Z = L.Blocks(torch.randint(0, 120, (Q, R), dtype=torch.uint8, device=DEV), torch.full((Q, 4), 127, dtype=torch.uint8, device=DEV), L.E4M3, R)
    X = L.sr_block_quantize(torch.ones((1, R), device=DEV), L.Quant(L.E4M3, 1.0, round_mode=L.RTN))
    out = L.sr_gemm_blocks(X, Z, dtype=torch.bfloat16)
    for at in (0, (1 << 27) - 300, Q - 1000):
        n = min(Q - at, 1000)
        part = L.Blocks(Z.codes[at:at + n].clone(), Z.exps[at:at + n].clone(), L.E4M3, R)
        assert torch.equal(out[:, at:at + n], L.sr_gemm_blocks(X, part, dtype=torch.bfloat16))
