"""Block-scaled quantizers, checkpoints and products on the GPU against their definition in 64 bits."""
import numpy as np
import pytest
import torch

import block_util as B
import oracle
from gpu_util import DEV, check_product, check_product_f8_pipeline, group_max_sum, host_src, say
from paper_2511_00874_amd import lib as L
from paper_2511_00874_amd import synth

pytestmark = pytest.mark.gpu

# one token, blocks that end inside a tile on either side, several tiles
SHAPES = [(1, 16), (1, 128), (3, 144), (17, 400), (127, 256), (129, 272), (300, 2064)]


def _source(shape, seed, bf16):
    """Rows and columns of very different sizes, a block of zeros, the type's extremes, infinities and NaN."""
    rng = np.random.default_rng(seed)
    x = rng.standard_normal(shape) * np.exp2(rng.integers(-30, 30, (shape[0], 1))) * np.exp2(rng.integers(-4, 4, (1, shape[1])))
    x = x.astype(np.float32)
    flat = x.reshape(-1)
    for i, v in enumerate((0.0, -0.0, np.inf, -np.inf, np.nan, 3.38e38, -3.38e38, 1e-42, -1e-38)):
        flat[(i * 7919 + seed) % flat.size] = v
    x[shape[0] // 2, :128] = 0.0
    t = torch.from_numpy(x).to(DEV)
    return t.to(torch.bfloat16) if bf16 else t


def _expect(b, codes, exps, what):
    assert np.array_equal(b.exps.cpu().numpy()[:, :exps.shape[1]].astype(np.int64) - 127, exps), what
    got = b.codes.cpu().numpy()
    assert np.array_equal(got[:, :codes.shape[1]], codes), what
    assert not got[:, codes.shape[1]:-(-codes.shape[1] // 16) * 16].any(), what  # the padding that products rely on


@pytest.mark.parametrize("shape", SHAPES)
@pytest.mark.parametrize("kind", [L.E4M3, L.E5M2])
@pytest.mark.parametrize("mode", [L.RTN, L.SR])
@pytest.mark.parametrize("bf16", [False, True])
def test_quantize_both_layouts(shape, kind, mode, bf16):
    say("block_quantize", shape, kind, mode, bf16)
    t = _source(shape, 3, bf16)
    x = B.wide(t)
    q = L.Quant(kind, 1.0, seed=11, counter_offset=2**33 + 5, round_mode=mode)
    rows, turned = L.sr_block_quantize(t, q, layout=L.BOTH)
    want = [B.block_codes(x, kind, mode, 11, 2**33 + 5, turned=way) for way in (False, True)]
    _expect(rows, *want[0], "rows")
    _expect(turned, *want[1], "turned")
    _expect(L.sr_block_quantize(t, q), *want[0], "rows alone")
    _expect(L.sr_block_quantize(t, q, layout=L.TURNED), *want[1], "turned alone")


@pytest.mark.parametrize("shape", SHAPES)
@pytest.mark.parametrize("kind,to", [(L.E4M3, L.E4M3), (L.E5M2, L.E5M2), (L.E4M3, L.E5M2), (L.E5M2, L.E4M3)])
def test_turn_and_restore(shape, kind, to):
    say("block_turn", shape, kind, to)
    t = _source(shape, 5, True)
    b = L.sr_block_quantize(t, L.Quant(kind, 1.0, round_mode=L.RTN))
    v = B.values(b)
    for dtype in (torch.float32, torch.bfloat16):
        got = B.wide(b.values(dtype))
        assert np.array_equal(got, v, equal_nan=True)
    for mode in (L.RTN, L.SR):
        _expect(L.sr_block_turn(b, L.Quant(to, 1.0, seed=4, counter_offset=9, round_mode=mode)),
                *B.block_codes(v, to, mode, 4, 9, turned=True), "turn")


def test_turning_a_checkpoint_mostly_moves_exponents():
    # values of 16 binades in both directions: what was exact in a block along the rows is exact in one along the columns, unless it
    # is below the normal numbers of the new block
    rng = np.random.default_rng(0)
    b = B.make(rng.standard_normal((256, 256)) * np.exp2(rng.integers(-4, 4, (256, 1))), L.E4M3, DEV)
    turned = L.sr_block_turn(b)
    v, w = B.values(b), B.values(turned).T
    e = turned.exps.cpu().numpy()[:, :2].astype(np.int64) - 127
    normal = np.abs(v) >= 2.0**-6 * 2.0**B.over_columns(e, 256).T
    assert normal.mean() > 0.9 and np.array_equal(v[normal], w[normal])


def test_rounding_is_unbiased_and_nearest_is_not():
    x = torch.full((4096, 128), 1.03, device=DEV)
    x[:, 0] = 448.0  # the scale of every block is 1: 1.03 lies between 1 and 1.125
    q = L.Quant(L.E4M3, 1.0, seed=2)
    sr = B.values(L.sr_block_quantize(x, q))[:, 1:]
    assert set(np.unique(sr)) == {1.0, 1.125}
    n, p = sr.size, 0.03 / 0.125
    assert abs((sr == 1.125).mean() - p) < 5 * np.sqrt(p * (1 - p) / n)
    assert (B.values(L.sr_block_quantize(x, L.RTN_E4M3))[:, 1:] == 1.0).all()


def test_a_counter_on_the_device_and_another_stream():
    t = synth.gaussian_torch((300, 256), 1.0, 0, DEV)
    at = torch.tensor([77], dtype=torch.int64, device=DEV)
    want = L.sr_block_quantize(t, L.Quant(L.E5M2, 1.0, seed=5, counter_offset=77), layout=L.BOTH)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = L.sr_block_quantize(t, L.Quant(L.E5M2, 1.0, seed=5, counter_offset=at), layout=L.BOTH)
    side.synchronize()
    for g, w in zip(got, want):
        assert B.same(g, w)


def test_nothing_to_do():
    q = L.Quant(L.E4M3, 1.0, round_mode=L.RTN)
    empty = torch.empty((0, 256), device=DEV)
    rows, turned = L.sr_block_quantize(empty, q, layout=L.BOTH)
    assert rows.shape == (0, 256) and turned.shape == (256, 0)
    assert L.sr_block_turn(rows).shape == (256, 0) and rows.values().shape == (0, 256)
    Z = L.sr_block_quantize(synth.gaussian_torch((48, 256), 1.0, 0, DEV), q)
    assert L.sr_gemm_blocks(rows, Z).shape == (0, 48)
    out = torch.full((256, 48), 3.0, device=DEV)  # a contraction over no tokens
    none = L.sr_block_quantize(torch.empty((0, 48), device=DEV), q, layout=L.TURNED)
    assert torch.equal(L.sr_gemm_blocks(turned, none, beta=1.0, out=out), torch.full_like(out, 3.0))
    assert torch.equal(L.sr_gemm_blocks(turned, none, out=out), torch.zeros_like(out))


# ---- products -------------------------------------------------------------------------------------------------------
PRODUCTS = [(1, 16, 16), (1, 2048, 5632), (3, 80, 144), (16, 48, 128), (17, 130, 1040), (33, 257, 777), (64, 192, 2064), (65, 63, 1),
            (113, 384, 400), (130, 127, 2063), (257, 513, 640), (300, 1000, 1296)]


def _operands(P, Q, R, kx, kz, seed=0):
    rng = np.random.default_rng(seed)
    x = rng.standard_normal((P, R)) * np.exp2(rng.integers(-6, 6, (P, 1))) * np.exp2(np.arange(R) // 128 % 5)
    z = rng.standard_normal((Q, R)) * 0.02 * np.exp2(rng.integers(-6, 6, (Q, 1)))
    if P > 2:
        x[P // 2] = 0.0
    return B.make(x, kx, DEV), B.make(z, kz, DEV)


@pytest.mark.parametrize("dims", PRODUCTS)
@pytest.mark.parametrize("kinds", [(L.E4M3, L.E4M3), (L.E5M2, L.E4M3), (L.E4M3, L.E5M2), (L.E5M2, L.E5M2)])
def test_product_exact(dims, kinds):
    say("gemm_blocks", dims, kinds)
    X, Z = _operands(*dims, *kinds)
    x, z = B.values(X), B.values(Z)
    ref, ab = x @ z.T, np.abs(x) @ np.abs(z).T
    check_product(B.wide(L.sr_gemm_blocks(X, Z)), ref, ab, "f32")
    got = B.wide(L.sr_gemm_blocks(X, Z, dtype=torch.bfloat16))
    assert np.all(np.abs(got - ref) <= 1e-5 * ab + 2.0**-8 * np.abs(ref)), "bf16"
    base = synth.gaussian_torch(dims[:2], 1.0, 1, DEV)
    out = base.clone()
    L.sr_gemm_blocks(X, Z, alpha=0.5, beta=1.0, out=out)
    check_product(B.wide(out), 0.5 * ref + B.wide(base), 0.5 * ab + np.abs(B.wide(base)), "beta")


@pytest.mark.parametrize("dims", PRODUCTS)
@pytest.mark.parametrize("kinds", [(L.E4M3, L.E4M3), (L.E5M2, L.E4M3), (L.E4M3, L.E5M2), (L.E5M2, L.E5M2)])
def test_product_on_the_fp8_pipeline(dims, kinds):
    say("gemm_blocks f8", dims, kinds)
    X, Z = _operands(*dims, *kinds, seed=1)
    x, z = B.values(X), B.values(Z)
    ref, ab = x @ z.T, np.abs(x) @ np.abs(z).T
    check_product_f8_pipeline(B.wide(L.sr_gemm_blocks(X, Z, f8_pipeline=True)), ref, group_max_sum(x, z, 1.0), ab, "f32")


def test_product_of_exact_integers():
    # small whole numbers in every place: any misplaced code, scale or row changes the result
    rng = np.random.default_rng(4)
    for P, Q, R in ((5, 96, 640), (200, 272, 1168), (300, 700, 513), (2321, 3950, 1168)):  # (the last: whole tiles, and tiles in slices)
        say("integers", P, Q, R)
        x = rng.integers(-8, 9, (P, R)) * np.exp2((np.arange(R) // 128) % 3) * np.exp2(np.arange(P) % 5)[:, None]
        z = rng.integers(-8, 9, (Q, R)) * np.exp2((np.arange(R) // 128) % 2) * np.exp2(np.arange(Q) % 3)[:, None]
        X, Z = B.make(x, L.E4M3, DEV), B.make(z, L.E4M3, DEV)
        for f8 in (False, True):
            assert np.array_equal(B.wide(L.sr_gemm_blocks(X, Z, f8_pipeline=f8)), x @ z.T), (P, Q, R, f8)


def test_product_carries_infinities_and_nan_of_their_rows_only():
    rng = np.random.default_rng(5)
    for P in (3, 200):
        x = rng.standard_normal((P, 400))
        X, Z = B.make(x, L.E4M3, DEV), B.make(rng.standard_normal((80, 400)), L.E4M3, DEV)
        X.codes[1, 17] = 0x7F
        for f8 in (False, True):
            got = B.wide(L.sr_gemm_blocks(X, Z, f8_pipeline=f8))
            assert np.isnan(got[1]).all() and np.isfinite(np.delete(got, 1, 0)).all()


def test_product_is_the_same_every_time():
    X, Z = _operands(200, 528, 5648, L.E4M3, L.E4M3)
    first = L.sr_gemm_blocks(X, Z)
    for _ in range(3):
        assert torch.equal(L.sr_gemm_blocks(X, Z), first)


def test_operands_beyond_4_gib():
    # offsets of rows and of scales past 32 bits: X is 2^21 + 77 rows of 2064
    M, K = (1 << 21) + 77, 2064
    q = L.Quant(L.E4M3, 1.0, round_mode=L.RTN)
    t = torch.empty((M, K), dtype=torch.bfloat16, device=DEV)
    for r in range(0, M, 1 << 18):
        t[r:r + (1 << 18)].normal_(generator=torch.Generator(device=DEV).manual_seed(r))
    Z = L.sr_block_quantize(synth.gaussian_torch((32, K), 0.02, 1, DEV), q)
    rows, turned = L.sr_block_quantize(t, q, layout=L.BOTH)
    at = M - 300
    part = L.sr_block_quantize(t[at:].contiguous(), q)
    assert torch.equal(rows.codes[at:, :K], part.codes[:, :K]) and torch.equal(rows.exps[at:, :17], part.exps[:, :17])
    assert (M - 77) % 128 == 0
    x = B.wide(t[-77 - 128:])  # the last whole block of rows and the ragged one
    codes, exps = B.block_codes(x, L.E4M3, turned=True)
    assert np.array_equal(turned.codes[:, M - 77 - 128:M].cpu().numpy(), codes)
    assert np.array_equal(turned.exps[:, (M - 77) // 128 - 1:M // 128 + 1].cpu().numpy().astype(np.int64) - 127, exps)
    del turned, t
    for f8 in (False, True):
        out = L.sr_gemm_blocks(rows, Z, dtype=torch.bfloat16, f8_pipeline=f8)
        few = L.Blocks(rows.codes[at:, :K].contiguous(),  # (rows without gaps)
                       rows.exps[at:].contiguous(), L.E4M3, K)
        assert torch.equal(out[at:], L.sr_gemm_blocks(few, Z, dtype=torch.bfloat16, f8_pipeline=f8))
    back = L.sr_block_turn(rows)
    first = (M - 77) // 128 - 1
    v = B.values(L.Blocks(rows.codes[first * 128:].contiguous(), rows.exps[first * 128:].contiguous(), L.E4M3, K))
    codes, exps = B.block_codes(v, L.E4M3, turned=True)
    assert np.array_equal(back.codes[:, first * 128:M].cpu().numpy(), codes)
    assert np.array_equal(back.exps[:, first:first + 2].cpu().numpy().astype(np.int64) - 127, exps)
