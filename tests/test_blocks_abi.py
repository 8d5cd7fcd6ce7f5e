"""Refusals of the block-scaled operators: every call below is rejected before anything is launched (no GPU here)."""
import ctypes as C

import pytest
import torch


@pytest.fixture(scope="module")
def lib():
    from paper_2511_00874_amd import build
    if build.stale():
        build.build()
    from paper_2511_00874_amd import lib as L
    return L


BUF = 0x1000  # never dereferenced
OK, NULL, SHAPE, FORMAT, ALIGN, WORKSPACE, UNSUPPORTED = 0, -1, -2, -3, -4, -5, -6


def _q(lib, kind=3, rnd=1, flags=0, counter=0):
    return C.byref(lib.srq_quant(kind, rnd, 0.0, flags, None, 0, counter))  # (a scale of 0: ignored)


def _bad_quantizers(lib):
    return [(None, NULL), (_q(lib, kind=1), UNSUPPORTED), (_q(lib, kind=5), UNSUPPORTED), (_q(lib, kind=0), UNSUPPORTED),
            (_q(lib, kind=9), FORMAT), (_q(lib, kind=-1), FORMAT), (_q(lib, rnd=2), FORMAT), (_q(lib, flags=1), FORMAT),
            (_q(lib, flags=8), FORMAT), (_q(lib, flags=2), ALIGN), (_q(lib, flags=2, counter=12), ALIGN)]


def test_pitches(lib):
    assert [lib.raw.sr_block_pitch(n) for n in (0, 1, 16, 17, 2048)] == [0, 16, 16, 32, 2048]
    assert [lib.raw.sr_block_scale_pitch(n) for n in (0, 1, 128, 129, 512, 513, 2048)] == [0, 4, 4, 4, 4, 8, 16]


def test_quantize(lib):
    f = lib.raw.sr_block_quantize
    for q, want in _bad_quantizers(lib):
        assert f(BUF, BUF, BUF, BUF, BUF, 0, 4, 32, q, None) == want
    q = _q(lib)
    assert f(BUF, BUF, None, None, BUF, 2, 4, 32, q, None) == FORMAT
    assert f(BUF, BUF, None, None, BUF, 0, 4, 24, q, None) == ALIGN
    assert f(BUF, BUF, None, None, BUF, 0, 1 << 31, 32, q, None) == SHAPE
    assert f(BUF, BUF, None, None, BUF, 0, 1 << 30, 1 << 20, q, None) == SHAPE
    assert f(None, None, None, None, BUF, 0, 4, 32, q, None) == NULL
    assert f(BUF, None, None, None, BUF, 0, 4, 32, q, None) == NULL
    assert f(BUF, BUF, BUF, None, BUF, 0, 4, 32, q, None) == NULL
    assert f(BUF, BUF, None, None, None, 0, 4, 32, q, None) == NULL
    assert f(BUF + 8, BUF, None, None, BUF, 0, 4, 32, q, None) == ALIGN
    assert f(BUF, BUF + 2, None, None, BUF, 0, 4, 32, q, None) == ALIGN
    assert f(BUF, BUF, None, None, BUF + 4, 0, 4, 32, q, None) == ALIGN
    assert f(None, None, None, None, None, 0, 0, 32, q, None) == OK and f(None, None, None, None, None, 0, 4, 0, q, None) == OK


def test_turn_and_restore(lib):
    f, g = lib.raw.sr_block_turn, lib.raw.sr_block_restore
    for q, want in _bad_quantizers(lib):
        assert f(BUF, BUF, BUF, BUF, 3, 4, 32, q, None) == want
    q = _q(lib)
    assert f(BUF, BUF, BUF, BUF, 1, 4, 32, q, None) == UNSUPPORTED and f(BUF, BUF, BUF, BUF, 77, 4, 32, q, None) == FORMAT
    assert f(BUF, BUF, BUF, BUF, 3, 4, 40, q, None) == ALIGN
    for i in range(4):
        args = [BUF] * 4
        args[i] = None
        assert f(*args, 3, 4, 32, q, None) == NULL
    assert g(BUF, 0, BUF, BUF, 1, 4, 32, None) == UNSUPPORTED and g(BUF, 3, BUF, BUF, 3, 4, 32, None) == FORMAT
    assert g(None, 0, BUF, BUF, 3, 4, 32, None) == NULL and g(BUF, 0, BUF, None, 3, 4, 32, None) == NULL
    assert g(BUF + 8, 0, BUF, BUF, 3, 4, 32, None) == ALIGN and g(BUF, 0, BUF, BUF, 3, 4, 8, None) == ALIGN
    assert g(None, 0, None, None, 3, 0, 32, None) == OK and f(None, None, None, None, 3, 0, 32, q, None) == OK


def test_product(lib):
    def f(out=BUF, dtype=0, X=BUF, sx=BUF, kx=3, Z=BUF, sz=BUF, kz=3, P=64, Q=64, R=64, alpha=1.0, beta=0.0, flags=0, ws=BUF, n=1 << 40):
        return lib.raw.sr_gemm_blocks(out, dtype, X, sx, kx, Z, sz, kz, P, Q, R, alpha, beta, flags, ws, n, None)

    assert f(kx=1) == f(kz=6) == UNSUPPORTED and f(kx=99) == FORMAT
    assert f(dtype=2) == f(flags=2) == f(alpha=float("inf")) == f(alpha=float("nan")) == FORMAT
    assert f(beta=0.5) == f(beta=1.0, dtype=1) == UNSUPPORTED
    assert f(R=(1 << 22) + 1) == f(P=1 << 31) == f(P=1 << 30, Q=1 << 30) == SHAPE
    assert f(out=None) == f(X=None) == f(sx=None) == f(Z=None) == f(sz=None) == NULL
    assert f(out=BUF + 4) == f(X=BUF + 8) == f(Z=BUF + 1) == f(sx=BUF + 2) == f(sz=BUF + 1) == ALIGN
    assert f(P=0, out=None) == f(Q=0, out=None) == OK
    for flags in (0, 1):  # few tiles and a long contraction are cut in slices
        need = lib.raw.sr_gemm_blocks_workspace_bytes(1009, 2048, 65536, flags)
        if need:
            assert f(P=1009, Q=2048, R=65536, flags=flags, ws=None) == f(P=1009, Q=2048, R=65536, flags=flags, n=need - 1) == WORKSPACE


def test_gated(lib):
    def f(h=BUF, hs=BUF, gu=BUF, gs=BUF, X=BUF, sx=BUF, W=BUF, sw=BUF, M=8, F=256, K=64, act=0, qh=_q(lib), qgu=_q(lib), flags=0, ws=BUF, n=1 << 40):
        return lib.raw.sr_gated_fwd(h, hs, gu, gs, X, sx, W, sw, M, F, K, act, qh, qgu, flags, ws, n, None)

    for q, want in _bad_quantizers(lib)[1:]:
        assert f(qh=q) == f(qgu=q) == want
    assert f(qh=_q(lib, kind=4)) == f(qgu=_q(lib, kind=4)) == UNSUPPORTED  # (E4M3 alone)
    assert f(act=2) == f(flags=4) == FORMAT
    assert f(F=0) == f(K=0) == f(K=1 << 23) == f(M=1 << 31) == SHAPE
    assert f(F=192) == f(K=72) == ALIGN
    assert f(h=None) == f(hs=None) == f(gu=None) == f(gs=None) == f(X=None) == f(sx=None) == f(W=None) == f(sw=None) == NULL
    assert f(h=BUF + 8) == f(h=BUF + 8, qh=None) == f(gu=BUF + 4) == f(W=BUF + 8) == ALIGN
    assert f(M=0, h=None, X=None, W=None) == OK
    need = lib.raw.sr_gated_fwd_workspace_bytes(8, 256, 4096, 0)  # few rows: slices
    assert need and f(K=4096, ws=None) == f(K=4096, n=need - 1) == WORKSPACE and f(K=4096, ws=BUF + 8) == ALIGN

    def b(dz=BUF, ds=BUF, dt=BUF, dts=BUF, dH=BUF, dtype=0, gu=BUF, gs=BUF, M=8, F=256, act=0, q=_q(lib)):
        return lib.raw.sr_gated_bwd(dz, ds, dt, dts, dH, dtype, gu, gs, M, F, act, q, None)

    for q, want in _bad_quantizers(lib):
        assert b(q=q) == want
    assert b(dtype=5) == b(act=-1) == FORMAT and b(F=0) == b(M=1 << 31) == SHAPE and b(F=64) == ALIGN
    assert b(dz=None) == b(ds=None) == b(dt=None) == b(dts=None) == b(dH=None) == b(gu=None) == b(gs=None) == NULL
    assert b(dH=BUF + 2) == b(dt=BUF + 8) == ALIGN and b(M=0, dH=None) == OK


def test_norm(lib):
    def f(y=BUF, ys=BUF, h=BUF, rstd=BUF, x=BUF, r=BUF, g=BUF, dtype=0, M=4, D=64, eps=1e-5, q=_q(lib)):
        return lib.raw.sr_rmsnorm_fwd(y, ys, h, rstd, x, r, g, dtype, M, D, eps, q, None)

    for q, want in _bad_quantizers(lib)[1:]:
        assert f(q=q) == want
    assert f(dtype=9) == f(eps=0.0) == f(eps=-1.0) == f(eps=float("nan")) == f(eps=float("inf")) == FORMAT
    assert f(D=0) == f(M=1 << 31) == SHAPE and f(D=24) == ALIGN and f(D=16400) == UNSUPPORTED
    assert f(y=None) == f(ys=None) == f(h=None) == f(rstd=None) == f(x=None) == f(g=None) == NULL
    assert f(y=BUF + 4, q=None) == f(x=BUF + 8) == f(r=BUF + 8) == f(g=BUF + 4) == ALIGN
    assert f(M=0, y=None, x=None) == OK

    def b(dx=BUF, dg=BUF, dy=BUF, dh=BUF, h=BUF, rstd=BUF, g=BUF, dtype=0, M=4, D=64, beta=0.0, ws=BUF, n=1 << 30):
        return lib.raw.sr_rmsnorm_bwd(dx, dg, dy, dh, h, rstd, g, dtype, M, D, beta, ws, n, None)

    assert b(dtype=-1) == FORMAT and b(beta=0.5) == b(D=16400) == UNSUPPORTED and b(D=0) == SHAPE and b(D=8) == ALIGN
    assert b(dx=None) == b(dg=None) == b(dy=None) == b(h=None) == b(rstd=None) == b(g=None) == NULL
    assert b(dx=BUF + 8) == b(dh=BUF + 8) == b(dg=BUF + 2) == ALIGN
    need = lib.raw.sr_rmsnorm_bwd_workspace_bytes(4, 64)
    assert need and b(ws=None) == b(n=need - 1) == WORKSPACE


def test_the_bindings_refuse_parts_that_do_not_fit(lib):
    b = lib.Blocks.empty(4, 272, lib.E4M3, "cpu")
    with pytest.raises(RuntimeError):
        b.values()  # host memory
    for codes, exps in ((b.codes[:, :256], b.exps), (b.codes, b.exps[:, :3]), (b.codes.view(torch.int8), b.exps), (b.codes[:3], b.exps)):
        with pytest.raises(ValueError):
            lib.Blocks(codes, exps, lib.E4M3, 272).values()
    with pytest.raises(ValueError):
        lib.sr_gemm_blocks(b, lib.Blocks.empty(4, 256, lib.E4M3, "cpu"))
