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
    assert [lib.raw.sr_block_pitch(n) for n in (0, 1, 128, 129, 2048)] == [0, 128, 128, 256, 2048]
    assert [lib.raw.sr_block_scale_pitch(n) for n in (0, 1, 128, 129, 512, 513, 2048)] == [0, 4, 4, 4, 4, 8, 16]


def test_quantize(lib):
    def f(c=BUF, p=32, s=BUF, ct=BUF, pt=16, st=BUF, x=BUF, dtype=0, M=4, K=32, q=_q(lib)):
        return lib.raw.sr_block_quantize(c, p, s, ct, pt, st, x, dtype, M, K, q, None)

    for q, want in _bad_quantizers(lib):
        assert f(q=q) == want
    assert f(dtype=2) == FORMAT and f(K=24) == ALIGN
    assert f(M=1 << 31) == f(M=1 << 29, K=1 << 20) == f(K=(1 << 21) + 16, p=1 << 22) == f(p=(1 << 22) + 16) == SHAPE
    assert f(c=None, ct=None) == f(s=None) == f(st=None) == f(x=None) == NULL
    assert f(c=BUF + 8) == f(s=BUF + 2) == f(ct=BUF + 4) == f(x=BUF + 4) == f(p=40) == f(pt=20) == ALIGN
    assert f(p=16) == f(M=17, pt=16) == SHAPE  # rows that do not hold their values
    assert f(c=None, ct=None, x=None, M=0) == f(c=None, ct=None, x=None, K=0) == OK


def test_turn_and_restore(lib):
    def f(ct=BUF, pt=16, st=BUF, c=BUF, p=32, s=BUF, kind=3, M=4, K=32, q=_q(lib)):
        return lib.raw.sr_block_turn(ct, pt, st, c, p, s, kind, M, K, q, None)

    for q, want in _bad_quantizers(lib):
        assert f(q=q) == want
    assert f(kind=1) == UNSUPPORTED and f(kind=77) == FORMAT and f(K=40) == f(p=24) == ALIGN
    assert f(ct=None) == f(st=None) == f(c=None) == f(s=None) == NULL and f(p=16) == f(M=20) == SHAPE
    assert f(ct=None, st=None, c=None, s=None, M=0) == OK

    def g(x=BUF, dtype=0, c=BUF, p=32, s=BUF, kind=3, M=4, K=32):
        return lib.raw.sr_block_restore(x, dtype, c, p, s, kind, M, K, None)

    assert g(kind=1) == UNSUPPORTED and g(dtype=3) == FORMAT and g(x=None) == g(s=None) == g(c=None) == NULL
    assert g(x=BUF + 8) == g(K=8) == g(p=36) == ALIGN and g(p=16) == SHAPE and g(x=None, c=None, s=None, M=0) == OK


def test_product(lib):
    def f(out=BUF, dtype=0, X=BUF, px=None, sx=BUF, kx=3, Z=BUF, pz=None, sz=BUF, kz=3, P=64, Q=64, R=64, alpha=1.0, beta=0.0,
          flags=0, ws=BUF, n=1 << 40):
        least = (R + 15) // 16 * 16
        return lib.raw.sr_gemm_blocks(out, dtype, X, px or least, sx, kx, Z, pz or least, sz, kz, P, Q, R, alpha, beta, flags, ws, n, None)

    assert f(kx=1) == f(kz=6) == UNSUPPORTED and f(kx=99) == FORMAT
    assert f(dtype=2) == f(flags=2) == f(alpha=float("inf")) == f(alpha=float("nan")) == FORMAT
    assert f(beta=0.5) == f(beta=1.0, dtype=1) == UNSUPPORTED
    assert f(R=(1 << 22) + 1) == f(P=1 << 31) == f(P=1 << 29, Q=1 << 29) == SHAPE
    assert f(out=None) == f(X=None) == f(sx=None) == f(Z=None) == f(sz=None) == NULL
    assert f(out=BUF + 4) == f(X=BUF + 8) == f(Z=BUF + 1) == f(sx=BUF + 2) == f(sz=BUF + 1) == f(px=72) == ALIGN
    assert f(px=48) == f(pz=(1 << 22) + 16) == SHAPE
    assert f(P=0, out=None) == f(Q=0, out=None) == OK
    for flags in (0, 1):  # few tiles and a long contraction are cut in slices
        need = lib.raw.sr_gemm_blocks_workspace_bytes(1009, 2048, 65536, flags)
        if need:
            assert f(P=1009, Q=2048, R=65536, flags=flags, ws=None) == f(P=1009, Q=2048, R=65536, flags=flags, n=need - 1) == WORKSPACE


def test_gated(lib):
    def f(h=BUF, hs=BUF, gu=BUF, gs=BUF, X=BUF, px=None, sx=BUF, W=BUF, pw=None, sw=BUF, M=8, F=256, K=64, act=0, qh=_q(lib), qgu=_q(lib), flags=0, ws=BUF, n=1 << 40):
        return lib.raw.sr_gated_fwd(h, hs, gu, gs, X, px or K, sx, W, pw or K, sw, M, F, K, act, qh, qgu, flags, ws, n, None)

    for q, want in _bad_quantizers(lib)[1:]:
        assert f(qh=q) == f(qgu=q) == want
    assert f(qh=_q(lib, kind=4)) == f(qgu=_q(lib, kind=4)) == UNSUPPORTED  # (E4M3 alone)
    assert f(act=2) == f(flags=4) == FORMAT
    assert f(F=0) == f(K=0) == f(K=1 << 23) == f(M=1 << 31) == SHAPE
    assert f(F=192) == f(K=72) == f(px=72) == ALIGN and f(pw=48) == f(pw=(1 << 22) + 16) == SHAPE
    assert f(h=None) == f(hs=None) == f(gu=None) == f(gs=None) == f(X=None) == f(sx=None) == f(W=None) == f(sw=None) == NULL
    assert f(h=BUF + 8) == f(h=BUF + 8, qh=None) == f(gu=BUF + 4) == f(W=BUF + 8) == ALIGN
    assert f(M=0, h=None, X=None, W=None) == OK
    need = lib.raw.sr_gated_fwd_workspace_bytes(80, 256, 4096, 0)  # few tiles: slices
    assert need and f(M=80, K=4096, ws=None) == f(M=80, K=4096, n=need - 1) == WORKSPACE and f(M=80, K=4096, ws=BUF + 8) == ALIGN
    assert lib.raw.sr_gated_fwd_workspace_bytes(16, 256, 4096, 0) == 16 * 512 * 4  # few rows: the sums
    assert lib.raw.sr_gemm_blocks_workspace_bytes(16, 256, 4096, 0) == 0

    def b(dz=BUF, ds=BUF, dt=BUF, pt=16, dts=BUF, dH=BUF, dtype=0, gu=BUF, gs=BUF, M=8, F=256, act=0, q=_q(lib)):
        return lib.raw.sr_gated_bwd(dz, ds, dt, pt, dts, dH, dtype, gu, gs, M, F, act, q, None)

    for q, want in _bad_quantizers(lib):
        assert b(q=q) == want
    assert b(dtype=5) == b(act=-1) == FORMAT and b(F=0) == b(M=1 << 31) == SHAPE and b(F=64) == ALIGN
    assert b(dz=None) == b(ds=None) == b(dt=None) == b(dts=None) == b(dH=None) == b(gu=None) == b(gs=None) == NULL
    assert b(dH=BUF + 2) == b(dt=BUF + 8) == b(pt=24) == ALIGN and b(M=17) == SHAPE and b(M=0, dH=None) == OK


def test_norm(lib):
    def f(y=BUF, py=64, ys=BUF, h=BUF, rstd=BUF, x=BUF, r=BUF, g=BUF, dtype=0, M=4, D=64, eps=1e-5, q=_q(lib)):
        return lib.raw.sr_rmsnorm_fwd(y, py, ys, h, rstd, x, r, g, dtype, M, D, eps, q, None)

    for q, want in _bad_quantizers(lib)[1:]:
        assert f(q=q) == want
    assert f(dtype=9) == f(eps=0.0) == f(eps=-1.0) == f(eps=float("nan")) == f(eps=float("inf")) == FORMAT
    assert f(D=0) == f(M=1 << 31) == SHAPE and f(D=24) == ALIGN and f(D=16400) == UNSUPPORTED
    assert f(y=None) == f(ys=None) == f(h=None) == f(rstd=None) == f(x=None) == f(g=None) == NULL
    assert f(y=BUF + 4, q=None) == f(x=BUF + 8) == f(r=BUF + 8) == f(g=BUF + 4) == f(py=72) == ALIGN and f(py=48) == SHAPE
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
    for codes, exps in ((b.codes[:, :256], b.exps), (b.codes[:, :280], b.exps), (b.codes, b.exps[:, :3]), (b.codes.view(torch.int8), b.exps), (b.codes[:3], b.exps)):
        with pytest.raises(ValueError):
            lib.Blocks(codes, exps, lib.E4M3, 272).values()
    with pytest.raises(ValueError):
        lib.sr_gemm_blocks(b, lib.Blocks.empty(4, 256, lib.E4M3, "cpu"))
