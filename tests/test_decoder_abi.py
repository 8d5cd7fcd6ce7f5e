"""Refusals of attention, embedding and AdamW: every call below is rejected before anything is launched (no GPU here)."""
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


def test_struct_layouts_match_the_header(lib):
    assert C.sizeof(lib.srq_heads) == 24 and lib.srq_heads.head.offset == 16
    assert C.sizeof(lib.srq_attention) == 80 and lib.srq_attention.offsets_q.offset == 48 and lib.srq_attention.scale.offset == 72
    assert C.sizeof(lib.srq_adamw_tensor) == 80 and lib.srq_adamw_tensor.n.offset == 48 and lib.srq_adamw_tensor.state_kind.offset == 76
    assert C.sizeof(lib.srq_adamw) == 72 and lib.srq_adamw.step.offset == 32 and lib.srq_adamw.counter_dev.offset == 64


def _shape(lib, **other):
    a = {"sequences": 2, "rows_q": 200, "rows_k": 200, "heads_q": 4, "heads_kv": 2, "dim": 64, "offsets_q": None, "offsets_k": None, "lengths_k": None,
         "scale": 0.125, "causal": 1} | other
    return lib.srq_attention(*[a[n] for n, _ in lib.srq_attention._fields_])


BAD_SHAPES = [({"scale": 0.0}, FORMAT), ({"scale": -1.0}, FORMAT), ({"scale": float("nan")}, FORMAT), ({"scale": float("inf")}, FORMAT), ({"causal": 2}, FORMAT),
              ({"sequences": 0}, SHAPE), ({"heads_q": 0}, SHAPE), ({"heads_kv": 0}, SHAPE), ({"dim": 0}, SHAPE), ({"heads_kv": 3}, SHAPE), ({"heads_q": 1}, SHAPE),
              ({"rows_q": 1 << 31}, SHAPE), ({"rows_k": 1 << 31}, SHAPE), ({"sequences": 1 << 31}, SHAPE), ({"heads_q": 1 << 20, "heads_kv": 1}, SHAPE),
              ({"rows_q": 1 << 29, "rows_k": 1 << 29, "heads_q": 64}, SHAPE), ({"rows_q": 201}, SHAPE), ({"rows_k": 201}, SHAPE),
              ({"offsets_q": BUF, "rows_k": 100}, SHAPE), ({"offsets_q": BUF, "offsets_k": None, "rows_q": 201}, SHAPE), ({"offsets_k": BUF, "rows_q": 201}, SHAPE),
              ({"dim": 60}, ALIGN), ({"offsets_q": BUF + 2}, ALIGN), ({"lengths_k": BUF + 1}, ALIGN), ({"dim": 136}, UNSUPPORTED), ({"dim": 256}, UNSUPPORTED)]


def _heads(lib, p=BUF, row=512, head=64):
    return lib.srq_heads(p, row, head)


def test_attention(lib):
    def f(o=_heads(lib), lse=BUF, q=_heads(lib), k=_heads(lib), v=_heads(lib), ws=BUF, n=1 << 40, **other):
        return lib.raw.sr_attention_fwd(o, lse, q, k, v, _shape(lib, **other), ws, n, None)

    for other, want in BAD_SHAPES:
        assert f(**other) == want, other
        assert lib.raw.sr_attention_fwd_workspace_bytes(_shape(lib, **other)) == lib.raw.sr_attention_bwd_workspace_bytes(_shape(lib, **other)) == 0
    assert lib.raw.sr_attention_fwd(None, BUF, None, None, None, None, None, 0, None) == NULL
    names = ("o", "q", "k", "v")
    for n in names:
        assert f(**{n: None}) == f(**{n: _heads(lib, p=None)}) == NULL, n
        assert f(**{n: _heads(lib, p=BUF + 8)}) == f(**{n: _heads(lib, row=516)}) == f(**{n: _heads(lib, head=68)}) == ALIGN, n
        assert f(**{n: _heads(lib, row=56)}) == f(**{n: _heads(lib, row=(1 << 22) + 8)}) == SHAPE, n
    assert f(lse=None) == NULL and f(lse=BUF + 2) == ALIGN
    # the result: no two values at one place
    assert f(o=_heads(lib, head=0)) == f(o=_heads(lib, head=56)) == f(o=_heads(lib, row=128)) == f(o=_heads(lib, row=64, head=199 * 64)) == SHAPE
    assert f(rows_q=0, o=_heads(lib, p=None), q=_heads(lib, p=None), lse=None) == OK
    # few rows over many: chunks, for a second launch
    few = {"rows_q": 2, "rows_k": 2 * 4096}
    need = lib.raw.sr_attention_fwd_workspace_bytes(_shape(lib, **few))
    assert need and f(ws=None, **few) == f(n=need - 1, **few) == WORKSPACE and f(ws=BUF + 8, **few) == ALIGN

    def b(dq=_heads(lib), dk=_heads(lib), dv=_heads(lib), do=_heads(lib), q=_heads(lib), k=_heads(lib), v=_heads(lib), o=_heads(lib), lse=BUF, ws=BUF, n=1 << 40,
          **other):
        return lib.raw.sr_attention_bwd(dq, dk, dv, do, q, k, v, o, lse, _shape(lib, **other), ws, n, None)

    for other, want in BAD_SHAPES:
        assert b(**other) == want, other
    for n in ("dq", "dk", "dv", "do", "q", "k", "v", "o"):
        assert b(**{n: None}) == b(**{n: _heads(lib, p=None)}) == NULL and b(**{n: _heads(lib, p=BUF + 4)}) == ALIGN and b(**{n: _heads(lib, row=48)}) == SHAPE, n
    for n in ("dq", "dk", "dv"):
        assert b(**{n: _heads(lib, head=0)}) == SHAPE
    assert b(lse=None) == NULL and b(lse=BUF + 1) == ALIGN
    need = lib.raw.sr_attention_bwd_workspace_bytes(_shape(lib))
    assert need and b(ws=None) == b(n=need - 1) == WORKSPACE and b(ws=BUF + 4) == ALIGN
    none = _heads(lib, p=None)
    assert b(rows_q=0, rows_k=0, dq=none, dk=none, dv=none, do=none, q=none, k=none, v=none, o=none, lse=None, ws=None, n=0) == OK


def test_embedding(lib):
    def f(out=BUF, od=0, t=BUF, td=0, ids=BUF, size=8, M=4, V=10, D=64, scale=1.0):
        return lib.raw.sr_embedding_fwd(out, od, t, td, ids, size, M, V, D, scale, None)

    assert f(od=2) == f(td=-1) == f(size=2) == f(scale=float("nan")) == f(scale=float("inf")) == FORMAT
    assert f(V=0) == f(D=0) == f(M=1 << 31) == f(V=1 << 31) == SHAPE and f(D=12) == ALIGN
    assert f(out=None) == f(t=None) == f(ids=None) == NULL
    assert f(out=BUF + 8) == f(t=BUF + 4) == f(ids=BUF + 4) == f(ids=BUF + 2, size=4) == ALIGN
    assert f(M=0, out=None, t=None, ids=None) == OK

    def b(dt=BUF, dy=BUF, d=0, ids=BUF, size=8, M=4, V=10, D=64, scale=1.0, pad=-1, beta=0.0, ws=BUF, n=1 << 40):
        return lib.raw.sr_embedding_bwd(dt, dy, d, ids, size, M, V, D, scale, pad, beta, ws, n, None)

    assert b(d=2) == b(size=1) == b(scale=float("nan")) == b(pad=-2) == FORMAT and b(beta=0.5) == UNSUPPORTED
    assert b(V=0) == b(D=0) == b(M=1 << 31) == b(D=1 << 23) == b(M=1 << 29, D=1 << 20) == SHAPE and b(D=20) == ALIGN
    assert b(dt=None) == b(dy=None) == b(ids=None) == NULL and b(dt=BUF + 8) == b(dy=BUF + 4) == b(ids=BUF + 4) == ALIGN
    need = lib.raw.sr_embedding_bwd_workspace_bytes(4, 64)
    assert need and b(ws=None) == b(n=need - 1) == WORKSPACE and b(ws=BUF + 4) == ALIGN
    assert lib.raw.sr_embedding_bwd_workspace_bytes(0, 64) == 0


def test_adamw(lib):
    def t(w=0x10000, g=0x20000, m=0x30000, v=0x40000, ms=0x50000, vs=0x60000, n=100, counter=0, decay=0.0, wd=0, gd=0, kind=0):
        return lib.srq_adamw_tensor(w, g, m, v, ms, vs, n, counter, decay, wd, gd, kind)

    def f(*ts, count=None, b1=0.9, b2=0.95, lr=1e-3, eps=1e-8, rnd=0, reserved=0, step=1, ld=None, sd=None, cd=None):
        o = lib.srq_adamw(b1, b2, lr, eps, rnd, reserved, step, 0, ld, sd, cd)
        return lib.raw.sr_adamw((lib.srq_adamw_tensor * max(len(ts), 1))(*ts), len(ts) if count is None else count, o, None)

    nan, inf = float("nan"), float("inf")
    assert lib.raw.sr_adamw(None, 1, lib.srq_adamw(0.9, 0.9, 1.0, 0.0, 0, 0, 1, 0, None, None, None), None) == NULL
    assert lib.raw.sr_adamw((lib.srq_adamw_tensor * 1)(t()), 1, None, None) == NULL
    assert f(t(), count=-1) == SHAPE and f(t(n=1 << 41)) == SHAPE
    assert f(t(), b1=1.0) == f(t(), b1=-0.1) == f(t(), b2=nan) == f(t(), lr=inf) == f(t(), eps=-1.0) == f(t(), eps=nan) == f(t(), rnd=2) == FORMAT
    assert f(t(), reserved=1) == f(t(), step=0) == f(t(decay=nan)) == f(t(wd=2)) == f(t(gd=-1)) == f(t(kind=9)) == f(t(kind=-1)) == FORMAT
    assert f(t(kind=4)) == f(t(kind=1)) == UNSUPPORTED
    for n in ("w", "g", "m", "v"):
        assert f(t(**{n: None})) == NULL and f(t(**{n: 0x70008})) == ALIGN
    assert f(t(kind=3, ms=None)) == f(t(kind=3, vs=None)) == NULL
    assert f(t(), ld=BUF + 2) == f(t(), sd=BUF + 4) == f(t(), cd=BUF + 4) == ALIGN
    # memory that two tensors, or two parts of one, would write
    far = {"w": 0x110000, "g": 0x120000, "m": 0x130000, "v": 0x140000}
    assert f(t(), t()) == f(t(), t(**far | {"w": 0x10000 + 384})) == f(t(), t(**far | {"m": 0x40000})) == f(t(m=0x10000)) == UNSUPPORTED
    far |= {"ms": 0x150000, "vs": 0x160000, "kind": 3}
    assert f(t(kind=3), t(**far | {"vs": 0x60000})) == f(t(kind=3, ms=0x30000)) == f(t(kind=3, ms=0x60000)) == UNSUPPORTED
    assert f() == f(t(n=0, w=None, g=None, m=None, v=None)) == OK


def test_the_bindings_refuse_tensors_that_do_not_fit(lib):
    q = torch.zeros((4, 2, 64), dtype=torch.bfloat16)
    with pytest.raises(RuntimeError):
        lib.sr_attention_fwd(q, q, q)  # host memory
    with pytest.raises(TypeError):
        lib.sr_attention_fwd(q.float(), q, q)
    with pytest.raises(ValueError):
        lib.sr_attention_fwd(q, q, q, offsets=torch.zeros(3, dtype=torch.int64))
    with pytest.raises(ValueError):
        lib.sr_attention_fwd(q, q, q, sequences=2, lengths_k=torch.zeros(3, dtype=torch.int32))
    with pytest.raises(TypeError):
        lib.sr_embedding_fwd(torch.zeros((4, 8)), torch.zeros(3))
    with pytest.raises(ValueError):
        lib.AdamWTensor.zeros(torch.zeros(4), torch.zeros(5)).c()
    with pytest.raises(ValueError):
        lib.AdamWTensor.zeros(torch.zeros(4), torch.zeros(4), bits=16)
    with pytest.raises(TypeError):
        lib.AdamWTensor(torch.zeros(4), torch.zeros(4), torch.zeros(4, dtype=torch.uint8), torch.zeros(4)).c()
    t = lib.AdamWTensor.zeros(torch.zeros(200), torch.zeros(200), bits=8)
    t.v_scales = t.v_scales[:1]
    with pytest.raises(ValueError):
        t.c()
