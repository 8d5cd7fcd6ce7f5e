"""Thin ctypes binding over libsrq.so: same names as include/srq.h, argument marshalling only.

PyTorch is used for device memory and streams; every step of the path runs in the HIP
kernels.  There is no fallback: if the library is not built this module raises on import.
"""
import ctypes as C
import os

import torch  # first: its HIP runtime must be the one the library binds to

HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(HERE, "libsrq.so")

OK, ERR_WORKSPACE = 0, -5
F32, BF16 = 0, 1
NONE, INT8, INT4, E4M3, E5M2, E4M2, E4M1, E4M0 = 0, 1, 2, 3, 4, 5, 6, 7
SR, RTN = 0, 1
OP_FWD, OP_BWD_DATA, OP_BWD_WEIGHT, OP_BWD, OP_FWD_STASH, OP_BWD_STASHED = 0, 1, 2, 3, 4, 5
OP_FWD_WEIGHT_ONLY, OP_BWD_DATA_WEIGHT_ONLY = 6, 7
FLAG_F8_PIPELINE, FLAG_COUNTER_DEV, FLAG_QUANTIZE_ONCE = 1, 2, 4
PHASE_QUANTIZE, PHASE_PRODUCT, PHASE_BOTH = 1, 2, 3
ROWS, TURNED, BOTH = 1, 2, 3  # layouts of a block-scaled matrix that sr_block_quantize writes
ACT_SILU, ACT_GELU = 0, 1
KIND_NAMES = {INT8: "int8", INT4: "int4", E4M3: "e4m3", E5M2: "e5m2", E4M2: "e4m2", E4M1: "e4m1", E4M0: "e4m0"}
QMAX = {INT8: 127.0, INT4: 7.0, E4M3: 448.0, E5M2: 57344.0, E4M2: 448.0, E4M1: 384.0, E4M0: 256.0}


class srq_quant(C.Structure):
    _fields_ = [("kind", C.c_int32), ("round", C.c_int32), ("scale", C.c_float),
                ("flags", C.c_uint32), ("scale_dev", C.c_void_p), ("seed", C.c_uint64),
                ("counter_offset", C.c_uint64)]


class srq_absmax_req(C.Structure):
    _fields_ = [("x", C.c_void_p), ("dtype", C.c_int32), ("kind", C.c_int32), ("n", C.c_size_t),
                ("scale_out_dev", C.c_void_p)]


class srq_heads(C.Structure):
    _fields_ = [("p", C.c_void_p), ("row", C.c_size_t), ("head", C.c_size_t)]


class srq_attention(C.Structure):
    _fields_ = [(n, C.c_size_t) for n in ("sequences", "rows_q", "rows_k", "heads_q", "heads_kv", "dim")] + \
               [(n, C.c_void_p) for n in ("offsets_q", "offsets_k", "lengths_k")] + [("scale", C.c_float), ("causal", C.c_int32)]


class srq_adamw_tensor(C.Structure):
    _fields_ = [(n, C.c_void_p) for n in ("w", "g", "m", "v", "m_scales", "v_scales")] + \
               [("n", C.c_size_t), ("counter_offset", C.c_uint64), ("weight_decay", C.c_float), ("w_dtype", C.c_int32), ("g_dtype", C.c_int32),
                ("state_kind", C.c_int32)]


class srq_adamw(C.Structure):
    _fields_ = [("beta1", C.c_double), ("beta2", C.c_double), ("lr", C.c_float), ("eps", C.c_float), ("round", C.c_int32), ("reserved", C.c_uint32),
                ("step", C.c_uint64), ("seed", C.c_uint64), ("lr_dev", C.c_void_p), ("step_dev", C.c_void_p), ("counter_dev", C.c_void_p)]


if not os.path.exists(LIB_PATH):
    raise ImportError(
        f"{LIB_PATH} is missing: build it with `python -m paper_2511_00874_amd.build` "
        "(there is no CPU fallback)")
_lib = C.CDLL(LIB_PATH)

_vp, _sz, _qp = C.c_void_p, C.c_size_t, C.POINTER(srq_quant)
_lib.sr_absmax_scale.argtypes = [_vp, _vp, C.c_int, _sz, C.c_int, _vp]
_lib.sr_absmax_scales.argtypes = [C.POINTER(srq_absmax_req), C.c_int, _vp, _sz, _vp]
_lib.sr_absmax_workspace_bytes.argtypes = [C.POINTER(srq_absmax_req), C.c_int]
_lib.sr_absmax_workspace_bytes.restype = _sz
_lib.sr_quantize.argtypes = [_vp, _vp, C.c_int, _sz, _sz, C.c_int, _qp, _vp]
_lib.sr_gemm_codes.argtypes = [_vp, _vp, C.c_int, _vp, C.c_int, _sz, _sz, _sz, C.c_float, C.c_float,
                               _vp, _sz, _vp]
_lib.sr_gemm_workspace_bytes.argtypes = [_sz, _sz, _sz]
_lib.sr_gemm_workspace_bytes.restype = _sz
_lib.sr_gemm_bf16.argtypes = [_vp, _vp, _vp, _sz, _sz, _sz, C.c_float, C.c_float, _vp, _sz, _vp]
_lib.sr_gemm_bf16_workspace_bytes.argtypes = [_sz, _sz, _sz]
_lib.sr_gemm_bf16_workspace_bytes.restype = _sz
_lib.sr_gemm_e5m2.argtypes = _lib.sr_gemm_bf16.argtypes
_lib.sr_gemm_e5m2_workspace_bytes.argtypes = [_sz, _sz, _sz]
_lib.sr_gemm_e5m2_workspace_bytes.restype = _sz
_lib.sr_linear_fwd.argtypes = [_vp, _vp, C.c_int, _vp, C.c_int, _sz, _sz, _sz, _qp, _qp, _vp, _sz, _vp]
_lib.sr_linear_bwd_data.argtypes = _lib.sr_linear_fwd.argtypes
_lib.sr_linear_fwd_static.argtypes = [_vp, _vp, C.c_int, _vp, C.c_int, _sz, _sz, _sz, _qp, _qp, _vp]
_lib.sr_linear_fwd_fused.argtypes = _lib.sr_linear_fwd_static.argtypes
_lib.sr_linear_fwd_phase.argtypes = [_vp, _vp, C.c_int, _vp, C.c_int, _sz, _sz, _sz, _qp, _qp, _vp, _sz, C.c_int, _vp]
_lib.sr_linear_fwd_static_limit.argtypes = []
_lib.sr_linear_fwd_static_limit.restype = _sz
_lib.sr_linear_bwd_weight.argtypes = [_vp, _vp, C.c_int, _vp, C.c_int, _sz, _sz, _sz, _qp, _qp,
                                      C.c_float, _vp, _sz, _vp]
_lib.sr_linear_bwd.argtypes = [_vp, _vp, _vp, C.c_int, _vp, C.c_int, _vp, C.c_int, _sz, _sz, _sz, _qp, _qp, _qp,
                               C.c_float, _vp, _sz, _vp]
_lib.sr_linear_bwd_phase.argtypes = [_vp, _vp, _vp, C.c_int, _vp, C.c_int, _vp, C.c_int, _sz, _sz, _sz, _qp, _qp, _qp,
                                     C.c_float, _vp, _sz, C.c_int, _vp]
_lib.sr_linear_workspace_bytes.argtypes = [C.c_int, _sz, _sz, _sz]
_lib.sr_linear_workspace_bytes.restype = _sz
_lib.sr_linear_stash_bytes.argtypes = [_sz, _sz, _sz]
_lib.sr_linear_stash_bytes.restype = _sz
_lib.sr_linear_fwd_stash.argtypes = [_vp, _vp, C.c_int, _vp, C.c_int, _sz, _sz, _sz, _qp, _qp, _qp, _qp, _vp, _sz, _vp, _sz, _vp]
_lib.sr_linear_bwd_stashed.argtypes = [_vp, _vp, _vp, C.c_int, _sz, _sz, _sz, _qp, _qp, _qp, _vp, _sz, C.c_float, _vp, _sz, _vp]
_lib.sr_linear_fwd_stash_phase.argtypes = [_vp, _vp, C.c_int, _vp, C.c_int, _sz, _sz, _sz, _qp, _qp, _qp, _qp, _vp, _sz, _vp, _sz,
                                           C.c_int, _vp]
_lib.sr_linear_bwd_stashed_phase.argtypes = [_vp, _vp, _vp, C.c_int, _sz, _sz, _sz, _qp, _qp, _qp, _vp, _sz, C.c_float, _vp, _sz,
                                             C.c_int, _vp]
_lib.sr_update_bf16.argtypes = [_vp, _vp, C.c_float, _sz, C.c_int, C.c_uint64, C.c_uint64, _vp]
_lib.sr_block_pitch.argtypes = _lib.sr_block_scale_pitch.argtypes = [_sz]
_lib.sr_block_quantize.argtypes = [_vp, _sz, _vp, _vp, _sz, _vp, _vp, C.c_int, _sz, _sz, _qp, _vp]
_lib.sr_block_turn.argtypes = [_vp, _sz, _vp, _vp, _sz, _vp, C.c_int, _sz, _sz, _qp, _vp]
_lib.sr_block_restore.argtypes = [_vp, C.c_int, _vp, _sz, _vp, C.c_int, _sz, _sz, _vp]
_lib.sr_gemm_blocks.argtypes = [_vp, C.c_int, _vp, _sz, _vp, C.c_int, _vp, _sz, _vp, C.c_int, _sz, _sz, _sz, C.c_float, C.c_float,
                                C.c_uint32, _vp, _sz, _vp]
_lib.sr_gemm_blocks_workspace_bytes.argtypes = [_sz, _sz, _sz, C.c_uint32]
_lib.sr_gated_fwd.argtypes = [_vp, _vp, _vp, _vp, _vp, _sz, _vp, _vp, _sz, _vp, _sz, _sz, _sz, C.c_int, _qp, _qp, C.c_uint32, _vp, _sz, _vp]
_lib.sr_gated_fwd_workspace_bytes.argtypes = [_sz, _sz, _sz, C.c_uint32]
_lib.sr_gated_bwd.argtypes = [_vp, _vp, _vp, _sz, _vp, _vp, C.c_int, _vp, _vp, _sz, _sz, C.c_int, _qp, _vp]
_lib.sr_rmsnorm_fwd.argtypes = [_vp, _sz, _vp, _vp, _vp, _vp, _vp, _vp, C.c_int, _sz, _sz, C.c_float, _qp, _vp]
_lib.sr_rmsnorm_bwd.argtypes = [_vp, _vp, _vp, _vp, _vp, _vp, _vp, C.c_int, _sz, _sz, C.c_float, _vp, _sz, _vp]
_lib.sr_rmsnorm_bwd_workspace_bytes.argtypes = [_sz, _sz]
_hp, _ap = C.POINTER(srq_heads), C.POINTER(srq_attention)
_lib.sr_attention_fwd.argtypes = [_hp, _vp, _hp, _hp, _hp, _ap, _vp, _sz, _vp]
_lib.sr_attention_bwd.argtypes = [_hp] * 8 + [_vp, _ap, _vp, _sz, _vp]
_lib.sr_attention_fwd_workspace_bytes.argtypes = _lib.sr_attention_bwd_workspace_bytes.argtypes = [_ap]
_lib.sr_embedding_fwd.argtypes = [_vp, C.c_int, _vp, C.c_int, _vp, C.c_int, _sz, _sz, _sz, C.c_float, _vp]
_lib.sr_embedding_bwd.argtypes = [_vp, _vp, C.c_int, _vp, C.c_int, _sz, _sz, _sz, C.c_float, C.c_int64, C.c_float, _vp, _sz, _vp]
_lib.sr_embedding_bwd_workspace_bytes.argtypes = [_sz, _sz]
_lib.sr_adamw.argtypes = [C.POINTER(srq_adamw_tensor), C.c_int, C.POINTER(srq_adamw), _vp]
for _n in ("sr_block_pitch", "sr_block_scale_pitch", "sr_gemm_blocks_workspace_bytes", "sr_gated_fwd_workspace_bytes",
           "sr_rmsnorm_bwd_workspace_bytes", "sr_attention_fwd_workspace_bytes", "sr_attention_bwd_workspace_bytes",
           "sr_embedding_bwd_workspace_bytes"):
    getattr(_lib, _n).restype = _sz
_lib.sr_status_string.argtypes = [C.c_int]
_lib.sr_status_string.restype = C.c_char_p
for _n in ("sr_linear_fwd_static", "sr_linear_fwd_fused", "sr_linear_fwd_phase", "sr_linear_bwd_phase", "sr_absmax_scale", "sr_absmax_scales", "sr_quantize", "sr_gemm_codes", "sr_gemm_bf16", "sr_gemm_e5m2", "sr_linear_fwd", "sr_linear_bwd_data",
           "sr_linear_bwd_weight", "sr_linear_bwd", "sr_update_bf16", "sr_linear_fwd_stash", "sr_linear_bwd_stashed",
           "sr_linear_fwd_stash_phase", "sr_linear_bwd_stashed_phase", "sr_block_quantize", "sr_block_turn", "sr_block_restore",
           "sr_gemm_blocks", "sr_gated_fwd", "sr_gated_bwd", "sr_rmsnorm_fwd", "sr_rmsnorm_bwd", "sr_attention_fwd", "sr_attention_bwd",
           "sr_embedding_fwd", "sr_embedding_bwd", "sr_adamw"):
    getattr(_lib, _n).restype = C.c_int

EXPORTS = ["sr_absmax_scale", "sr_absmax_scales", "sr_absmax_workspace_bytes", "sr_quantize", "sr_gemm_codes", "sr_gemm_workspace_bytes", "sr_gemm_bf16", "sr_gemm_bf16_workspace_bytes", "sr_gemm_e5m2", "sr_gemm_e5m2_workspace_bytes",
           "sr_linear_fwd", "sr_linear_bwd_data", "sr_linear_bwd_weight", "sr_linear_bwd",
           "sr_linear_workspace_bytes", "sr_linear_stash_bytes", "sr_linear_fwd_stash", "sr_linear_bwd_stashed",
           "sr_update_bf16", "sr_status_string", "sr_linear_fwd_static", "sr_linear_fwd_static_limit",
           "sr_linear_fwd_fused", "sr_linear_fwd_phase", "sr_linear_bwd_phase", "sr_linear_fwd_stash_phase",
           "sr_linear_bwd_stashed_phase",
           "sr_block_pitch", "sr_block_scale_pitch", "sr_block_quantize", "sr_block_turn", "sr_block_restore", "sr_gemm_blocks",
           "sr_gemm_blocks_workspace_bytes", "sr_gated_fwd", "sr_gated_fwd_workspace_bytes", "sr_gated_bwd", "sr_rmsnorm_fwd", "sr_rmsnorm_bwd",
           "sr_rmsnorm_bwd_workspace_bytes", "sr_attention_fwd", "sr_attention_fwd_workspace_bytes", "sr_attention_bwd",
           "sr_attention_bwd_workspace_bytes", "sr_embedding_fwd", "sr_embedding_bwd", "sr_embedding_bwd_workspace_bytes", "sr_adamw"]

raw = _lib  # the C entry points themselves, for tests of the error paths


class SrqError(RuntimeError):
    def __init__(self, status):
        self.status = status
        super().__init__(f"srq status {status}: {_lib.sr_status_string(status).decode()}")


def _check(status):
    if status != OK:
        raise SrqError(status)


def status_string(status):
    return _lib.sr_status_string(status).decode()


def _dtype(t):
    if t.dtype == torch.float32:
        return F32
    if t.dtype == torch.bfloat16:
        return BF16
    raise TypeError("source tensors must be float32 or bfloat16")


def _dev(t):
    if not t.is_cuda:
        raise RuntimeError("srq needs device tensors: there is no CPU path")
    if not t.is_contiguous():
        raise ValueError("tensors must be dense row-major")
    return t.data_ptr()


# The handle of the current device's current stream.  torch.cuda.current_stream().cuda_stream makes a stream object and
# looks up the device for it (4 us a call, as much as a kernel launch); the raw handle comes without either where this torch
# has the two calls.
if hasattr(torch._C, "_cuda_getDevice") and hasattr(torch._C, "_cuda_getCurrentRawStream"):
    _current_device, _current_raw_stream = torch._C._cuda_getDevice, torch._C._cuda_getCurrentRawStream

    def _stream():
        return _current_raw_stream(_current_device())
else:
    _current_device = torch.cuda.current_device

    def _stream():
        return torch.cuda.current_stream().cuda_stream


class Quant:
    """One quantizer (Delta, eps): format, per-tensor scale (float or 1-element device tensor),
    rounding mode and position in the Philox stream."""

    def __init__(self, kind, scale, seed=0, counter_offset=0, round_mode=SR, flags=0):
        self.kind, self.scale, self.seed = kind, scale, seed
        self.counter_offset, self.round_mode, self.flags = counter_offset, round_mode, flags

    def c(self):
        scale, offset, flags = self.scale, self.counter_offset, self.flags
        if isinstance(scale, torch.Tensor):
            value, scale_dev = 0.0, _dev(scale)
        else:
            value, scale_dev = float(scale), None
        if isinstance(offset, torch.Tensor):
            # a 1-element int64 device tensor: the kernels read the offset when they run
            assert offset.dtype == torch.int64 and offset.numel() == 1
            flags |= FLAG_COUNTER_DEV
            offset = _dev(offset)
        else:
            offset &= 2**64 - 1
        return srq_quant(self.kind, self.round_mode, value, flags, scale_dev, self.seed & (2**64 - 1), offset)


def _q(q):
    """A quantizer as the C entry points take it; one that is marshalled already stays as it is."""
    return q if type(q) is srq_quant else q.c()


def sr_absmax_scale(x, kind, out=None):
    """Device tensor holding max|x| / Qmax(kind) (1 if x is all zero)."""
    if out is None:
        out = torch.empty(1, dtype=torch.float32, device=x.device)
    _check(_lib.sr_absmax_scale(_dev(out), _dev(x), _dtype(x), x.numel(), kind, _stream()))
    return out


class AbsmaxBatch:
    """Prepared sr_absmax_scales call: requests [(tensor, kind, out 1-element tensor)], marshalled once."""

    def __init__(self, requests):
        self.keep = requests
        self.count = len(requests)
        self.reqs = (srq_absmax_req * self.count)()
        for r, (x, kind, out) in zip(self.reqs, requests):
            r.x, r.dtype, r.kind, r.n, r.scale_out_dev = _dev(x), _dtype(x), kind, x.numel(), _dev(out)
        need = _lib.sr_absmax_workspace_bytes(self.reqs, self.count)
        self.ws = torch.empty(max(need, 4), dtype=torch.uint8, device=requests[0][0].device)

    def run(self):
        _check(_lib.sr_absmax_scales(self.reqs, self.count, _dev(self.ws), self.ws.numel(), _stream()))


def sr_absmax_scales(requests):
    """requests: [(tensor, kind, out 1-element device tensor)]; all scales in two launches."""
    AbsmaxBatch(requests).run()


def absmax_scales(pairs):
    """The scales of [(tensor, kind)] in two launches: one tensor that holds them in order (a view of its own for each
    costs as much as a launch)."""
    count = len(pairs)
    out = torch.empty(count, dtype=torch.float32, device=pairs[0][0].device)
    at = _dev(out)
    reqs = (srq_absmax_req * count)(*[(_dev(x), _dtype(x), kind, x.numel(), at + 4 * i) for i, (x, kind) in enumerate(pairs)])
    need = _lib.sr_absmax_workspace_bytes(reqs, count)
    ws = torch.empty(max(need, 4), dtype=torch.uint8, device=out.device)
    _check(_lib.sr_absmax_scales(reqs, count, ws.data_ptr(), ws.numel(), _stream()))
    return out


def sr_linear_stash_bytes(M, N, K):
    return _lib.sr_linear_stash_bytes(M, N, K)


def sr_linear_fwd_stash(A, W, qA, qW, qA_bwd, qW_bwd, stash=None, out=None, workspace=None, phase=PHASE_BOTH):
    """Alg. 1 that also saves Q(A; qA_bwd)^T and Q(W; qW_bwd)^T in code form: returns (Y, stash).
    `phase`: the quantizer launch, the product, or both (the halves take the same out, stash, workspace)."""
    M, K = A.shape
    N = W.shape[0]
    if out is None:
        out = torch.empty((M, N), dtype=torch.float32, device=A.device)
    if stash is None:
        stash = torch.empty(sr_linear_stash_bytes(M, N, K), dtype=torch.uint8, device=A.device)
    ws = _ws(OP_FWD_STASH, M, N, K, workspace, A.device)
    _check(_lib.sr_linear_fwd_stash_phase(_dev(out), _dev(A), _dtype(A), _dev(W), _dtype(W), M, N, K, _q(qA),
                                          _q(qW), _q(qA_bwd), _q(qW_bwd), _dev(stash),
                                          stash.numel(), _dev(ws), ws.numel(), phase, _stream()))
    return out, stash


def sr_linear_bwd_stashed(dY, stash, K, qdY, qW, qA, out_dA=None, out_dW=None, beta=0.0, workspace=None,
                          phase=PHASE_BOTH):
    """Alg. 2 from the stash of sr_linear_fwd_stash: (dA, dW); only dY is read.  `phase` as above."""
    M, N = dY.shape
    if out_dA is None:
        out_dA = torch.empty((M, K), dtype=torch.float32, device=dY.device)
    if out_dW is None:
        out_dW = torch.empty((N, K), dtype=torch.float32, device=dY.device)
    ws = _ws(OP_BWD_STASHED, M, N, K, workspace, dY.device)
    _check(_lib.sr_linear_bwd_stashed_phase(_dev(out_dA), _dev(out_dW), _dev(dY), _dtype(dY), M, N, K, _q(qdY),
                                            _q(qW), _q(qA), _dev(stash), stash.numel(), beta, _dev(ws),
                                            ws.numel(), phase, _stream()))
    return out_dA, out_dW


def sr_update_bf16(w, g, eta, seed=0, counter_offset=0, round_mode=SR):
    """Eq. 10 in place: w (bfloat16 tensor) <- Q(w - eta * g), g float32 of the same size."""
    assert w.dtype == torch.bfloat16 and g.dtype == torch.float32 and w.numel() == g.numel()
    assert w.is_contiguous() and g.is_contiguous()
    _check(_lib.sr_update_bf16(_dev(w), _dev(g), float(eta), w.numel(), round_mode, seed, counter_offset, _stream()))
    return w


def sr_quantize(x, q, transpose_out=False, out=None):
    """Codes of x (2-D, or 1-D treated as one row): uint8, packed two per byte for INT4."""
    rows, cols = (1, x.numel()) if x.dim() == 1 else x.shape
    n = rows * cols
    nbytes = n // 2 if q.kind == INT4 else n
    if out is None:
        out = torch.empty(max(nbytes, 1), dtype=torch.uint8, device=x.device)[:nbytes]
    _check(_lib.sr_quantize(_dev(out), _dev(x), _dtype(x), rows, cols, int(bool(transpose_out)),
                            _q(q), _stream()))
    return out


def sr_gemm_workspace_bytes(P, Q, R):
    return _lib.sr_gemm_workspace_bytes(P, Q, R)


def sr_gemm_codes(X, kindX, Z, kindZ, alpha=1.0, out=None, beta=0.0, workspace=None):
    """out (P,Q) = alpha * X (P,R) . Z (Q,R)^T on codes, one byte per element."""
    P, R = X.shape
    Q = Z.shape[0]
    if out is None:
        out = torch.empty((P, Q), dtype=torch.float32, device=X.device)
    need = sr_gemm_workspace_bytes(P, Q, R)
    if workspace is None and need:
        workspace = torch.empty(need, dtype=torch.uint8, device=X.device)
    _check(_lib.sr_gemm_codes(_dev(out), _dev(X), kindX, _dev(Z), kindZ, P, Q, R, alpha, beta,
                              _dev(workspace) if workspace is not None else None,
                              workspace.numel() if workspace is not None else 0, _stream()))
    return out


def sr_gemm_bf16(X, Z, alpha=1.0, out=None, beta=0.0, workspace=None):
    """out (P,Q) = alpha * X (P,R) . Z (Q,R)^T for bfloat16 operands."""
    P, R = X.shape
    Q = Z.shape[0]
    if out is None:
        out = torch.empty((P, Q), dtype=torch.float32, device=X.device)
    need = _lib.sr_gemm_bf16_workspace_bytes(P, Q, R)
    if workspace is None and need:
        workspace = torch.empty(need, dtype=torch.uint8, device=X.device)
    _check(_lib.sr_gemm_bf16(_dev(out), _dev(X), _dev(Z), P, Q, R, alpha, beta,
                             _dev(workspace) if workspace is not None else None,
                             workspace.numel() if workspace is not None else 0, _stream()))
    return out


def sr_gemm_e5m2(X, Z, alpha=1.0, beta=0.0, out=None, workspace=None):
    """out (P,Q) = alpha * X Z^T for uint8 matrices of E5M2 codes: exact products, binary32 sums."""
    P, R = X.shape
    Q = Z.shape[0]
    if out is None:
        out = torch.empty((P, Q), dtype=torch.float32, device=X.device)
    need = _lib.sr_gemm_e5m2_workspace_bytes(P, Q, R)
    if workspace is None and need:
        workspace = torch.empty(need, dtype=torch.uint8, device=X.device)
    _check(_lib.sr_gemm_e5m2(_dev(out), _dev(X), _dev(Z), P, Q, R, alpha, beta,
                             _dev(workspace) if workspace is not None else None,
                             workspace.numel() if workspace is not None else 0, _stream()))
    return out


def sr_linear_workspace_bytes(op, M, N, K):
    return _lib.sr_linear_workspace_bytes(op, M, N, K)


def _ws(op, M, N, K, workspace, device):
    if workspace is None:
        workspace = torch.empty(sr_linear_workspace_bytes(op, M, N, K), dtype=torch.uint8, device=device)
    return workspace


def sr_linear_fwd(A, W, qA, qW, out=None, workspace=None, phase=None):
    """Alg. 1: Y (M,N) = Q(A) Q(W)^T, A (M,K), W (N,K).  qA = Quant(NONE, 1.0): A as it is
    (weight-only objective, Sec. 3.2).  phase = PHASE_QUANTIZE / PHASE_PRODUCT: one half of the call
    (sr_linear_fwd_phase); `out` and `workspace` are then required."""
    M, K = A.shape
    N = W.shape[0]
    if phase is not None:
        _check(_lib.sr_linear_fwd_phase(_dev(out), _dev(A), _dtype(A), _dev(W), _dtype(W), M, N, K, _q(qA),
                                        _q(qW), _dev(workspace), workspace.numel(), phase, _stream()))
        return out
    if out is None:
        out = torch.empty((M, N), dtype=torch.float32, device=A.device)
    ws = _ws(OP_FWD_WEIGHT_ONLY if qA.kind == NONE else OP_FWD, M, N, K, workspace, A.device)
    _check(_lib.sr_linear_fwd(_dev(out), _dev(A), _dtype(A), _dev(W), _dtype(W), M, N, K,
                              _q(qA), _q(qW), _dev(ws), ws.numel(), _stream()))
    return out


def sr_linear_fwd_static(A, W, qA, qW, out):
    """sr_linear_fwd with the library's static scratch array as workspace; `out` is required (this
    call is for callers that may not allocate)."""
    M, K = A.shape
    N = W.shape[0]
    _check(_lib.sr_linear_fwd_static(_dev(out), _dev(A), _dtype(A), _dev(W), _dtype(W), M, N, K,
                                     _q(qA), _q(qW), _stream()))
    return out


def sr_linear_fwd_fused(A, W, qA, qW, out=None):
    """Alg. 1 with the quantizers inside the product kernel (no workspace, no codes in memory)."""
    M, K = A.shape
    N = W.shape[0]
    if out is None:
        out = torch.empty((M, N), dtype=torch.float32, device=A.device)
    _check(_lib.sr_linear_fwd_fused(_dev(out), _dev(A), _dtype(A), _dev(W), _dtype(W), M, N, K,
                                    _q(qA), _q(qW), _stream()))
    return out


def sr_linear_bwd_data(dY, W, qdY, qW, out=None, workspace=None):
    """Alg. 2: dA (M,K) = Q(dY) Q(W), dY (M,N), W (N,K).  qdY = Quant(NONE, 1.0): dY as it is."""
    M, N = dY.shape
    K = W.shape[1]
    if out is None:
        out = torch.empty((M, K), dtype=torch.float32, device=dY.device)
    ws = _ws(OP_BWD_DATA_WEIGHT_ONLY if qdY.kind == NONE else OP_BWD_DATA, M, N, K, workspace, dY.device)
    _check(_lib.sr_linear_bwd_data(_dev(out), _dev(dY), _dtype(dY), _dev(W), _dtype(W), M, N, K,
                                   _q(qdY), _q(qW), _dev(ws), ws.numel(), _stream()))
    return out


def sr_linear_bwd_weight(dY, A, qdY, qA, out=None, beta=0.0, workspace=None):
    """Alg. 2: dW (N,K) = beta * dW + Q(dY)^T Q(A), dY (M,N), A (M,K)."""
    M, N = dY.shape
    K = A.shape[1]
    if out is None:
        out = torch.empty((N, K), dtype=torch.float32, device=dY.device)
    ws = _ws(OP_BWD_WEIGHT, M, N, K, workspace, dY.device)
    _check(_lib.sr_linear_bwd_weight(_dev(out), _dev(dY), _dtype(dY), _dev(A), _dtype(A), M, N, K,
                                     _q(qdY), _q(qA), beta, _dev(ws), ws.numel(),
                                     _stream()))
    return out


def sr_linear_bwd(dY, W, A, qdY, qW, qA, out_dA=None, out_dW=None, beta=0.0, workspace=None, phase=None):
    """Alg. 2 in one call: (dA, dW), with dY read and quantized once.  phase = PHASE_QUANTIZE /
    PHASE_PRODUCT: one half of the call (sr_linear_bwd_phase); outputs and workspace are then required."""
    M, N = dY.shape
    K = W.shape[1]
    if phase is not None:
        _check(_lib.sr_linear_bwd_phase(_dev(out_dA), _dev(out_dW), _dev(dY), _dtype(dY), _dev(W), _dtype(W), _dev(A),
                                        _dtype(A), M, N, K, _q(qdY), _q(qW), _q(qA), beta,
                                        _dev(workspace), workspace.numel(), phase, _stream()))
        return out_dA, out_dW
    if out_dA is None:
        out_dA = torch.empty((M, K), dtype=torch.float32, device=dY.device)
    if out_dW is None:
        out_dW = torch.empty((N, K), dtype=torch.float32, device=dY.device)
    ws = _ws(OP_BWD, M, N, K, workspace, dY.device)
    _check(_lib.sr_linear_bwd(_dev(out_dA), _dev(out_dW), _dev(dY), _dtype(dY), _dev(W), _dtype(W), _dev(A),
                              _dtype(A), M, N, K, _q(qdY), _q(qW), _q(qA), beta,
                              _dev(ws), ws.numel(), _stream()))
    return out_dA, out_dW


# ---- block-scaled matrices -----------------------------------------------------------------------
RTN_E4M3 = Quant(E4M3, 1.0, round_mode=RTN).c()  # nearest, one scale a block: the usual quantizer of a forward pass
_U8 = torch.uint8


class Blocks:
    """A block-scaled matrix (include/srq.h) of `cols` columns: `codes` uint8, a row in each (at least cols bytes rounded up to 16, a multiple of
    16); `exps` uint8, for every 128 columns of a row the biased exponent of their scale, rows of a multiple of 4; both dense.
    kind: E4M3 or E5M2."""

    __slots__ = ("codes", "exps", "kind", "cols")

    def __init__(self, codes, exps, kind, cols):
        self.codes, self.exps, self.kind, self.cols = codes, exps, kind, cols

    @property
    def shape(self):
        return self.codes.shape[0], self.cols

    @staticmethod
    def empty(rows, cols, kind, device):
        """Room for one, rows of codes in whole cache lines."""
        return Blocks(torch.empty((rows, (cols + 127) // 128 * 128), dtype=_U8, device=device),
                      torch.empty((rows, (cols + 511) // 512 * 4), dtype=_U8, device=device), kind, cols)

    def values(self, dtype=torch.float32):
        return sr_block_restore(self, dtype)


def _blocks(b, rows=None, cols=None):
    """The addresses of a block-scaled matrix's parts and its pitch (codes, pitch, scales); rows, cols: what the call expects of its shape."""
    codes, exps = b.codes, b.exps
    n, pitch = codes.shape
    if (codes.dtype is not _U8 or exps.dtype is not _U8 or pitch & 15 or pitch < b.cols
            or exps.shape != (n, (b.cols + 511) // 512 * 4)):
        raise ValueError("the parts of a block-scaled matrix do not fit together")
    if (rows is not None and n != rows) or (cols is not None and b.cols != cols):
        raise ValueError(f"block-scaled matrix of {n} x {b.cols} where {rows} x {cols} is wanted")
    return _dev(codes), pitch, _dev(exps)


def _room(b):
    """The same of one that Blocks.empty made."""
    return b.codes.data_ptr(), b.codes.shape[1], b.exps.data_ptr()


def _like(t, shape, dtype, what):
    if t.shape != shape or t.dtype is not dtype:
        raise ValueError(f"{what} must be {tuple(shape)} of {dtype}")
    return _dev(t)


def _scratch(workspace, need, device):
    """(address, bytes) of the caller's workspace, or of one made here if it gave none."""
    if workspace is None:
        if not need:
            return None, 0
        workspace = torch.empty(need, dtype=_U8, device=device)
        return workspace.data_ptr(), need
    return _dev(workspace), workspace.numel() * workspace.element_size()


def sr_block_quantize(x, q, layout=ROWS):
    """x (M, K) in block-scaled form by q (its scale is ignored): along the rows, turned (K, M), or both of them from one pass."""
    M, K = x.shape
    none = (None, 0, None)
    rows = Blocks.empty(M, K, q.kind, x.device) if layout & ROWS else None
    turned = Blocks.empty(K, M, q.kind, x.device) if layout & TURNED else None
    _check(_lib.sr_block_quantize(*(none if rows is None else _room(rows)), *(none if turned is None else _room(turned)), _dev(x), _dtype(x),
                                  M, K, _q(q), _stream()))
    return (rows, turned) if layout == BOTH else rows or turned


def sr_block_turn(b, q=None):
    """A block-scaled matrix (M, K) turned (K, M), blocks along its rows; q: to its format (default: the same, nearest)."""
    M, K = b.shape
    if q is None:
        q = srq_quant(b.kind, RTN, 1.0)
    src = _blocks(b)
    out = Blocks.empty(K, M, q.kind, b.codes.device)
    _check(_lib.sr_block_turn(*_room(out), *src, b.kind, M, K, _q(q), _stream()))
    return out


def sr_block_restore(b, dtype=torch.float32):
    """The values of a block-scaled matrix."""
    src = _blocks(b)
    out = torch.empty(b.shape, dtype=dtype, device=b.codes.device)
    _check(_lib.sr_block_restore(out.data_ptr(), _dtype(out), *src, b.kind, *b.shape, _stream()))
    return out


def sr_gemm_blocks(X, Z, alpha=1.0, beta=0.0, out=None, dtype=torch.float32, f8_pipeline=False, workspace=None):
    """out (P, Q) = alpha * X Z^T (+ out) for block-scaled X (P, R) and Z (Q, R), float32 or bfloat16; f8_pipeline: on the fp8
    matrix pipeline (hardware-rounded group sums, as stated in the header)."""
    R = X.cols
    z = _blocks(Z, cols=R)
    x = _blocks(X)
    P, Q = X.codes.shape[0], Z.codes.shape[0]
    if out is None:
        if beta:
            raise ValueError("beta needs an out to add to")
        out = torch.empty((P, Q), dtype=dtype, device=X.codes.device)
        at = out.data_ptr()
    else:
        at = _like(out, (P, Q), out.dtype, "out")
    flags = FLAG_F8_PIPELINE if f8_pipeline else 0
    need = 0 if workspace is not None else _lib.sr_gemm_blocks_workspace_bytes(P, Q, R, flags)
    ws, size = _scratch(workspace, need, out.device)
    _check(_lib.sr_gemm_blocks(at, _dtype(out), *x, X.kind, *z, Z.kind, P, Q, R, alpha, beta, flags, ws, size, _stream()))
    return out


def sr_gated_fwd(X, W, act=ACT_SILU, qh=None, qgu=None, f8_pipeline=False, workspace=None):
    """H = act(X Wg^T) * (X Wu^T) for block-scaled X (M, K) and W (2F, K) = [Wg; Wu]: (H, checkpoint).  H block-scaled by qh, bfloat16
    if it is None; the checkpoint [G | U] (M, 2F) block-scaled by qgu, None without."""
    M, K = X.codes.shape[0], X.cols
    F = W.codes.shape[0] // 2
    x = _blocks(X)
    w = _blocks(W, 2 * F, K)
    if X.kind != E4M3 or W.kind != E4M3:
        raise ValueError("the gated block takes E4M3")
    dev = X.codes.device
    if qh is None:
        h = torch.empty((M, F), dtype=torch.bfloat16, device=dev)
        at, es = h.data_ptr(), None
    else:
        h = Blocks.empty(M, F, qh.kind, dev)
        at, _, es = _room(h)
    gu, keep, ks = None, None, None
    if qgu is not None:
        gu = Blocks.empty(M, 2 * F, qgu.kind, dev)
        keep, _, ks = _room(gu)
    flags = FLAG_F8_PIPELINE if f8_pipeline else 0
    need = 0 if workspace is not None else _lib.sr_gated_fwd_workspace_bytes(M, F, K, flags)
    ws, size = _scratch(workspace, need, dev)
    _check(_lib.sr_gated_fwd(at, es, keep, ks, *x, *w, M, F, K, act, None if qh is None else _q(qh), None if qgu is None else _q(qgu), flags,
                             ws, size, _stream()))
    return h, gu


def sr_gated_bwd(dH, gu, q, act=ACT_SILU):
    """dZ = [dG | dU] (M, 2F) from dH (M, F) and the checkpoint of sr_gated_fwd, block-scaled by q: (along its rows, turned)."""
    M, F = dH.shape
    at, pitch, es = _blocks(gu, M, 2 * F)
    if gu.kind != E4M3 or pitch != 2 * F:
        raise ValueError("the gated block's checkpoint is E4M3, without gaps")
    rows, turned = Blocks.empty(M, 2 * F, q.kind, dH.device), Blocks.empty(2 * F, M, q.kind, dH.device)
    _check(_lib.sr_gated_bwd(rows.codes.data_ptr(), rows.exps.data_ptr(), *_room(turned), _dev(dH), _dtype(dH), at, es, M, F, act, _q(q),
                             _stream()))
    return rows, turned


def sr_rmsnorm_fwd(x, gamma, eps, residual=None, q=None):
    """h = x + residual, y = h / sqrt(mean(h^2) + eps) * gamma: (y, h, rstd).  y block-scaled by q, or of x's dtype if it is None; h is
    x itself without a residual; gamma float32."""
    M, D = x.shape
    g = _like(gamma, (D,), torch.float32, "gamma")
    dev = x.device
    rstd = torch.empty(M, dtype=torch.float32, device=dev)
    if residual is None:
        h, r, ha = x, None, None
    else:
        r = _like(residual, x.shape, x.dtype, "residual")
        h = torch.empty_like(x)
        ha = h.data_ptr()
    if q is None:
        y = torch.empty_like(x)
        out = y.data_ptr(), 0, None
    else:
        y = Blocks.empty(M, D, q.kind, dev)
        out = _room(y)
    _check(_lib.sr_rmsnorm_fwd(*out, ha, rstd.data_ptr(), _dev(x), r, g, _dtype(x), M, D, eps, None if q is None else _q(q), _stream()))
    return y, h, rstd


def sr_rmsnorm_bwd(dy, h, rstd, gamma, dh=None, out_dx=None, out_dgamma=None, beta=0.0, workspace=None):
    """(dx, dgamma): dx the gradient of x and of the residual, dh (optional) what reaches h from behind the norm;
    dgamma = its sum over the rows + beta * out_dgamma."""
    M, D = dy.shape
    hp, gp = _like(h, dy.shape, dy.dtype, "h"), _like(gamma, (D,), torch.float32, "gamma")
    rp, dp = _like(rstd, (M,), torch.float32, "rstd"), None if dh is None else _like(dh, dy.shape, dy.dtype, "dh")
    if out_dx is None:
        out_dx = torch.empty_like(dy)
        xp = out_dx.data_ptr()
    else:
        xp = _like(out_dx, dy.shape, dy.dtype, "out_dx")
    if out_dgamma is None:
        if beta:
            raise ValueError("beta needs an out_dgamma to add to")
        out_dgamma = torch.empty(D, dtype=torch.float32, device=dy.device)
        op = out_dgamma.data_ptr()
    else:
        op = _like(out_dgamma, (D,), torch.float32, "out_dgamma")
    need = 0 if workspace is not None else _lib.sr_rmsnorm_bwd_workspace_bytes(M, D)
    ws, size = _scratch(workspace, need, dy.device)
    _check(_lib.sr_rmsnorm_bwd(xp, op, _dev(dy), dp, hp, rp, gp, _dtype(dy), M, D, beta, ws, size, _stream()))
    return out_dx, out_dgamma


# ---- a decoder around its products -----------------------------------------------------------------
def _here(t, what):
    if t.is_cuda and t.get_device() != _current_device():
        raise RuntimeError(f"{what} is not on the current device, on whose stream the call would run")
    return t


def _heads(t, rows, heads, dim, what):
    """A tensor (rows, heads, dim) of bfloat16 as the C interface takes it; only the values of a head have to be neighbours."""
    if t.dtype is not torch.bfloat16:
        raise TypeError(f"{what} must be bfloat16")
    if not t.is_cuda:
        raise RuntimeError("srq needs device tensors: there is no CPU path")
    if t.get_device() != _current_device():
        _here(t, what)
    if t.shape != (rows, heads, dim):
        raise ValueError(f"{what} must be {(rows, heads, dim)}")
    row, head, one = t.stride()
    if one != 1 and dim > 1:
        raise ValueError(f"{what}: the values of a head must be neighbours")
    return srq_heads(t.data_ptr(), row, head)


def _int32(t, n, what):
    if t is None:
        return None
    if t.dtype is not torch.int32 or t.shape != (n,):
        raise ValueError(f"{what} must be {n} int32 values")
    return _dev(_here(t, what))


def _attention(q, k, scale, causal, sequences, offsets, offsets_k, lengths_k):
    T, H, D = q.shape
    if offsets is not None:
        sequences = offsets.shape[0] - 1
    elif offsets_k is not None:
        sequences = offsets_k.shape[0] - 1
    return srq_attention(sequences, T, k.shape[0], H, k.shape[1], D, _int32(offsets, sequences + 1, "offsets"),
                         _int32(offsets_k, sequences + 1, "offsets_k"), _int32(lengths_k, sequences, "lengths_k"),
                         D ** -0.5 if scale is None else scale, int(bool(causal)))


def sr_attention_fwd(q, k, v, scale=None, causal=True, sequences=1, offsets=None, offsets_k=None, lengths_k=None, out=None, workspace=None):
    """softmax(scale q k^T) v of q (T, heads, D), k and v (S, key heads, D), bfloat16: (o (T, heads, D), lse (heads, T)).  Rows belong together as
    sequences: `sequences` equal ones, or from offsets (int32, one more than sequences) on; offsets_k for k and v where they differ, lengths_k how
    many of a sequence's rows of k and v count.  scale: 1 / sqrt(D) if it is None.  Rows of no sequence are not written: in results made here they
    hold what the memory held."""
    T, H, D = q.shape
    S, G = k.shape[:2]
    a = _attention(q, k, scale, causal, sequences, offsets, offsets_k, lengths_k)
    heads = _heads(q, T, H, D, "q"), _heads(k, S, G, D, "k"), _heads(v, S, G, D, "v")
    if out is None:
        out = torch.empty((T, H, D), dtype=torch.bfloat16, device=q.device)
    lse = torch.empty((H, T), dtype=torch.float32, device=q.device)
    args = _heads(out, T, H, D, "out"), lse.data_ptr(), *heads, a
    ws, size = (None, 0) if workspace is None else _scratch(workspace, 0, q.device)
    status = _lib.sr_attention_fwd(*args, ws, size, _stream())
    if status == ERR_WORKSPACE and workspace is None:  # (most calls want none, and are spared the question)
        ws, size = _scratch(None, _lib.sr_attention_fwd_workspace_bytes(a), q.device)
        status = _lib.sr_attention_fwd(*args, ws, size, _stream())
    _check(status)
    return out, lse


def sr_attention_bwd(do, q, k, v, o, lse, scale=None, causal=True, sequences=1, offsets=None, offsets_k=None, lengths_k=None, out_dq=None, out_dk=None,
                     out_dv=None, workspace=None):
    """(dq, dk, dv) from the output gradient, what sr_attention_fwd took and gave.  Rows of no sequence, and of k and v behind lengths_k, are not written: in
    results made here they hold what the memory held."""
    T, H, D = q.shape
    S, G = k.shape[:2]
    a = _attention(q, k, scale, causal, sequences, offsets, offsets_k, lengths_k)
    kv = _heads(k, S, G, D, "k"), _heads(v, S, G, D, "v")
    reads = _heads(do, T, H, D, "do"), _heads(q, T, H, D, "q"), *kv, _heads(o, T, H, D, "o")
    lp = _like(_here(lse, "lse"), (H, T), torch.float32, "lse")
    if out_dq is None:
        out_dq = torch.empty((T, H, D), dtype=torch.bfloat16, device=q.device)
    if out_dk is None:
        out_dk = torch.empty((S, G, D), dtype=torch.bfloat16, device=q.device)
    if out_dv is None:
        out_dv = torch.empty((S, G, D), dtype=torch.bfloat16, device=q.device)
    need = 0 if workspace is not None else _lib.sr_attention_bwd_workspace_bytes(a)
    ws, size = _scratch(workspace, need, q.device)
    _check(_lib.sr_attention_bwd(_heads(out_dq, T, H, D, "out_dq"), _heads(out_dk, S, G, D, "out_dk"), _heads(out_dv, S, G, D, "out_dv"), *reads, lp, a, ws,
                                 size, _stream()))
    return out_dq, out_dk, out_dv


def _ids(ids):
    if ids.dtype is torch.int64:
        return _dev(_here(ids, "ids")), 8
    if ids.dtype is torch.int32:
        return _dev(_here(ids, "ids")), 4
    raise TypeError("ids must be int32 or int64")


def sr_embedding_fwd(table, ids, scale=1.0, dtype=None, out=None):
    """scale * table[ids]: (M, D) of ids (M,) and table (V, D), of dtype (default: the table's)."""
    V, D = table.shape
    at, size = _ids(ids)
    M = ids.numel()
    if out is None:
        out = torch.empty((M, D), dtype=dtype or table.dtype, device=table.device)
        to = out.data_ptr()
    else:
        to = _like(_here(out, "out"), (M, D), dtype or out.dtype, "out")
    _check(_lib.sr_embedding_fwd(to, _dtype(out), _dev(_here(table, "table")), _dtype(table), at, size, M, V, D, scale, _stream()))
    return out


def sr_embedding_bwd(dy, ids, V, scale=1.0, padding=-1, beta=0.0, out=None, workspace=None):
    """The gradient (V, D), float32, of a table from that of its rows, dy (M, D): scale * the sum of each id's rows + beta * out; without the places whose
    id is `padding`."""
    M, D = dy.shape
    at, size = _ids(ids)
    if ids.numel() != M:
        raise ValueError(f"{ids.numel()} ids for {M} rows")
    if out is None:
        if beta:
            raise ValueError("beta needs an out to add to")
        out = torch.empty((V, D), dtype=torch.float32, device=dy.device)
        to = out.data_ptr()
    else:
        to = _like(_here(out, "out"), (V, D), torch.float32, "out")
    need = 0 if workspace is not None else _lib.sr_embedding_bwd_workspace_bytes(M, D)
    ws, n = _scratch(workspace, need, dy.device)
    _check(_lib.sr_embedding_bwd(to, _dev(_here(dy, "dy")), _dtype(dy), at, size, M, V, D, scale, padding, beta, ws, n, _stream()))
    return out


class AdamWTensor:
    """One tensor of an AdamW step: weights w (float32 or bfloat16), gradient g, moments m and v, all of one size and dense.  Moments are float32, or uint8
    codes with m_scales and v_scales (uint8, one for every 128 values; zeros to begin with): then `second()` is the square of what v holds."""

    __slots__ = ("w", "g", "m", "v", "m_scales", "v_scales", "weight_decay", "counter_offset")

    def __init__(self, w, g, m, v, m_scales=None, v_scales=None, weight_decay=0.0, counter_offset=0):
        self.w, self.g, self.m, self.v, self.m_scales, self.v_scales = w, g, m, v, m_scales, v_scales
        self.weight_decay, self.counter_offset = weight_decay, counter_offset

    @staticmethod
    def zeros(w, g, bits=32, **more):
        """With moments of zeros, in 32 or 8 bits."""
        if bits not in (8, 32):
            raise ValueError("moments are held in 32 or 8 bits")
        n, dev = w.numel(), w.device
        if bits == 32:
            return AdamWTensor(w, g, *(torch.zeros(n, dtype=torch.float32, device=dev) for _ in range(2)), **more)
        return AdamWTensor(w, g, *(torch.zeros(n, dtype=_U8, device=dev) for _ in range(2)),
                           *(torch.zeros((n + 127) // 128, dtype=_U8, device=dev) for _ in range(2)), **more)

    def blocks(self):
        """Blocks of the random stream that a step with stochastic rounding uses."""
        return 3 * ((self.w.numel() + 7) // 8)

    def _values(self, x, scales):
        if scales is None:
            return x.reshape(-1).clone()
        return torch.ldexp(x.reshape(-1).view(torch.float8_e4m3fn).float(), (scales.int() - 127).repeat_interleave(128)[:x.numel()])

    def first(self):
        """The first moment, float32 (for checkpoints and tests: plain torch)."""
        return self._values(self.m, self.m_scales)

    def second(self):
        """The second moment, float32."""
        v = self._values(self.v, self.v_scales)
        return v if self.v_scales is None else v.square()

    def c(self):
        w, g, m, v, ms, vs = self.w, self.g, self.m, self.v, self.m_scales, self.v_scales
        n, narrow = w.numel(), ms is not None
        if not (g.numel() == m.numel() == v.numel() == n):
            what, t = next((what, t) for what, t in (("g", g), ("m", m), ("v", v)) if t.numel() != n)
            raise ValueError(f"{what} has {t.numel()} values, w {n}")
        state = _U8 if narrow else torch.float32
        if m.dtype is not state or v.dtype is not state or (vs is not None) != narrow:
            raise TypeError("moments are float32, or uint8 codes with their scales")
        if narrow and (ms.dtype is not _U8 or vs.dtype is not _U8 or not (ms.numel() == vs.numel() == (n + 127) // 128)):
            raise ValueError("one scale (uint8) for every 128 values")
        return srq_adamw_tensor(_dev(w), _dev(g), _dev(m), _dev(v), _dev(ms) if narrow else None, _dev(vs) if narrow else None, n,
                                self.counter_offset & (2**64 - 1), self.weight_decay, _dtype(w), _dtype(g), E4M3 if narrow else NONE)

    def on(self, device):
        """Whether all of it is there."""
        return self.w.get_device() == self.g.get_device() == self.m.get_device() == self.v.get_device() == device and (
            self.m_scales is None or self.m_scales.get_device() == self.v_scales.get_device() == device)


def _scalar_dev(x, dtype):
    """The address of a 1-element tensor on the device, None of a number."""
    if not isinstance(x, torch.Tensor):
        return None
    if x.dtype is not dtype or x.numel() != 1:
        raise ValueError(f"a 1-element tensor of {dtype}")
    return _dev(_here(x, "a value on the device"))


class AdamWBatch:
    """Prepared sr_adamw call on a list of AdamWTensor, marshalled once: the tensors stay where they are."""

    def __init__(self, tensors):
        self.keep = list(tensors)
        self.count = len(self.keep)
        self.list = (srq_adamw_tensor * max(self.count, 1))(*[t.c() for t in self.keep])
        self.device = self.keep[0].w.get_device() if self.count else None
        if not all([t.on(self.device) for t in self.keep]):
            raise RuntimeError("the tensors of a step are on one device")

    def run(self, lr, step, betas=(0.9, 0.999), eps=1e-8, round_mode=SR, seed=0, counter=None):
        """One step, in place.  lr and step: numbers, or 1-element tensors on the device (float32, int64) that are read when the kernels run; counter: such a
        tensor (int64) that is added to every tensor's counter_offset."""
        if self.device is not None and self.device != _current_device():
            raise RuntimeError("the tensors are not on the current device, on whose stream the call would run")
        ld, sd = _scalar_dev(lr, torch.float32), _scalar_dev(step, torch.int64)
        o = srq_adamw(betas[0], betas[1], 0.0 if ld else lr, eps, round_mode, 0, 0 if sd else step, seed & (2**64 - 1), ld, sd,
                      None if counter is None else _scalar_dev(counter, torch.int64))
        _check(_lib.sr_adamw(self.list, self.count, o, _stream()))


def sr_adamw(tensors, lr, step, **how):
    """One step of AdamW on a list of AdamWTensor (AdamWBatch.run)."""
    AdamWBatch(tensors).run(lr, step, **how)
