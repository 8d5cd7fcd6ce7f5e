"""Training with the SR-quantized linear layer: an autograd face of Alg. 1 / Alg. 2 and the
weight update of Eq. 10, plus a small decoder whose linears all go through it, and a gated feed-forward
block on block-scaled operands (norm, both products, activation and their backward passes).

Only the linears, the gated block and the weight update are this library's; embedding, layer norm, attention,
GELU and the loss are plain PyTorch operators (they are not quantized in the paper's method,
Sec. 3.1: the quantization sites are the inputs of the matrix products).
"""
import torch
import torch.nn.functional as F

from . import lib as L

# Rows per call: keeps every operand matrix of the products below the library's 2 GiB limit for
# the widest layer used here (32000 outputs in the two-byte form).  Token chunks are independent
# in Y and dA; dW accumulates over them (beta = 1), which is also how micro-batches accumulate.
MAX_ROWS = 16384
MASK64 = 2**64 - 1
NOQ = L.Quant(L.NONE, 1.0)  # the identity quantizer of the weight-only objective


def _rows(t, r0, r1):
    """Rows r0 .. r1 - 1 of t; t itself where that is all of them (a view costs as much as a kernel launch)."""
    return t if r0 == 0 and r1 == t.shape[0] else t[r0:r1]


def _matrix(x, cols):
    """x as a dense binary32 matrix of `cols` columns; x itself where it is one (each of the three steps costs as much as a
    launch, also where it changes nothing)."""
    if x.dim() == 2 and x.shape[1] == cols and x.dtype is torch.float32 and x.is_contiguous():
        return x
    return x.reshape(-1, cols).contiguous().float()


def _quant(scales, i, kind, rounding, seed, position):
    """The quantizer with the i-th of `scales`, in the form of the C interface: for calls while `scales` lives.  A position held on
    the device (a 1-element int64 tensor) stays there and is read when the kernels run."""
    if isinstance(position, torch.Tensor):
        return L.Quant(kind, scales[i:i + 1], seed, position, rounding)
    return L.srq_quant(kind, rounding, 0.0, 0, scales.data_ptr() + 4 * i, seed & MASK64, position & MASK64)


class SRLinearFn(torch.autograd.Function):
    """Everything the backward pass of ONE forward call needs travels on the autograd context:
    the saved activation -- as the codes of its backward quantizer when the forward pass can write
    them (the stash of sr_linear_fwd_stash: integer forward formats), else in binary32 -- the
    stream positions drawn for the backward quantizers of A and W, the scales found for them and (objectives that share one quantized weight copy between the
    passes) the weight quantizer itself.  A second forward of the same layer before the first
    backward therefore cannot disturb the first one's gradients."""

    @staticmethod
    def forward(ctx, x, layer):
        ctx.layer = layer
        ctx.shape = x.shape
        a = _matrix(x, x.shape[-1])
        y, ctx.saved = layer._forward(a)
        if "stash" not in ctx.saved:  # the backward pass quantizes (or multiplies) the activation itself
            ctx.save_for_backward(a)
        return y if x.dim() == 2 else y.reshape(*x.shape[:-1], layer.out_features)

    @staticmethod
    def backward(ctx, dy):
        a = ctx.saved_tensors[0] if ctx.saved_tensors else None
        layer = ctx.layer
        da = layer._backward(_matrix(dy, layer.out_features), a, ctx.saved)
        return da if len(ctx.shape) == 2 else da.reshape(ctx.shape), None


OBJECTIVES = ("five", "weight_only", "qat")


class SRLinear(torch.nn.Module):
    """y = Q(x) Q(W)^T with the five quantizers of Alg. 1 / Alg. 2 (per-tensor absmax scales,
    fresh stream positions every call); W is held in bfloat16 and updated by Eq. 10.

    The weight gradient is kept by the layer (`self.dW`, float32, accumulated over backward
    calls until `update`), not handed to autograd: the update consumes it in place.

    objective:
      "five"         all five quantizers independent (Alg. 1 / Alg. 2 in general form): A and W
                     to `fwd_kind` in the forward pass, A, W and dY to `bwd_kind` in the backward.
      "weight_only"  Sec. 3.2: only the weights are quantized (to `fwd_kind`, one quantized copy
                     per forward call, used again in its backward pass); activations and
                     gradients stay in binary32, so the weight gradient dY^T A has no quantized
                     operand and is a plain matrix product.
      "qat"          Sec. 3.3 (Fig. 3), the estimator whose expectation is the gradient of the
                     quantization-aware objective (Eq. 6-7): the forward pass multiplies the
                     unquantized activation by Q(W); the backward pass uses the SAME quantized
                     weights (same thresholds: one copy per mini-batch) and stochastically
                     rounds the saved activation and the output gradient.  One format
                     (`bwd_kind`) for all four quantizers, as in the paper (one Delta).
    weight_only=True is kept as a synonym of objective="weight_only"."""

    def __init__(self, in_features, out_features, seed, fwd_kind=L.INT8, bwd_kind=L.E5M2, device="cuda:0",
                 init_std=0.02, round_mode=L.SR, weight_only=False, objective=None):
        super().__init__()
        self.in_features, self.out_features = in_features, out_features
        g = torch.Generator(device=device).manual_seed(seed)
        w = torch.randn((out_features, in_features), device=device, generator=g) * init_std
        self.weight = w.to(torch.bfloat16)           # not an nn.Parameter: autograd never sees it
        self.dW = torch.zeros((out_features, in_features), dtype=torch.float32, device=device)
        self.have_grad = False
        self.objective = objective or ("weight_only" if weight_only else "five")
        assert self.objective in OBJECTIVES
        self.weight_only = self.objective == "weight_only"
        if self.objective == "qat":
            fwd_kind = bwd_kind  # one Delta: the weights are quantized once, for both passes
        self.kinds = {"A_fwd": fwd_kind, "W_fwd": fwd_kind, "A_bwd": bwd_kind, "W_bwd": bwd_kind, "dY_bwd": bwd_kind}
        self.seed, self.position, self.round_mode = seed, 0, round_mode
        self.ws = None

    def __setattr__(self, name, value):
        # Module's own looks for parameters, buffers and modules first, 1.4 us; an attribute that is there is none of these, and a
        # number does not become one
        if type(value) in (int, bool) and name in self.__dict__:
            object.__setattr__(self, name, value)
        else:
            super().__setattr__(name, value)

    _sizes = None  # bytes that calls of so many rows need

    def _size(self, op, M):
        """Bytes of workspace for a call of M rows, or of its stash (op None).  A query plans the products anew: up to 256
        answers are kept."""
        sizes = self._sizes
        if sizes is None or len(sizes) >= 256:
            sizes = self._sizes = {}
        key = (op, M, self.out_features, self.in_features)
        need = sizes.get(key)
        if need is None:
            need = sizes[key] = L.sr_linear_stash_bytes(*key[1:]) if op is None else L.sr_linear_workspace_bytes(*key)
        return need

    def _q(self, name, scales, i, position):
        return _quant(scales, i, self.kinds[name], self.round_mode, self.seed, position)

    @staticmethod
    def _q_saved(saved):
        """The weights' quantizer of a forward pass for its backward pass (everything but the address of its scale is kept)."""
        return _quant(saved["scales"], *saved["w"])

    def _workspace(self, op, M):
        need = self._size(op, M)
        if self.ws is None or self.ws.numel() < need:
            self.ws = torch.empty(need, dtype=torch.uint8, device=self.weight.device)
        return self.ws

    # -- objectives that multiply an unquantized activation by Q(W) in the forward pass ---------
    def _forward_unquantized_a(self, a):
        M, K = a.shape
        N = self.out_features
        w = self.weight
        qat = self.objective == "qat"
        pairs = [(w, self.kinds["W_fwd"])]            # W, and (qat) A for the backward pass
        if qat:
            pairs.append((a, self.kinds["A_bwd"]))
        sc = L.absmax_scales(pairs)
        qw = self._q("W_fwd", sc, 0, self.position)   # the same copy serves the backward pass
        saved = {"scales": sc, "w": (0, self.kinds["W_fwd"], self.round_mode, self.seed, self.position)}
        pos_a = self.position + (N * K + 7) // 8      # (a new position, also where it is a tensor: the old one is kept above)
        if qat:
            saved["a"] = 1, pos_a
        self.position = pos_a + (M * K + 7) // 8 if qat else pos_a
        y = torch.empty((M, N), dtype=torch.float32, device=a.device)
        for r0 in range(0, M, MAX_ROWS):
            r1 = min(M, r0 + MAX_ROWS)
            L.sr_linear_fwd(_rows(a, r0, r1), w, NOQ, qw, out=_rows(y, r0, r1),
                            workspace=self._workspace(L.OP_FWD_WEIGHT_ONLY, r1 - r0))
        return y, saved

    def _backward_weight_only(self, dy, a, saved):
        M, N = dy.shape
        da = torch.empty((M, self.in_features), dtype=torch.float32, device=dy.device)
        qw = self._q_saved(saved)
        for r0 in range(0, M, MAX_ROWS):
            r1 = min(M, r0 + MAX_ROWS)
            L.sr_linear_bwd_data(_rows(dy, r0, r1), self.weight, NOQ, qw, out=_rows(da, r0, r1),
                                 workspace=self._workspace(L.OP_BWD_DATA_WEIGHT_ONLY, r1 - r0))
        if self.have_grad:
            self.dW.addmm_(dy.t(), a)
        else:
            torch.mm(dy.t(), a, out=self.dW)
        self.have_grad = True
        return da

    def _forward(self, a):
        if self.objective != "five":
            return self._forward_unquantized_a(a)
        M, K = a.shape
        N = self.out_features
        w = self.weight
        sc = L.absmax_scales([(a, self.kinds["A_fwd"]), (w, self.kinds["W_fwd"]), (a, self.kinds["A_bwd"]),
                              (w, self.kinds["W_bwd"])])
        # every tensor gets its own stretch of the stream (in blocks of 8 elements); a chunk that
        # starts at row r0 continues where the rows before it would have drawn, so the codes do
        # not depend on the chunking.  The backward quantizers of A and W get theirs now.
        a_blocks, w_blocks = (M * K + 7) // 8, (N * K + 7) // 8
        pos_w = self.position
        pos_a = pos_w + w_blocks
        pos_a_bwd = pos_a + a_blocks
        pos_w_bwd = pos_a_bwd + a_blocks
        self.position = pos_w_bwd + w_blocks
        qw, qw_bwd = self._q("W_fwd", sc, 1, pos_w), self._q("W_bwd", sc, 3, pos_w_bwd)
        saved = {"scales": sc, "a": (2, pos_a_bwd), "w": (3, self.kinds["W_bwd"], self.round_mode, self.seed, pos_w_bwd)}
        y = torch.empty((M, N), dtype=torch.float32, device=a.device)
        # integer forward formats: the same pass over A and W also writes the codes of their backward
        # quantizers (one stash per chunk of rows), and the activation itself need not be kept
        stash = self.kinds["A_fwd"] in (L.INT8, L.INT4)
        if stash:
            saved["stash"] = []
        for r0 in range(0, M, MAX_ROWS):
            r1 = min(M, r0 + MAX_ROWS)
            qa = self._q("A_fwd", sc, 0, pos_a + (r0 * K) // 8)
            if stash:
                qa_bwd = self._q("A_bwd", sc, 2, pos_a_bwd + (r0 * K) // 8)
                st = torch.empty(self._size(None, r1 - r0), dtype=torch.uint8, device=a.device)
                L.sr_linear_fwd_stash(_rows(a, r0, r1), w, qa, qw, qa_bwd, qw_bwd, stash=st, out=_rows(y, r0, r1),
                                      workspace=self._workspace(L.OP_FWD_STASH, r1 - r0))
                saved["stash"].append(st)
            else:
                L.sr_linear_fwd(_rows(a, r0, r1), w, qa, qw, out=_rows(y, r0, r1),
                                workspace=self._workspace(L.OP_FWD, r1 - r0))
        return y, saved

    def _backward(self, dy, a, saved):
        if self.weight_only:
            return self._backward_weight_only(dy, a, saved)
        # "five" and "qat" differ only in where the weight quantizer comes from: its own draw, or
        # the forward pass's (Fig. 3: W_hat is shared by the two passes)
        M, N = dy.shape
        K = self.in_features
        w = self.weight
        sdy = L.absmax_scales([(dy, self.kinds["dY_bwd"])])
        da = torch.empty((M, K), dtype=torch.float32, device=dy.device)
        pos_dy = self.position
        self.position = pos_dy + (M * N + 7) // 8
        scales, (i_a, pos_a), qw = saved["scales"], saved["a"], self._q_saved(saved)
        for i, r0 in enumerate(range(0, M, MAX_ROWS)):
            r1 = min(M, r0 + MAX_ROWS)
            qdy = self._q("dY_bwd", sdy, 0, pos_dy + (r0 * N) // 8)
            qa = self._q("A_bwd", scales, i_a, pos_a + (r0 * K) // 8)
            beta = 1.0 if self.have_grad else 0.0
            if "stash" in saved:
                L.sr_linear_bwd_stashed(_rows(dy, r0, r1), saved["stash"][i], K, qdy, qw, qa,
                                        out_dA=_rows(da, r0, r1), out_dW=self.dW, beta=beta, workspace=self._workspace(L.OP_BWD_STASHED, r1 - r0))
            else:
                L.sr_linear_bwd(_rows(dy, r0, r1), w, _rows(a, r0, r1), qdy, qw, qa,
                                out_dA=_rows(da, r0, r1), out_dW=self.dW, beta=beta, workspace=self._workspace(L.OP_BWD, r1 - r0))
            self.have_grad = True
        return da

    def forward(self, x):
        return SRLinearFn.apply(x, self)

    def update(self, lr):
        """Eq. 10: W <- Q_SR(W - lr * dW) on the bfloat16 grid; clears the accumulated gradient."""
        if self.have_grad:
            L.sr_update_bf16(self.weight.view(-1), self.dW.view(-1), lr, seed=self.seed, counter_offset=self.position,
                             round_mode=self.round_mode)
            self.position += (self.weight.numel() + 7) // 8
            self.have_grad = False


class GatedMLPFn(torch.autograd.Function):
    """What the backward pass reads is saved with the graph: 8-bit codes of the norm's result, of G and U and of H, the weights turned, the
    residual stream and rstd.  It goes when the backward pass is done, also where a result that holds on to the graph stays."""

    @staticmethod
    def forward(ctx, x, residual, gamma, layer):
        ctx.layer, ctx.shape = layer, x.shape
        ctx.set_materialize_grads(False)  # (a zero dh would be written and read)
        d = layer.features
        a, r = x.reshape(-1, d).contiguous(), residual.reshape(-1, d).contiguous()
        y, h, kept = layer._forward(a, r, gamma.detach(), True)
        ctx.forms = [(k.kind, k.cols) if isinstance(k, L.Blocks) else None for k in kept]
        ctx.save_for_backward(h, gamma, *(t for k in kept for t in ((k.codes, k.exps) if isinstance(k, L.Blocks) else (k,))))
        return y.view(x.shape), h.view(x.shape)

    @staticmethod
    @torch.autograd.function.once_differentiable  # (the kernels' gradients have none of their own)
    def backward(ctx, dy, dh):
        h, gamma, *parts = ctx.saved_tensors
        parts = iter(parts)
        kept = [next(parts) if form is None else L.Blocks(next(parts), next(parts), *form) for form in ctx.forms]
        d = ctx.layer.features
        dy = torch.zeros_like(h) if dy is None else dy.reshape(-1, d).contiguous()
        if dh is not None:
            dh = dh.reshape(-1, d).contiguous()
        dx, dgamma = ctx.layer._backward(dy, dh, h, gamma, kept)
        dx = dx.view(ctx.shape)
        return dx, dx, dgamma, None


class GatedMLP(torch.nn.Module):
    """h = x + residual;  y = Wd (act(Wg n) * (Wu n)),  n = h / sqrt(mean(h^2) + eps) * gamma:  (y, h) of (x, residual), float32 or bfloat16.

    Products run on block-scaled operands (a power of two for every 128 values): E4M3 in the forward pass, `grad_kind` for the output
    gradients, rounded to nearest forward and stochastically backward (`round_fwd`, `round_bwd`).  Kept for the backward pass are the
    operands themselves and [G | U], a byte a value each.  Weights are held in bfloat16, [Wg; Wu] in `w_in` (2F x d) and Wd in `w_out` (d x F), their
    gradients in binary32 in `dw_in` and `dw_out` until `update` applies Eq. 10.  f8_pipeline: the fp8 matrix pipeline for products with
    bfloat16 results.  `freeze()` keeps the weights' codes for calls without gradients, token by token say."""

    def __init__(self, features, hidden, seed, act=L.ACT_SILU, eps=1e-5, grad_kind=L.E5M2, round_fwd=L.RTN, round_bwd=L.SR, f8_pipeline=False,
                 device="cuda:0", init_std=0.02):
        super().__init__()
        if features % 16 or hidden % 128:
            raise ValueError("features must be a multiple of 16, hidden of 128")
        self.features, self.hidden, self.act, self.eps = features, hidden, act, eps
        self.grad_kind, self.round_fwd, self.round_bwd, self.f8_pipeline = grad_kind, round_fwd, round_bwd, f8_pipeline
        self.gamma = torch.nn.Parameter(torch.ones(features, device=device))
        g = torch.Generator(device=device).manual_seed(seed)
        self.w_in = (torch.randn((2 * hidden, features), device=device, generator=g) * init_std).to(torch.bfloat16)
        self.w_out = (torch.randn((features, hidden), device=device, generator=g) * init_std).to(torch.bfloat16)
        self.dw_in = torch.zeros((2 * hidden, features), dtype=torch.float32, device=device)
        self.dw_out = torch.zeros((features, hidden), dtype=torch.float32, device=device)
        self.have_grad = False
        self.seed, self.position = seed, 0
        self.frozen = None

    def _q(self, kind, mode, count):
        """A quantizer with its own stretch of the stream, for `count` values."""
        at = self.position
        self.position = at + (count + 7) // 8  # (a new position, also where it is a tensor on the device: the quantizer keeps the old one)
        return L.Quant(kind, 1.0, seed=self.seed, counter_offset=at, round_mode=mode)

    def _weights(self, layout):
        return [L.sr_block_quantize(w, self._q(L.E4M3, self.round_fwd, w.numel()), layout) for w in (self.w_in, self.w_out)]

    def _forward(self, x, residual, gamma, keep):
        M, d = x.shape
        f = self.hidden
        q = [self._q(L.E4M3, self.round_fwd, M * n) for n in (d, f, 2 * f)]
        n, h, rstd = L.sr_rmsnorm_fwd(x, gamma, self.eps, residual=residual, q=q[0])
        if keep:
            (w_in, w_in_t), (w_out, w_out_t) = self._weights(L.BOTH)
        else:
            w_in, w_out = self.frozen or self._weights(L.ROWS)
        hidden, gu = L.sr_gated_fwd(n, w_in, self.act, qh=q[1], qgu=q[2] if keep else None)
        f8 = self.f8_pipeline and x.dtype is torch.bfloat16
        y = L.sr_gemm_blocks(hidden, w_out, dtype=x.dtype, f8_pipeline=f8)
        return y, h, (n, rstd, hidden, gu, w_in_t, w_out_t) if keep else None

    def _backward(self, dy, dh, h, gamma, kept):
        n, rstd, hidden, gu, w_in_t, w_out_t = kept
        M, d = dy.shape
        f8 = self.f8_pipeline and dy.dtype is torch.bfloat16
        beta = 1.0 if self.have_grad else 0.0
        rows, turned = L.sr_block_quantize(dy, self._q(self.grad_kind, self.round_bwd, M * d), L.BOTH)
        L.sr_gemm_blocks(turned, L.sr_block_turn(hidden), beta=beta, out=self.dw_out)
        dhidden = L.sr_gemm_blocks(rows, w_out_t, dtype=dy.dtype, f8_pipeline=f8)
        rows, turned = L.sr_gated_bwd(dhidden, gu, self._q(self.grad_kind, self.round_bwd, M * 2 * self.hidden), self.act)
        L.sr_gemm_blocks(turned, L.sr_block_turn(n), beta=beta, out=self.dw_in)
        dn = L.sr_gemm_blocks(rows, w_in_t, dtype=dy.dtype, f8_pipeline=f8)
        self.have_grad = True
        return L.sr_rmsnorm_bwd(dn, h, rstd, gamma, dh=dh)

    def forward(self, x, residual):
        if torch.is_grad_enabled():
            return GatedMLPFn.apply(x, residual, self.gamma, self)
        d = self.features
        y, h, _ = self._forward(x.reshape(-1, d).contiguous(), residual.reshape(-1, d).contiguous(), self.gamma.detach(), False)
        return y.view(x.shape), h.view(x.shape)

    def freeze(self):
        """The weights' codes once, for the calls without gradients until the next update."""
        self.frozen = self._weights(L.ROWS)
        return self

    def update(self, lr):
        """Eq. 10 on both weights, as SRLinear.update; clears the accumulated gradients."""
        if self.have_grad:
            for w, g in ((self.w_in, self.dw_in), (self.w_out, self.dw_out)):
                L.sr_update_bf16(w.view(-1), g.view(-1), lr, seed=self.seed, counter_offset=self.position, round_mode=self.round_bwd)
                self.position += (w.numel() + 7) // 8
            self.have_grad = False
            self.frozen = None


class Block(torch.nn.Module):
    """ffn: "gelu" (two SR linears around a GELU, layer norm in front) or "gated" (GatedMLP, which takes the residual's addition and the
    norm along; its quantizers are its own, whatever the objective of the SR linears)."""

    def __init__(self, d, heads, seed, device, objective="five", ffn="gelu"):
        super().__init__()
        self.heads = heads
        assert ffn in ("gelu", "gated")
        self.ln1 = torch.nn.LayerNorm(d, device=device)
        self.ln2 = torch.nn.LayerNorm(d, device=device) if ffn == "gelu" else None
        self.qkv = SRLinear(d, 3 * d, seed, device=device, objective=objective)
        self.proj = SRLinear(d, d, seed + 1, device=device, objective=objective)
        self.mlp = None
        if ffn == "gated":
            self.mlp = GatedMLP(d, (8 * d // 3 + 127) // 128 * 128, seed + 2, device=device)
            return
        self.fc1 = SRLinear(d, 4 * d, seed + 2, device=device, objective=objective)
        self.fc2 = SRLinear(4 * d, d, seed + 3, device=device, objective=objective)

    def forward(self, x):
        B, T, d = x.shape
        q, k, v = self.qkv(self.ln1(x)).view(B, T, 3, self.heads, d // self.heads).permute(2, 0, 3, 1, 4)
        att = F.scaled_dot_product_attention(q.bfloat16(), k.bfloat16(), v.bfloat16(), is_causal=True).float()
        a = self.proj(att.transpose(1, 2).reshape(B, T, d))
        if self.mlp is not None:
            y, h = self.mlp(a, x)
            return h + y
        x = x + a
        return x + self.fc2(F.gelu(self.fc1(self.ln2(x))))


class Decoder(torch.nn.Module):
    """Pre-norm decoder: token + position embedding, `layers` blocks, final norm, output head."""

    def __init__(self, vocab=32000, d=768, heads=12, layers=12, seq=1024, seed=1, device="cuda:0", weight_only=False,
                 objective=None, ffn="gelu"):
        super().__init__()
        objective = objective or ("weight_only" if weight_only else "five")
        self.tok = torch.nn.Embedding(vocab, d, device=device)
        self.pos = torch.nn.Embedding(seq, d, device=device)
        torch.nn.init.normal_(self.tok.weight, std=0.02)
        torch.nn.init.normal_(self.pos.weight, std=0.02)
        self.blocks = torch.nn.ModuleList([Block(d, heads, seed + 10 * i, device, objective, ffn) for i in range(layers)])
        self.ln = torch.nn.LayerNorm(d, device=device)
        self.head = SRLinear(d, vocab, seed + 10 * layers, device=device, objective=objective)

    def sr_linears(self):
        return [m for m in self.modules() if isinstance(m, SRLinear)]

    def gated_mlps(self):
        return [m for m in self.modules() if isinstance(m, GatedMLP)]

    def forward(self, ids):
        B, T = ids.shape
        x = self.tok(ids) + self.pos(torch.arange(T, device=ids.device))
        for blk in self.blocks:
            x = blk(x)
        return self.head(self.ln(x))


def _gated_mlps(model):
    """The gated blocks of a model, which need not be a Decoder nor know of them."""
    return model.gated_mlps() if hasattr(model, "gated_mlps") else []


def train_step(model, ids, targets, lr, micro_batches=1):
    """One mini-batch step: forward and backward over `micro_batches` slices of the batch (weight
    gradients accumulate inside the SR linears, the others in .grad), then the updates: Eq. 10 for
    the SR linears and gated blocks, plain SGD for the float32 parameters.  Returns the mean loss (device tensor)."""
    total = None
    for ids_mb, tgt_mb in zip(ids.chunk(micro_batches), targets.chunk(micro_batches)):
        logits = model(ids_mb)
        loss = F.cross_entropy(logits.view(-1, logits.shape[-1]), tgt_mb.reshape(-1)) / micro_batches
        loss.backward()
        total = loss.detach() if total is None else total + loss.detach()
    for m in model.sr_linears() + _gated_mlps(model):
        m.update(lr)
    with torch.no_grad():
        for p in model.parameters():
            if p.grad is not None:
                p.add_(p.grad, alpha=-lr)
                p.grad = None
    return total


def flops_per_token(model):
    """6 x (parameters of the SR linears and gated blocks): forward + the two backward products."""
    return 6.0 * (sum(m.in_features * m.out_features for m in model.sr_linears()) +
                  sum(3 * m.features * m.hidden for m in _gated_mlps(model)))


__all__ = ["SRLinear", "GatedMLP", "Decoder", "train_step", "flops_per_token", "MAX_ROWS"]
