"""The block-scaled 8-bit operators: what is timed of them, in plain torch operations and through the library.

A matrix in block-scaled form is held as one byte a value (E4M3 or E5M2) and one power of two, stored as its biased
exponent, for every 128 consecutive values of a row.  "op" of a case says which use it stands for:

  norm_fwd   residual addition and root-mean-square norm of M tokens, the result in block-scaled form
  norm_bwd   its backward pass: gradients of the inputs and of the gain
  store      a tensor to block-scaled form, along its rows and turned (what the three products of a layer take)
  turn       an 8-bit activation checkpoint, blocks along its rows, to the turned operand of a weight gradient
  product    X Z^T of two block-scaled matrices
  gated_fwd  both projections of a gated feed-forward block, activation and product: H, and G and U as 8-bit checkpoint
  gated_bwd  its backward pass from that checkpoint: the gradients of G and U, along rows and turned

Sizes are tokens M, out features N, in features K (gated: F hidden features).  8-bit results are returned as they are held:
8-bit floats, and the scales as powers of two.
"""
import math

import torch

own = False
DEV = "cuda:0"
BLOCK = 128
EPS = 1e-5
E4M3, E5M2 = "e4m3", "e5m2"
GRID = {E4M3: (448.0, 3, -6, 9, torch.float8_e4m3fn), E5M2: (57344.0, 2, -14, 16, torch.float8_e5m2)}
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


def listed():
    return [
        # one token of a sequence being generated, in front of a projection of the 2048-wide layer
        {"name": "norm_token", "op": "norm_fwd", "M": 1, "K": 2048, "type": "bf16"},
        # a training batch of 16 sequences of 1024 tokens through the same layer
        {"name": "norm_16k", "op": "norm_fwd", "M": 16384, "K": 2048, "type": "bf16"},
        # backward pass of an odd batch, residual stream in binary32
        {"name": "norm_bwd_ragged", "op": "norm_bwd", "M": 8191, "K": 2048, "type": "f32"},
        # an output gradient rounded stochastically, for both backward products
        {"name": "store_grad_16k", "op": "store", "M": 16384, "K": 2048, "type": "bf16", "kind": E5M2, "sr": True},
        # the hidden activations of an odd batch, from their checkpoint to the operand of the down projection's gradient
        {"name": "turn_hidden_ragged", "op": "turn", "M": 12289, "K": 5632, "kind": E4M3},
        # down projection of one token
        {"name": "product_token", "op": "product", "M": 1, "N": 2048, "K": 5632, "x": E4M3, "out": "bf16", "f8": True},
        # the same of a short, odd prompt
        {"name": "product_prompt", "op": "product", "M": 1009, "N": 2048, "K": 5632, "x": E4M3, "out": "bf16", "f8": True},
        # weight gradient of gate and up projections, binary32 sums of exact products
        {"name": "product_weight_grad", "op": "product", "M": 11264, "N": 2048, "K": 16384, "x": E5M2, "out": "f32", "f8": False},
        # gated block: one token, a batch of requests, a training batch
        {"name": "gated_token", "op": "gated_fwd", "M": 1, "F": 5632, "K": 2048, "act": "silu", "keep": False, "f8": True},
        {"name": "gated_requests", "op": "gated_fwd", "M": 113, "F": 5632, "K": 2048, "act": "gelu", "keep": False, "f8": True},
        {"name": "gated_16k", "op": "gated_fwd", "M": 16384, "F": 5632, "K": 2048, "act": "silu", "keep": True, "f8": True},
        # its backward pass, gradients rounded stochastically
        {"name": "gated_bwd_16k", "op": "gated_bwd", "M": 16384, "F": 5632, "type": "bf16", "act": "silu", "kind": E5M2, "sr": True},
    ]


def _log(rng, lo, hi, multiple=1):
    v = math.exp(rng.uniform(math.log(lo), math.log(hi)))
    return max(multiple, int(v / multiple + 0.5) * multiple)


def draw(rng):
    op = rng.choice(["norm_fwd", "norm_bwd", "store", "turn", "product", "product", "product", "gated_fwd", "gated_fwd", "gated_bwd"])
    while True:
        M = _log(rng, 1, 16384)
        if op in ("norm_fwd", "norm_bwd"):
            return {"op": op, "M": M, "K": _log(rng, 512, 8192, 16), "type": rng.choice(["bf16", "f32"])}
        if op == "store":
            return {"op": op, "M": M, "K": _log(rng, 512, 5632, 16), "type": rng.choice(["bf16", "f32"]),
                    "kind": rng.choice([E4M3, E5M2]), "sr": rng.random() < 0.5}
        if op == "turn":
            return {"op": op, "M": M, "K": _log(rng, 512, 5632, 16), "kind": rng.choice([E4M3, E5M2])}
        if op == "product":
            f8 = rng.random() < 0.6
            N, K = _log(rng, 128, 11264, 16), _log(rng, 128, 16384, 16)
            if M * N * K <= 11264 * 2048 * 16384:
                return {"op": op, "M": M, "N": N, "K": K, "x": rng.choice([E4M3, E4M3, E5M2]), "out": "bf16" if f8 else "f32", "f8": f8}
            continue
        F = _log(rng, 256, 5632, 128)
        act = rng.choice(["silu", "silu", "gelu"])
        if op == "gated_fwd":
            return {"op": op, "M": M, "F": F, "K": _log(rng, 256, 4096, 16) if F <= 2816 else _log(rng, 256, 2048, 16), "act": act,
                    "keep": rng.random() < 0.5, "f8": rng.random() < 0.7}
        return {"op": op, "M": M, "F": F, "type": rng.choice(["bf16", "f32"]), "act": act, "kind": rng.choice([E4M3, E5M2]),
                "sr": rng.random() < 0.5}


# ---- inputs ---------------------------------------------------------------------------------------------------------
def _gauss(g, shape, std=1.0):
    return torch.randn(shape, generator=g, device=DEV) * std


def _activations(g, M, K):
    """Channels of different strength, as a trained layer's, and a few outliers."""
    x = _gauss(g, (M, K)) * torch.exp(_gauss(g, (1, K), 0.5))
    return torch.where(torch.rand((M, K), generator=g, device=DEV) < 1e-3, x * 20.0, x)


def _gradients(g, M, K):
    """Tokens whose losses differ by orders of magnitude."""
    return _gauss(g, (M, K), 1e-3) * torch.exp(_gauss(g, (M, 1), 1.5))


def _held(x, kind):
    """A matrix as a program holds it between the calls: codes with rows of a multiple of 16 bytes, exponents of 4."""
    codes, scales = _to_blocks(x, kind)
    c = torch.zeros((x.shape[0], -(-x.shape[1] // 16) * 16), dtype=torch.uint8, device=DEV)
    c[:, :x.shape[1]] = codes.view(torch.uint8)
    e = torch.zeros((x.shape[0], -(-scales.shape[1] // 4) * 4), dtype=torch.uint8, device=DEV)
    e[:, :scales.shape[1]] = scales.view(torch.uint8)
    return {"codes": c, "exps": e, "kind": kind, "cols": x.shape[1]}


def prepare(case, seed):
    g = torch.Generator(device=DEV).manual_seed(seed)
    op, s = case["op"], dict(case)
    M = case["M"]
    if op in ("norm_fwd", "norm_bwd"):
        K, t = case["K"], TYPES[case["type"]]
        s["gamma"] = 1.0 + _gauss(g, (K,), 0.1)
        s["x"], s["res"] = _activations(g, M, K).to(t), _gauss(g, (M, K), 3.0).to(t)
        if op == "norm_bwd":
            s["h"] = s["x"]
            s["rstd"] = torch.rsqrt(s["h"].float().square().mean(1) + EPS)
            s["dy"], s["dh"] = _gradients(g, M, K).to(t), _gradients(g, M, K).to(t)
    elif op == "store":
        s["x"], s["seed"] = _gradients(g, M, case["K"]).to(TYPES[case["type"]]), seed
    elif op == "turn":
        s["x"] = _held(_activations(g, M, case["K"]), case["kind"])
    elif op == "product":
        s["X"] = _held(_activations(g, M, case["K"]) if case["x"] == E4M3 else _gradients(g, M, case["K"]), case["x"])
        s["Z"] = _held(_gauss(g, (case["N"], case["K"]), 0.02), E4M3)
    elif op == "gated_fwd":
        s["X"] = _held(_activations(g, M, case["K"]), E4M3)
        s["W"] = _held(_gauss(g, (2 * case["F"], case["K"]), 0.02), E4M3)
    else:
        s["gu"] = _held(_gauss(g, (M, 2 * case["F"])), E4M3)
        s["dH"], s["seed"] = _gradients(g, M, case["F"]).to(TYPES[case["type"]]), seed
    return s


# ---- the plain forms ------------------------------------------------------------------------------------------------
def _philox(n, seed):
    """The 16 random bits of elements 0 .. n - 1 (n a multiple of 8): Philox4x32-10, block i / 8, slice i % 8."""
    lo32 = 0xFFFFFFFF
    i = torch.arange(n // 8, device=DEV, dtype=torch.int64)
    c = [i & lo32, i >> 32, torch.zeros_like(i), torch.zeros_like(i)]
    k0, k1 = seed & lo32, (seed >> 32) & lo32
    for _ in range(10):
        p0, p1 = c[0] * 0xD2511F53, c[2] * 0xCD9E8D57
        c = [((p1 >> 32) & lo32) ^ c[1] ^ k0, p1 & lo32, ((p0 >> 32) & lo32) ^ c[3] ^ k1, p0 & lo32]
        k0, k1 = (k0 + 0x9E3779B9) & lo32, (k1 + 0xBB67AE85) & lo32
    return torch.stack([h for w in c for h in (w & 0xFFFF, w >> 16)], 1).view(-1)


def _to_blocks(x, kind, bits=None):
    """x (R x C, binary32) -> codes as 8-bit floats (R x C), scales (R x blocks of 128 columns) as powers of two."""
    qmax, m, emin, top, f8 = GRID[kind]
    R, C = x.shape
    nb = -(-C // BLOCK)
    t = torch.nn.functional.pad(x, (0, nb * BLOCK - C)).view(R, nb, BLOCK)
    amax = t.abs().amax(2)
    frac, e = torch.frexp(amax)
    e = torch.where(amax == 0, 0, (e - top + (frac > 0.875).int()).clamp(min=-100))
    t = torch.ldexp(t, -e[:, :, None]).clamp(-qmax, qmax).view(R, nb * BLOCK)[:, :C]
    d = (torch.frexp(t)[1] - 1).clamp(min=emin) - m
    y = torch.ldexp(t, -d)
    q = torch.floor(y)
    threshold = 0.5 if bits is None else (bits.float() + 0.5) / 65536.0
    q = q + (y - q >= threshold).float()
    return (torch.ldexp(q, d) + 0.0).to(f8), (e + 127).to(torch.uint8).view(torch.float8_e8m0fnu)


def _values(b, dtype=torch.float32):
    codes = b["codes"][:, :b["cols"]].view(GRID[b["kind"]][4]).to(dtype)
    scales = torch.ldexp(torch.ones((), dtype=dtype, device=DEV), b["exps"].int() - 127)
    return codes * scales.repeat_interleave(BLOCK, 1)[:, :b["cols"]]


def _both_layouts(x, kind, sr, seed):
    bits = _philox(x.numel(), seed).view(x.shape) if sr else None
    return [*_to_blocks(x, kind, bits), *_to_blocks(x.t().contiguous(), kind, None if bits is None else bits.t())]


def _act(g, name):
    """The activation and its derivative."""
    if name == "silu":
        s = torch.sigmoid(g)
        return g * s, s * (1.0 + g * (1.0 - s))
    p = 0.5 * (1.0 + torch.erf(g * math.sqrt(0.5)))
    return g * p, p + g * torch.exp(-0.5 * g * g) * (1.0 / math.sqrt(2.0 * math.pi))


def _plain(s):
    op = s["op"]
    if op == "norm_fwd":
        h = (s["x"].float() + s["res"].float()).to(s["x"].dtype)
        v = h.float()
        rstd = 1.0 / torch.sqrt(v.square().mean(1) + EPS)
        return [*_to_blocks(v * rstd[:, None] * s["gamma"], E4M3), h, rstd]
    if op == "norm_bwd":
        dy, xhat = s["dy"].float(), s["h"].float() * s["rstd"][:, None]
        d = dy * s["gamma"]
        dx = s["rstd"][:, None] * (d - xhat * (d * xhat).mean(1, keepdim=True)) + s["dh"].float()
        return [dx.to(s["h"].dtype), (dy * xhat).sum(0)]
    if op == "store":
        return _both_layouts(s["x"].float(), s["kind"], s["sr"], s["seed"])
    if op == "turn":
        return [*_to_blocks(_values(s["x"]).t().contiguous(), s["kind"])]
    if op == "product":
        return (_values(s["X"]) @ _values(s["Z"]).t()).to(TYPES[s["out"]])
    if op == "gated_fwd":
        gu = _values(s["X"]) @ _values(s["W"]).t()
        g, u = gu[:, :s["F"]], gu[:, s["F"]:]
        h = _to_blocks(_act(g, s["act"])[0] * u, E4M3)
        return [*h, *_to_blocks(gu, E4M3)] if s["keep"] else [*h]
    gu, dh = _values(s["gu"]), s["dH"].float()
    a, da = _act(gu[:, :s["F"]], s["act"])
    return _both_layouts(torch.cat([dh * gu[:, s["F"]:] * da, dh * a], 1), s["kind"], s["sr"], s["seed"])


# ---- the library ----------------------------------------------------------------------------------------------------
def _shown(b):
    """Codes and scales of the library's block-scaled matrix, without copies."""
    from paper_2511_00874_amd import lib as L
    return [b.codes[:, :b.cols].view(torch.float8_e4m3fn if b.kind == L.E4M3 else torch.float8_e5m2),
            b.exps[:, :-(-b.cols // BLOCK)].view(torch.float8_e8m0fnu)]


def _library(s):
    from paper_2511_00874_amd import lib as L
    op, kinds = s["op"], {E4M3: L.E4M3, E5M2: L.E5M2}

    def blocks(b):
        return L.Blocks(b["codes"], b["exps"], kinds[b["kind"]], b["cols"])

    def quant():
        return L.Quant(kinds[s["kind"]], 1.0, seed=s["seed"], round_mode=L.SR if s["sr"] else L.RTN)

    if op == "norm_fwd":
        y, h, rstd = L.sr_rmsnorm_fwd(s["x"], s["gamma"], EPS, residual=s["res"], q=L.RTN_E4M3)
        return [*_shown(y), h, rstd]
    if op == "norm_bwd":
        return [*L.sr_rmsnorm_bwd(s["dy"], s["h"], s["rstd"], s["gamma"], dh=s["dh"])]
    if op == "store":
        rows, turned = L.sr_block_quantize(s["x"], quant(), layout=L.BOTH)
        return [*_shown(rows), *_shown(turned)]
    if op == "turn":
        return _shown(L.sr_block_turn(blocks(s["x"])))
    if op == "product":
        return L.sr_gemm_blocks(blocks(s["X"]), blocks(s["Z"]), dtype=TYPES[s["out"]], f8_pipeline=s["f8"])
    act = L.ACT_SILU if s["act"] == "silu" else L.ACT_GELU
    if op == "gated_fwd":
        h, gu = L.sr_gated_fwd(blocks(s["X"]), blocks(s["W"]), act=act, qh=L.RTN_E4M3, qgu=L.RTN_E4M3 if s["keep"] else None,
                               f8_pipeline=s["f8"])
        return [*_shown(h), *_shown(gu)] if s["keep"] else _shown(h)
    rows, turned = L.sr_gated_bwd(s["dH"], blocks(s["gu"]), quant(), act=act)
    return [*_shown(rows), *_shown(turned)]


def run(state):
    return _library(state) if own else _plain(state)


# ---- the definitions in 64 bits -------------------------------------------------------------------------------------
def _scaled64(v, kind):
    """v in units of its blocks' scales, not rounded to 8 bits, and the scales: the least powers of two that fit."""
    R, C = v.shape
    nb, qmax = -(-C // BLOCK), GRID[kind][0]
    w = torch.zeros((R, nb * BLOCK), dtype=torch.float64, device=DEV)
    w[:, :C] = v
    top = w.view(R, nb, BLOCK).abs().max(2).values
    e = torch.ceil(torch.log2(top / qmax))
    e = torch.where(torch.exp2(e) * qmax < top, e + 1, torch.where(torch.exp2(e - 1) * qmax >= top, e - 1, e))
    scale = torch.where(top == 0, 1.0, torch.exp2(e.clamp(min=-100)))
    return [(w.view(R, nb, BLOCK) / scale[:, :, None]).view(R, nb * BLOCK)[:, :C], scale]


def _decoded64(b):
    """Value of every code by the bits of its format."""
    _, m, emin, _, _ = GRID[b["kind"]]
    c = b["codes"][:, :b["cols"]].long()
    field, frac = (c & 127) >> m, (c & ((1 << m) - 1)).double()
    mag = torch.where(field == 0, frac, frac + (1 << m)) * torch.exp2(field.clamp(min=1).double() - 1 + emin - m)
    at = torch.arange(b["cols"], device=DEV) // BLOCK
    return torch.where(c >= 128, -mag, mag) * torch.exp2(b["exps"].double() - 127)[:, at]


def _act64(g, name):
    if name == "silu":
        q = torch.exp(-g)
        return g / (1 + q), (1 + q + g * q) / (1 + q) ** 2
    c = torch.special.erfc(-g / math.sqrt(2)) / 2
    return g * c, c + g * torch.exp(-g * g / 2) / math.sqrt(2 * math.pi)


def exact(case, seed):
    s, op = prepare(case, seed), case["op"]
    if op == "norm_fwd":
        h = (s["x"].double() + s["res"].double()).to(s["x"].dtype).double()  # (the norm is that of the stored sum)
        rstd = (h.pow(2).sum(1) / h.shape[1] + EPS).pow(-0.5)
        return [*_scaled64(h * rstd[:, None] * s["gamma"].double(), E4M3), s["x"].double() + s["res"].double(), rstd]
    if op == "norm_bwd":
        dy, h, r, w = s["dy"].double(), s["h"].double(), s["rstd"].double()[:, None], s["gamma"].double()
        along = (dy * w * h).sum(1, keepdim=True) / h.shape[1]
        return [r * dy * w - h * r ** 3 * along + s["dh"].double(), (dy * h * r).sum(0)]
    if op == "store":
        v = s["x"].double()
        return [*_scaled64(v, s["kind"]), *_scaled64(v.t(), s["kind"])]
    if op == "turn":
        return _scaled64(_decoded64(s["x"]).t(), s["kind"])
    if op == "product":
        return _decoded64(s["X"]) @ _decoded64(s["Z"]).t()
    F = case["F"]
    if op == "gated_fwd":
        x, w = _decoded64(s["X"]), _decoded64(s["W"])
        g, u = x @ w[:F].t(), x @ w[F:].t()
        h = _scaled64(_act64(g, case["act"])[0] * u, E4M3)
        return [*h, *_scaled64(torch.cat([g, u], 1), E4M3)] if case["keep"] else h
    gu, dh = _decoded64(s["gu"]), s["dH"].double()
    a, da = _act64(gu[:, :F], case["act"])
    v = torch.cat([dh * gu[:, F:] * da, dh * a], 1)
    return [*_scaled64(v, case["kind"]), *_scaled64(v.t(), case["kind"])]


# ---- what a pass cannot do without ----------------------------------------------------------------------------------
def work(case):
    op, M = case["op"], case["M"]
    es = {"bf16": 2, "f32": 4}.get(case.get("type"), 0)

    def held(rows, cols):
        return rows * cols + rows * -(-cols // BLOCK)

    if op == "norm_fwd":
        K = case["K"]
        return {"bytes": 3 * es * M * K + held(M, K) + 4 * K + 4 * M, "flops": 6.0 * M * K}
    if op == "norm_bwd":
        K = case["K"]
        return {"bytes": 4 * es * M * K + 8 * K + 4 * M, "flops": 10.0 * M * K}
    if op == "store":
        K = case["K"]
        return {"bytes": es * M * K + held(M, K) + held(K, M), "flops": 8.0 * M * K}
    if op == "turn":
        K = case["K"]
        return {"bytes": held(M, K) + held(K, M), "flops": 4.0 * M * K}
    if op == "product":
        N, K = case["N"], case["K"]
        return {"bytes": held(M, K) + held(N, K) + M * N * (2 if case["out"] == "bf16" else 4), "flops": 2.0 * M * N * K}
    F = case["F"]
    if op == "gated_fwd":
        K = case["K"]
        return {"bytes": held(M, K) + held(2 * F, K) + held(M, F) * (3 if case["keep"] else 1), "flops": 4.0 * M * F * K}
    return {"bytes": es * M * F + held(M, 2 * F) + held(M, 2 * F) + held(2 * F, M), "flops": 20.0 * M * F}
