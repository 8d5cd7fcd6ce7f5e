"""Attention, embedding and AdamW: what is timed of them, in plain torch operations and through the library.

They are the parts of a decoder's training step, and of serving it, around the quantized linears and the gated block.  "op" of a case:

  attention       softmax(Q K^T / sqrt(D), causal) V over sequences packed back to back, query heads in groups that share a key head;
                  with "capacity": one new query a sequence over a cache of that many rows a sequence, of which some are filled
  attention_step  the same, and the gradients of Q, K and V from that of the result
  embed           rows of a table, scaled
  embed_grad      the gradient of the table from that of the rows
  adamw           one step over many tensors: weights in bfloat16 (rounded stochastically) or binary32, both moments in binary32 or in 8 bits
                  (E4M3 and a power of two for every 128 values; the second moment as its root)

What is held in 8 bits is returned as it is held: 8-bit floats, and the scales as powers of two.
"""
import math
import random

import torch

own = False
DEV = "cuda:0"
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
BLOCK = 128
LR, BETA1, BETA2, EPS, STEP = 3e-4, 0.9, 0.95, 1e-8, 1000
INF = float("inf")


def listed():
    return [
        # four sequences being generated by the 768-wide model: one token each, caches of its 1024 positions
        {"name": "attention_token", "op": "attention", "seqs": 4, "capacity": 1024, "heads": 12, "kv": 12, "D": 64},
        # one token for each of 24 long conversations, four query heads to a key head
        {"name": "attention_tokens_long", "op": "attention", "seqs": 24, "capacity": 32768, "heads": 16, "kv": 4, "D": 128},
        # prompts of all lengths packed into one batch, in the 2048-wide layer
        {"name": "attention_prompts", "op": "attention", "seqs": 23, "longest": 1999, "heads": 32, "kv": 8, "D": 64},
        # one long document
        {"name": "attention_document", "op": "attention", "seqs": 1, "longest": 16384, "heads": 16, "kv": 4, "D": 128},
        # the 768-wide decoder's training batch
        {"name": "attention_step_768", "op": "attention_step", "seqs": 8, "longest": 1024, "equal": True, "heads": 12, "kv": 12, "D": 64},
        # training on packed documents, the 2048-wide layer with shared key heads
        {"name": "attention_step_packed", "op": "attention_step", "seqs": 9, "longest": 4095, "heads": 16, "kv": 4, "D": 128},
        # the next tokens of a few sequences
        {"name": "embed_token", "op": "embed", "M": 7, "V": 32000, "K": 2048, "table": "bf16", "type": "bf16", "scale": 1.0},
        # gradient of the 768-wide decoder's table, an odd batch
        {"name": "embed_grad_768", "op": "embed_grad", "M": 8191, "V": 32000, "K": 768, "type": "f32", "scale": 1.0},
        # the largest batch of the 2048-wide layer, scaled embedding
        {"name": "embed_grad_64k", "op": "embed_grad", "M": 65536, "V": 32000, "K": 2048, "type": "bf16", "scale": math.sqrt(2048)},
        # gains and offsets of the 768-wide decoder's norms: small tensors, where the launch is all there is
        {"name": "adamw_norms", "op": "adamw", "tensors": 50, "least": 768, "most": 768, "w": "f32", "g": "f32", "bits": 32},
        # the linears of that decoder
        {"name": "adamw_768", "op": "adamw", "layers": 12, "d": 768, "f": 0, "w": "bf16", "g": "f32", "bits": 32},
        # four layers of the 2048-wide model with both moments in 8 bits
        {"name": "adamw_2048_8bit", "op": "adamw", "layers": 4, "d": 2048, "f": 5632, "w": "bf16", "g": "f32", "bits": 8},
    ]


def _log(rng, lo, hi, multiple=1):
    v = math.exp(rng.uniform(math.log(lo), math.log(hi)))
    return max(multiple, int(v / multiple + 0.5) * multiple)


def draw(rng):
    op = rng.choice(["attention", "attention", "token", "token", "attention_step", "attention_step", "embed", "embed_grad", "embed_grad", "adamw", "adamw"])
    while True:
        if op in ("attention", "token", "attention_step"):
            kv, group, D = rng.choice([1, 2, 4, 8, 12]), rng.choice([1, 1, 2, 4, 8]), rng.choice([64, 64, 128, 128, 80, 96])
            if kv * group > 32:
                continue
            c = {"op": "attention" if op == "token" else op, "heads": kv * group, "kv": kv, "D": D}
            if op == "token":
                c |= {"seqs": _log(rng, 1, 64), "capacity": _log(rng, 128, 32768)}
                if c["seqs"] * c["capacity"] * kv * D <= 24 * 32768 * 4 * 128:
                    return c
            else:
                c |= {"seqs": _log(rng, 1, 32), "longest": _log(rng, 16, 16384 if op == "attention" else 8192)}
                pairs = c["seqs"] * c["longest"] ** 2 * c["heads"]
                if pairs <= (16 * 16384 ** 2 if op == "attention" else 9 * 16 * 4095 ** 2):
                    return c
        elif op == "embed":
            return {"op": op, "M": _log(rng, 1, 65536), "V": _log(rng, 1000, 131072), "K": _log(rng, 64, 4096, 8), "table": rng.choice(["bf16", "f32"]),
                    "type": rng.choice(["bf16", "f32"]), "scale": rng.choice([1.0, 16.0, 45.25])}
        elif op == "embed_grad":
            c = {"op": op, "M": _log(rng, 1, 65536), "V": _log(rng, 1000, 131072), "K": _log(rng, 64, 4096, 8), "type": rng.choice(["bf16", "f32"]),
                 "scale": rng.choice([1.0, 16.0, 45.25])}
            if (c["M"] + c["V"]) * c["K"] <= 97536 * 2048:
                return c
        else:
            c = {"op": op, "tensors": _log(rng, 1, 200), "least": rng.choice([1, 64, 768]), "most": _log(rng, 1000, 16 << 20), "w": rng.choice(["bf16", "f32"]),
                 "g": rng.choice(["f32", "f32", "bf16"]), "bits": rng.choice([8, 32])}
            if sum(_sizes(c)) <= 200 << 20:
                return c


# ---- sizes that a case stands for -----------------------------------------------------------------------------------
def _lengths(case):
    """Rows of every sequence: the longest, others from one row on (filled rows of every cache)."""
    most = case.get("capacity") or case["longest"]
    if case.get("equal"):
        return [most] * case["seqs"]
    rng = random.Random(most * 1000 + case["seqs"])
    n = [most] + [_log(rng, max(1, most // 64), most) for _ in range(case["seqs"] - 1)]
    rng.shuffle(n)
    return n


def _sizes(case):
    """Values of every tensor of an optimizer step."""
    if "layers" in case:
        d, f = case["d"], case["f"]
        return ([d * d] * 4 + [d * f] * 3 if f else [3 * d * d, d * d, 4 * d * d, 4 * d * d]) * case["layers"]
    rng = random.Random(case["most"] * 1000 + case["tensors"])
    return [case["most"]] + [_log(rng, case["least"], case["most"]) for _ in range(case["tensors"] - 1)]


def _places(case):
    """Where each tensor begins in the flat buffers (whole blocks of 128), and their length."""
    at, places = 0, []
    for n in _sizes(case):
        places.append(at)
        at += -(-n // BLOCK) * BLOCK
    return places, at


# ---- inputs ---------------------------------------------------------------------------------------------------------
def _gauss(g, shape, std=1.0):
    return torch.randn(shape, generator=g, device=DEV) * std


def _heads(g, rows, heads, D, channels):
    """Projections of tokens: channels of different strength, some with an offset."""
    return _gauss(g, (rows, heads, D)) * torch.exp(_gauss(g, (1, heads, D), 0.3)) + _gauss(g, (1, heads, D), channels)


def _gradients(g, shape):
    """Tokens whose losses differ by orders of magnitude."""
    return _gauss(g, shape, 1e-3) * torch.exp(_gauss(g, (shape[0],) + (1,) * (len(shape) - 1), 1.5))


def prepare(case, seed):
    g = torch.Generator(device=DEV).manual_seed(seed)
    op, s = case["op"], dict(case)
    if op in ("attention", "attention_step"):
        H, kv, D, n = case["heads"], case["kv"], case["D"], _lengths(case)
        s["n"] = n
        if "capacity" in case:
            s["q"] = _heads(g, case["seqs"], H, D, 0.3).bfloat16()
            s["keys"], s["values"] = (_heads(g, case["seqs"] * case["capacity"], kv, D, 0.5).bfloat16() for _ in range(2))
            s["lengths"] = torch.tensor(n, dtype=torch.int32, device=DEV)
        else:
            s["qkv"] = torch.cat([_heads(g, sum(n), H, D, 0.3), _heads(g, sum(n), kv, D, 0.5), _heads(g, sum(n), kv, D, 0.3)], 1).bfloat16()
            ends = [0]
            for v in n:
                ends.append(ends[-1] + v)
            s["offsets"] = torch.tensor(ends, dtype=torch.int32, device=DEV)
        if op == "attention_step":
            s["do"] = _gradients(g, (sum(n), H, D)).bfloat16()
    elif op in ("embed", "embed_grad"):
        V, M, K = case["V"], case["M"], case["K"]
        often = 1.0 / (torch.arange(V, device=DEV) + 2.7)  # the frequencies of words
        s["ids"] = torch.multinomial(often, M, replacement=True, generator=g)
        if op == "embed":
            s["rows"] = _gauss(g, (V, K), 0.02).to(TYPES[case["table"]])
        else:
            s["dy"] = _gradients(g, (M, K)).to(TYPES[case["type"]])
    else:
        places, total = _places(case)
        s["places"], s["n"], s["seed"] = places, _sizes(case), seed
        live = torch.zeros(total + 1, dtype=torch.int32, device=DEV)
        live[torch.tensor(places, device=DEV)] += 1
        live.index_add_(0, torch.tensor([a + n for a, n in zip(places, s["n"])], device=DEV), torch.full((len(places),), -1, dtype=torch.int32, device=DEV))
        live = torch.cumsum(live, 0)[:total].float()  # ones where a tensor has values, zeros between them
        size = 1e-4 * torch.exp(_gauss(g, (total,))) * live
        s["w"] = (_gauss(g, (total,), 0.02) * live).to(TYPES[case["w"]])
        s["g"] = (_gauss(g, (total,)) * size).to(TYPES[case["g"]])
        s["m"], s["v"] = _gauss(g, (total,), 0.3) * size, size * size * (0.3 + torch.rand(total, generator=g, device=DEV))
        if case["bits"] == 8:
            (s["m"], s["m_scales"]), (s["v"], s["v_scales"]) = (_held(x) for x in (s["m"], torch.sqrt(s["v"])))
    return s


# ---- the plain forms ------------------------------------------------------------------------------------------------
def _padded(s):
    """Q (B, kv, group * Lq, D), K and V (B, kv, Lk, D) in binary32, every sequence filled up to the longest; what sees what (B, 1, group * Lq, Lk); and the
    places (sequence, row) of the packed rows."""
    H, kv, D, B = s["heads"], s["kv"], s["D"], s["seqs"]
    group = H // kv
    if "capacity" in s:
        seen = torch.arange(s["capacity"], device=DEV) < s["lengths"][:, None]
        q = s["q"].float().view(B, kv, group, D)
        k, v = (s[x].float().view(B, s["capacity"], kv, D).transpose(1, 2).contiguous() for x in ("keys", "values"))
        return q, k, v, seen[:, None, None, :].expand(B, 1, group, s["capacity"]), None
    first, L = s["offsets"][:-1].long(), max(s["n"])
    n = s["offsets"][1:].long() - first
    row = torch.arange(L, device=DEV)
    at = (first[:, None] + row).clamp(max=s["qkv"].shape[0] - 1)  # (B, L)
    x = s["qkv"].float()[at]                                   # (B, L, heads, D)
    q = x[:, :, :H].reshape(B, L, kv, group, D).permute(0, 2, 3, 1, 4).reshape(B, kv, group * L, D)
    k, v = (x[:, :, a:a + kv].transpose(1, 2).contiguous() for a in (H, H + kv))
    mine = (row < n[:, None])[:, None, :]                      # keys of the sequence
    seen = ((row[None, :] <= row[:, None])[None] & mine)       # (B, L, L)
    flat = (torch.arange(B, device=DEV)[:, None].expand(B, L)[row < n[:, None]], row[None].expand(B, L)[row < n[:, None]])
    return q, k, v, seen[:, None].repeat(1, 1, group, 1), flat


def _packed(x, s, flat, heads):
    """(B, kv, group * L, D) back to (rows, heads, D)."""
    B, kv, D = x.shape[0], s["kv"], x.shape[-1]
    x = x.view(B, kv, heads // kv, -1, D).reshape(B, heads, -1, D)
    return x[:, :, 0] if flat is None else x[flat[0], :, flat[1]]


def _attention(s, step):
    q, k, v, seen, flat = _padded(s)
    scale = 1.0 / math.sqrt(s["D"])
    p = torch.matmul(q, k.transpose(2, 3).contiguous()).mul_(scale).masked_fill_(~seen, -INF)
    top = p.amax(3, keepdim=True)
    top = torch.where(top == -INF, 0.0, top)
    p = p.sub_(top).exp_()
    total = p.sum(3, keepdim=True)
    p = p.div_(torch.where(total == 0, 1.0, total))
    o = _packed(torch.matmul(p, v), s, flat, s["heads"])
    out = [o.bfloat16(), _packed(top + torch.log(total), s, flat, s["heads"])[..., 0].t().contiguous()]
    if not step:
        return out
    B, L, kv, group, D = s["seqs"], max(s["n"]), s["kv"], s["heads"] // s["kv"], s["D"]
    do = torch.zeros((B, s["heads"], L, D), device=DEV)
    do[flat[0], :, flat[1]] = s["do"].float()
    do = do.view(B, kv, group * L, D)
    dv = torch.matmul(p.transpose(2, 3).contiguous(), do)
    dp = torch.matmul(do, v.transpose(2, 3).contiguous())
    ds = dp.sub_((dp * p).sum(3, keepdim=True)).mul_(p).mul_(scale)
    dq, dk = torch.matmul(ds, k), torch.matmul(ds.transpose(2, 3).contiguous(), q)
    return out + [_packed(dq, s, flat, s["heads"]).bfloat16(), _packed(dk, s, flat, kv).bfloat16(), _packed(dv, s, flat, kv).bfloat16()]


def _philox(block, seed):
    """The 16 random bits of the eight elements of every block: Philox4x32-10."""
    lo32 = 0xFFFFFFFF
    c = [block & lo32, block >> 32, torch.zeros_like(block), torch.zeros_like(block)]
    k0, k1 = seed & lo32, (seed >> 32) & lo32
    for _ in range(10):
        p0, p1 = c[0] * 0xD2511F53, c[2] * 0xCD9E8D57
        c = [((p1 >> 32) & lo32) ^ c[1] ^ k0, p1 & lo32, ((p0 >> 32) & lo32) ^ c[3] ^ k1, p0 & lo32]
        k0, k1 = (k0 + 0x9E3779B9) & lo32, (k1 + 0xBB67AE85) & lo32
    return torch.stack([h for w in c for h in (w & 0xFFFF, w >> 16)], 1).view(-1)


def _block_scale(x):
    """Exponents (blocks of 128 along the flat axis) of the least powers of two e with max|x| <= 448 2^e."""
    amax = x.view(-1, BLOCK).abs().amax(1)
    frac, e = torch.frexp(amax)
    return torch.where(amax == 0, 0, (e - 9 + (frac > 0.875).int()).clamp(min=-100))


def _held(x, bits=None, root_of=None):
    """x as codes and scales.  bits: rounded stochastically by them, else to nearest; root_of: x is the root of these, whose expectation is kept: between
    two neighbours by where the square lies between theirs, and never from above zero to zero."""
    e = _block_scale(x)
    by = e.repeat_interleave(BLOCK)
    t = torch.ldexp(x, -by)
    d = (torch.frexp(t)[1] - 1).clamp(min=-6) - 3
    y = torch.ldexp(t, -d)
    q = torch.floor(y)
    threshold = 0.5 if bits is None else (bits.float() + 0.5) / 65536.0
    if root_of is None:
        q = q + (y - q >= threshold).float()
    else:
        u = torch.ldexp(torch.ldexp(root_of, -2 * by), -2 * d)
        q = q + (u - q * q >= threshold * (2.0 * q + 1.0)).float()
        q = torch.where((q == 0) & (root_of > 0), 1.0, q)
    return (torch.ldexp(q, d) + 0.0).to(torch.float8_e4m3fn).view(torch.uint8), (e + 127).to(torch.uint8)


def _values(codes, scales):
    return torch.ldexp(codes.view(torch.float8_e4m3fn).float(), (scales.int() - 127).repeat_interleave(BLOCK))


def _to_bf16(x, bits):
    """Stochastically rounded: the chance of the neighbour above is the distance from the one below."""
    u = x.contiguous().view(torch.int32).long() & 0xFFFFFFFF
    mag, negative = u & 0x7FFFFFFF, u >> 31
    mag = ((mag + torch.where(negative == 1, bits, 65535 - bits)) >> 16) << 16
    return torch.where(negative == 1, -1.0, 1.0) * mag.to(torch.int32).view(torch.float32) + 0.0


def _adamw(s):
    total, sizes = s["w"].numel(), torch.tensor(s["n"], device=DEV)
    groups, eights = -(-sizes // BLOCK) * (BLOCK // 8), (sizes + 7) // 8
    first = 3 * (torch.cumsum(eights, 0) - eights)             # every tensor's stretch of the random stream: weights, first, second moment
    place = torch.cumsum(groups, 0) - groups
    block = (torch.arange(total // 8, device=DEV) - place.repeat_interleave(groups)) + first.repeat_interleave(groups)
    more = eights.repeat_interleave(groups)
    g, w = s["g"].float(), s["w"].float()
    m, v = (s["m"], s["v"]) if s["bits"] == 32 else (_values(s["m"], s["m_scales"]), _values(s["v"], s["v_scales"]).square())
    m = m * BETA1 + g * (1.0 - BETA1)
    v = v * BETA2 + (g * g) * (1.0 - BETA2)
    c1, c2 = 1.0 - BETA1 ** STEP, 1.0 - BETA2 ** STEP
    update = (m / c1) / (torch.sqrt(v / c2) + EPS)
    w = w - LR * (update + 0.1 * w)
    s["w"].copy_(w if s["w"].dtype is torch.float32 else _to_bf16(w, _philox(block, s["seed"])))
    if s["bits"] == 32:
        s["m"].copy_(m)
        s["v"].copy_(v)
        return [s["w"], s["m"], s["v"]]
    for x, (codes, scales) in (("m", _held(m, _philox(block + more, s["seed"]))),
                               ("v", _held(torch.sqrt(v), _philox(block + 2 * more, s["seed"]), root_of=v))):
        s[x].copy_(codes)
        s[x + "_scales"].copy_(scales)
    return _shown(s)


def _shown(s):
    return [s["w"]] + [s[x].view(t) for x in ("m", "v") for x, t in ((x, torch.float8_e4m3fn), (x + "_scales", torch.float8_e8m0fnu))]


def _plain(s):
    op = s["op"]
    if op in ("attention", "attention_step"):
        return _attention(s, op == "attention_step")
    if op == "embed":
        return (s["rows"][s["ids"]].float() * s["scale"]).to(TYPES[s["type"]])
    if op == "embed_grad":  # sums of neighbours in the order of the tokens, as differences of running sums (of thousands of terms: in 64 bits)
        ids, order = torch.sort(s["ids"], stable=True)
        total = torch.zeros((ids.numel() + 1, s["K"]), dtype=torch.float64, device=DEV)
        torch.cumsum(s["dy"].double()[order], 0, out=total[1:])
        first, last = (torch.searchsorted(ids, torch.arange(s["V"], device=DEV), right=r) for r in (False, True))
        return ((total[last] - total[first]) * s["scale"]).float()
    return _adamw(s)


# ---- the library ----------------------------------------------------------------------------------------------------
def _library(s):
    from paper_2511_00874_amd import lib as L
    op = s["op"]
    if op in ("attention", "attention_step"):
        if "capacity" in s:
            return [*L.sr_attention_fwd(s["q"], s["keys"], s["values"], sequences=s["seqs"], lengths_k=s["lengths"])]
        H, kv = s["heads"], s["kv"]
        q, k, v = s["qkv"][:, :H], s["qkv"][:, H:H + kv], s["qkv"][:, H + kv:]
        how = {"sequences": s["seqs"]} if s.get("equal") else {"offsets": s["offsets"]}
        o, lse = L.sr_attention_fwd(q, k, v, **how)
        return [o, lse] if op == "attention" else [o, lse, *L.sr_attention_bwd(s["do"], q, k, v, o, lse, **how)]
    if op == "embed":
        return L.sr_embedding_fwd(s["rows"], s["ids"], scale=s["scale"], dtype=TYPES[s["type"]])
    if op == "embed_grad":
        return L.sr_embedding_bwd(s["dy"], s["ids"], s["V"], scale=s["scale"])
    if "batch" not in s:  # the list of tensors, which a training loop makes once: weights, gradients and moments stay where they are
        at, batch = 0, []
        for a, n in zip(s["places"], s["n"]):
            held = {} if s["bits"] == 32 else {x + "_scales": s[x + "_scales"][a // BLOCK:][:-(-n // BLOCK)] for x in ("m", "v")}
            batch.append(L.AdamWTensor(*(s[x][a:a + n] for x in ("w", "g", "m", "v")), weight_decay=0.1, counter_offset=at, **held))
            at += 3 * ((n + 7) // 8)
        s["batch"] = L.AdamWBatch(batch)
    s["batch"].run(LR, STEP, betas=(BETA1, BETA2), eps=EPS, seed=s["seed"])
    return [s["w"], s["m"], s["v"]] if s["bits"] == 32 else _shown(s)


def run(state):
    return _library(state) if own else _plain(state)


# ---- the definitions in 64 bits -------------------------------------------------------------------------------------
def _exact_attention(s, step):
    H, kv, D = s["heads"], s["kv"], s["D"]
    results, first = [], 0
    for b, n in enumerate(s["n"]):
        if "capacity" in s:
            parts = s["q"][b:b + 1], *(s[x].view(-1, s["capacity"], kv, D)[b, :n] for x in ("keys", "values"))
        else:
            x = s["qkv"][first:first + n]
            parts = x[:, :H], x[:, H:H + kv], x[:, H + kv:]
        q, k, v = (p.double().transpose(0, 1).contiguous() for p in parts)
        hidden = torch.ones((q.shape[1], n), dtype=torch.bool, device=DEV).triu(n - q.shape[1] + 1)
        rows = []
        for h in range(kv):  # a key head with its queries
            qh, kh, vh = (t.detach().requires_grad_(step) for t in (q[h * (H // kv):(h + 1) * (H // kv)], k[h], v[h]))
            a = (qh @ kh.t().contiguous() / math.sqrt(D)).masked_fill(hidden, -INF)
            lse = torch.logsumexp(a, 2)
            o = torch.exp(a - lse[..., None]) @ vh
            r = [o.detach(), lse.detach()]
            if step:
                do = s["do"][first:first + n, h * (H // kv):(h + 1) * (H // kv)].double().transpose(0, 1).contiguous()
                r += torch.autograd.grad(o, (qh, kh, vh), do)
            rows.append(r)
            del a, o, lse
        first += q.shape[1]
        results.append([torch.cat([r[0] for r in rows]).transpose(0, 1), torch.cat([r[1] for r in rows])] +
                       ([torch.cat([r[2] for r in rows]).transpose(0, 1), *(torch.stack([r[i] for r in rows], 1) for i in (3, 4))] if step else []))
    return [torch.cat([r[i] for r in results], 1 if i == 1 else 0) for i in range(len(results[0]))]


def _units64(v):
    """v (flat, whole blocks) in units of its blocks' scales, not rounded, and the scales: the least powers of two that fit."""
    w = v.view(-1, BLOCK)
    top = w.abs().max(1).values
    e = torch.ceil(torch.log2(top / 448))
    e = torch.where(torch.exp2(e) * 448 < top, e + 1, torch.where(torch.exp2(e - 1) * 448 >= top, e - 1, e))
    scale = torch.where(top == 0, 1.0, torch.exp2(e.clamp(min=-100)))
    return [(w / scale[:, None]).view(-1), scale]


def _code64(codes, scales):
    """Value of every code by the bits of E4M3."""
    c = codes.long()
    field, frac = (c >> 3) & 15, (c & 7).double()
    mag = torch.where(field == 0, frac / 8 * 2.0 ** -6, (1 + frac / 8) * torch.exp2(field.double() - 7))
    return torch.where(c >= 128, -mag, mag) * torch.exp2(scales.double() - 127).repeat_interleave(BLOCK)


def exact(case, seed):
    s, op = prepare(case, seed), case["op"]
    if op in ("attention", "attention_step"):
        return _exact_attention(s, op == "attention_step")
    if op == "embed":
        return torch.index_select(s["rows"], 0, s["ids"]).double() * s["scale"]
    if op == "embed_grad":
        order = torch.argsort(s["ids"], stable=True)
        total = torch.cumsum(torch.nn.functional.pad(torch.bincount(s["ids"], minlength=s["V"]), (1, 0)), 0).tolist()
        out = torch.zeros((s["V"], s["K"]), dtype=torch.float64, device=DEV)
        for i in sorted(set(s["ids"].tolist())):
            out[i] = s["dy"][order[total[i]:total[i + 1]]].double().sum(0) * s["scale"]
        return out
    w, g = s["w"].double(), s["g"].double()
    m, v = (s["m"].double(), s["v"].double()) if case["bits"] == 32 else (_code64(s["m"], s["m_scales"]), _code64(s["v"], s["v_scales"]).pow(2))
    m, v = m + (g - m) * (1 - BETA1), v + (g * g - v) * (1 - BETA2)
    hat = m / -math.expm1(STEP * math.log(BETA1)), v / -math.expm1(STEP * math.log(BETA2))
    w = w * (1 - LR * 0.1) - LR * hat[0] / (hat[1].sqrt() + EPS)
    return [w, m, v] if case["bits"] == 32 else [w, *_units64(m), *_units64(v.sqrt())]


# ---- what a pass cannot do without ----------------------------------------------------------------------------------
def work(case):
    op = case["op"]
    es = {"bf16": 2, "f32": 4}
    if op in ("attention", "attention_step"):
        H, kv, D, n = case["heads"], case["kv"], case["D"], _lengths(case)
        token = "capacity" in case
        rows, keys = len(n) if token else sum(n), sum(n)
        pairs = H * (keys if token else sum(v * (v + 1) // 2 for v in n))
        forward = {"bytes": 2 * D * (2 * H * rows + 2 * kv * keys) + 4 * H * rows, "flops": 4.0 * D * pairs}
        if op == "attention":
            return forward
        return {"bytes": forward["bytes"] + 2 * D * (2 * H * rows + 2 * kv * keys), "flops": 14.0 * D * pairs}
    if op == "embed":
        M, K = case["M"], case["K"]
        return {"bytes": min(M, case["V"]) * K * es[case["table"]] + M * K * es[case["type"]] + 8 * M, "flops": 1.0 * M * K}
    if op == "embed_grad":
        M, K = case["M"], case["K"]
        return {"bytes": M * K * es[case["type"]] + 8 * M + 4 * case["V"] * K, "flops": 1.0 * M * K}
    n = sum(_sizes(case))
    held = 8 * n if case["bits"] == 32 else 2 * (n + n // BLOCK)
    return {"bytes": 2 * held + n * (2 * es[case["w"]] + es[case["g"]]), "flops": 15.0 * n}
