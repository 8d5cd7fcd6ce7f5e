"""AdamW over many tensors, against its definition in 64 bits and the rounding rules of the formats it stores."""
import numpy as np
import pytest
import torch

import block_util as B
import oracle
from gpu_util import DEV, host_src, say
from paper_2511_00874_amd import lib as L

pytestmark = pytest.mark.gpu
U = 2.0**-24
BETAS, EPS = (0.9, 0.95), 1e-8


def _tensor(n, seed, w, g, bits, offset=0, decay=0.1):
    rng = np.random.default_rng(seed)
    size = 1e-3 * np.exp(2 * rng.standard_normal(n))
    f = lambda x, t: torch.from_numpy(x).to(DEV).to(t)  # noqa: E731
    m, v = 0.3 * size * rng.standard_normal(n), size * size * (0.2 + rng.random(n))
    t = L.AdamWTensor.zeros(f(0.02 * rng.standard_normal(n), w), f(size * rng.standard_normal(n), g), bits, weight_decay=decay, counter_offset=offset)
    if bits == 32:
        t.m.copy_(f(m, torch.float32))
        t.v.copy_(f(v, torch.float32))
    else:
        for x, scales, val in ((t.m, t.m_scales, m), (t.v, t.v_scales, np.sqrt(v))):
            codes, e = B.block_codes(val[None], L.E4M3)
            x.copy_(torch.from_numpy(codes.reshape(-1)))
            scales.copy_(torch.from_numpy((e.reshape(-1) + 127).astype(np.uint8)))
    return t


def _want(t, lr, step):
    """w, m, v after a step and how far each may be off before it is rounded for storage."""
    w, g, m, v = B.wide(t.w), B.wide(t.g), B.wide(t.first()), B.wide(t.second())
    b1, b2 = BETAS
    m1, v1 = b1 * m + (1 - b1) * g, b2 * v + (1 - b2) * g * g
    em, ev = 4 * U * (np.abs(b1 * m) + np.abs((1 - b1) * g)), 6 * U * v1
    c1, c2 = 1 - b1**step, 1 - b2**step
    root = np.sqrt(v1 / c2) + EPS
    update = m1 / c1 / root
    # 1 - beta^step as expm1 of step log(beta), both rounded: off by step |log beta| beta^step / (1 - beta^step) roundings, at most one, and expm1's few
    eu = em / c1 / root + np.abs(update) * 24 * U
    w1 = w - lr * (update + t.weight_decay * w)
    return (w1, m1, v1), (lr * (eu + 4 * U * (np.abs(update) + np.abs(t.weight_decay * w))) + 2 * U * (np.abs(w) + np.abs(w1)), em, ev)


def _blocks(codes, scales):
    e = np.zeros((1, -(-scales.numel() // 4) * 4), np.uint8)
    e[0, :scales.numel()] = scales.cpu().numpy()
    n = codes.numel()
    c = np.zeros((1, -(-n // 16) * 16), np.uint8)
    c[0, :n] = codes.cpu().numpy()
    return L.Blocks(torch.from_numpy(c), torch.from_numpy(e), L.E4M3, n)


def _check(t, want, err, sr, what):
    (w, m, v), (ew, em, ev) = want, err
    got = B.wide(t.w)
    if t.w.dtype is torch.float32:
        assert np.all(np.abs(got - w) <= ew), what
    else:
        step = 2.0**(np.floor(np.log2(np.maximum(np.abs(w) + ew, 1e-30))) - 7)
        assert np.all(np.abs(got - w) <= (step if sr else step / 2) + ew), what
    if t.m_scales is None:
        assert np.all(np.abs(B.wide(t.m) - m) <= em) and np.all(np.abs(B.wide(t.v) - v) <= ev), what
        return
    B.check_blocks(_blocks(t.m, t.m_scales), m[None], em[None], (what, "m"), sr)
    # the root is rounded by squares: nearest too is one of the two neighbours, and nothing above zero becomes zero
    root = np.sqrt(v)
    least = 2.0**-9 * 2.0**(t.v_scales.cpu().numpy().astype(int) - 127).repeat(128)[:v.size]
    got = np.sqrt(B.wide(t.second()))
    assert np.all((got > 0) == (v > 0)), what
    B.check_blocks(_blocks(t.v, t.v_scales), root[None], (ev / np.maximum(root, 1e-30) + U * root + (got <= least * 1.001) * least)[None], (what, "v"), True)


SIZES = [1, 7, 8, 127, 128, 129, 768, 2047, 2048, 2049, 5000, 70001]


@pytest.mark.parametrize("w", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("g", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("bits", [8, 32])
@pytest.mark.parametrize("mode", [L.SR, L.RTN])
def test_step(w, g, bits, mode):
    say("adamw", w, g, bits, mode)
    ts = [_tensor(n, i, w, g, bits, offset=1000 * i, decay=0.1 * (i % 3)) for i, n in enumerate(SIZES)]
    for step in (1, 2, 1000):
        want = [_want(t, 1e-3, step) for t in ts]
        L.sr_adamw(ts, 1e-3, step, betas=BETAS, eps=EPS, round_mode=mode, seed=5)
        for t, (x, e) in zip(ts, want):
            _check(t, x, e, mode == L.SR, (t.w.numel(), step))


def test_a_list_is_its_tensors_one_by_one():
    # over a hundred tensors of all kinds: several launches
    def some():
        rng = np.random.default_rng(0)
        kinds = [(a, b, c) for a in (torch.float32, torch.bfloat16) for b in (torch.float32, torch.bfloat16) for c in (8, 32)]
        return [_tensor(int(rng.integers(0, 5000)), i, *kinds[int(rng.integers(0, 8)) if i < 40 else i % 2], offset=i << 20) for i in range(260)]
    a, b = some(), some()
    L.sr_adamw(a, 1e-3, 7, seed=3)
    for t in b:
        L.sr_adamw([t], 1e-3, 7, seed=3)
    for i, (x, y) in enumerate(zip(a, b)):
        assert torch.equal(x.w, y.w) and torch.equal(x.m, y.m) and torch.equal(x.v, y.v), i
        assert x.m_scales is None or (torch.equal(x.m_scales, y.m_scales) and torch.equal(x.v_scales, y.v_scales)), i


def test_bfloat16_weights_take_the_thresholds_of_the_update():
    # without moments and decay the step is w - lr * sign-like update: with beta1 = beta2 = 0 it is g / (|g| + eps); its rounding is sr_update_bf16's
    n = 4099
    rng = np.random.default_rng(1)
    w0 = torch.from_numpy(rng.standard_normal(n)).to(DEV).bfloat16()
    g = torch.from_numpy(np.sign(rng.standard_normal(n))).float().to(DEV)
    t = L.AdamWTensor.zeros(w0.clone(), g, 32, counter_offset=77)
    lr = 0.0012345
    L.sr_adamw([t], lr, 1, betas=(0.0, 0.0), eps=0.0, seed=9)  # update = sign(g) exactly
    want = oracle.update_bf16(host_src(w0), g.cpu().numpy(), np.float32(lr), 9, 77)
    assert np.array_equal(host_src(t.w), np.asarray(want).view(np.uint16).reshape(-1))


@pytest.mark.parametrize("mode", [L.SR, L.RTN])
def test_codes_of_the_moments(mode):
    # first moment: the codes of the block quantizer; second: by squares, with thresholds of their own stretch of the stream
    n = 128 * 33 + 40
    t = _tensor(n, 4, torch.float32, torch.float32, 8, offset=50)
    w = L.AdamWTensor.zeros(t.w.clone(), t.g, 32, weight_decay=t.weight_decay)
    w.m.copy_(t.first())
    w.v.copy_(t.second())
    L.sr_adamw([t], 1e-3, 3, betas=BETAS, round_mode=mode, seed=11)
    L.sr_adamw([w], 1e-3, 3, betas=BETAS, round_mode=mode, seed=11)
    assert torch.equal(t.w, w.w)  # from the moments before they are rounded
    groups = (n + 7) // 8
    padded = torch.zeros(-(-n // 16) * 16, device=DEV)
    padded[:n] = w.m
    b = L.sr_block_quantize(padded[None], L.Quant(L.E4M3, 1.0, seed=11, counter_offset=50 + groups, round_mode=mode))
    assert torch.equal(b.codes[0, :n], t.m) and torch.equal(b.exps[0, :t.m_scales.numel()], t.m_scales)
    v = B.wide(w.v)
    e = B.block_exponents(np.sqrt(v)[None], L.E4M3)
    assert np.array_equal(t.v_scales.cpu().numpy().astype(int) - 127, e[0])
    scale = 2.0**e[0].repeat(128)[:n].astype(float)
    grid = oracle.decode_array(L.E4M3, np.arange(127, dtype=np.uint8)).astype(float)  # ascending
    r = np.sqrt(v) / scale
    low = np.clip(np.searchsorted(grid, r, side="right") - 1, 0, 125)
    a, c = grid[low], grid[low + 1]
    part = (r * r - a * a) / (c * c - a * a)
    eps = np.array([0.5 if mode == L.RTN else oracle.eps_from_r16(oracle.r16(11, 50 + 2 * groups, i)) for i in range(n)])
    code = low + (part >= eps)
    code = np.where((code == 0) & (v > 0), 1, code)
    sure = np.abs(part - eps) > 1e-4  # (binary32: part is known to a few 2^-17)
    got = t.v.cpu().numpy().astype(int)
    assert np.array_equal(got[sure], code[sure]) and sure.mean() > 0.99
    assert np.all(np.abs(got - code) <= 1)


def test_stochastic_rounding_keeps_the_second_moment():
    # one value in all places, the block's scale set by one of them: the mean of the squares is the value (4 sigma of 2^17 draws)
    n = 1 << 17
    v0 = np.float32(0.37**2)
    t = L.AdamWTensor.zeros(torch.zeros(n, device=DEV), torch.zeros(n, device=DEV), 8)
    g = torch.full((n,), 0.37, device=DEV)
    g[::128] = 1.0
    t.g = g
    L.sr_adamw([t], 0.0, 1, betas=(0.0, 0.0), seed=2)
    got = B.wide(t.second()).reshape(-1, 128)[:, 1:].reshape(-1)
    lo, hi = got.min(), got.max()
    assert lo < v0 < hi and len(np.unique(got)) == 2
    assert abs(got.mean() - v0) <= 4 * (hi - lo) / 2 / np.sqrt(got.size) + 1e-6


def test_state_of_zeros_and_gradients_of_zero():
    for bits in (8, 32):
        t = L.AdamWTensor.zeros(torch.ones(300, device=DEV), torch.zeros(300, device=DEV), bits)
        L.sr_adamw([t], 1e-2, 1)
        assert (t.w == 1).all() and not t.first().any() and not t.second().any()


def test_what_is_not_finite_keeps_to_its_value():
    for bits in (8, 32):
        t = _tensor(1000, 1, torch.float32, torch.float32, bits)
        t.g[5], t.g[300] = float("nan"), float("inf")
        L.sr_adamw([t], 1e-3, 2, betas=BETAS)
        bad = [i for i in range(1000) if not torch.isfinite(t.w[i])]
        assert bad == [5, 300]


def test_values_on_the_device_and_replay():
    # lr, step and stream position read when the kernels run: a captured step replayed is the steps themselves
    def make():
        return [_tensor(5000, 1, torch.bfloat16, torch.float32, 8), _tensor(900, 2, torch.float32, torch.float32, 32, offset=3000)]
    a, b = make(), make()
    used = sum(t.blocks() for t in a)
    lr, step, pos = torch.zeros(1, device=DEV), torch.zeros(1, dtype=torch.int64, device=DEV), torch.zeros(1, dtype=torch.int64, device=DEV)
    batch = L.AdamWBatch(a)
    lr.fill_(1e-3)
    step.fill_(1)
    keep = [[x.clone() for x in (t.w, t.m, t.v)] + ([t.m_scales.clone(), t.v_scales.clone()] if t.m_scales is not None else []) for t in a]
    batch.run(lr, step, betas=BETAS, seed=4, counter=pos)
    torch.cuda.synchronize()
    for t, k in zip(a, keep):
        for x, y in zip((t.w, t.m, t.v, t.m_scales, t.v_scales), k):
            x.copy_(y)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        batch.run(lr, step, betas=BETAS, seed=4, counter=pos)
    for i in range(1, 5):
        lr.fill_(1e-3 / i)
        step.fill_(i)
        pos.fill_(used * i)
        graph.replay()
        torch.cuda.synchronize()
        for t in b:
            t.counter_offset += used
        L.sr_adamw(b, 1e-3 / i, i, betas=BETAS, seed=4)
        for x, y in zip(a, b):
            assert torch.equal(x.w, y.w) and torch.equal(x.m, y.m) and torch.equal(x.v, y.v), i


def test_nothing():
    L.sr_adamw([], 1e-3, 1)
    t = L.AdamWTensor.zeros(torch.empty(0, device=DEV), torch.empty(0, device=DEV))
    L.sr_adamw([t], 1e-3, 1)
