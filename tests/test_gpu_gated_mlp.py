"""The gated feed-forward block through autograd: a training step and single tokens, against the block written out in binary64."""
import numpy as np
import pytest
import torch

import block_util as B
from gpu_util import DEV, say
from paper_2511_00874_amd import lib as L
from paper_2511_00874_amd import train

pytestmark = pytest.mark.gpu


def _forward64(x, r, gamma, w_in, w_out, act, eps):
    h = x + r
    rstd = 1.0 / np.sqrt((h * h).mean(1, keepdims=True) + eps)
    n = h * rstd * gamma
    gu = n @ w_in.T
    f = w_in.shape[0] // 2
    a, da = B.act64(gu[:, :f], act)
    return h, rstd, n, gu, a, da, a * gu[:, f:], (a * gu[:, f:]) @ w_out.T


def _backward64(dy, dh, state, gamma, w_in, w_out):
    h, rstd, n, gu, a, da, hidden, _ = state
    f = gu.shape[1] // 2
    dhid = dy @ w_out
    dz = np.concatenate([dhid * gu[:, f:] * da, dhid * a], 1)
    dn = dz @ w_in
    xhat = h * rstd
    d = dn * gamma
    dx = rstd * (d - xhat * (d * xhat).mean(1, keepdims=True)) + dh
    return dx, (dn * xhat).sum(0), dz.T @ n, dy.T @ hidden


def _near(got, want, tol, what):
    got = B.wide(got).reshape(want.shape)
    rel = np.linalg.norm(got - want) / np.linalg.norm(want)
    assert rel < tol, (what, rel)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("act", [L.ACT_SILU, L.ACT_GELU])
@pytest.mark.parametrize("f8", [False, True])
def test_step_against_the_block_in_64_bits(dtype, act, f8):
    say("gated mlp", dtype, act, f8)
    M, d, f = 333, 272, 384
    layer = train.GatedMLP(d, f, 3, act=act, device=DEV, init_std=0.08, f8_pipeline=f8)
    g = torch.Generator(device=DEV).manual_seed(1)
    x, r, dy, dh = (torch.randn((M, d), generator=g, device=DEV).to(dtype) for _ in range(4))
    with torch.no_grad():
        layer.gamma.add_(0.1 * torch.randn(d, generator=g, device=DEV))
    x.requires_grad_()
    r.requires_grad_()
    y, h = layer(x, r)
    torch.autograd.backward([y, h], [dy, dh])
    w_in, w_out, gamma = B.wide(layer.w_in), B.wide(layer.w_out), B.wide(layer.gamma)
    state = _forward64(B.wide(x), B.wide(r), gamma, w_in, w_out, act, layer.eps)
    dx, dgamma, dw_in, dw_out = _backward64(B.wide(dy), B.wide(dh), state, gamma, w_in, w_out)
    # rounding to E4M3 to nearest leaves 2^-4 / sqrt(3) at most of a value, uniformly 0.027 of a tensor; to E5M2 stochastically 0.075.
    # A product's operands add in squares: y has three such roundings behind it (n, W twice over, H), a gradient up to six of which two of E5M2.
    _near(h, state[0], 0.005, "h")
    _near(y, state[-1], 0.027 * 4, "y")
    own = dx - B.wide(dh)
    for t in (x.grad, r.grad):
        _near(torch.from_numpy(B.wide(t) - B.wide(dh)), own, 0.16 + (0.02 if dtype is torch.bfloat16 else 0.0), "dx")
    _near(layer.gamma.grad, dgamma, 0.16, "dgamma")
    _near(layer.dw_in, dw_in, 0.16, "dW in")
    _near(layer.dw_out, dw_out, 0.12, "dW out")
    # a second pass adds to the gradients; the update consumes them
    first = layer.dw_out.clone()
    y, h = layer(x, r)
    torch.autograd.backward([y, h], [dy, dh])
    _near(layer.dw_out, 2 * dw_out, 0.12, "dW out, two passes")
    assert not torch.equal(layer.dw_out, 2 * first)  # (new thresholds)
    before = layer.w_out.clone()
    layer.update(0.01)
    step = B.wide(before) - 0.01 * 2 * dw_out
    _near(layer.w_out, step, 0.01 + 0.12 * np.linalg.norm(0.02 * dw_out) / np.linalg.norm(step), "update")
    assert not layer.have_grad


def test_gradients_of_the_weights_are_unbiased():
    # stochastic rounding backward: the mean over thresholds approaches the gradient of the codes kept by the forward pass
    M, d, f = 128, 128, 128
    layer = train.GatedMLP(d, f, 5, device=DEV, init_std=0.08)
    g = torch.Generator(device=DEV).manual_seed(2)
    x, r, dy = (torch.randn((M, d), generator=g, device=DEV) for _ in range(3))
    one = torch.zeros_like(layer.dw_out)
    n = 200
    for _ in range(n):
        y, h = layer(x, r)
        y.backward(dy)
        if not one.any():
            one.copy_(layer.dw_out)
    mean = layer.dw_out / n
    _, _, (_, _, hidden, _, _, _) = layer._forward(x, r, layer.gamma.detach(), True)
    want = B.wide(dy).T @ B.values(hidden)
    _near(one, want, 0.1, "one step")
    _near(mean, want, 0.1 / np.sqrt(n) * 2 + 0.002, "mean")  # (the turned H is rounded once more where it falls below its block's normal numbers)


def test_single_tokens_and_frozen_weights():
    M, d, f = 9, 256, 384
    layer = train.GatedMLP(d, f, 3, device=DEV, init_std=0.08)
    g = torch.Generator(device=DEV).manual_seed(1)
    x, r = (torch.randn((M, d), generator=g, device=DEV).to(torch.bfloat16) for _ in range(2))
    with torch.no_grad():
        want, h = layer(x, r)
        layer.freeze()
        got = [layer(x[i:i + 1], r[i:i + 1]) for i in range(M)]
    # a row's result does not depend on the others beside it (round to nearest, the same kernels for up to sixteen rows)
    assert torch.equal(torch.cat([y for y, _ in got]), want) and torch.equal(torch.cat([k for _, k in got]), h)
    state = _forward64(B.wide(x), B.wide(r), 1.0, B.wide(layer.w_in), B.wide(layer.w_out), layer.act, layer.eps)
    _near(want, state[-1], 0.027 * 4, "y")


def test_decoder_with_gated_blocks_trains():
    torch.manual_seed(0)
    model = train.Decoder(vocab=512, d=128, heads=4, layers=2, seq=64, device=DEV, ffn="gated")
    ids = torch.randint(0, 512, (8, 65), generator=torch.Generator().manual_seed(3)).to(DEV)
    losses = [float(train.train_step(model, ids[:, :-1], ids[:, 1:], 0.5, micro_batches=2)) for _ in range(30)]
    assert losses[0] == pytest.approx(np.log(512), rel=0.05) and losses[-1] < losses[0] - 0.3
    assert len(model.gated_mlps()) == 2


def test_refusals():
    with pytest.raises(ValueError):
        train.GatedMLP(120, 256, 0, device=DEV)
    with pytest.raises(ValueError):
        train.GatedMLP(128, 192, 0, device=DEV)
    layer = train.GatedMLP(128, 128, 0, device=DEV)
    with pytest.raises(ValueError), torch.no_grad():
        layer(torch.zeros((4, 128), device=DEV), torch.zeros((4, 128), device=DEV, dtype=torch.bfloat16))


def test_a_step_in_a_graph_replays():
    M, d, f = 200, 128, 256
    layer = train.GatedMLP(d, f, 3, device=DEV)
    layer.freeze()
    x, r = torch.randn((M, d), device=DEV), torch.randn((M, d), device=DEV)
    with torch.no_grad():
        for _ in range(2):
            layer(x, r)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            y, h = layer(x, r)
        for k in range(3):
            x.copy_(torch.randn((M, d), device=DEV))
            graph.replay()
            torch.cuda.synchronize()
            want = layer(x, r)
            torch.cuda.synchronize()
            assert torch.equal(y, want[0]) and torch.equal(h, want[1])
