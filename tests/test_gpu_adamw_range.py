"""AdamW where gradients are far larger or smaller than usual, in both widths of the moments."""
import numpy as np
import pytest
import torch

import block_util as B
import oracle
from gpu_util import DEV, say
from paper_2511_00874_amd import lib as L

pytestmark = pytest.mark.gpu
U = 2.0**-24


@pytest.mark.parametrize("eps", [0.0, 1e-30])
@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("w", [torch.float32, torch.bfloat16])
def test_second_moments_below_the_normal_numbers(eps, bits, w):
    # squares of gradients of 2^-68 to 2^-60 lie on both sides of 2^-126; the step is m / root(v) all the same
    say("small second moments", eps, bits, w)
    rng = np.random.default_rng(0)
    n = 1000
    g = torch.from_numpy(rng.choice([-1.0, 1.0], n) * 2.0 ** rng.uniform(-68, -60, n)).float().to(DEV)
    g[::7] = 0.0
    t = L.AdamWTensor.zeros(torch.ones(n, device=DEV).to(w), g, bits)
    t.w[::7] = 0.0
    lr, b1, b2 = 0.25, 0.9, 0.95
    L.sr_adamw([t], lr, 1, betas=(b1, b2), eps=eps, round_mode=L.RTN)
    x = B.wide(g)
    live = x != 0
    v = (1 - b2) * x * x
    # the square, its product with 1 - beta2 and the sum are each rounded by 6 U together, or 2^-150 below the normal numbers: half as much of the root
    ev = 6 * U * v + 3 * 2.0**-150
    with np.errstate(divide="ignore", invalid="ignore"):
        update = np.where(live, x / (np.abs(x) + eps), 0.0)
        eu = np.abs(update) * (ev / v + 24 * U)
    got, want = B.wide(t.w), 1 - lr * update
    if w is torch.float32:
        assert np.all(np.abs(got - want)[live] <= (lr * eu + 2 * U * 2)[live])
    else:
        assert np.all(np.abs(got - want)[live] <= (lr * eu + 2.0**-8 * 2)[live])
    if eps:
        assert not got[~live].any()
    if bits == 32:
        assert np.all(np.abs(B.wide(t.v) - v) <= ev)


@pytest.mark.parametrize("mode", [L.SR, L.RTN])
@pytest.mark.parametrize("w", [torch.float32, torch.bfloat16])
def test_blocks_of_roots_of_any_size(mode, w):
    # a block of 128 for every binade from 2^-62, whose squares pass under binary32's normal numbers, to 2^63; without memory the root is |g| itself
    say("roots", mode, w)
    rng = np.random.default_rng(0)
    sizes = np.arange(-62, 63)
    g = (rng.uniform(0.01, 1.0, (len(sizes), 128)) * 2.0 ** sizes[:, None]).astype(np.float32)
    g[:, 5] = 0.0
    t = L.AdamWTensor.zeros(torch.zeros(g.size, device=DEV).to(w), torch.from_numpy(g.reshape(-1)).to(DEV), 8)
    L.sr_adamw([t], 0.0, 1, betas=(0.0, 0.0), round_mode=mode, seed=3)
    e = B.block_exponents(g.astype(float), L.E4M3)
    assert np.array_equal(t.v_scales.cpu().numpy().astype(int) - 127, e.reshape(-1))
    unit = 2.0 ** e.reshape(-1, 1)
    grid = oracle.decode_array(L.E4M3, np.arange(127, dtype=np.uint8)).astype(float)  # ascending
    got = t.v.cpu().numpy().reshape(g.shape).astype(int)
    # one of the two neighbours; the square is rounded on its way, below 2^-126 by up to 2^-150, which is half as much of the root, so that a root this near
    # a number of the grid may count as below it or above
    r = np.abs(g.astype(float)) / unit
    near = 2.0**-22 + 2.0**-150 / np.maximum(g.astype(float)**2, 2.0**-149)
    least, most = (np.clip(np.searchsorted(grid, r * (1 + off), side="right") - 1, 0, 125) for off in (-near, near))
    assert np.all((got >= least) & (got <= most + 1))
    assert np.all((got > 0) == (g != 0))
    if mode == L.RTN:  # the nearer square
        low = np.clip(np.searchsorted(grid, r, side="right") - 1, 0, 125)
        part = (r**2 - grid[low]**2) / (grid[low + 1]**2 - grid[low]**2)
        want = np.where((low == 0) & (r > 0), 1, low + (part >= 0.5))
        sure = np.abs(part - 0.5) > 1e-4 + 16 * near  # (the value is no more than sixteen steps of the squares)
        assert np.array_equal(got[sure], want[sure])


def test_large_gradients_through_the_steps():
    # moments in 8 bits follow those in 32 over steps with gradients of 1e13 in some blocks
    n = 128 * 8
    rng = np.random.default_rng(1)
    size = 10.0 ** np.repeat([-8, -3, 0, 5, 11, 12, 13, 17], 128)
    narrow, wide = (L.AdamWTensor.zeros(torch.zeros(n, device=DEV), torch.zeros(n, device=DEV), bits) for bits in (8, 32))
    for step in range(1, 6):
        g = torch.from_numpy(size * (1 + 0.1 * rng.standard_normal(n))).float().to(DEV)
        for t in (narrow, wide):
            t.g.copy_(g)
            L.sr_adamw([t], 1e-3, step, betas=(0.9, 0.95), round_mode=L.RTN)
    # stored m is off by 2^-4, the square of the stored root by 2^-3 (2 q + 1 of 2 q^2 at q = 8): carried through four steps by the betas, 11 % of the m of the
    # fifth and 25 % of its v, 12 % of the root, so that an update is within 1.11 / 0.88 of the other's: less than a third
    a, b = B.wide(narrow.w), B.wide(wide.w)
    assert np.all(np.abs(a - b) <= np.abs(b) / 3)
    assert np.all(np.abs(np.sqrt(B.wide(narrow.second())) - np.sqrt(B.wide(wide.second()))) <= np.sqrt(B.wide(wide.second())) / 3)
