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
