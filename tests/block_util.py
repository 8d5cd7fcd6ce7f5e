"""The block-scaled form written out for the tests: scales, codes and values in 64 bits on the host (no code of the library)."""
import numpy as np
import torch

import oracle
from paper_2511_00874_amd import lib as L

QMAX = {L.E4M3: 448.0, L.E5M2: 57344.0}
MBITS = {L.E4M3: 3, L.E5M2: 2}
EMIN = {L.E4M3: -6, L.E5M2: -14}
SPAN = 128


def wide(t):
    """A tensor's values as a float64 array."""
    return t.detach().cpu().double().numpy()


def block_exponents(x, kind):
    """Exponent of the scale of every 128 columns of a row of x (float64)."""
    rows, cols = x.shape
    nb = -(-cols // SPAN)
    a = np.zeros((rows, nb * SPAN))
    a[:, :cols] = np.where(np.isfinite(x), np.abs(x), 0.0)
    top = a.reshape(rows, nb, SPAN).max(2)
    e = np.zeros((rows, nb), dtype=np.int64)
    for k in range(-100, 129):  # the least that fits, by its definition
        e[(top > QMAX[kind] * 2.0**(k - 1)) & (top <= QMAX[kind] * 2.0**k)] = k
    e[(top > 0) & (top <= QMAX[kind] * 2.0**-100)] = -100
    return np.minimum(e, {L.E4M3: 119, L.E5M2: 112}[kind])  # the largest whose values all are binary32 numbers


def over_columns(e, cols):
    return np.repeat(e, SPAN, axis=1)[:, :cols]


def block_codes(x, kind, mode=oracle.RTN, seed=0, offset=0, turned=False):
    """(codes, exponents) of x by the oracle's Eq. 1; turned: of its transpose, with the thresholds of x's own order."""
    e = block_exponents(x.T if turned else x, kind)
    each = over_columns(e, x.shape[0] if turned else x.shape[1])
    each = each.T if turned else each
    with np.errstate(invalid="ignore"):
        t = (x * 2.0**-each.astype(np.float64)).astype(np.float32)  # exact, or far below the grid
    codes = oracle.quantize(t, kind, 1.0, seed, offset, mode)
    return (np.ascontiguousarray(codes.T) if turned else codes), e


def values(b):
    """The values of a block-scaled matrix of the library, float64, by the oracle's decode tables."""
    c = b.codes.cpu().numpy()[:, :b.cols]
    e = b.exps.cpu().numpy().astype(np.int64)[:, :-(-b.cols // SPAN)] - 127
    return oracle.decode_array(b.kind, c) * 2.0**over_columns(e, b.cols).astype(np.float64)


def same(a, b):
    """Equal codes and scales (what lies between the rows is nothing)."""
    n = -(-a.cols // SPAN)
    return (a.shape == b.shape and a.kind == b.kind and torch.equal(a.codes[:, :a.cols], b.codes[:, :b.cols])
            and torch.equal(a.exps[:, :n], b.exps[:, :n]))


def spacing(v, exps, kind):
    """Spacing of the scaled grid at v."""
    s = 2.0**over_columns(exps, v.shape[1]).astype(np.float64)
    t = np.minimum(np.abs(v) / s, QMAX[kind])
    e = np.maximum(np.floor(np.log2(np.maximum(t, 1e-300))), EMIN[kind])
    return s * 2.0**(e - MBITS[kind])


def check_blocks(b, want, err, what, sr=False):
    """Codes and scales of `want` (float64), which the library knows to within `err` (array): every scale is that of some value within
    it, and every code stands for a neighbour (nearest, or either one) of such a value."""
    e = b.exps.cpu().numpy().astype(np.int64)[:, :-(-b.cols // SPAN)] - 127
    least, most = np.maximum(np.abs(want) - err, 0.0), np.abs(want) + err
    low, high = block_exponents(least, b.kind), block_exponents(most, b.kind)
    zero = block_exponents(np.where(least > 0, 1.0, 0.0), b.kind) == 0  # blocks that may be all zeros, whose scale is 1
    assert np.all(((low <= e) & (e <= high)) | (zero & ((e == 0) | (e <= high)))), what
    got = values(b)
    step = spacing(np.abs(want) + err, e, b.kind)
    room = (step if sr else step / 2) + err
    # (a value whose block was scaled for a slightly smaller maximum saturates within err of it)
    bad = np.abs(got - want) > room * (1 + 1e-12)
    assert not bad.any(), (what, np.argwhere(bad)[:3], got[bad][:3], want[bad][:3], room[bad][:3])


def make(x, kind, device):
    """A block-scaled matrix on the device from host codes (nearest)."""
    x = np.asarray(x, dtype=np.float64)
    codes, e = block_codes(x, kind)
    b = L.Blocks.empty(*x.shape, kind, device)
    c = np.zeros(tuple(b.codes.shape), dtype=np.uint8)
    c[:, :x.shape[1]] = codes
    s = np.zeros(tuple(b.exps.shape), dtype=np.uint8)
    s[:, :e.shape[1]] = e + 127
    b.codes.copy_(torch.from_numpy(c))
    b.exps.copy_(torch.from_numpy(s))
    return b


def act64(g, act):
    """The activation and its derivative."""
    from scipy.special import erf
    if act == L.ACT_SILU:
        s = 1.0 / (1.0 + np.exp(-g))
        return g * s, s * (1.0 + g * (1.0 - s))
    p = 0.5 * (1.0 + erf(g / np.sqrt(2.0)))
    return g * p, p + g * np.exp(-0.5 * g * g) / np.sqrt(2.0 * np.pi)
