"""Attention over values near the largest of their type: a mean of values is no larger than they are, however many, and has to come out finite."""
import numpy as np
import pytest
import torch

import attention_util as A
from gpu_util import DEV, say
from paper_2511_00874_amd import lib as L

pytestmark = pytest.mark.gpu

# rows, keys, heads, key heads, what cuts them: whole tiles; tiles in pieces; few rows in one launch, and in chunks that a second one joins
FORMS = [(200, 200, 2, 1, {}), (1500, 1500, 2, 1, {}), (5, 5 * 1000, 4, 2, {"sequences": 5}), (2, 2 * 6000, 4, 4, {"sequences": 2}), (64, 3000, 2, 1, {})]


def _ints(x):
    return None if x is None else torch.tensor(x, dtype=torch.int32, device=DEV)


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("T,S,heads,kv,how", FORMS)
@pytest.mark.parametrize("same_sign", [True, False])
def test_large_values(D, T, S, heads, kv, how, same_sign):
    # sums of the weights, which are not divided by their sum before, would pass 2^128: bounds as everywhere
    say("large values", D, T, S, heads, kv, how, same_sign)
    q, k, v = (A.make((n, h, D), 80 + i, DEV) for i, (n, h) in enumerate(((T, heads), (S, kv), (S, kv))))
    v = v.abs() if same_sign else v
    v = (v.float().clamp(-4, 4) * 0.75e38).bfloat16()  # up to 3e38
    o, lse = L.sr_attention_fwd(q, k, v, causal=T == S, **how)
    want = A.forward(*(A.wide(x) for x in (q, k, v)), D ** -0.5, T == S, A.pairs(T, S, **how))
    assert torch.isfinite(o.float()).all() and want[0].max() > 1e37
    A.check(o, want[0], want[2], "o")
    A.check(lse, want[1], want[3], "lse")


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("T,S,heads,kv,how", FORMS)
def test_rows_and_channels_beside_large_values(D, T, S, heads, kv, how):
    # large values, infinities and NaN in some channels: the others are the same bits
    say("beside large values", D, T, S, heads, kv, how)
    q, k, v = (A.make((n, h, D), 90 + i, DEV) for i, (n, h) in enumerate(((T, heads), (S, kv), (S, kv))))
    o, lse = L.sr_attention_fwd(q, k, v, causal=T == S, **how)
    for bad in (3e38, -3e38, float("inf"), float("nan")):
        v2 = v.clone()
        v2[:, :, 3] = bad
        got = L.sr_attention_fwd(q, k, v2, causal=T == S, **how)
        rest = [c for c in range(D) if c != 3]
        assert torch.equal(got[0][..., rest], o[..., rest]) and torch.equal(got[1], lse), bad
        if abs(bad) < 1e39:
            value = v2[0, 0, 3].double()
            assert ((got[0][..., 3].double() - value).abs() <= 2 * A.H * value.abs()).all(), bad
    # one large place that only the last row sees
    if T == S:
        v2 = v.clone()
        v2[-1] = 3e38
        got = L.sr_attention_fwd(q, k, v2)
        assert torch.equal(got[0][:-1], o[:-1])


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("n", [64, 100, 129, 1500])
def test_keys_with_scores_of_minus_infinity(D, causal, n):
    # an infinite channel of a key, negative in every query: its weight is 0 in every row, so that the rest is as without it, and its own gradients are zeros
    heads, kv = 4, 2
    q, k, v, do = (A.make((n, h, D), 95 + i, DEV) for i, h in enumerate((heads, kv, kv, heads)))
    q[..., 5] = -1.0
    k[..., 5] = 0.0
    at = n // 2
    k2 = k.clone()
    k2[at, :, 5] = float("inf")
    keep = [i for i in range(n) if i != at]
    o, lse = L.sr_attention_fwd(q, k2, v, causal=causal)
    dq, dk, dv = L.sr_attention_bwd(do, q, k2, v, o, lse, causal=causal)
    assert torch.isfinite(o.float()).all() and torch.isfinite(lse[:, at + 1:] if causal else lse).all()
    assert not dk[at].any() and not dv[at].any()
    assert all(torch.isfinite(x.float()).all() for x in (dq, dk, dv))
    if not causal:  # the key left out altogether
        want = A.backward(*(A.wide(x) for x in (do, q, k[keep], v[keep])), D ** -0.5, False, A.pairs(n, n - 1))
        for g, w, e in zip((dq, dk[keep], dv[keep]), *want):
            A.check(g, w, e, "gradient")
