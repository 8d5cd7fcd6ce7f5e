"""Gradients of attention: dq hangs on what its row sees and on nothing else, and is as good where a few keys have all the weight."""
import numpy as np
import pytest
import torch

import attention_util as A
from gpu_util import DEV, say
from paper_2511_00874_amd import lib as L

pytestmark = pytest.mark.gpu
H, U = A.H, A.U


def _step(do, q, k, v, **how):
    o, lse = L.sr_attention_fwd(q, k, v, **how)
    return (o, lse, *L.sr_attention_bwd(do, q, k, v, o, lse, **how))


# places in every part of a tile of 128 rows and of 64 keys, rows whose tiles of keys are cut into pieces
PLACES = [(200, 97), (200, 64), (256, 192), (256, 129), (128, 1), (300, 250), (40, 39), (65, 33), (1500, 1490), (1500, 1345)]


@pytest.mark.parametrize("D", [64, 96, 128])
@pytest.mark.parametrize("n,at", PLACES)
def test_rows_do_not_depend_on_later_keys(D, n, at):
    say("later keys", D, n, at)
    heads, kv = 4, 2
    q, k, v, do = (A.make((n, h, D), i, DEV) for i, h in enumerate((heads, kv, kv, heads)))
    o, lse, dq, _, _ = _step(do, q, k, v)
    for bad in (1.0, 100.0, 1e4, 1e30, 3e38, float("inf"), float("nan")):
        for which in ("k", "v", "kv"):
            for channels in (slice(None), slice(3, 4)):
                k2, v2 = k.clone(), v.clone()
                if "k" in which:
                    k2[at:, :, channels] = bad
                if "v" in which:
                    v2[at:, :, channels] = bad
                got = _step(do, q, k2, v2)
                assert torch.equal(got[0][:at], o[:at]) and torch.equal(got[1][:, :at], lse[:, :at]), (bad, which, channels)
                assert torch.equal(got[2][:at], dq[:at]), (bad, which, channels)


def _dq(do, q, k, v, scale, causal, groups):
    """dq in 64 bits, and how far it may be off.

    With p and ds of the kernel off by binary32, e what delta, of o as it was rounded, is off by, and roundings to bfloat16 of at most H each, the weights are
    w_j = (ds_j + p_j e) (1 + H), p^_j = p_j (1 + H), and dq = scale sum w_j (k_j - B^) with B^ = sum p^ k / sum p^, which is off the mean B = sum p k by 2 H (1 + 2 H)
    sum p |k - B| at most.  The sum of ds is 0, so B^ may be taken off the keys of the definition too: dq is off by
    scale (|e| |B - B^| + H sum (|ds_j| + p_j |e|) |k_j - B^|), binary32's errors of p and ds times the keys, those of the sums, and its own rounding."""
    heads, D = q.shape[1:]
    g = heads // k.shape[1]
    o, lse, eo, el = A.forward(q, k, v, scale, causal, groups)
    out, err = np.full(q.shape, np.nan), np.zeros(q.shape)
    for q0, lq, k0, lk in groups:
        rq, rk = slice(q0, q0 + lq), slice(k0, k0 + lk)
        out[rq] = 0.0
        seen = np.ones((lq, lk), bool)
        if causal:
            seen = np.arange(lk)[None] <= np.arange(lq)[:, None] + lk - lq
        for h in range(heads):
            a, b, c, d = q[rq, h], k[rk, h // g], v[rk, h // g], do[rq, h]
            with np.errstate(invalid="ignore"):
                p = np.where(seen, np.exp(scale * (a @ b.T) - lse[h, rq][:, None]), 0.0)
            ep = 2 * (D + 4) * U * scale * np.where(seen, np.abs(a) @ np.abs(b).T, 0.0) + 64 * U + el[h, rq][:, None]
            dp = d @ c.T
            ds = p * (dp - (p * dp).sum(1)[:, None])
            e = (np.abs(d) * eo[rq, h]).sum(1)[:, None] + (D + 4) * U * (np.abs(d) * np.abs(o[rq, h])).sum(1)[:, None]
            e32 = ep * (np.abs(ds) + p * e) + p * (1 + ep) * (D + 4) * U * (np.abs(d) @ np.abs(c).T) + (lk + 8) * U * (np.abs(ds) + p * e)
            mean = p @ b
            for i in range(lq):
                s = seen[i]
                if not s.any():
                    continue
                away = np.abs(b[s] - mean[i])                                  # (keys seen, D)
                off = 2 * (H + ep[i, s].max()) * (1 + 2 * H) * (p[i, s] @ away)  # of the mean
                away = away + off
                er = e[i] * off + H * (1 + H) * ((np.abs(ds[i, s]) + p[i, s] * e[i]) @ away)
                er += e32[i, s] @ away + ((lk + 8) * U) * ((np.abs(ds[i, s]) + p[i, s] * e[i]) @ (np.abs(b[s]) + np.abs(mean[i])))
                out[q0 + i, h] = scale * ds[i, s] @ b[s]
                err[q0 + i, h] = scale * er
    err += H * (np.abs(np.nan_to_num(out)) + err) + 1e-37
    return out, err


@pytest.mark.parametrize("D", [64, 80, 128])
@pytest.mark.parametrize("size", [1.0, 3.0, 10.0])
@pytest.mark.parametrize("offset", [0.5, 8.0])
@pytest.mark.parametrize("causal,lengths", [(True, [300]), (True, [65, 256, 1]), (False, [100, 250]), (True, [1500])])
def test_peaked_scores(D, size, offset, causal, lengths):
    # queries so large that few keys have all the weight: a row's gradient is a small difference; keys with an offset beside which their differences are small
    say("peaked scores", D, size, offset, causal, lengths)
    heads, n = 2, sum(lengths)
    q, k, v, do = (A.make((n, heads, D), 60 + i, DEV) for i in range(4))
    q = (q.float() * size).bfloat16()
    k = (k.float() + offset * A.make((1, heads, D), 70, DEV).float()).bfloat16()
    v = (v.float() + A.make((1, heads, D), 71, DEV).float()).bfloat16()
    ends = np.cumsum([0] + lengths).tolist()
    got = _step(do, q, k, v, causal=causal, offsets=torch.tensor(ends, dtype=torch.int32, device=DEV))[2]
    want, err = _dq(*(A.wide(x) for x in (do, q, k, v)), D ** -0.5, causal, A.pairs(n, n, offsets=ends))
    print("largest share of the bound", float((np.abs(A.wide(got) - want) / err).max()), flush=True)
    A.check(got, want, err, "dq")
    # all together they are off by no more than the roundings of ds and of dq, each half a step at most, leave of the sums
    assert np.linalg.norm(A.wide(got) - want) <= 2 * H * np.linalg.norm(want)
