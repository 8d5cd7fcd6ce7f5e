"""Attention and its gradients by their definition in 64 bits on the host, and how far results may be off.

U = 2^-24 is half a step of binary32 relative to a value, H = 2^-8 of bfloat16.  A score is a sum of D products, each exact in binary32, so it is off
by at most e = (D + 4) U scale sum |q k| (the multiplications by scale and log2 e, and the subtraction of the maximum, of whose size the sum is, among
them).  Weights of the softmax are off by a factor within 2 e + 64 U (exponentials of binary32, the sum), and are rounded to bfloat16 for the product:
H more; the result is rounded once: H of it."""
import numpy as np
import torch

U, H = 2.0**-24, 2.0**-8


def wide(t):
    return t.detach().cpu().double().numpy()


def spans(rows, sequences, offsets):
    if offsets is None:
        per = rows // sequences
        return [(b * per, per) for b in range(sequences)]
    return [(a, max(0, b - a)) for a, b in zip(offsets[:-1], offsets[1:])]


def pairs(T, S, sequences=1, offsets=None, offsets_k=None, lengths_k=None):
    """(first row of q, rows, first row of k, rows) of every sequence."""
    ks = spans(S, sequences, offsets if offsets_k is None else offsets_k)
    if lengths_k is not None:
        ks = [(a, min(n, m)) for (a, n), m in zip(ks, lengths_k)]
    return [(*q, *k) for q, k in zip(spans(T, sequences, offsets), ks)]


def forward(q, k, v, scale, causal, groups):
    """Of float64 arrays q (T, heads, D), k and v (S, key heads, D): o, lse and how far each may be off; NaN in rows of no sequence."""
    T, heads, D = q.shape
    g = heads // k.shape[1]
    o, lse = np.full(q.shape, np.nan), np.full((heads, T), np.nan)
    eo, el = np.zeros(q.shape), np.zeros((heads, T))
    for q0, lq, k0, lk in groups:
        seen = np.ones((lq, lk), bool)
        if causal:
            seen = np.arange(lk)[None] <= np.arange(lq)[:, None] + lk - lq
        for h in range(heads):
            a, b, c = q[q0:q0 + lq, h], k[k0:k0 + lk, h // g], v[k0:k0 + lk, h // g]
            s = np.where(seen, scale * (a @ b.T), -np.inf)
            e = (D + 4) * U * scale * np.where(seen, np.abs(a) @ np.abs(b).T, 0.0).max(1, initial=0.0)
            top = np.where(seen.any(1), s.max(1, initial=-np.inf), 0.0)
            p = np.exp(s - top[:, None])
            total = p.sum(1)
            with np.errstate(divide="ignore"):
                lse[h, q0:q0 + lq] = np.where(seen.any(1), top + np.log(total), -np.inf)
            p = p / np.where(total == 0, 1.0, total)[:, None]
            r = p @ c
            o[q0:q0 + lq, h] = r
            eo[q0:q0 + lq, h] = (H + 2 * e + 64 * U)[:, None] * (p @ np.abs(c)) * (1 + H) + H * np.abs(r)
            el[h, q0:q0 + lq] = 2 * e + 64 * U * (1 + np.abs(np.where(seen.any(1), lse[h, q0:q0 + lq], 0.0)))
    return o, lse, eo, el


def backward(do, q, k, v, scale, causal, groups):
    """dq, dk, dv and how far each may be off."""
    heads, D = q.shape[1:]
    g = heads // k.shape[1]
    o, lse, eo, el = forward(q, k, v, scale, causal, groups)
    grads, errs = [np.full(x.shape, np.nan) for x in (q, k, v)], [np.zeros(x.shape) for x in (q, k, v)]
    for q0, lq, k0, lk in groups:
        rq, rk = slice(q0, q0 + lq), slice(k0, k0 + lk)
        grads[0][rq] = grads[1][rk] = grads[2][rk] = 0.0
        seen = np.ones((lq, lk), bool)
        if causal:
            seen = np.arange(lk)[None] <= np.arange(lq)[:, None] + lk - lq
        for h in range(heads):
            a, b, c, d = q[rq, h], k[rk, h // g], v[rk, h // g], do[rq, h]
            ep = 2 * (D + 4) * U * scale * np.where(seen, np.abs(a) @ np.abs(b).T, 0.0) + 64 * U + el[h, rq][:, None]
            with np.errstate(invalid="ignore"):
                p = np.where(seen, np.exp(scale * (a @ b.T) - lse[h, rq][:, None]), 0.0)
            dp = d @ c.T
            delta = np.nan_to_num((d * o[rq, h]).sum(1))
            # products of bfloat16 values in binary32; delta from the result as it was rounded
            edp = (D + 4) * U * (np.abs(d) @ np.abs(c).T)
            edelta = (np.abs(d) * eo[rq, h]).sum(1) + (D + 4) * U * (np.abs(d) * np.abs(np.nan_to_num(o[rq, h]))).sum(1)
            ds = p * (dp - delta[:, None])
            eds = (ep + H * (1 + H)) * np.abs(ds) + (1 + H) * p * (1 + ep) * (edp + edelta[:, None])
            sums = (lq + lk + 8) * U  # of at most so many terms each
            grads[0][rq, h] += scale * ds @ b
            errs[0][rq, h] += scale * ((eds + sums * np.abs(ds)) @ np.abs(b))
            # a row's errors, added up, are taken off times a mean of keys
            if lk:
                errs[0][rq, h] += scale * (eds + sums * np.abs(ds)).sum(1)[:, None] * np.abs(b).max(0)
            grads[1][rk, h // g] += scale * ds.T @ a
            errs[1][rk, h // g] += scale * ((eds + sums * np.abs(ds)).T @ np.abs(a))
            grads[2][rk, h // g] += p.T @ d
            errs[2][rk, h // g] += ((ep + H * (1 + H) + sums) * p).T @ np.abs(d)
    for x, e in zip(grads, errs):
        e += H * np.abs(np.nan_to_num(x)) + 1e-37
    return grads, errs


def check(got, want, err, what):
    """Where want is NaN nothing is said."""
    got = wide(got)
    fine = ~np.isnan(want)
    finite = fine & np.isfinite(want)
    assert np.array_equal(got[fine & ~finite], want[fine & ~finite]), what
    bad = finite & ~(np.abs(got - np.where(finite, want, 0.0)) <= err + 1e-37)
    assert not bad.any(), (what, np.argwhere(bad)[:3].tolist(), got[bad][:3], want[bad][:3], err[bad][:3])


def make(shape, seed, device, spread=0.5):
    """Heads with channels of different strength, bfloat16."""
    rng = np.random.default_rng(seed)
    x = rng.standard_normal(shape) * np.exp(spread * rng.standard_normal((1, *shape[1:])))
    return torch.from_numpy(x).to(device).to(torch.bfloat16)
