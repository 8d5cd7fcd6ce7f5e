"""Attention, forward and backward, against its definition in 64 bits."""
import numpy as np
import pytest
import torch

import attention_util as A
from gpu_util import DEV, say
from paper_2511_00874_amd import lib as L

pytestmark = pytest.mark.gpu


def _ints(x):
    return None if x is None else torch.tensor(x, dtype=torch.int32, device=DEV)


def _case(T, S, heads, kv, D, causal, seed, step, scale=None, **how):
    say("attention", T, S, heads, kv, D, causal, how)
    q, k, v, do = (A.make((n, h, D), seed + i, DEV) for i, (n, h) in enumerate(((T, heads), (S, kv), (S, kv), (T, heads))))
    groups = A.pairs(T, S, **how)
    dev = {n: x if n == "sequences" else _ints(x) for n, x in how.items()}
    o, lse = L.sr_attention_fwd(q, k, v, scale=scale, causal=causal, **dev)
    c = D ** -0.5 if scale is None else scale
    q64, k64, v64, d64 = (A.wide(t) for t in (q, k, v, do))
    want = A.forward(q64, k64, v64, c, causal, groups)
    A.check(o, want[0], want[2], "o")
    A.check(lse, want[1], want[3], "lse")
    if not step:
        return
    grads = L.sr_attention_bwd(do, q, k, v, o, lse, scale=scale, causal=causal, **dev)
    want, err = A.backward(d64, q64, k64, v64, c, causal, groups)
    for n, g, w, e in zip("qkv", grads, want, err):
        A.check(g, w, e, "d" + n)
    again = L.sr_attention_bwd(do, q, k, v, o, lse, scale=scale, causal=causal, **dev)
    for n, a, b, w in zip("qkv", grads, again, want):
        there = torch.from_numpy(~np.isnan(w)).to(DEV)
        assert torch.equal(a[there], b[there]), n


# one row; rows and keys that end inside a tile of 32, 64, 128; several tiles
@pytest.mark.parametrize("n", [1, 2, 31, 33, 64, 65, 127, 128, 129, 191, 300])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("causal", [True, False])
def test_one_sequence(n, D, causal):
    _case(n, n, 2, 1, D, causal, n, True)


@pytest.mark.parametrize("D", [8, 16, 40, 56, 72, 80, 96, 104, 120])
def test_head_sizes(D):
    _case(130, 130, 3, 3, D, True, D, True)


@pytest.mark.parametrize("heads,kv", [(1, 1), (8, 1), (12, 4), (40, 1), (9, 9)])
def test_groups_of_heads(heads, kv):
    _case(70, 70, heads, kv, 64, True, heads, True)


# packed sequences: of nothing, of one row, ending inside tiles; rows in front of the first and behind the last
PACKED = [[0, 5, 6, 6, 136, 200, 233], [3, 3, 67, 195, 196], [0, 0, 0, 1], [7, 300]]


@pytest.mark.parametrize("offsets", PACKED)
@pytest.mark.parametrize("D", [64, 96])
@pytest.mark.parametrize("causal", [True, False])
def test_packed(offsets, D, causal):
    _case(offsets[-1] + 5, offsets[-1] + 5, 4, 2, D, causal, len(offsets), True, offsets=offsets)


# tiles with many keys (or queries), few enough in all that they are cut into pieces
@pytest.mark.parametrize("D", [64, 80, 128])
@pytest.mark.parametrize("causal", [True, False])
def test_long_tiles_in_pieces(D, causal):
    _case(1500, 1500, 2, 1, D, causal, 1, True)
    _case(1301, 1301, 4, 1, D, causal, 2, True, offsets=[0, 100, 1250, 1301])
    _case(300, 1900, 2, 2, D, causal, 3, True, offsets=[0, 200, 300], offsets_k=[0, 1700, 1800])
    _case(1700, 200, 2, 2, D, causal, 4, True, offsets=[0, 1600, 1700], offsets_k=[50, 200, 200])
    _case(2 * 1000, 2 * 1000, 3, 1, D, causal, 5, True, sequences=2, lengths_k=[999, 1000])


def test_many_sequences():
    # more than the search looks at in one step, in one step of its second level, and many of no rows
    rng = np.random.default_rng(1)
    n = rng.integers(0, 4, 9000)
    n[rng.integers(0, 9000, 20)] = 150
    offsets = np.concatenate([[2], 2 + np.cumsum(n)]).tolist()
    T = offsets[-1] + 1
    say("many sequences", T)
    q, k, v = (A.make((T, 1, 8), i, DEV) for i in range(3))
    o, lse = L.sr_attention_fwd(q, k, v, offsets=_ints(offsets))
    want = A.forward(*(A.wide(t) for t in (q, k, v)), 8 ** -0.5, True, A.pairs(T, T, offsets=offsets))
    A.check(o, want[0], want[2], "o")
    A.check(lse, want[1], want[3], "lse")
    do = A.make((T, 1, 8), 3, DEV)
    grads = L.sr_attention_bwd(do, q, k, v, o, lse, offsets=_ints(offsets))
    want, err = A.backward(A.wide(do), *(A.wide(t) for t in (q, k, v)), 8 ** -0.5, True, A.pairs(T, T, offsets=offsets))
    for n, g, w, e in zip("qkv", grads, want, err):
        A.check(g, w, e, "d" + n)


# rows of q and of k that differ: fewer queries (a prompt that goes on), more (rows that see nothing), none of either
DIFFERENT = [([0, 3, 4, 74, 79], [0, 10, 210, 260, 260]), ([0, 128, 130, 130, 400], [1, 2, 300, 310, 350]), ([0, 200], [0, 70]), ([0, 40], [0, 333])]


@pytest.mark.parametrize("offsets,offsets_k", DIFFERENT)
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("D", [64, 128])
def test_rows_of_queries_and_keys_differ(offsets, offsets_k, causal, D):
    _case(offsets[-1], offsets_k[-1] + 3, 4, 2, D, causal, len(offsets), True, offsets=offsets, offsets_k=offsets_k)


@pytest.mark.parametrize("heads,kv,D", [(12, 12, 64), (16, 4, 128), (5, 1, 72), (64, 1, 64), (40, 1, 128)])
@pytest.mark.parametrize("S", [1, 40, 100, 1000, 3000])
def test_one_query_a_sequence_over_caches(heads, kv, D, S):
    B = 5
    lengths = [S, 0, 1, S // 2, min(S, 33)]
    _case(B, B * S, heads, kv, D, True, S, False, sequences=B, lengths_k=lengths)
    _case(B, B * S, heads, kv, D, False, S, S <= 100, sequences=B, lengths_k=lengths)


@pytest.mark.parametrize("rows", [2, 3, 7, 16, 33])
@pytest.mark.parametrize("causal", [True, False])
def test_few_queries_a_sequence_over_caches(rows, causal):
    _case(3 * rows, 3 * 700, 8, 2, 64, causal, rows, False, sequences=3, lengths_k=[700, rows - 1, 250])
    _case(3 * rows, 3 * 700, 6, 6, 128, causal, rows, False, sequences=3, lengths_k=[699, 2 * rows, 64])


def test_one_query_over_packed_keys():
    offsets = [4, 4, 5, 900, 4000]
    _case(4, 4100, 8, 2, 128, True, 0, True, sequences=4, offsets_k=offsets)


def test_equal_sequences_and_scale():
    _case(4 * 77, 4 * 77, 4, 4, 64, True, 5, True, scale=0.3, sequences=4)
    _case(3 * 20, 3 * 150, 2, 1, 128, False, 6, True, scale=1.0, sequences=3)
    _case(3 * 90, 3 * 31, 2, 1, 64, True, 7, True, scale=2.0, sequences=3, lengths_k=[31, 0, 5])


@pytest.mark.parametrize("size", [1.0, 30.0])
def test_large_scores(size):
    # scores of thousands: one key takes all; the running maximum moves often
    n, D = 200, 64
    q, k, v = (A.make((n, 2, D), i, DEV) for i in range(3))
    k = (k * size * torch.linspace(0.1, 1.0, n, device=DEV)[:, None, None]).bfloat16()
    o, lse = L.sr_attention_fwd(q, k, v)
    want = A.forward(*(A.wide(t) for t in (q, k, v)), 0.125, True, A.pairs(n, n))
    A.check(o, want[0], want[2], "o")
    A.check(lse, want[1], want[3], "lse")


def test_parts_of_one_matrix_and_heads_first():
    # q, k, v and their gradients as parts of what one projection writes; and tensors whose heads come before their rows
    T, heads, kv, D = 150, 4, 2, 64
    qkv = A.make((T, heads + 2 * kv, D), 0, DEV)
    parts = lambda x: (x[:, :heads], x[:, heads:heads + kv], x[:, heads + kv:])  # noqa: E731
    do = A.make((T, heads, D), 1, DEV)
    o, lse = L.sr_attention_fwd(*parts(qkv))
    dense = [p.contiguous() for p in parts(qkv)]
    o2, lse2 = L.sr_attention_fwd(*dense)
    assert torch.equal(o, o2) and torch.equal(lse, lse2)
    dqkv = torch.zeros_like(qkv)
    L.sr_attention_bwd(do, *parts(qkv), o, lse, **dict(zip(("out_dq", "out_dk", "out_dv"), parts(dqkv))))
    want = L.sr_attention_bwd(do, *dense, o, lse)
    assert all(torch.equal(a, b) for a, b in zip(parts(dqkv), want))
    first = [p.transpose(0, 1).contiguous().transpose(0, 1) for p in parts(qkv)]
    out = torch.empty((heads, T, D), dtype=torch.bfloat16, device=DEV).transpose(0, 1)
    o3, lse3 = L.sr_attention_fwd(*first, out=out)
    assert torch.equal(o3, o) and torch.equal(lse3, lse)
    # one key head for all as a view that repeats it: a stride of 0 between heads
    one = dense[1][:, :1]
    many = L.sr_attention_fwd(dense[0], one.expand(T, heads, D), dense[2][:, :1].expand(T, heads, D))
    assert torch.equal(many[0], L.sr_attention_fwd(dense[0], one, dense[2][:, :1])[0])


@pytest.mark.parametrize("D", [64, 80, 128])
def test_what_is_not_seen_has_no_part(D):
    # NaN and infinities in rows of no sequence, behind lengths_k, in the gaps between heads
    n, heads, kv = 140, 4, 2
    wide = torch.full((n + 60, heads + 2 * kv, 128), float("nan"), dtype=torch.bfloat16, device=DEV)
    x = A.make((n, heads + 2 * kv, D), 3, DEV)
    wide[20:20 + n, :, :D] = x
    wide[:20, ::2] = float("inf")
    parts = lambda y: (y[:, :heads, :D], y[:, heads:heads + kv, :D], y[:, heads + kv:, :D])  # noqa: E731
    offsets = _ints([20, 20 + 50, 20 + n])
    o, lse = L.sr_attention_fwd(*parts(wide), offsets=offsets)
    want = L.sr_attention_fwd(*parts(x), offsets=_ints([0, 50, n]))
    assert torch.equal(o[20:20 + n], want[0]) and torch.equal(lse[:, 20:20 + n], want[1])
    do = A.make((n + 60, heads, D), 4, DEV)
    do[:20] = do[20 + n:] = float("nan")
    got = L.sr_attention_bwd(do, *parts(wide), o, lse, offsets=offsets)
    grads = L.sr_attention_bwd(do[20:20 + n], *parts(x), *want, offsets=_ints([0, 50, n]))
    assert all(torch.equal(a[20:20 + n], b) for a, b in zip(got, grads))
    # caches that are filled in part
    keys, values = A.make((3 * 200, kv, D), 5, DEV), A.make((3 * 200, kv, D), 6, DEV)
    fill = [150, 0, 33]
    q = A.make((3, heads, D), 7, DEV)
    want = L.sr_attention_fwd(q, keys, values, sequences=3, lengths_k=_ints(fill))
    for b in range(3):
        keys[200 * b + fill[b]:200 * (b + 1)] = float("nan")
        values[200 * b + fill[b]:200 * (b + 1)] = float("inf")
    got = L.sr_attention_fwd(q, keys, values, sequences=3, lengths_k=_ints(fill))
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    assert not got[0][1].any() and torch.isinf(got[1][:, 1]).all()


@pytest.mark.parametrize("D", [64, 72, 128])
@pytest.mark.parametrize("n,at", [(200, 97), (200, 64), (65, 33), (300, 250), (40, 39)])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
def test_what_comes_later_has_no_part(D, n, at, bad):
    # a place that is not finite, in a sequence: rows before it, and what belongs to them, are as if it were not there
    heads, kv = 4, 2
    q, k, v, do = (A.make((n, h, D), i, DEV) for i, h in enumerate((heads, kv, kv, heads)))
    o, lse = L.sr_attention_fwd(q, k, v)
    dq, dk, dv = L.sr_attention_bwd(do, q, k, v, o, lse)
    for which in ("k", "v", "kv"):
        k2, v2 = k.clone(), v.clone()
        if "k" in which:
            k2[at, :, 3] = bad
        if "v" in which:
            v2[at:, :, 5] = bad
        o2, lse2 = L.sr_attention_fwd(q, k2, v2)
        assert torch.equal(o2[:at], o[:at]) and torch.equal(lse2[:, :at], lse[:, :at]), which
        if which == "v":  # channel 5 of every row that sees it, no other
            assert not torch.isfinite(o2[at:, :, 5]).any() and torch.equal(o2[at:, :, 6:], o[at:, :, 6:]) and torch.equal(o2[..., :5], o[..., :5])
            if bad != bad:
                assert torch.isnan(o2[at:, :, 5]).all()
            else:
                assert (o2[at:, :, 5] == bad).all()
        g = L.sr_attention_bwd(do, q, k2, v2, o2, lse2)
        assert torch.isfinite(g[0][:at].float()).all()
        err = (g[0][:at].float() - dq[:at].float()).abs().max() / dq[:at].float().abs().max()
        assert err <= 2.0**-6, which  # (the mean key that takes up rounding is another one)
    # rows of q and do that are not finite: keys behind them, which they do not see
    for which in ("q", "do"):
        x = {"q": q.clone(), "do": do.clone()}
        x[which][at, :, 7] = bad
        o2, lse2 = L.sr_attention_fwd(x["q"], k, v)
        rest = [i for i in range(n) if i != at]
        assert torch.equal(o2[rest], o[rest])
        g = L.sr_attention_bwd(x["do"], x["q"], k, v, o2, lse2)
        assert torch.equal(g[1][at + 1:], dk[at + 1:]) and torch.equal(g[2][at + 1:], dv[at + 1:]), which
        assert torch.equal(g[0][rest], dq[rest])
        if which == "do":  # channel 7 of dv of every key that it sees
            assert not torch.isfinite(g[2][:at + 1, :, 7]).any() and torch.equal(g[2][..., 8:], dv[..., 8:]) and torch.equal(g[2][..., :7], dv[..., :7])
    # a few queries over a cache
    few = L.sr_attention_fwd(q[-8:], k, v)
    v2 = v.clone()
    v2[n - 3:, :, 2] = bad
    got = L.sr_attention_fwd(q[-8:], k, v2)
    assert torch.equal(got[0][:5], few[0][:5]) and torch.equal(got[1], few[1])


def test_rows_of_no_sequence_are_left_as_they_were():
    T, heads, D = 100, 2, 64
    q, k, v, do = (A.make((T, heads, D), i, DEV) for i in range(4))
    offsets = _ints([10, 40, 77])
    out = torch.full((T, heads, D), 7.0, dtype=torch.bfloat16, device=DEV)
    _, lse = L.sr_attention_fwd(q, k, v, offsets=offsets, out=out)
    assert (out[:10] == 7).all() and (out[77:] == 7).all() and not (out[10:77] == 7).all(2).any()
    outs = {n: torch.full((T, heads, D), 7.0, dtype=torch.bfloat16, device=DEV) for n in ("out_dq", "out_dk", "out_dv")}
    L.sr_attention_bwd(do, q, k, v, out, lse, offsets=offsets, lengths_k=_ints([30, 20]), **outs)
    for n, x in outs.items():
        end = 77 if n == "out_dq" else 60
        assert (x[:10] == 7).all() and (x[end:] == 7).all() and not (x[10:end] == 7).all(2).any(), n


def test_gradients_against_differences():
    # of sum(o * c), by differences of the definition in 64 bits along random directions: bfloat16 weights and results leave the gradient to
    # within the bounds of its own check, summed over the direction
    T, heads, kv, D = 33, 4, 2, 64
    rng = np.random.default_rng(0)
    q, k, v, c = (A.make((T, n, D), 20 + i, DEV) for i, n in enumerate((heads, kv, kv, heads)))
    o, lse = L.sr_attention_fwd(q, k, v)
    grads = L.sr_attention_bwd(c, q, k, v, o, lse)
    x, c64 = [A.wide(t) for t in (q, k, v)], A.wide(c)
    _, err = A.backward(c64, *x, D ** -0.5, True, A.pairs(T, T))

    def loss(y):
        return (A.forward(*y, D ** -0.5, True, A.pairs(T, T))[0] * c64).sum()

    for i in range(3):
        u = rng.standard_normal(x[i].shape)
        t = 1e-5
        up, down = ([y + s * t * u if j == i else y for j, y in enumerate(x)] for s in (1, -1))
        num = (loss(up) - loss(down)) / (2 * t)
        own = (A.wide(grads[i]) * u).sum()
        assert abs(num - own) <= (err[i] * np.abs(u)).sum() + 1e-6 * abs(num)


def test_offsets_out_of_range_stay_within_the_tensors():
    # offsets and lengths are kept within the rows, whatever they hold: nothing outside is read or written (the results say nothing)
    T, heads, D = 64, 2, 64
    wide = torch.zeros((T + 128, heads, D), dtype=torch.bfloat16, device=DEV)
    q = wide[64:64 + T]
    for bad in ([-5, 10, 1000], [50, 20, 60], [2**31 - 1, -2**31, 5], [0, 64, 64]):
        o = torch.full((T + 128, heads, D), 3.0, dtype=torch.bfloat16, device=DEV)
        L.sr_attention_fwd(q, q, q, offsets=_ints(bad), lengths_k=_ints([2**31 - 1, -7]), out=o[64:64 + T])
        assert (o[:64] == 3).all() and (o[64 + T:] == 3).all()


def test_nothing():
    e = torch.empty((0, 4, 64), dtype=torch.bfloat16, device=DEV)
    o, lse = L.sr_attention_fwd(e, e, e)
    assert o.shape == (0, 4, 64) and lse.shape == (4, 0)
    assert all(g.shape == (0, 4, 64) for g in L.sr_attention_bwd(e, e, e, e, o, lse))
    q = A.make((3, 4, 64), 0, DEV)
    o, lse = L.sr_attention_fwd(q, e, e, causal=False)
    assert not o.any() and torch.isinf(lse).all()
    dq, dk, dv = L.sr_attention_bwd(q, q, e, e, o, lse)
    assert not dq.any() and dk.numel() == dv.numel() == 0
    dq, dk, dv = L.sr_attention_bwd(e, e, q, q, e, torch.empty((4, 0), device=DEV))
    assert not dk.any() and not dv.any()


@pytest.mark.parametrize("D", [64, 96, 128])
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("lengths", [[64, 1, 2, 33, 200], [47, 300], [1500], [7, 64, 65]])
def test_rows_that_see_few_keys(D, causal, lengths):
    # Their softmax hangs on a few keys, and ds = p (do v^T - delta) on differences.  With delta from p and dP themselves, 2^-24 being half a step of
    # binary32: p is off by 2^-18 of itself (the exponent, below 2^5 in size, and lse by 2^-19 each at most), do v^T and delta by 128 2^-24 of the sums a of |do| |v|;
    # ds is multiplied as two values of 8 bits, 2^-16: together |ds| is off by 2^-14 (|ds| + p (a + sum p a)) at most, dq by that times |k|, and its rounding.
    # The sum of ds, which is off 0 by as much, is taken off times the mean key of a tile of the sequence, no more than its largest.
    heads, n = 2, sum(lengths)
    q, k, v, do = (A.make((n, heads, D), 40 + i, DEV) for i in range(4))
    k = (k.float() + 2.0 * A.make((1, heads, D), 50, DEV).float()).bfloat16()
    v = (v.float() + 2.0 * A.make((1, heads, D), 51, DEV).float()).bfloat16()
    ends = np.cumsum([0] + lengths).tolist()
    o, lse = L.sr_attention_fwd(q, k, v, causal=causal, offsets=_ints(ends))
    got = A.wide(L.sr_attention_bwd(do, q, k, v, o, lse, causal=causal, offsets=_ints(ends))[0])
    q, k, v, do = (A.wide(x) for x in (q, k, v, do))
    scale, checked = D**-0.5, 0
    for first, m in zip(ends, lengths):
        for h in range(heads):
            for i in range(m if causal else m if m <= 64 else 0):
                seen = slice(first, first + (i + 1 if causal else m))
                if seen.stop - seen.start > 64:
                    continue
                x = scale * k[seen, h] @ q[first + i, h]
                p = np.exp(x - x.max()) / np.exp(x - x.max()).sum()
                dp, a = v[seen, h] @ do[first + i, h], np.abs(v[seen, h]) @ np.abs(do[first + i, h])
                ds = p * (dp - p @ dp)
                want = scale * ds @ k[seen, h]
                eds = 2.0**-14 * (np.abs(ds) + p * (a + p @ a))
                off = scale * (eds @ np.abs(k[seen, h]) + eds.sum() * np.abs(k[first:first + m, h]).max(0))
                assert (np.abs(got[first + i, h] - want) <= off + 2.0**-8 * (np.abs(want) + off)).all(), (m, h, i)
                checked += 1
    assert checked or not causal and min(lengths) > 64
