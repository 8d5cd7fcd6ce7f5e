"""Attention, embedding and AdamW where offsets pass 32 bits, and on tensors of another device than the current one."""
import pytest
import torch

pytestmark = pytest.mark.gpu
if torch.cuda.is_available():
    from paper_2511_00874_amd import lib as L

DEV = "cuda:0"


def test_a_cache_of_more_than_2_to_the_32_values():
    # 2^22 + 64 places of 8 heads of 128: the last sequence's lie behind 2^32 values
    S, heads, kv, D, n = 2**22 + 64, 16, 8, 128, 1000
    g = torch.Generator(device=DEV).manual_seed(1)
    keys, values = (torch.zeros((S, kv, D), dtype=torch.bfloat16, device=DEV) for _ in range(2))
    for x in (keys, values):
        x[S - n:] = torch.randn((n, kv, D), generator=g, device=DEV).bfloat16()
    for rows in (1, 70):
        q = torch.randn((rows, heads, D), generator=g, device=DEV).bfloat16()
        offsets, offsets_k = (torch.tensor(x, dtype=torch.int32, device=DEV) for x in ([0, rows], [S - n, S]))
        o, lse = L.sr_attention_fwd(q, keys, values, offsets=offsets, offsets_k=offsets_k)
        want, lse_want = L.sr_attention_fwd(q, keys[S - n:].clone(), values[S - n:].clone())
        # (pieces may be cut otherwise: a weight and a result in other roundings, 2^-9 each of what they are)
        assert (o.float() - want.float()).abs().max() <= 2.0**-7 * want.float().abs().max() and (lse - lse_want).abs().max() <= 2e-5
        grads = [torch.zeros_like(x) for x in (q, keys, values)]
        do = torch.randn((rows, heads, D), generator=g, device=DEV).bfloat16()
        L.sr_attention_bwd(do, q, keys, values, o, lse, offsets=offsets, offsets_k=offsets_k, out_dq=grads[0], out_dk=grads[1], out_dv=grads[2])
        plain = L.sr_attention_bwd(do, q, keys[S - n:].clone(), values[S - n:].clone(), o, lse)
        for a, b in zip((grads[0], grads[1][S - n:], grads[2][S - n:]), plain):
            assert (a.float() - b.float()).abs().max() <= 2.0**-7 * b.float().abs().max()
        assert not grads[1][:S - n].any() and not grads[2][:S - n].any()
        # the whole cache as one sequence: zeros before the last places
        o, lse = L.sr_attention_fwd(q[:1], keys, values)
        p = torch.softmax(torch.cat([(keys[S - n:, h // 2].double() @ q[0, h].double() * D**-0.5).view(1, n) for h in range(heads)]).double(), 1)
        z = torch.logsumexp(torch.stack([keys[S - n:, h // 2].double() @ q[0, h].double() * D**-0.5 for h in range(heads)]), 1)
        total = torch.logaddexp(z, torch.tensor(float(S - n), dtype=torch.float64, device=DEV).log())
        assert (lse[:, 0].double() - total).abs().max() <= 2e-5 * total.abs().max()
        exact = torch.stack([p[h] @ values[S - n:, h // 2].double() * torch.exp(z[h] - total[h]) for h in range(heads)])
        size = torch.stack([p[h] @ values[S - n:, h // 2].double().abs() * torch.exp(z[h] - total[h]) for h in range(heads)])
        # weights and the result rounded to 8 bits; sums of lse in binary32
        assert ((o[0].double() - exact).abs() <= 2.0**-7 * size + 2.0**-8 * exact.abs()).all()


def test_a_table_of_more_than_2_to_the_32_values():
    V, D = 2**18 + 100, 2**14 + 8
    table = torch.empty((V, D), dtype=torch.bfloat16, device=DEV)
    g = torch.Generator(device=DEV).manual_seed(2)
    ids = torch.tensor([V - 1, 3, V - 1, 2**18, V - 50, 0], device=DEV)
    for i in ids.unique().tolist():
        table[i] = torch.randn(D, generator=g, device=DEV).bfloat16()
    assert torch.equal(L.sr_embedding_fwd(table, ids), table[ids])
    del table
    dy = torch.randn((6, D), generator=g, device=DEV)
    d = L.sr_embedding_bwd(dy, ids, V)
    want = {V - 1: dy[0] + dy[2], 3: dy[1], 2**18: dy[3], V - 50: dy[4], 0: dy[5]}
    for i, row in want.items():
        assert torch.equal(d[i], row)
        d[i] = 0
    assert not d[:V // 2].any() and not d[V // 2:].any()


def test_a_batch_of_more_than_2_to_the_32_values():
    M, V, D = 2**18 + 100, 300, 2**14 + 8
    ids = torch.arange(M, device=DEV) % (V - 1)
    ids[M - 7:] = V - 1
    dy = torch.zeros((M, D), dtype=torch.bfloat16, device=DEV)
    last = torch.randint(-8, 9, (7, D), device=DEV).bfloat16()
    dy[M - 7:] = last
    d = L.sr_embedding_bwd(dy, ids, V)
    assert torch.equal(d[V - 1], last.float().sum(0)) and not d[:V - 1].any()


@pytest.mark.parametrize("bits", [8, 32])
def test_a_tensor_of_more_than_2_to_the_32_values(bits):
    n, part = 2**32 + 128 * 5 + 24, 128 * 3 + 24
    g = torch.Generator(device=DEV).manual_seed(3)
    w = torch.zeros(n, dtype=torch.bfloat16, device=DEV)
    grad = torch.zeros(n, dtype=torch.bfloat16, device=DEV)
    w[-part:] = torch.randn(part, generator=g, device=DEV).bfloat16()
    grad[-part:] = torch.randn(part, generator=g, device=DEV).bfloat16()
    small = L.AdamWTensor.zeros(w[-part:].clone(), grad[-part:].clone(), bits)
    large = L.AdamWTensor.zeros(w, grad, bits)
    for step in (1, 2):
        for t in (small, large):
            L.sr_adamw([t], 0.1, step, round_mode=L.RTN)
    for a, b in ((small.w, large.w), (small.m, large.m), (small.v, large.v)):
        assert torch.equal(a, b[-part:]) and not b[:128].any() and not b[n - part - 128:n - part].any()
    if bits == 8:
        assert torch.equal(small.m_scales, large.m_scales[-4:]) and torch.equal(small.v_scales, large.v_scales[-4:])


def test_tensors_of_another_device_are_refused(monkeypatch):
    # (seen from the second of two devices; nothing is launched)
    q = torch.zeros((16, 2, 64), dtype=torch.bfloat16, device=DEV)
    ids, table = torch.zeros(4, dtype=torch.int64, device=DEV), torch.zeros((8, 8), device=DEV)
    batch = L.AdamWBatch([L.AdamWTensor.zeros(table, table.clone())])
    monkeypatch.setattr(L, "_current_device", lambda: 1)
    for call in (lambda: L.sr_attention_fwd(q, q, q), lambda: L.sr_attention_bwd(q, q, q, q, q, table), lambda: L.sr_embedding_fwd(table, ids),
                 lambda: L.sr_embedding_bwd(table[:4], ids, 8), lambda: batch.run(0.1, 1)):
        with pytest.raises(RuntimeError, match="current device"):
            call()


def test_backward_with_offsets_out_of_range_stays_within_the_tensors():
    T, heads, D = 64, 2, 64
    wide = torch.zeros((T + 128, heads, D), dtype=torch.bfloat16, device=DEV)
    q, lse = wide[64:64 + T], torch.zeros((heads, T), device=DEV)
    for bad in ([-5, 10, 1000], [50, 20, 60], [2**31 - 1, -2**31, 5], [0, 64, 64]):
        grads = [torch.full((T + 128, heads, D), 3.0, dtype=torch.bfloat16, device=DEV) for _ in range(3)]
        offsets, lengths = (torch.tensor(x, dtype=torch.int32, device=DEV) for x in (bad, [2**31 - 1, -7]))
        L.sr_attention_bwd(q, q, q, q, q, lse, offsets=offsets, lengths_k=lengths, **{n: x[64:64 + T] for n, x in zip(("out_dq", "out_dk", "out_dv"), grads)})
        for x in grads:
            assert (x[:64] == 3).all() and (x[64 + T:] == 3).all()
