"""Attention, embedding and AdamW through autograd and the decoder: what the modules give is what the calls beneath them give."""
import numpy as np
import pytest
import torch
import torch.nn.functional as F

import attention_util as A
from gpu_util import DEV, say
from paper_2511_00874_amd import lib as L
from paper_2511_00874_amd import train

pytestmark = pytest.mark.gpu


def test_attention_gradients_through_autograd():
    T, heads, kv, D = 130, 4, 2, 64
    offsets = torch.tensor([3, 60, 120], dtype=torch.int32, device=DEV)
    qkv = A.make((T, heads + 2 * kv, D), 0, DEV).requires_grad_()
    o = train.attention(qkv, heads, kv, offsets=offsets)
    do = A.make((T, heads, D), 1, DEV)
    o.backward(do)
    parts = [A.wide(x) for x in (qkv[:, :heads], qkv[:, heads:heads + kv], qkv[:, heads + kv:])]
    want, err = A.backward(A.wide(do), *parts, D ** -0.5, True, A.pairs(T, T, offsets=[3, 60, 120]))
    grad = qkv.grad
    for g, w, e in zip((grad[:, :heads], grad[:, heads:heads + kv], grad[:, heads + kv:]), want, err):
        A.check(g, w, e, "gradient")
    # rows of no sequence: zeros, forward and backward
    for x in (o.detach(), grad):
        assert not x[:3].any() and not x[120:].any()
    with pytest.raises(RuntimeError):  # (the kernels' gradients have none of their own)
        torch.autograd.grad(train.attention(qkv, heads, kv).float().sum(), qkv, create_graph=True)[0].float().sum().backward()


def test_two_graphs_of_one_layer_do_not_meet():
    qkv = A.make((70, 6, 64), 0, DEV).requires_grad_()
    a, b = train.attention(qkv, 2, 2), train.attention(qkv * 2, 2, 2)
    do = A.make((70, 2, 64), 1, DEV)
    g2, = torch.autograd.grad(b, qkv, do)
    g1, = torch.autograd.grad(a, qkv, do)
    one = train.attention(qkv, 2, 2)
    assert torch.equal(g1, torch.autograd.grad(one, qkv, do)[0])
    two = train.attention(qkv * 2, 2, 2)
    assert torch.equal(g2, torch.autograd.grad(two, qkv, do)[0])


def test_embedding_gradients_through_autograd():
    table = train.Embedding(50, 24, scale=3.0, padding=7, device=DEV)
    ids = torch.randint(0, 50, (5, 9), device=DEV, generator=torch.Generator(device=DEV).manual_seed(0))
    ids[0, 0] = 7
    y = table(ids)
    assert torch.equal(y, table.weight[ids] * 3.0)
    c = torch.randn_like(y)
    (y * c).sum().backward()
    want = torch.zeros((50, 24), dtype=torch.float64).index_add_(0, ids.cpu().view(-1), c.cpu().double().view(-1, 24)) * 3.0
    want[7] = 0.0
    # a sum of at most 45 terms and a product
    size = torch.zeros((50, 24), dtype=torch.float64).index_add_(0, ids.cpu().view(-1), c.cpu().double().view(-1, 24).abs()) * 3.0
    assert ((table.weight.grad.cpu().double() - want).abs() <= 50 * 2.0**-24 * size).all()


def _tiny(seed=5, **how):
    torch.manual_seed(seed)
    m = train.Decoder(vocab=96, d=64, heads=4, layers=2, seq=40, seed=seed, device=DEV, attention="packed", embedding="sorted", **how)
    for lin in m.sr_linears():
        lin.round_mode = L.RTN  # (a pass is the same wherever its stretches of the stream are)
    return m


@pytest.mark.parametrize("kv_heads", [None, 2])
@pytest.mark.parametrize("ffn", ["gelu", "gated"])
def test_decoder_is_its_parts(kv_heads, ffn):
    m = _tiny(kv_heads=kv_heads, ffn=ffn)
    for g in m.gated_mlps():
        g.round_bwd = L.RTN
    ids = torch.randint(0, 96, (4, 20), device=DEV, generator=torch.Generator(device=DEV).manual_seed(1))
    logits = m(ids)
    x = L.sr_embedding_fwd(m.tok.weight.detach(), ids.view(-1)).view(4, 20, 64) + L.sr_embedding_fwd(m.pos.weight.detach(), torch.arange(20, device=DEV))
    x0 = x.clone().requires_grad_()
    h = x0
    kv = kv_heads or 4
    for b in m.blocks:
        qkv = b.qkv(b.ln1(h)).bfloat16().view(80, 4 + 2 * kv, 16)
        a = b.proj(train.attention(qkv, 4, kv, sequences=4).view(4, 20, 64).float())
        if b.mlp is not None:
            y, r = b.mlp(a, h)
            h = r + y
        else:
            h = h + a
            h = h + b.fc2(F.gelu(b.fc1(b.ln2(h))))
    by_hand = m.head(m.ln(h))
    assert torch.equal(logits, by_hand)
    dy = torch.randn_like(logits) * 1e-2
    logits.backward(dy)
    grads = [p.grad.clone() for p in (m.tok.weight, m.pos.weight)]
    dx, = torch.autograd.grad(by_hand, x0, dy)
    assert torch.equal(grads[0], L.sr_embedding_bwd(dx.reshape(80, 64), ids.view(-1), 96))
    assert torch.equal(grads[1], L.sr_embedding_bwd(dx.sum(0), torch.arange(20, device=DEV), 40))


def test_packed_batches():
    # sequences packed back to back are the sequences: attention, positions (per-tensor scales keep the linears from being so, row by row)
    lengths = [1, 17, 5, 25]  # (the linears take whole sixteens of rows)
    offsets = torch.tensor(np.cumsum([0] + lengths), dtype=torch.int32, device=DEV)
    T = sum(lengths)
    m = _tiny()
    ids = torch.randint(0, 96, (T,), device=DEV, generator=torch.Generator(device=DEV).manual_seed(2))
    logits = m(ids, offsets)
    assert logits.shape == (T, 96)
    x = (m.tok(ids) + m.pos(torch.cat([torch.arange(n, device=DEV) for n in lengths]))).unsqueeze(0)
    for b in m.blocks:
        x = b(x, offsets)
    assert torch.equal(logits, m.head(m.ln(x)).squeeze(0))
    logits.square().mean().backward()
    assert all(p.grad is not None and torch.isfinite(p.grad).all() for p in m.parameters())
    # what comes after a place, and what belongs to other sequences, has no part in its attention
    qkv = A.make((T, 12, 16), 3, DEV)
    o = train.attention(qkv, 4, offsets=offsets)
    for a, n in zip(offsets.tolist(), lengths):
        assert torch.equal(o[a:a + n], train.attention(qkv[a:a + n].contiguous(), 4))
    with pytest.raises(ValueError):
        train.Decoder(vocab=96, d=64, heads=4, layers=1, seq=40, device=DEV)(ids, offsets)
    with pytest.raises(ValueError):
        train.Decoder(vocab=96, d=64, heads=4, layers=1, seq=40, device=DEV, kv_heads=2)


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("ffn", ["gelu", "gated"])
def test_training_steps(bits, ffn):
    say("training steps", bits, ffn)
    m = _tiny(ffn=ffn, kv_heads=2)
    opt = train.AdamW(m, lr=1e-3, bits=bits, seed=3)
    ids = torch.randint(0, 96, (4, 20), device=DEV, generator=torch.Generator(device=DEV).manual_seed(1))
    assert len(opt.tensors()) == len(m.sr_linears()) + 2 * len(m.gated_mlps()) + len(list(m.parameters()))
    for step in range(1, 4):
        loss = F.cross_entropy(m(ids).view(-1, 96), ids.view(-1))
        loss.backward()
        # the step is one call on every tensor and its gradient
        copies = []
        for x, t in opt.owned + opt.params:
            g = t.g if isinstance(x, (train.SRLinear, train.GatedMLP)) else x.grad
            copies.append(L.AdamWTensor(t.w.clone(), g.clone(), t.m.clone(), t.v.clone(), *(None if s is None else s.clone() for s in (t.m_scales, t.v_scales)),
                                        weight_decay=t.weight_decay))
        opt.step()
        for c, t in zip(copies, opt.tensors()):
            c.counter_offset = t.counter_offset
            L.sr_adamw([c], 1e-3, step, betas=opt.betas, eps=opt.eps, seed=3)
            assert torch.equal(c.w, t.w) and torch.equal(c.m, t.m) and torch.equal(c.v, t.v)
        assert all(p.grad is None for p in m.parameters()) and not any(x.have_grad for x in m.sr_linears() + m.gated_mlps())
        assert torch.isfinite(loss)
    places = [(t.counter_offset, t.counter_offset + t.blocks()) for t in opt.tensors()]
    assert all(a[1] <= b[0] for a, b in zip(sorted(places), sorted(places)[1:]))  # every tensor draws for itself
    # a saved state goes on where it was
    state = opt.state_dict()
    state["tensors"] = [[x.clone() for x in t] for t in state["tensors"]]
    other = train.AdamW(m, bits=bits, seed=3)
    other.load_state_dict(state)
    assert other.steps == 3 and all(torch.equal(a.m, b.m) and torch.equal(a.v, b.v) for a, b in zip(opt.tensors(), other.tensors()))
    with pytest.raises(ValueError):
        train.AdamW(m, bits=40 - bits).load_state_dict(state)


def test_train_step_with_an_optimizer():
    m = _tiny()
    opt = train.AdamW(m, bits=8)
    ids = torch.randint(0, 96, (4, 24), device=DEV, generator=torch.Generator(device=DEV).manual_seed(1))
    before = [t.w.clone() for t in opt.tensors()]
    loss = train.train_step(m, ids, ids, 1e-3, micro_batches=2, optimizer=opt)
    assert torch.isfinite(loss) and opt.steps == 1
    assert all(not torch.equal(a, t.w) for a, t in zip(before, opt.tensors()) if t.w.numel() > 1000)


def test_captured_step():
    # lookup, attention, both backward passes and the optimizer recorded in one graph, replayed with other ids between eager work
    T, V, D, heads = 96, 40, 64, 1
    g = torch.Generator(device=DEV).manual_seed(0)
    ids = torch.randint(0, V, (T,), device=DEV, generator=g)
    table = (torch.randn((V, D), device=DEV, generator=g)).bfloat16()
    do = torch.randn((T, heads, D), device=DEV, generator=g).bfloat16()
    offsets = torch.tensor([0, 50, T], dtype=torch.int32, device=DEV)
    step, pos = torch.ones(1, dtype=torch.int64, device=DEV), torch.zeros(1, dtype=torch.int64, device=DEV)
    grad = torch.zeros((V, D), device=DEV)

    def make():
        return L.AdamWBatch([L.AdamWTensor.zeros(table.clone().view(-1), grad.view(-1), 8)])

    def run(batch, step, pos):
        w = batch.keep[0].w.view(V, D)
        x = L.sr_embedding_fwd(w, ids).view(T, heads, D)
        o, lse = L.sr_attention_fwd(x, x, x, offsets=offsets)
        dq, dk, dv = L.sr_attention_bwd(do, x, x, x, o, lse, offsets=offsets)
        L.sr_embedding_bwd((dq.float() + dk.float() + dv.float()).view(T, D), ids, V, out=grad)
        batch.run(1e-2, step, counter=pos)
        return o

    a, b = make(), make()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        run(make(), step, pos)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        o = run(a, step, pos)
    for i in range(1, 5):
        step.fill_(i)
        pos.fill_(1000 * i)
        ids.copy_(torch.randint(0, V, (T,), device=DEV, generator=g))
        offsets[1] = 10 * i
        graph.replay()
        torch.cuda.synchronize()
        got = [x.clone() for x in (o, grad, a.keep[0].w, a.keep[0].m, a.keep[0].v)]
        want = [run(b, step, pos), grad, b.keep[0].w, b.keep[0].m, b.keep[0].v]
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(got, want)), i


def test_calls_on_two_streams():
    q, k, v = (A.make((600, 4, 64), i, DEV) for i in range(3))
    one = L.sr_attention_fwd(q, k, v)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    outs = []
    for _ in range(4):
        for s in streams:
            with torch.cuda.stream(s):
                outs.append(L.sr_attention_fwd(q, k, v))
    torch.cuda.synchronize()
    assert all(torch.equal(o[0], one[0]) and torch.equal(o[1], one[1]) for o in outs)
