"""Calls that use a workspace, on two streams at once: each has its own, whatever the other does in between."""
import pytest
import torch

import attention_util as A
from gpu_util import DEV, say
from paper_2511_00874_amd import lib as L

pytestmark = pytest.mark.gpu


def _shape(q, k, **how):
    return L._attention(q, k, None, how.get("causal", True), how.get("sequences", 1), None, None, None)


def _attention(T, S, heads, kv, D, step, **how):
    def make(seed):
        return tuple(A.make((n, h, D), seed + i, DEV) for i, (n, h) in enumerate(((T, heads), (S, kv), (S, kv), (T, heads))))

    def run(x):
        o, lse = L.sr_attention_fwd(*x[:3], **how)
        return (o, lse, *L.sr_attention_bwd(x[3], *x[:3], o, lse, **how)) if step else (o, lse)

    def need(x):
        a = _shape(x[0], x[1], **how)
        return (L._lib.sr_attention_bwd_workspace_bytes if step else L._lib.sr_attention_fwd_workspace_bytes)(a)
    return make, run, need


def _embedding(M, V, K):
    def make(seed):
        g = torch.Generator(device=DEV).manual_seed(seed)
        return torch.randn((M, K), device=DEV, generator=g), torch.randint(0, V, (M,), device=DEV, generator=g)
    return make, lambda x: (L.sr_embedding_bwd(x[0], x[1], V),), lambda x: L._lib.sr_embedding_bwd_workspace_bytes(M, K)


CASES = {"keys in pieces": _attention(2000, 2000, 2, 1, 64, False), "chunks of a cache": _attention(2, 2 * 8000, 4, 4, 128, False, sequences=2),
         "backward 64": _attention(1500, 1500, 2, 1, 64, True), "backward 128": _attention(300, 300, 4, 2, 128, True),
         "table by ranks": _embedding(5000, 900, 64), "table by digits": _embedding(20000, 5000, 32)}


@pytest.mark.parametrize("name", CASES)
def test_two_streams(name):
    say("two streams", name)
    make, run, need = CASES[name]
    inputs = [make(100 * i) for i in range(2)]
    assert all(need(x) > 0 for x in inputs)
    want = [run(x) for x in inputs]
    assert not torch.equal(want[0][0], want[1][0])
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    got = [[], []]
    for _ in range(6):
        for i, s in enumerate(streams):
            with torch.cuda.stream(s):
                got[i].append(run(inputs[i]))
    torch.cuda.synchronize()
    for i in range(2):
        for r in got[i]:
            assert all(torch.equal(x, y) for x, y in zip(r, want[i])), i


def test_two_graphs_replayed_at_once():
    # captured calls keep the workspace that they were recorded with: two graphs have one each
    streams, graphs, outs, want = [torch.cuda.Stream() for _ in range(2)], [], [], []
    make, run, need = CASES["backward 128"]
    inputs = [make(100 * i) for i in range(2)]
    assert need(inputs[0]) > 0
    for x, s in zip(inputs, streams):
        s.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(s):
            run(x)
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=s):
            outs.append(run(x))
        graphs.append(g)
        want.append(run(x))
    for _ in range(4):
        for o in outs:
            for t in o:
                t.zero_()
        torch.cuda.synchronize()
        for g, s in zip(graphs, streams):
            with torch.cuda.stream(s):
                g.replay()
        torch.cuda.synchronize()
        for o, w in zip(outs, want):
            assert all(torch.equal(x, y) for x, y in zip(o, w))
