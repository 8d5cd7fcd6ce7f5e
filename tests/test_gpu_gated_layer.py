"""GatedMLP with its stream position on the device, in a captured training step, and what autograd keeps of it."""
import pytest
import torch

from gpu_util import DEV, say
from paper_2511_00874_amd import lib as L
from paper_2511_00874_amd import train

pytestmark = pytest.mark.gpu
M, D, F = 96, 64, 128


def _inputs():
    g = torch.Generator(device=DEV).manual_seed(2)
    return tuple(torch.randn((M, D), device=DEV, generator=g) for _ in range(4))


def _layer(position):
    layer = train.GatedMLP(D, F, 9, device=DEV, round_fwd=L.SR, init_std=0.08)
    layer.position = position
    return layer


def _step(layer, x0, r0, dy, dh):
    x, r = x0.clone().requires_grad_(), r0.clone().requires_grad_()
    layer.gamma.grad, layer.have_grad = None, False
    y, h = layer(x, r)
    torch.autograd.backward([y, h], [dy, dh])
    return y.detach(), h.detach(), x.grad, r.grad, layer.gamma.grad, layer.dw_in, layer.dw_out


def test_a_position_on_the_device_gives_what_the_same_number_gives():
    say("gated mlp, device position")
    data = _inputs()
    host = _layer(1000)
    want = _step(host, *data)
    device = _layer(torch.tensor([1000], dtype=torch.int64, device=DEV))
    got = _step(device, *data)
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    assert int(device.position) == host.position
    other = _step(_layer(1001), *data)
    assert not torch.equal(other[0], want[0]) and not torch.equal(other[5], want[5])


def test_a_captured_step_draws_from_where_its_position_is_when_replayed():
    data = _inputs()
    at = torch.tensor([1000], dtype=torch.int64, device=DEV)
    layer = _layer(at)
    graph, stream = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        _step(layer, *data)  # warm up on the capture stream
        torch.cuda.synchronize()
        layer.position = at
        graph.capture_begin()
        got = _step(layer, *data)
        at.copy_(layer.position)  # the next replay goes on from here
        graph.capture_end()
    torch.cuda.synchronize()
    for position in (1000, None, None, 7, 1000):
        if position is not None:
            at.fill_(position)
        begin = int(at)
        graph.replay()
        torch.cuda.synchronize()
        plain = _layer(begin)
        want = _step(plain, *data)
        assert all(torch.equal(a, b) for a, b in zip(got, want)), begin
        assert int(at) == plain.position
        torch.cuda.synchronize()
