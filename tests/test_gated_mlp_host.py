"""The host side of GatedMLP: which quantizers its calls get, and what a training step asks of a model."""
import weakref

import pytest
import torch

from paper_2511_00874_amd import lib as L
from paper_2511_00874_amd import train

COUNTS = (40, 7, 4096, 1)


def _drawn(position):
    layer = train.GatedMLP(32, 128, 7, device="cpu")
    layer.position = position
    return [layer._q(L.E4M3, L.SR, n) for n in COUNTS], layer


def test_a_position_on_the_device_is_another_for_every_quantizer():
    want, host = _drawn(1000)
    assert [q.counter_offset for q in want] == [1000, 1005, 1006, 1518] and host.position == 1519
    at = torch.tensor([1000], dtype=torch.int64)
    got, layer = _drawn(at)
    assert all(isinstance(q.counter_offset, torch.Tensor) for q in got)  # (marshalled as device counters)
    assert [int(q.counter_offset) for q in got] == [q.counter_offset for q in want]
    assert int(layer.position) == host.position and int(at) == 1000  # (the caller's tensor is left as it was)


def test_a_training_step_takes_models_that_know_of_linears_alone():
    class Model(torch.nn.Module):
        def __init__(self):
            super().__init__()
            self.table = torch.nn.Embedding(11, 11)

        def sr_linears(self):
            return []

        def forward(self, ids):
            return self.table(ids)

    model = Model()
    ids = torch.arange(10)[None]
    losses = [float(train.train_step(model, ids, ids + 1, 1.0)) for _ in range(3)]
    assert losses[2] < losses[1] < losses[0]
    assert train.flops_per_token(model) == 0.0


def _plain_layer():
    """A block whose passes are plain operators on the CPU, and the tensors and gradients that they were given."""
    layer = train.GatedMLP(32, 128, 7, device="cpu")
    layer.seen = {}

    def forward(x, residual, gamma, keep):
        h = x + residual
        blocks = [L.Blocks(torch.full((len(x), 16 * (i + 1)), i, dtype=torch.uint8), torch.full((len(x), 4), 10 + i, dtype=torch.uint8), L.E4M3,
                           16 * (i + 1)) for i in range(5)]
        kept = blocks[0], torch.full((len(x),), 2.0), *blocks[1:]
        layer.seen["kept"] = [weakref.ref(t) for b in blocks for t in (b.codes, b.exps)] + [weakref.ref(kept[1])]
        layer.seen["forms"] = [(b.kind, b.cols, b.codes.clone(), b.exps.clone()) for b in blocks]
        return h * gamma, h, kept

    def backward(dy, dh, h, gamma, kept):
        n, rstd, *blocks = kept
        layer.seen["back"] = [(b.kind, b.cols, b.codes.clone(), b.exps.clone()) for b in (n, *blocks)]
        layer.seen["dh"] = dh
        assert torch.equal(rstd, torch.full((len(h),), 2.0))
        return dy * gamma + (0 if dh is None else dh), (dy * h).sum(0)

    layer._forward, layer._backward = forward, backward
    return layer


def _pass(layer):
    x, r = (torch.randn((6, 32), requires_grad=True) for _ in range(2))
    y, h = layer(x, r)
    return x, r, y, h


def test_what_a_pass_keeps_goes_with_its_backward_pass():
    layer = _plain_layer()
    x, r, y, h = _pass(layer)
    assert all(t() is not None for t in layer.seen["kept"])
    (y + h).sum().backward()
    for a, b in zip(layer.seen["back"], layer.seen["forms"]):
        assert a[:2] == b[:2] and torch.equal(a[2], b[2]) and torch.equal(a[3], b[3])
    # y and h are still here, and with them the graph
    assert y.grad_fn is not None and not any(t() is not None for t in layer.seen["kept"])
    assert torch.equal(x.grad, torch.full((6, 32), 2.0)) and torch.equal(r.grad, x.grad)


def test_what_a_pass_keeps_is_seen_by_hooks_of_saved_tensors():
    layer, seen = _plain_layer(), []

    def pack(t):
        seen.append(t.data_ptr())
        return t.clone()

    with torch.autograd.graph.saved_tensors_hooks(pack, lambda t: t):
        x, r, y, h = _pass(layer)
        kept = {t().data_ptr() for t in layer.seen["kept"] if t() is not None}
    assert kept <= set(seen) and len(seen) >= 13
    (y + h).sum().backward()
    assert torch.equal(x.grad, torch.full((6, 32), 2.0))


def test_a_second_derivative_is_refused():
    layer = _plain_layer()
    x, r, y, h = _pass(layer)
    (dx,) = torch.autograd.grad((y * y).sum(), x, create_graph=True)
    with pytest.raises(RuntimeError):
        (dx * dx).sum().backward()


def test_a_result_that_is_not_used_has_no_gradient_to_read():
    layer = _plain_layer()
    x, r, y, h = _pass(layer)
    y.sum().backward()
    assert layer.seen["dh"] is None and torch.equal(x.grad, torch.ones((6, 32)))
    x, r, y, h = _pass(layer)
    layer.gamma.grad = None
    h.sum().backward()
    assert torch.equal(layer.seen["dh"], torch.ones((6, 32))) and torch.equal(r.grad, torch.ones((6, 32)))
    assert torch.equal(layer.gamma.grad, torch.zeros(32))
