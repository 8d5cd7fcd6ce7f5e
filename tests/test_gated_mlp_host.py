"""The host side of GatedMLP: which quantizers its calls get, and what a training step asks of a model."""
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
