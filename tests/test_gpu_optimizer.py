"""The AdamW of a model: which memory a step is made in, and what it counts."""
import pytest
import torch

from gpu_util import DEV
from paper_2511_00874_amd import lib as L
from paper_2511_00874_amd import train

pytestmark = pytest.mark.gpu


class Two(torch.nn.Module):
    """An SR linear, a gated block and a matrix of plain parameters."""

    def __init__(self):
        super().__init__()
        self.lin = train.SRLinear(16, 32, 1, device=DEV)
        self.mlp = train.GatedMLP(16, 128, 2, device=DEV)
        self.matrix = torch.nn.Parameter(torch.randn((5, 7), device=DEV))

    def sr_linears(self):
        return [self.lin]

    def gated_mlps(self):
        return [self.mlp]

    def fill(self, seed, lin=True, mlp=True, matrix=True):
        """Gradients, as a backward pass leaves them."""
        g = torch.Generator(device=DEV).manual_seed(seed)
        rand = lambda x: torch.randn(x.shape, device=DEV, generator=g)  # noqa: E731
        if lin:
            self.lin.dW.copy_(rand(self.lin.dW))
            self.lin.have_grad = True
        if mlp:
            self.mlp.dw_in.copy_(rand(self.mlp.dw_in))
            self.mlp.dw_out.copy_(rand(self.mlp.dw_out))
            self.mlp.have_grad = True
            self.mlp.gamma.grad = rand(self.mlp.gamma)
        if matrix:
            self.matrix.grad = rand(self.matrix)


def _weights(m):
    return [m.lin.weight, m.mlp.w_in, m.mlp.w_out, m.mlp.gamma.detach(), m.matrix.detach()]


@pytest.mark.parametrize("bits", [32, 8])
def test_weights_assigned_anew(bits):
    # a weight or gradient in other memory than when the optimizer was made, as after loading a checkpoint: the step is made there
    a, b = Two(), Two()
    b.load_state_dict(a.state_dict())
    opts = [train.AdamW(m, lr=1e-2, bits=bits) for m in (a, b)]
    for m, o in zip((a, b), opts):
        m.fill(0)
        o.step()
    old = [w.clone() for w in _weights(a)]
    kept = _weights(a)
    a.lin.weight = a.lin.weight.clone()
    a.lin.dW = torch.zeros_like(a.lin.dW)
    a.mlp.w_in, a.mlp.w_out = a.mlp.w_in.clone(), a.mlp.w_out.clone()
    a.mlp.dw_in, a.mlp.dw_out = torch.zeros_like(a.mlp.dw_in), torch.zeros_like(a.mlp.dw_out)
    a.mlp.gamma.data, a.matrix.data = a.mlp.gamma.data.clone(), a.matrix.data.clone()
    for m, o in zip((a, b), opts):
        m.fill(1)
        o.step()
    for x, y, was, memory in zip(_weights(a), _weights(b), old, kept):
        assert torch.equal(x, y) and not torch.equal(x, was)
        assert torch.equal(memory, was)  # (what it was in before is left alone)
    # of another size: refused, with the state as it was
    a.fill(2)
    a.matrix.data, a.matrix.grad = torch.zeros((5, 8), device=DEV), None
    a.matrix.grad = torch.zeros((5, 8), device=DEV)
    before = opts[0].steps, opts[0].position
    with pytest.raises(ValueError):
        opts[0].step()
    assert (opts[0].steps, opts[0].position) == before and a.lin.have_grad
