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


@pytest.mark.parametrize("bits", [32, 8])
def test_a_weight_counts_its_own_steps(bits):
    # what has no gradient at some steps is corrected by the steps that it made, as if it were alone
    m = Two()
    o = train.AdamW(m, lr=1e-2, bits=bits, round_mode=L.RTN)
    who = [(True, False, True), (True, True, False), (False, True, True), (True, True, True)]
    names = ("lin", "mlp", "matrix")
    of = {"lin": [0], "mlp": [1, 2, 3], "matrix": [4]}
    alone = [L.AdamWTensor.zeros(w.clone(), torch.empty(w.shape, device=DEV), bits, weight_decay=0.1 if w.dim() > 1 else 0.0) for w in _weights(m)]
    counts = [0] * 5

    def step(i, parts):
        m.fill(i, **dict(zip(names, parts)))
        grads = [m.lin.dW, m.mlp.dw_in, m.mlp.dw_out, m.mlp.gamma.grad, m.matrix.grad]
        for k in [k for name, there in zip(names, parts) if there for k in of[name]]:
            counts[k] += 1
            alone[k].g.copy_(grads[k])
            L.sr_adamw([alone[k]], 1e-2, counts[k], betas=o.betas, eps=o.eps, round_mode=L.RTN)
        o.step()
        assert all(torch.equal(w, t.w) for w, t in zip(_weights(m), alone)), (i, parts)

    for i, parts in enumerate(who):
        step(i, parts)
    assert counts == [3, 3, 3, 3, 3] and o.steps == 4
    state = o.state_dict()
    saved = state | {"tensors": [[x.clone() for x in t] for t in state["tensors"]], "counts": list(state["counts"])}
    o = train.AdamW(m, lr=1e-2, bits=bits, round_mode=L.RTN)
    o.load_state_dict(saved)
    assert o.state_dict()["counts"] == counts
    step(10, (True, False, False))
    step(11, (True, True, True))
    # a state from before weights had counts of their own: all have made all steps
    del saved["counts"]
    o.load_state_dict(saved)
    assert o.state_dict()["counts"] == [4] * 5
    with pytest.raises(ValueError):
        o.load_state_dict(saved | {"counts": [1, 2]})
