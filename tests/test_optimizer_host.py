"""OrthogonalMomentum without a GPU: what it does around the orthogonalised update, with another operation in its place."""
import os
import re

import pytest
import torch

from paper_2202_08556_amd import optim
from paper_2202_08556_amd.node_classifier import NodeClassifier, optimizers

README = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "README.md")


@pytest.fixture
def as_it_is(monkeypatch):
    """orthogonalise hands its update back; what it was given is kept."""
    given = []

    def same(update, *_):
        given.append(update)
        return update.clone()

    monkeypatch.setattr(optim, "orthogonalise", same)
    return given


def step(shape, **kw):
    p = torch.nn.Parameter(torch.zeros(shape))
    p.grad = torch.ones(shape)
    optim.OrthogonalMomentum([p], lr=1.0, momentum=0.0, nesterov=False, **kw).step()
    return float(-p.detach().flatten()[0])


def test_factor_by_the_axis_of_the_outputs(as_it_is):
    """max(1, outputs / inputs)^(1/2), for weights (out, in) and (in, out)."""
    assert step((8, 2)) == 2.0 and step((2, 8)) == 1.0 and step((3, 8, 2)) == 2.0
    assert step((8, 2), out_axis=-1) == 1.0 and step((2, 8), out_axis=-1) == 2.0 and step((3, 2, 8), out_axis=-1) == 2.0
    for bad in (0, 1, -3, None):
        with pytest.raises(ValueError):
            step((2, 8), out_axis=bad)


def test_factor_of_the_framework_s_own_weights(as_it_is):
    """A layer that widens takes the larger step, one that narrows does not: their weights are (in, out)."""
    model = NodeClassifier(4, 8, 3)
    before = {n: p.detach().clone() for n, p in model.named_parameters()}
    for p in model.parameters():
        p.grad = torch.ones_like(p)
    optimizers(model, lr=1.0)[0].step()
    moved = {n: float((before[n] - p.detach()).flatten()[0]) for n, p in model.named_parameters() if p.dim() == 2 and "blocks" in n}
    update = 1.0 + 0.95                                      # gradient 1 and the momentum's share of it
    for name, by in (("w_up", 2.0), ("w_gate", 2.0), ("w_down", 1.0), ("conv.weight", 1.0)):
        got = [v for n, v in moved.items() if n.endswith(name)]
        assert len(got) == 2 and all(abs(v - by * update) < 1e-5 for v in got), (name, got)


def test_states_saved_without_the_choice(as_it_is):
    p = torch.nn.Parameter(torch.zeros(2, 8))
    opt = optim.OrthogonalMomentum([p], lr=1.0)
    saved = opt.state_dict()
    del saved["param_groups"][0]["out_axis"]
    opt.load_state_dict(saved)
    p.grad = torch.ones(2, 8)
    opt.step()
    assert opt.param_groups[0]["out_axis"] == -2 and float(-p.detach()[0, 0]) == pytest.approx(1.95)


def test_the_readme_s_optimizer():
    """The line of README.md runs as it is written, on a model with vectors among its blocks' parameters."""
    line, = re.findall(r"^step = (optim\..*?)(?:  +#.*)?$", open(README).read(), flags=re.M)
    model = NodeClassifier(4, 8, 3, norm="rms")
    step = eval(line, {"optim": optim, "model": model})
    assert all(p.dim() == 2 for g in step.param_groups for p in g["params"]) and step.param_groups[0]["out_axis"] == -1


def test_momentum_is_held_in_32_bits(as_it_is):
    """bfloat16 weights: 200 steps of one gradient bring a momentum of 0.99 to (1 - 0.99^200) / 0.01 times it, off by no more than
    a rounding to 32 bits a step; what is orthogonalised has the weight's type and one rounding.  Also after saving and loading."""
    p = torch.nn.Parameter(torch.zeros(2, 8, dtype=torch.bfloat16))
    opt = optim.OrthogonalMomentum([p], lr=1e-3, momentum=0.99, nesterov=False)
    g = torch.linspace(0.5, 1.5, 16).view(2, 8).to(torch.bfloat16)
    for k in range(200):
        if k == 100:
            other = torch.nn.Parameter(p.detach().clone())
            again = optim.OrthogonalMomentum([other], lr=1e-3, momentum=0.99, nesterov=False)
            again.load_state_dict(opt.state_dict())
            p, opt = other, again
        p.grad = g.clone()
        opt.step()
    want = g.double() * (1 - 0.99 ** 200) / 0.01
    held = opt.state[p]["momentum"]
    assert held.dtype == torch.float32 and ((held.double() - want).abs() <= 200 * 2.0 ** -24 * want).all()
    last = as_it_is[-1]
    assert last.dtype == torch.bfloat16 and ((last[0].double() - want).abs() <= (2.0 ** -8 + 2.0 ** -16) * want).all()


def test_more_matrices_than_a_call_takes(as_it_is):
    """Weights of one shape go in as few calls as take 65535 matrices at most each."""
    params = [torch.nn.Parameter(torch.zeros(30000, 1, 2)) for _ in range(5)]
    for i, p in enumerate(params):
        p.grad = torch.full_like(p, float(i + 1))
    optim.OrthogonalMomentum(params, lr=1.0, momentum=0.0, nesterov=False).step()
    assert [u.shape[0] * u.shape[1] for u in as_it_is] == [60000, 60000, 30000]
    assert all((p.detach() == -(i + 1.0)).all() for i, p in enumerate(params))
