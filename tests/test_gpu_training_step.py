"""RMS norm, the cross entropy of a linear layer and orthogonalised updates as a training step has them together, and where torch
does more around an operation than differentiate it backwards (a mode, a subclass, recomputation)."""
import pytest
import torch

from paper_2202_08556_amd import layers, node_classifier, optim
from paper_2202_08556_amd.node_classifier import NodeClassifier, batch_of_graphs, label_step, optimizers

pytestmark = pytest.mark.gpu


class Marked(torch.Tensor):
    pass


def calls():
    g = torch.Generator(device="cuda").manual_seed(3)
    r = lambda *s: torch.randn(*s, generator=g, device="cuda")          # noqa: E731
    target = torch.randint(-5, 41, (40,), generator=g, device="cuda")
    wide = torch.randint(-5, 700, (40,), generator=g, device="cuda")
    return {
        "rms": ((r(40, 24), r(24)), lambda x, w: layers.rms_norm(x, w)),
        "rms_residual": ((r(40, 24), r(24), r(40, 24)), lambda x, w, s: sum(layers.rms_norm(x, w, residual=s))),
        "cross_entropy": ((r(40, 24), r(24, 41), r(41)), lambda x, w, b: layers.linear_cross_entropy(x, w, target, bias=b)),
        "cross_entropy_wide": ((r(40, 24), r(24, 700)), lambda x, w: layers.linear_cross_entropy(x, w, wide, reduction="none")),
    }


def run(operands, f):
    leaves = [t.detach().requires_grad_(True) for t in operands]
    y = f(*leaves)
    return [y.detach(), *torch.autograd.grad(y, leaves, torch.ones_like(y))]


@pytest.mark.parametrize("name", list(calls() if torch.cuda.is_available() else ["rms"]))
def test_modes_and_subclasses(name):
    from torch.overrides import TorchFunctionMode

    class Through(TorchFunctionMode):
        def __torch_function__(self, func, types, args=(), kwargs=None):
            return func(*args, **(kwargs or {}))

    operands, f = calls()[name]
    want = run(operands, f)
    with Through():
        got = run(operands, f)
    assert all(torch.equal(p, q) for p, q in zip(got, want))
    marked = operands[0].as_subclass(Marked).detach().requires_grad_(True)
    y = f(marked, *operands[1:])
    g, = torch.autograd.grad(y, marked, torch.ones_like(y))
    assert torch.equal(y.detach().as_subclass(torch.Tensor), want[0]) and torch.equal(g.as_subclass(torch.Tensor), want[1])


@pytest.mark.parametrize("name", list(calls() if torch.cuda.is_available() else ["rms"]))
def test_recomputed_and_accumulated(name):
    from torch.utils.checkpoint import checkpoint
    operands, f = calls()[name]
    want = run(operands, f)
    leaves = [t.detach().requires_grad_(True) for t in operands]
    y = checkpoint(f, *leaves, use_reentrant=False)
    y.backward(torch.ones_like(y))
    f(*leaves).sum().backward()
    assert torch.equal(y.detach(), want[0])
    # a sum of the same numbers twice, each rounded once
    assert all(torch.allclose(t.grad, 2 * w, rtol=1e-6, atol=1e-7) for t, w in zip(leaves, want[1:]))


def test_used_twice():
    """The same tensor as x and residual, and a weight that two calls share: gradients add up."""
    operands, _ = calls()["rms_residual"]
    x, w = operands[0].clone().requires_grad_(True), operands[1].clone().requires_grad_(True)
    y, s = layers.rms_norm(x, w, residual=x)
    (y.sum() + layers.rms_norm(s, w).sum()).backward()
    X, W = x.detach().double().requires_grad_(True), w.detach().double().requires_grad_(True)
    n = lambda t: t * torch.rsqrt(t.square().mean(-1, keepdim=True) + 1e-6) * W             # noqa: E731
    (n(2 * X).sum() + n(2 * X).sum()).backward()
    assert torch.allclose(x.grad.double(), X.grad, rtol=1e-4, atol=1e-5) and torch.allclose(w.grad.double(), W.grad, rtol=1e-4, atol=1e-4)


def test_two_streams_at_once():
    """Calls of the same sizes on two streams have scratch memory of their own."""
    g = torch.Generator(device="cuda").manual_seed(5)
    r = lambda *s: torch.randn(*s, generator=g, device="cuda")          # noqa: E731
    sets = [(r(500, 96), r(96, 900), torch.randint(0, 900, (500,), generator=g, device="cuda"), r(300, 200)) for _ in range(2)]

    def step(x, w, t, u):
        x, w = x.detach().requires_grad_(True), w.detach().requires_grad_(True)
        loss = layers.linear_cross_entropy(x, w, t)
        return [loss.detach(), *torch.autograd.grad(loss, (x, w)), optim.orthogonalise(u)]

    want = [step(*s) for s in sets]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in sets]
    got = [None, None]
    for _ in range(5):
        for i, stream in enumerate(streams):
            stream.wait_stream(torch.cuda.current_stream())
            with torch.cuda.stream(stream):
                got[i] = step(*sets[i])
        torch.cuda.synchronize()
        assert all(torch.equal(p, q) for a, b in zip(got, want) for p, q in zip(a, b))


def test_gradients_of_the_labelled_model():
    """The loss without logits against the logits' own: (A . h) . W + b and A . (h . W) + b are the same numbers up to rounding."""
    torch.manual_seed(0)
    graph, offsets = batch_of_graphs(30, 12.0, seed=2)
    X = torch.randn(graph.m, 16, device="cuda")
    model = NodeClassifier(16, 32, 11, norm="rms").cuda()
    target = torch.randint(-4, 11, (graph.m,), device="cuda")
    names = [n for n, _ in model.named_parameters()]
    loss = model.loss(graph, X, target, offsets)
    got = torch.autograd.grad(loss, list(model.parameters()))
    logits = model(graph, X, offsets)
    ref = torch.nn.functional.cross_entropy(logits, target.clamp(min=-1), ignore_index=-1)
    want = torch.autograd.grad(ref, list(model.parameters()))
    assert abs(float(loss.detach() - ref.detach())) < 1e-5
    for n, a, b in zip(names, got, want):
        assert float((a - b).norm()) <= 1e-4 * float(b.norm()) + 1e-6, n


def test_steps_of_the_labelled_model():
    torch.manual_seed(0)
    graph, offsets = batch_of_graphs(30, 12.0, seed=2)
    X = torch.randn(graph.m, 16, device="cuda")
    model = NodeClassifier(16, 32, 11, norm="rms").cuda()
    target = torch.randint(-4, 11, (graph.m,), device="cuda")
    both = optimizers(model)
    before = [p.detach().clone() for p in model.parameters()]
    for _ in range(3):
        assert torch.isfinite(label_step(model, both, graph, X, offsets, target))
    assert all(torch.isfinite(p).all() and not torch.equal(p, q) for p, q in zip(model.parameters(), before))
    with torch.no_grad():
        one = model.blocks[0].per_node(torch.randn(1, 32, device="cuda"))
    assert one.shape == (1, 32)


def test_command(monkeypatch, capsys):
    monkeypatch.setattr("sys.argv", ["node_classifier", "--graphs", "20", "--hidden", "32", "--steps", "12", "--labels", "0.5"])
    node_classifier.main()
    assert "ms a step" in capsys.readouterr().out
