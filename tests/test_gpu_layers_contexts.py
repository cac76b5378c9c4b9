"""The layers where torch does more around an operation than differentiate it backwards (a mode, a subclass), and where it
recomputes or accumulates: the same results."""
import pytest
import torch

from paper_2202_08556_amd import layers

pytestmark = pytest.mark.gpu


class Marked(torch.Tensor):
    pass


def calls():
    g = torch.Generator(device="cuda").manual_seed(1)
    r = lambda *s: torch.randn(*s, generator=g, device="cuda")          # noqa: E731
    offsets = torch.tensor([0, 3, 3, 40], dtype=torch.int32, device="cuda")
    index = torch.randint(0, 41, (40, 5), generator=g, device="cuda")
    top = r(40, 5)
    return {
        "group_norm": ((r(40, 24), r(24), r(24)), lambda x, w, b: layers.group_norm(x, 3, w, b, activation="silu", offsets=offsets)),
        "plain_norm": ((r(40, 24),), lambda x: layers.group_norm(x, 3)),
        "gated": ((r(40, 24), r(24, 56), r(24, 56), r(56, 24)), layers.gated_feed_forward),
        "distill": ((r(40, 41),), lambda z: layers.distill_loss(z, index, top, 2.0, "none")),
    }


def run(operands, f):
    leaves = [t.detach().requires_grad_(True) for t in operands]
    y = f(*leaves)
    return [y.detach(), *torch.autograd.grad(y, leaves, torch.ones_like(y))]


@pytest.mark.parametrize("name", ["group_norm", "plain_norm", "gated", "distill"])
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


@pytest.mark.parametrize("name", ["group_norm", "gated", "distill"])
def test_recomputed_and_accumulated(name):
    from torch.utils.checkpoint import checkpoint
    operands, f = calls()[name]
    want = run(operands, f)
    leaves = [t.detach().requires_grad_(True) for t in operands]
    y = checkpoint(f, *leaves, use_reentrant=False)
    y.backward(torch.ones_like(y))
    f(*leaves).sum().backward()
    assert torch.equal(y.detach(), want[0])
    assert all(torch.allclose(t.grad, 2 * w, rtol=1e-5, atol=1e-6) for t, w in zip(leaves, want[1:]))


def test_a_graph_is_used_once():
    operands, f = calls()["group_norm"]
    x = operands[0].requires_grad_(True)
    y = f(x, *operands[1:])
    torch.autograd.grad(y.sum(), x)
    with pytest.raises(RuntimeError):
        torch.autograd.grad(y.sum(), x)


def test_changed_operands_are_noticed():
    operands, f = calls()["gated"]
    leaves = [t.detach().requires_grad_(True) for t in operands]
    y = f(*leaves)
    with torch.no_grad():
        leaves[3].mul_(2)
    with pytest.raises(RuntimeError, match="modified"):
        y.sum().backward()


@pytest.mark.parametrize("name,kept", [("group_norm", 40 * 24 + 2 * 24 + 4 + 3 * 3 * 2), ("gated", 40 * 24 + 3 * 24 * 56 + 3 * 40 * 56),
                                       ("distill", 40 * 41 + 2 * 40 * 5 + 2 * 40)])
def test_hooks_see_all_that_is_kept(name, kept):
    """What waits for the backward pass goes through the hooks for saved tensors and nothing stays beside them: offloaded and
    brought back, the same results.  kept: operands and statistics; operands, u, v and a."""
    operands, f = calls()[name]
    want = run(operands, f)
    packed = []

    def pack(t):
        packed.append(t.numel())
        return t.detach().cpu()

    with torch.autograd.graph.saved_tensors_hooks(pack, lambda t: t.cuda()):
        got = run(operands, f)
    assert all(torch.equal(p, q) for p, q in zip(got, want))
    assert sum(packed) == kept


def test_recomputation_keeps_nothing_of_the_block():
    """The gated block's hidden numbers (u, v, a: 20 MB each) are not held between forward and backward under checkpoint."""
    from torch.utils.checkpoint import checkpoint
    x, wg, wu, wd = (torch.randn(s, device="cuda").requires_grad_(True) for s in ((5000, 16), (16, 1024), (16, 1024), (1024, 16)))
    layers.gated_feed_forward(x, wg, wu, wd).sum().backward()
    torch.cuda.synchronize()
    before = torch.cuda.memory_allocated()
    y = checkpoint(layers.gated_feed_forward, x, wg, wu, wd, use_reentrant=False)
    assert torch.cuda.memory_allocated() - before < 5000 * 1024 * 4
    y.sum().backward()


@pytest.mark.parametrize("name", ["group_norm", "gated", "distill"])
def test_function_transforms_and_forward_mode_are_refused(name):
    operands, f = calls()[name]
    with pytest.raises(RuntimeError):
        torch.func.vmap(lambda x: f(x, *operands[1:]))(operands[0].expand(2, *operands[0].shape))
    with torch.autograd.forward_ad.dual_level():
        x = torch.autograd.forward_ad.make_dual(operands[0], torch.ones_like(operands[0]))
        with pytest.raises(RuntimeError):
            f(x, *operands[1:])
