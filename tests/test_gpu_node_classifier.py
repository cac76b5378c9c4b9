"""The model of node_classifier.py, whose layers run together, against the same model in plain torch operations in 64 bits."""
import pytest
import torch

from paper_2202_08556_amd import node_classifier as nc

pytestmark = pytest.mark.gpu


def plain(model, A, X, offsets, top_index, top_logits, T):
    """Loss of the model in 64 bits, differentiable in the parameters given by name."""
    F = torch.nn.functional
    p = {k: v.detach().double().requires_grad_(True) for k, v in model.named_parameters()}
    conv = lambda h, name: A @ (h @ p[name + ".weight"]) + p[name + ".bias"]        # noqa: E731

    def norm(h, name, groups, each):
        w, b = p[name + ".weight"], p[name + ".bias"]
        bounds = offsets.tolist()
        parts = h.split(1) if each else [h[i:j] for i, j in zip(bounds, bounds[1:]) if j > i]
        out = []
        for q in parts:
            v = q.unflatten(1, (groups, -1))
            v = (v - v.mean((0, 2), keepdim=True)) / (v.var((0, 2), correction=0, keepdim=True) + 1e-5).sqrt()
            out.append(v.flatten(1))
        return torch.cat(out) * w + b

    h = conv(X.double(), "conv_in")
    for i, block in enumerate(model.blocks):
        n = f"blocks.{i}."
        h = h + conv(F.silu(norm(h, n + "norm_graph", block.norm_graph.groups, False)), n + "conv")
        x = norm(h, n + "norm_node", block.norm_node.groups, True)
        f = n + "feed_forward."
        h = h + (F.silu(x @ p[f + "w_gate"]) * (x @ p[f + "w_up"])) @ p[f + "w_down"]
    z = conv(h, "conv_out") / T
    t = (top_logits.double() / T).log_softmax(1)
    loss = (T * T * (t.exp() * (t - z.log_softmax(1).gather(1, top_index.long()))).sum(1)).mean()
    return loss, p


def test_model_and_gradients():
    """Everything is of order 1 and some twenty layers deep; float32 sums of up to 256 terms are off by some 1e-6 of their
    size, so 1e-4 leaves room for what the layers after them make of that."""
    torch.manual_seed(3)
    graph, offsets = nc.batch_of_graphs(12, 9.0, seed=4)
    X = torch.randn(graph.m, 20, device="cuda")
    model = nc.NodeClassifier(20, 32, 41, blocks=2, groups=4).cuda()
    top = nc.best_classes(nc.NodeClassifier(20, 48, 41, groups=4).cuda(), graph, X, offsets, 5)
    loss = nc.layers.distill_loss(model(graph, X, offsets), *top, 2.0)
    loss.backward()
    A = torch.sparse_csr_tensor(graph.rowptr, graph.colind, graph.vals.double(), (graph.m, graph.m)).to_dense()
    want, p = plain(model, A, X, offsets, *top, 2.0)
    want.backward()
    assert abs(float(loss.detach()) - float(want.detach())) <= 1e-4 * float(want.detach())
    for name, q in model.named_parameters():
        g = p[name].grad
        assert float((q.grad.double() - g).norm()) <= 1e-4 * float(g.norm()) + 1e-9, name


def test_training_lowers_the_loss():
    torch.manual_seed(5)
    graph, offsets = nc.batch_of_graphs(60, 15.0, seed=6)
    X = torch.randn(graph.m, 16, device="cuda")
    top = nc.best_classes(nc.NodeClassifier(16, 64, 11).cuda(), graph, X, offsets, 4)
    model = nc.NodeClassifier(16, 32, 11).cuda()
    optimizer = torch.optim.Adam(model.parameters(), lr=3e-3)
    losses = [float(nc.train_step(model, optimizer, graph, X, offsets, *top)) for _ in range(40)]
    assert losses[-1] < 0.5 * losses[0]


def test_one_node_is_a_row_of_all():
    """A node by itself (the path for single tokens) and among all others (matrix cores): sums in another order."""
    torch.manual_seed(7)
    block = nc.Block(64, 8).cuda()
    h = torch.randn(500, 64, device="cuda")
    with torch.no_grad():
        every, one = block.per_node(h), block.per_node(h[123])
    assert torch.allclose(every[123], one, rtol=1e-5, atol=1e-5)
