"""A residual model of node features trained by distillation or on labels: aggregation, group norm with an activation, gated
feed-forward blocks and the loss of a teacher's best classes or of the nodes' own, together.

    h = A . (X . W) + b
    h = h + A . (norm_silu(h) . W) + b          statistics over each graph of the batch
    h = h + feed_forward(norm(h))               statistics over each node
    logits = A . (h . W) + b

`python -m paper_2202_08556_amd.node_classifier` trains a small model on a batch of random graphs against a wider
teacher's best classes, then classifies single nodes, and prints the loss and the time of a step.  With `--labels SHARE` it
trains on the classes of that share of the nodes instead: the nodes' norm is the root-mean-square one, which adds the residual,
the loss is taken from (A . h) . W + b without the logits, and the weights' updates are orthogonalised.
"""
from __future__ import annotations

import argparse
import time

import numpy as np
import torch

from . import generators, layers
from .gcn import GraphConv, SparseGraph, aggregate
from .optim import OrthogonalMomentum


class Block(torch.nn.Module):
    """norm: that of the nodes by themselves, "group" or "rms"."""

    def __init__(self, hidden: int, groups: int, norm: str = "group"):
        super().__init__()
        if norm not in ("group", "rms"):
            raise ValueError(f"norm must be 'group' or 'rms', not {norm!r}")
        self.norm_graph = layers.GroupNorm(groups, hidden, activation="silu")
        self.conv = GraphConv(hidden, hidden, relu=False)
        self.norm_node = layers.GroupNorm(groups, hidden) if norm == "group" else layers.RMSNorm(hidden)
        self.feed_forward = layers.GatedFeedForward(hidden, 4 * hidden)

    def forward(self, graph: SparseGraph, h: torch.Tensor, offsets: torch.Tensor | None) -> torch.Tensor:
        more = self.conv(graph, self.norm_graph(h, offsets))
        if isinstance(self.norm_node, layers.RMSNorm):
            y, h = self.norm_node(more, residual=h)
            return h + self.feed_forward(y)
        return self.per_node(h + more)

    def per_node(self, h: torch.Tensor) -> torch.Tensor:
        """What a node's features go through by themselves, for one node or many."""
        if isinstance(self.norm_node, layers.RMSNorm):
            return h + self.feed_forward(self.norm_node(h))
        return h + self.feed_forward(self.norm_node(h.unsqueeze(-2)).squeeze(-2))


class NodeClassifier(torch.nn.Module):
    """Logits of the nodes of a graph, or of a batch of graphs side by side (offsets: int32, where each begins)."""

    def __init__(self, features: int, hidden: int, classes: int, blocks: int = 2, groups: int = 8, norm: str = "group"):
        super().__init__()
        self.conv_in = GraphConv(features, hidden, relu=False)
        self.blocks = torch.nn.ModuleList(Block(hidden, groups, norm) for _ in range(blocks))
        self.conv_out = GraphConv(hidden, classes, relu=False)

    def hidden(self, graph: SparseGraph, X: torch.Tensor, offsets: torch.Tensor | None = None) -> torch.Tensor:
        h = self.conv_in(graph, X)
        for block in self.blocks:
            h = block(graph, h, offsets)
        return h

    def forward(self, graph: SparseGraph, X: torch.Tensor, offsets: torch.Tensor | None = None) -> torch.Tensor:
        return self.conv_out(graph, self.hidden(graph, X, offsets))

    def loss(self, graph: SparseGraph, X: torch.Tensor, target: torch.Tensor, offsets: torch.Tensor | None = None) -> torch.Tensor:
        """Mean cross entropy of the nodes that have a class (target: -1 for the others)."""
        h = aggregate(graph, self.hidden(graph, X, offsets))
        return layers.linear_cross_entropy(h, self.conv_out.weight, target, bias=self.conv_out.bias)


def batch_of_graphs(graphs: int, mean: float, seed: int, device="cuda:0") -> tuple[SparseGraph, torch.Tensor]:
    """Random graphs of about `mean` nodes on one block-diagonal matrix (rows averaged), and their offsets."""
    rng = np.random.default_rng(seed)
    nodes = rng.poisson(mean, graphs)
    offsets = np.concatenate([[0], nodes.cumsum()]).astype(np.int32)
    rowptr, colind, vals = [0], [], []
    for first, n in zip(offsets, nodes):
        for i in range(n):
            near = np.unique(np.concatenate([[i], rng.integers(0, n, 3)]))
            colind.append(first + near)
            vals.append(np.full(near.size, 1.0 / near.size))
            rowptr.append(rowptr[-1] + near.size)
    m = int(offsets[-1])
    matrix = generators.CSR(m, m, np.array(rowptr, np.int32), np.concatenate(colind).astype(np.int32),
                            np.concatenate(vals).astype(np.float32))
    return SparseGraph.from_numpy(matrix, device), torch.from_numpy(offsets).to(device)


def best_classes(teacher: NodeClassifier, graph: SparseGraph, X: torch.Tensor, offsets: torch.Tensor, best: int):
    """(classes, logits) of the teacher's best per node: what is kept of it."""
    with torch.no_grad():
        top = teacher(graph, X, offsets).topk(best, dim=1)
    return top.indices.to(torch.int32), top.values


def train_step(model: NodeClassifier, optimizer: torch.optim.Optimizer, graph: SparseGraph, X: torch.Tensor, offsets: torch.Tensor,
               top_index: torch.Tensor, top_logits: torch.Tensor, temperature: float = 2.0) -> torch.Tensor:
    optimizer.zero_grad(set_to_none=True)
    loss = layers.distill_loss(model(graph, X, offsets), top_index, top_logits, temperature)
    loss.backward()
    optimizer.step()
    return loss.detach()


def optimizers(model: NodeClassifier, lr: float = 0.02) -> list[torch.optim.Optimizer]:
    """Orthogonalised updates for the blocks' matrices, Adam for everything else."""
    matrices = [p for p in model.blocks.parameters() if p.dim() == 2]
    ids = {id(p) for p in matrices}
    return [OrthogonalMomentum(matrices, lr=lr, out_axis=-1), torch.optim.Adam([p for p in model.parameters() if id(p) not in ids], lr=3e-3)]


def label_step(model: NodeClassifier, optimizers: list[torch.optim.Optimizer], graph: SparseGraph, X: torch.Tensor, offsets: torch.Tensor,
               target: torch.Tensor) -> torch.Tensor:
    for o in optimizers:
        o.zero_grad(set_to_none=True)
    loss = model.loss(graph, X, target, offsets)
    loss.backward()
    for o in optimizers:
        o.step()
    return loss.detach()


def main() -> None:
    p = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    p.add_argument("--graphs", type=int, default=400)
    p.add_argument("--features", type=int, default=32)
    p.add_argument("--hidden", type=int, default=64)
    p.add_argument("--classes", type=int, default=41)
    p.add_argument("--best", type=int, default=8)
    p.add_argument("--steps", type=int, default=60)
    p.add_argument("--labels", type=float, default=0.0, metavar="SHARE")
    a = p.parse_args()
    torch.manual_seed(0)
    graph, offsets = batch_of_graphs(a.graphs, 23.0, seed=1)
    X = torch.randn(graph.m, a.features, device="cuda")
    teacher = NodeClassifier(a.features, 2 * a.hidden, a.classes).cuda()
    top = best_classes(teacher, graph, X, offsets, a.best)
    model = NodeClassifier(a.features, a.hidden, a.classes, norm="rms" if a.labels else "group").cuda()
    if a.labels:
        target = torch.where(torch.rand(graph.m, device="cuda") < a.labels, top[0][:, 0], -1)
        both = optimizers(model)
    else:
        optimizer = torch.optim.Adam(model.parameters(), lr=3e-3)
    for step in range(a.steps):
        if step == 10:                                       # the first steps build what later ones find
            torch.cuda.synchronize()
            began = time.perf_counter()
        if a.labels:
            loss = label_step(model, both, graph, X, offsets, target)
        else:
            loss = train_step(model, optimizer, graph, X, offsets, *top)
        if step % 10 == 0:
            print(f"step {step}: loss {float(loss):.4f}", flush=True)
    torch.cuda.synchronize()
    if a.steps > 10:
        print(f"{graph.m} nodes in {a.graphs} graphs, {1e3 * (time.perf_counter() - began) / (a.steps - 10):.2f} ms a step")
    with torch.no_grad():
        one = torch.randn(1, a.hidden, device="cuda")
        print("one node's block:", tuple(model.blocks[0].per_node(one).shape))


if __name__ == "__main__":
    main()
