"""Trains a student of a GraphSAGE teacher on prepared hyperbatches, through the
framework's public entry points alone.

The graph's features are kept as 4-bit rows (a third of the fp16 bytes), which the
graph gathers unchanged.  Each step:

  prepare / fetch       a hyperbatch: sampled blocks and the nodes' 4-bit rows;
  teacher               a GraphSAGE-mean layer over each hop of the hyperbatch, on the
                        rows read back to fp16 (mx4_dequantize), and a linear head: its
                        top logits of each target node;
  student               for the target nodes alone, without their neighbourhoods: the
                        4-bit rows times 4-bit weights (mx4_linear, a frozen
                        projection) plus a learned, scaled embedding of the node
                        (embedding_lookup), then a linear head;
  loss and gradient     distillation from the teacher's top logits
                        (distill_loss_grad);
  update                the head by its dense gradient, the embedding table by the rows
                        of its gradient (embedding_grad_rows); nothing is read back.

    python examples/train_student.py [--steps 50] [--nodes 20000]
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

from agnes_inputs import synth  # noqa: E402
from paper_2601_01473_gb300 import Graph, ops  # noqa: E402


class Student:
    def __init__(self, nodes, dim, hidden, classes, device, seed=3):
        g = torch.Generator(device=device).manual_seed(seed)

        def normal(*shape, scale):
            return torch.randn(shape, generator=g, device=device) * scale

        self.dim, self.scale = dim, hidden ** 0.5
        self.projection = ops.mx4_quantize(normal(hidden, dim, scale=dim ** -0.5))
        self.bias = torch.zeros(hidden, device=device)
        self.table = normal(nodes, hidden, scale=0.02 / self.scale)
        self.head = normal(classes, hidden, scale=hidden ** -0.5)

    def step(self, rows, ids, teacher, index, temperature, lr):
        """One step on the 4-bit rows and ids of the target nodes; returns their
        losses."""
        hidden = ops.mx4_linear(rows, self.projection, self.dim, self.bias)
        hidden += ops.embedding_lookup(self.table, ids, self.scale)
        logits = hidden @ self.head.t()
        loss, grad = ops.distill_loss_grad(logits, teacher, index, 1.0 / ids.numel(), temperature,
                                           out=logits)
        g = ops.embedding_grad_rows(grad @ self.head, ids, self.table.shape[0], self.scale)
        self.head.addmm_(grad.t(), hidden, alpha=-lr)
        self.table.index_add_(0, g.ids.clamp(min=0), g.rows, alpha=-lr)
        return loss


class Teacher:
    """GraphSAGE layers with a linear head, here with fixed random weights."""

    def __init__(self, dim, hidden, classes, hops, device, seed=4):
        g = torch.Generator(device=device).manual_seed(seed)
        self.layers = []
        for _ in range(hops):
            self.layers.append((torch.randn(hidden, 2 * dim, generator=g, device=device)
                                / (2 * dim) ** 0.5).half())
            dim = hidden
        self.head = torch.randn(classes, hidden, generator=g, device=device) * 2

    def top_logits(self, graph, x, targets, top):
        """The top logits of every target node of the last hyperbatch."""
        hops = len(self.layers)
        for hop in range(hops - 1, -1, -1):  # the gathered rows are the outermost hop's
            x = graph.sage_mean_layer(hop, x, self.layers[hops - 1 - hop],
                                      out_dtype=torch.float16)
        logits = x[:, :targets].reshape(-1, x.shape[2]).float() @ self.head.t()
        return logits.topk(top, 1)


def train(steps=50, nodes=20_000, dim=128, hidden=128, classes=172, top=8, minibatches=4,
          targets=256, temperature=2.0, lr=0.5, device="cuda:0", report=None):
    """Returns the mean loss of each step."""
    device = torch.device(device)
    offsets, indices = synth.rmat_csr(nodes, 10, 0.57, 0.19, 0.19, seed=5,
                                      offsets_dtype=torch.int64)
    features = synth.normal_features(nodes, dim, torch.float16, seed=6).to(device)
    packed = ops.mx4_quantize(features)
    student = Student(nodes, dim, hidden, classes, device)
    teacher = Teacher(dim, hidden, classes, 2, device)
    pool = torch.arange(min(nodes, 4 * minibatches * targets), dtype=torch.int32)
    losses = []
    with Graph(offsets.to(device), indices.to(device), packed.view(torch.float16),
               adj_block_bytes=64 * 1024, feat_block_bytes=64 * 1024) as graph:
        for step in range(steps):
            ids = synth.hyperbatch_targets(pool, minibatches, targets, 7, step).to(device)
            graph.prepare(ids, [10, 5], 11, step * minibatches)
            hb = graph.fetch_all()
            H, capacity, _ = hb.feats.shape
            x = ops.mx4_dequantize(hb.feats.view(H * capacity, -1), dim, torch.float16)
            t, index = teacher.top_logits(graph, x.view(H, capacity, dim), targets, top)
            # the target nodes are the first of each minibatch's nodes
            rows = hb.feats[:, :targets].reshape(H * targets, -1)
            loss = student.step(rows, ids.view(-1), t, index, temperature, lr)
            losses.append(loss.mean())
            if report and step % report == 0:
                print(f"step {step}: loss {float(losses[-1]):.4f}")
        ops.check()
    return [float(v) for v in losses]


if __name__ == "__main__":
    p = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawTextHelpFormatter)
    p.add_argument("--steps", type=int, default=50)
    p.add_argument("--nodes", type=int, default=20_000)
    a = p.parse_args()
    losses = train(steps=a.steps, nodes=a.nodes, report=10)
    print(f"loss {losses[0]:.4f} -> {losses[-1]:.4f}")
