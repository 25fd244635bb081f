"""Trains a deeper student on prepared hyperbatches: a residual network over the target
nodes' 8-bit features whose layers run in 8 bits and keep their activations in 8 bits for
the backward pass, through the framework's public entry points alone.

The graph's features are kept as 8-bit rows, which the graph gathers unchanged.  A block is

  next  = norm(x)                        residual_norm, straight to 8-bit rows
  u     = next @ W1.T + b1               int8_linear
  a     = silu(u[:, :h]) * u[:, h:]      activation, u kept in 8 bits, a to 8-bit rows
  out   = a @ W2.T + b2                  int8_linear
  x     = x + gate * norm(out)           residual_norm, with the next block's norm

and its backward pass takes the 8-bit rows: residual_norm_grad, int8_linear_grad_weight and
int8_linear_grad_input, activation_grad.  Weights are fp32 and rounded to 8 bits after
every update (roundings have the identity's gradient).  The teacher and the loss are those
of train_student.py.

    python examples/train_deep_student.py [--steps 50] [--nodes 20000] [--blocks 2]
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
sys.path.insert(0, os.path.dirname(os.path.abspath(__file__)))

from agnes_inputs import synth  # noqa: E402
from paper_2601_01473_gb300 import Graph, ops  # noqa: E402
from train_student import Teacher  # noqa: E402


class Layer:
    """fp32 weights with their 8-bit form, and a bias."""

    def __init__(self, width, dim, g, device, scale=1.0):
        self.dim = dim
        self.weight = torch.randn((width, dim), generator=g, device=device) * (scale * dim ** -0.5)
        self.bias = torch.zeros(width, device=device)
        self.rows8 = ops.int8_quantize(self.weight)

    def __call__(self, x8, dtype):
        return ops.int8_linear(x8, self.rows8, self.dim, self.bias, out_dtype=dtype)

    def backward(self, grad, x8, input_too=True):
        """(gradients to the weights and the bias, to the input)"""
        d = ops.int8_linear_grad_weight(grad, x8, self.dim)
        return d, ops.int8_linear_grad_input(grad, self.rows8, self.dim) if input_too else None

    def update(self, d, lr):
        self.weight.add_(d.weight, alpha=-lr)
        self.bias.add_(d.bias, alpha=-lr)
        ops.int8_quantize(self.weight, out=self.rows8)


class DeepStudent:
    def __init__(self, dim, hidden, inner, classes, blocks, device, seed=3,
                 dtype=torch.bfloat16):
        g = torch.Generator(device=device).manual_seed(seed)
        ones = lambda: torch.ones(hidden, device=device)  # noqa: E731
        self.dtype, self.blocks = dtype, blocks
        self.inner = inner
        self.first = Layer(hidden, dim, g, device)
        self.up = [Layer(2 * inner, hidden, g, device) for _ in range(blocks)]
        self.down = [Layer(hidden, inner, g, device) for _ in range(blocks)]
        self.before = [ones() for _ in range(blocks + 1)]  # each block's, then the head's
        self.after = [ones() for _ in range(blocks)]
        self.gate = [ones() * 0.5 for _ in range(blocks)]
        self.head = torch.randn((classes, hidden), generator=g, device=device) * hidden ** -0.5

    def forward(self, rows):
        """The logits of 8-bit feature rows, and what the backward pass takes."""
        x = self.first(rows, torch.float32)  # the residual stays in fp32
        n8 = ops.residual_norm(x, before=self.before[0], rows8=True).next
        kept = [(rows, x, n8)]
        for i in range(self.blocks):
            u = self.up[i](n8, self.dtype)
            a8, u8 = ops.activation(u, "silu", gated=True, rows8=True)
            out = self.down[i](a8, self.dtype)
            last = i + 1 == self.blocks
            x, n = ops.residual_norm(x, out, gate=self.gate[i], after=self.after[i],
                                     before=self.before[i + 1], rows8=not last)
            kept.append((u8, a8, out, x, n))
            n8 = n
        return n.float() @ self.head.t(), kept

    def backward(self, grad, kept):
        """The gradients to every parameter, from the one to the logits."""
        n = kept[-1][4]
        d = {"head": grad.t() @ n.float()}
        d_next, d_sum = (grad @ self.head).to(self.dtype), None
        for i in reversed(range(self.blocks)):
            u8, a8, out, x, _ = kept[i + 1]
            n8 = kept[i][-1]
            r = ops.residual_norm_grad(d_next, d_sum, x, out, gate=self.gate[i],
                                       after=self.after[i], before=self.before[i + 1])
            d[f"gate{i}"], d[f"after{i}"], d[f"before{i + 1}"] = r.gate, r.after, r.before
            d_sum = r.x
            d[f"down{i}"], d_a = self.down[i].backward(r.branch, a8)
            d_u = ops.activation_grad(d_a, u8, "silu", gated=True)
            d[f"up{i}"], d_next = self.up[i].backward(d_u, n8)
        rows, x, _ = kept[0]
        r = ops.residual_norm_grad(d_next, d_sum, x, before=self.before[0])
        d["before0"] = r.before
        d["first"], _ = self.first.backward(r.x, rows, input_too=False)
        return d

    def step(self, rows, teacher, index, temperature, lr):
        """One step on the 8-bit rows of the target nodes; returns their losses."""
        logits, kept = self.forward(rows)
        loss, grad = ops.distill_loss_grad(logits, teacher, index, 1.0 / rows.shape[0], temperature,
                                           out=logits)
        d = self.backward(grad, kept)
        self.head.add_(d["head"], alpha=-lr)
        self.first.update(d["first"], lr)
        for i in range(self.blocks):
            self.up[i].update(d[f"up{i}"], lr)
            self.down[i].update(d[f"down{i}"], lr)
            self.gate[i].add_(d[f"gate{i}"], alpha=-lr)
            self.after[i].add_(d[f"after{i}"], alpha=-lr)
        for i in range(self.blocks + 1):
            self.before[i].add_(d[f"before{i}"], alpha=-lr)
        return loss


def train(steps=50, nodes=20_000, dim=128, hidden=128, inner=192, classes=172, top=8, blocks=2,
          minibatches=4, targets=256, temperature=2.0, lr=0.1, device="cuda:0", report=None):
    """Returns the mean loss of each step."""
    device = torch.device(device)
    offsets, indices = synth.rmat_csr(nodes, 10, 0.57, 0.19, 0.19, seed=5,
                                      offsets_dtype=torch.int64)
    features = synth.normal_features(nodes, dim, torch.float16, seed=6).to(device)
    packed = ops.int8_quantize(features)
    student = DeepStudent(dim, hidden, inner, classes, blocks, device)
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
            x = ops.int8_dequantize(hb.feats.view(H * capacity, -1), dim, torch.float16)
            t, index = teacher.top_logits(graph, x.view(H, capacity, dim), targets, top)
            # the target nodes are the first of each minibatch's nodes
            rows = hb.feats[:, :targets].reshape(H * targets, -1)
            loss = student.step(rows, t, index, temperature, lr)
            losses.append(loss.mean())
            if report and step % report == 0:
                print(f"step {step}: loss {float(losses[-1]):.4f}")
        ops.check()
    return [float(v) for v in losses]


if __name__ == "__main__":
    p = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawTextHelpFormatter)
    p.add_argument("--steps", type=int, default=50)
    p.add_argument("--nodes", type=int, default=20_000)
    p.add_argument("--blocks", type=int, default=2)
    a = p.parse_args()
    losses = train(steps=a.steps, nodes=a.nodes, blocks=a.blocks, report=10)
    print(f"loss {losses[0]:.4f} -> {losses[-1]:.4f}")
