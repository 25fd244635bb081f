"""The example that trains a student with the operators, run as it stands, and its
step against the same step in plain PyTorch."""
import importlib.util
import os

import pytest
import torch

from ops_support import gen
from paper_2601_01473_gb300 import ops

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def _example():
    spec = importlib.util.spec_from_file_location(
        "train_student", os.path.join(ROOT, "examples", "train_student.py"))
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


def test_the_example_imports():
    assert callable(_example().train)


@pytest.mark.gpu
def test_the_student_learns(cuda_device):
    losses = _example().train(steps=30, nodes=5000, targets=64)
    assert all(0 <= v < 100 for v in losses)
    # seeded: the loss falls by more than a step's noise
    assert sum(losses[-5:]) < 0.8 * sum(losses[:5])


@pytest.mark.gpu
def test_a_step_is_the_step_of_plain_pytorch(cuda_device):
    m = _example()
    s = m.Student(500, 96, 64, 40, cuda_device)
    g = gen(1)
    rows = ops.mx4_quantize(torch.randn(120, 96, generator=g).to(cuda_device))
    ids = torch.randint(-1, 500, (120,), generator=g).to(cuda_device)
    t = torch.randn(120, 6, generator=g).to(cuda_device)
    index = torch.rand(120, 40, generator=g).argsort(1)[:, :6].to(cuda_device)
    T, lr = 2.0, 0.5
    table, head = (v.double().clone().requires_grad_() for v in (s.table, s.head))
    x = ops.mx4_dequantize(rows, 96).double()
    w = ops.mx4_dequantize(s.projection, 96).double()
    emb = torch.where((ids >= 0)[:, None], table[ids.clamp(min=0)], 0.0) * s.scale
    log_q = torch.log_softmax((x @ w.t() + emb) @ head.t() / T, 1)
    log_p = torch.log_softmax(t.double() / T, 1)
    ref = T * T * (log_p.exp() * (log_p - log_q.gather(1, index))).sum(1)
    ref.mean().backward()
    want_table, want_head = table - lr * table.grad, head - lr * head.grad
    loss = s.step(rows, ids, t, index, T, lr)
    # fp32 products of up to 96 and 64 terms each way: a few hundred roundings
    for got, want in ((loss, ref), (s.table, want_table), (s.head, want_head)):
        off = (got.double() - want).abs().max()
        assert off <= 500 * 2.0 ** -24 * want.abs().max(), float(off)
