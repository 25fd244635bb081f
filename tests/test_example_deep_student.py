"""The example that trains a residual student in 8 bits, run as it stands, and the gradients
of its step against those of plain PyTorch in 64 bits."""
import importlib.util
import os

import pytest
import torch

from ops_support import gen
from paper_2601_01473_gb300 import ops

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def _example():
    spec = importlib.util.spec_from_file_location(
        "train_deep_student", os.path.join(ROOT, "examples", "train_deep_student.py"))
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


def test_the_example_imports():
    assert callable(_example().train)


@pytest.mark.gpu
def test_the_example_runs(cuda_device):
    losses = _example().train(steps=5, nodes=5000, targets=64)
    assert all(0 <= v < 100 for v in losses)


def _as(value, now):
    """`now`, with the gradient of `value`."""
    return value + (now - value).detach()


def _norm(v, w):
    return v * (v.square().mean(1, keepdim=True) + 1e-5).rsqrt() * w


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("rows", [5, 333])
def test_the_gradients_are_those_of_plain_pytorch(cuda_device, dtype, rows):
    m = _example()
    dim, hidden, inner, classes, blocks = 60, 72, 40, 19, 2
    s = m.DeepStudent(dim, hidden, inner, classes, blocks, cuda_device, dtype=dtype)
    g = gen(1)
    x8 = ops.int8_quantize(torch.randn(rows, dim, generator=g).to(cuda_device))
    logits, kept = s.forward(x8)
    grad = torch.randn(rows, classes, generator=g).to(cuda_device) / rows
    got = s.backward(grad, kept)

    leaf = lambda t: t.double().requires_grad_()  # noqa: E731
    # layers at the values of their 8-bit forms, whose gradient is the weights'
    value = lambda t8, n: ops.int8_dequantize(t8, n).double()  # noqa: E731
    leaves = {"head": leaf(s.head)}
    for name, layers in (("up", s.up), ("down", s.down), ("first", [s.first])):
        for i, layer in enumerate(layers):
            key = name if name == "first" else f"{name}{i}"
            leaves[key] = leaf(value(layer.rows8, layer.dim))
            leaves[key + "bias"] = leaf(layer.bias)
    for name in ("before", "after", "gate"):
        for i, v in enumerate(getattr(s, name)):
            leaves[f"{name}{i}"] = leaf(v)

    def linear(name, v):
        return v @ leaves[name].t() + leaves[name + "bias"]

    # each rounding and each stored tensor at the value that the step had
    rows8, x_now, n8 = kept[0]
    x = _as(linear("first", value(rows8, dim)), x_now.double())
    n = _as(_norm(x, leaves["before0"]), value(n8, hidden))
    for i in range(blocks):
        u8, a8, out_now, x_now, n_now = kept[i + 1]
        half = u8.shape[1] // 2
        u = _as(linear(f"up{i}", n), torch.cat((value(u8[:, :half], inner),
                                                value(u8[:, half:], inner)), 1))
        a = torch.nn.functional.silu(u[:, :inner]) * u[:, inner:]
        a = _as(a, value(a8, inner))
        out = _as(linear(f"down{i}", a), out_now.double())
        x = x + leaves[f"gate{i}"] * _norm(out, leaves[f"after{i}"])
        x = _as(x, x_now.double())
        n = _norm(x, leaves[f"before{i + 1}"])
        n = _as(n, n_now.double() if i + 1 == blocks else value(n_now, hidden))
    want_logits = n @ leaves["head"].t()
    assert (logits - want_logits).abs().max() <= 200 * 2.0 ** -24 * want_logits.abs().max()
    (want_logits * grad.double()).sum().backward()
    # Some hundred fp32 roundings on the way to each gradient, relative to its largest; the
    # gradients that pass between the operators in bfloat16 are rounded to 2^-8 of themselves,
    # some ten times over from the logits to the first layer.
    unit = 1000 * 2.0 ** -24 if dtype == torch.float32 else 20 * 2.0 ** -8
    for key, v in got.items():
        pairs = [(v, leaves[key])] if isinstance(v, torch.Tensor) else \
            [(v.weight, leaves[key]), (v.bias, leaves[key + "bias"])]
        for y, ref in pairs:
            off = (y.double() - ref.grad).abs().max()
            assert off <= unit * ref.grad.abs().max(), (key, float(off / ref.grad.abs().max()))
    ops.check()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_a_step_changes_every_parameter_by_its_gradient(cuda_device, dtype):
    m = _example()
    rows, lr = 70, 0.25
    new = lambda: m.DeepStudent(60, 72, 40, 19, 2, cuda_device, dtype=dtype)  # noqa: E731
    s, before = new(), new()
    g = gen(2)
    x8 = ops.int8_quantize(torch.randn(rows, 60, generator=g).to(cuda_device))
    teacher = torch.randn(rows, 4, generator=g).to(cuda_device)
    index = torch.randint(0, 19, (rows, 4), generator=g).to(cuda_device)
    loss = s.step(x8, teacher, index, 2.0, lr)
    logits, kept = before.forward(x8)
    want_loss, grad = ops.distill_loss_grad(logits, teacher, index, 1.0 / rows, 2.0)
    assert torch.equal(loss, want_loss)
    d = before.backward(grad, kept)

    def changed(new_value, old, by):
        assert by.abs().max() > 0
        # a product and a sum, each rounded
        off = (new_value.double() - (old.double() - lr * by.double())).abs()
        assert (off <= 2.0 ** -23 * (old.abs() + lr * by.abs())).all()

    changed(s.head, before.head, d["head"])
    layers = [("first", s.first, before.first)]
    for name in ("up", "down"):
        layers += [(f"{name}{i}", *pair) for i, pair in
                   enumerate(zip(getattr(s, name), getattr(before, name)))]
    for key, layer, old in layers:
        changed(layer.weight, old.weight, d[key].weight)
        changed(layer.bias, old.bias, d[key].bias)
        assert torch.equal(layer.rows8, ops.int8_quantize(layer.weight))
    for name in ("before", "after", "gate"):
        for i, (v, old) in enumerate(zip(getattr(s, name), getattr(before, name))):
            changed(v, old, d[f"{name}{i}"])
    ops.check()
