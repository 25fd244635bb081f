"""Nonlinearities that keep their input in 8 bits (include/agnes_ops.h) against their
formulas in 64 bits."""
import math

import pytest
import torch

from ops_support import FLOATS, U32, assert_within, gen, rounding
from paper_2601_01473_gb300 import ops
from test_ops_int8 import reference_rows, reference_values, row_bytes, values

KINDS = ["relu", "silu", "gelu"]
LEAST = 1e-36  # a reciprocal of more than 2^126 is zero


def formula(v, f):
    """(f(v), f'(v)) in 64 bits, and how far fp32 may be off either."""
    a = v.abs()
    if f == "relu":
        return v.clamp(min=0), (v > 0).double(), torch.zeros_like(v), torch.zeros_like(v)
    if f == "silu":
        # exp to 2 units, 1 + e, a reciprocal to 2 units: p to 9 halves; then two products and a
        # sum for the slope p (1 + v (1 - p)), whose 1 - p carries p's own error
        p = torch.sigmoid(v)
        slope = p * (1 + v * (1 - p))
        return v * p, slope, 11 * U32 * a * p + LEAST * (1 + a), \
            20 * U32 * p * (1 + a) + LEAST * (1 + a)
    # the distribution function to 5 units; exp(-v^2 / 2) to 2 units and v^2 / 2 rounded twice,
    # which counts v^2 units
    p = 0.5 * torch.special.erfc(-v / math.sqrt(2))
    phi = torch.exp(-v * v / 2) / math.sqrt(2 * math.pi)
    return v * p, p + v * phi, 12 * U32 * a * p + LEAST, \
        U32 * (12 * p + a * phi * (v * v + 12)) + LEAST


def check(got, ref, off, dtype):
    assert got.dtype == dtype
    assert_within(got, ref, off + U32 * ref.abs() + 1.01 * rounding(ref, dtype))


def _case(dev, rows, dim, dtype, f, gated, seed=0):
    n = 2 * dim if gated else dim
    x = (values(rows, n, seed) / 4).to(dtype)
    d = torch.randn(rows, dim, generator=gen(seed + 1)).to(dtype)
    y, kept = ops.activation(x.to(dev), f, gated=gated)
    v = x.double()
    value, _, off, _ = formula(v[:, :dim], f)
    if gated:
        value, off = value * v[:, dim:], off * v[:, dim:].abs()
    check(y, value, off, dtype)
    # what is kept: the rows of each half
    rb = row_bytes(dim)
    halves = [reference_rows(x[:, i:i + dim]) for i in range(0, n, dim)]
    assert torch.equal(kept.cpu(), torch.cat(halves, 1))
    assert kept.shape == (rows, rb * len(halves))
    k = [reference_values(h, dim) for h in halves]
    value, slope, off, slope_off = formula(k[0], f)
    got = ops.activation_grad(d.to(dev), kept, f, gated=gated)
    dd = d.double()
    if gated:
        ref = torch.cat((dd * slope * k[1], dd * value), 1)
        bound = torch.cat((dd.abs() * slope_off * k[1].abs(), dd.abs() * off), 1)
    else:
        ref, bound = dd * slope, dd.abs() * slope_off
    check(got, ref, bound + 3 * U32 * ref.abs(), dtype)
    return x, d, kept, y


# ---- without a GPU --------------------------------------------------------------------

def test_refusals():
    from paper_2601_01473_gb300 import build
    build.build()
    x = torch.zeros(2, 8)
    with pytest.raises(ValueError, match="CUDA device"):
        ops.activation(x)
    with pytest.raises(TypeError, match="2-D"):
        ops.activation(torch.zeros(8))
    L = ops.lib()
    forward = [None, 0, 8, 4, 8, 1, 0, None, 0, 8, None, 0, None]
    assert L.agnes_activation(*forward) == 1 and b"NULL" in L.agnes_last_error(None)
    # a stride, a size, a nonlinearity, gated (rows of 16 then), a type, out's stride, its type
    for at, value, status in ((2, 7, 1), (3, -1, 1), (4, 0, 1), (4, (1 << 17) + 1, 2), (5, 3, 1),
                              (5, -1, 1), (6, 2, 1), (6, 1, 1), (1, 3, 1), (9, 7, 1), (8, 1, 1),
                              (8, 3, 1)):
        bad = list(forward)
        bad[at] = value
        assert L.agnes_activation(*bad) == status, (at, value)
    forward[3] = 0
    assert L.agnes_activation(*forward) == 0
    back = [None, 0, 8, None, 16, 4, 8, 1, 0, None, 0, 8, None]
    assert L.agnes_activation_grad(*back) == 1
    for at, value in ((1, 4), (2, 7), (4, 8), (4, 24), (5, -1), (6, 0), (7, 9), (8, 5), (8, 1),
                      (10, 3), (11, 7)):
        bad = list(back)
        bad[at] = value
        assert L.agnes_activation_grad(*bad) == 1, (at, value)


@pytest.mark.parametrize("f", KINDS)
def test_the_formulas_slopes_are_those_of_differences(f):
    v = torch.linspace(-6, 6, 1001, dtype=torch.float64) + 0.0037
    h = 1e-6
    slope = (formula(v + h, f)[0] - formula(v - h, f)[0]) / (2 * h)
    assert (slope - formula(v, f)[1]).abs().max() < 1e-8


# ---- on a GPU ----------------------------------------------------------------------------

@pytest.mark.gpu
@pytest.mark.parametrize("dtype", FLOATS)
@pytest.mark.parametrize("f", KINDS)
@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("rows,dim", [(1, 1), (3, 7), (33, 128), (9, 301), (40, 64), (2, 1000),
                                      (5, 4096), (2, 8192), (3, 8200), (2, 9001)])
def test_forward_and_backward(cuda_device, dtype, f, gated, rows, dim):
    _case(cuda_device, rows, dim, dtype, f, gated)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", FLOATS)
@pytest.mark.parametrize("f", KINDS)
def test_over_the_whole_range(cuda_device, dtype, f):
    v = torch.cat((torch.linspace(-110, 110, 4001), torch.tensor([0.0, -0.0, 1e-30, -1e-30])))
    x = v.to(dtype)[:, None]  # a row each: kept to 2^-8 or so of itself
    y, kept = ops.activation(x.to(cuda_device), f)
    value, _, off, _ = formula(x.double(), f)
    check(y, value, off, dtype)
    k = ops.int8_dequantize(kept, 1).double().cpu()
    got = ops.activation_grad(torch.ones(len(v), 1, device=cuda_device), kept, f)
    _, slope, _, off = formula(k, f)
    check(got, slope, off, torch.float32)


@pytest.mark.gpu
@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("dtype", FLOATS)
def test_serving_and_8bit_outputs(cuda_device, dtype, gated):
    for rows, dim in ((1, 301), (50, 256), (3, 8200)):
        x = (values(rows, dim * (1 + gated), 3) / 4).to(dtype).to(cuda_device)
        for f in KINDS:
            y, kept = ops.activation(x, f, gated=gated)
            alone, none = ops.activation(x, f, gated=gated, keep=False)
            assert none is None and torch.equal(alone, y)
            y8, kept8 = ops.activation(x, f, gated=gated, rows8=True)
            assert torch.equal(kept8, kept)
            alone8, _ = ops.activation(x, f, gated=gated, rows8=True, keep=False)
            assert torch.equal(alone8, y8)
            if dtype == torch.float32:  # y has not been rounded
                assert torch.equal(y8, ops.int8_quantize(y))
            back = ops.int8_dequantize(y8, dim).double().cpu()
            want = y.double().cpu()
            step = want.abs().amax(1, keepdim=True) / 127 * 1.01
            unit = 0 if dtype == torch.float32 else rounding(want, dtype)
            assert ((back - want).abs() <= 0.501 * step + unit).all()


@pytest.mark.gpu
def test_strides_and_outputs(cuda_device):
    rows, dim = 30, 104
    x, d, kept, y = _case(cuda_device, rows, dim, torch.float16, "silu", True)
    want = ops.activation_grad(d.to(cuda_device), kept, "silu", gated=True)
    for first in (0, 1, 8):
        wide = torch.full((rows + 2, 2 * dim + 24), math.nan, dtype=torch.float16,
                          device=cuda_device)
        wide[1:-1, first:first + 2 * dim] = x.to(cuda_device)
        got, got_kept = ops.activation(wide[1:-1, first:first + 2 * dim], "silu", gated=True)
        assert torch.equal(got, y) and torch.equal(got_kept, kept)
        wide = torch.full((rows + 2, dim + 24), math.nan, dtype=torch.float16, device=cuda_device)
        wide[1:-1, first:first + dim] = d.to(cuda_device)
        kept_wide = torch.full((rows, kept.shape[1] + 32), 9, dtype=torch.uint8,
                               device=cuda_device)
        kept_wide[:, 16:-16] = kept
        out = torch.full((rows, 2 * dim + 16), 7.0, dtype=torch.float16, device=cuda_device)
        ops.activation_grad(wide[1:-1, first:first + dim], kept_wide[:, 16:-16], "silu", gated=True,
                            out=out[:, first:first + 2 * dim])
        assert torch.equal(out[:, first:first + 2 * dim], want)
        assert (out[:, :first] == 7).all() and (out[:, first + 2 * dim:] == 7).all()
    for out in FLOATS:
        got = ops.activation_grad(d.to(cuda_device), kept, "silu", gated=True, out_dtype=out)
        assert got.dtype == out
    empty, none = ops.activation(x[:0].to(cuda_device))
    assert empty.shape == (0, 2 * dim) and none.shape == (0, row_bytes(2 * dim))
    assert ops.activation_grad(d[:0].to(cuda_device), kept[:0], gated=True).shape == (0, 2 * dim)
    with pytest.raises(ValueError, match="halves"):
        ops.activation(x[:, :7].to(cuda_device), gated=True)
    with pytest.raises(ValueError, match="relu"):
        ops.activation(x.to(cuda_device), "tanh")
    with pytest.raises(ValueError, match="rows"):
        ops.activation_grad(d[:4].to(cuda_device), kept, gated=True)
    with pytest.raises(ValueError, match="bytes"):
        ops.activation_grad(d.to(cuda_device), kept)


@pytest.mark.gpu
@pytest.mark.parametrize("f", KINDS)
def test_a_row_with_a_nan_or_infinity(cuda_device, f):
    x = values(6, 64, 1)
    x[1, 5], x[2, 7], x[3, 9] = math.nan, math.inf, -math.inf
    x[4] = 0
    y, kept = ops.activation(x.to(cuda_device), f)
    y = y.cpu()
    assert y[1, 5].isnan() and y[2, 7] == math.inf
    fine = torch.isfinite(x)
    assert y[fine].isfinite().all() and (y[4] == 0).all()
    g = ops.activation_grad(torch.ones(6, 64, device=cuda_device), kept, f).cpu()
    assert g[1:4].isnan().all() and g[0].isfinite().all() and g[4:].isfinite().all()
    y8, _ = ops.activation(x.to(cuda_device), f, rows8=True)
    back = ops.int8_dequantize(y8, 64).cpu()
    assert back[1:3].isnan().all() and back[0].isfinite().all() and (back[4] == 0).all()


@pytest.mark.gpu
def test_gradients_are_those_of_differences(cuda_device):
    """Of the formula over a step around the kept values."""
    x = values(8, 96, 2)
    for f in ("silu", "gelu"):
        _, kept = ops.activation(x.to(cuda_device), f)
        k = ops.int8_dequantize(kept, 96).double().cpu()
        h = 1e-5
        want = (formula(k + h, f)[0] - formula(k - h, f)[0]) / (2 * h)
        got = ops.activation_grad(torch.ones(8, 96, device=cuda_device), kept, f).double().cpu()
        # the third derivatives are below 1, so the difference is within h^2
        assert ((got - want).abs() <= 1e-9 + formula(k, f)[3] + 4 * U32).all()


@pytest.mark.gpu
def test_streams_and_graphs(cuda_device):
    x = values(500, 512, 3).to(cuda_device)
    d = torch.randn(500, 256, generator=gen(1)).to(cuda_device)

    def run(**stream):
        y, kept = ops.activation(x, "gelu", gated=True, **stream)
        return y, kept, ops.activation_grad(d, kept, "gelu", gated=True, **stream)
    ref = run()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = run(stream=side)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, ref))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = run()
    graph.replay()
    assert all(torch.equal(a, b) for a, b in zip(got, ref))


@pytest.mark.gpu
def test_offsets_past_32_bits(cuda_device):
    rows, dim = 2_200_000, 1000  # 2.2e9 values
    part = (values(3, dim, 5) / 4).half()
    at = [0, 2_147_484, rows - 1]
    x = torch.zeros(rows, dim, dtype=torch.float16, device=cuda_device)
    x[at] = part.to(cuda_device)
    y, kept = ops.activation(x, "gelu")
    want, want_kept = ops.activation(part.to(cuda_device), "gelu")
    assert torch.equal(y[at], want) and torch.equal(kept[at], want_kept)
    assert int((y != 0).any(1).sum()) == 3
    g = ops.activation_grad(x, kept, "gelu")
    assert torch.equal(g[at], ops.activation_grad(part.to(cuda_device), want_kept, "gelu"))
    assert int((g != 0).any(1).sum()) == 3


@pytest.mark.gpu
@pytest.mark.parametrize("dim", [64, 61])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("f", KINDS)
def test_gradient_at_the_largest_numbers(cuda_device, dtype, f, dim):
    x = values(4, 2 * dim, 1).to(dtype)
    x[1, 5], x[2, 7] = torch.finfo(dtype).max, torch.finfo(dtype).min
    x[1, dim + 5], x[3, dim + 9] = torch.finfo(dtype).max, torch.finfo(dtype).min
    d = values(4, dim, 2).to(dtype)
    d[1, 5], d[2, 7], d[3, 9] = 0, 2.0 ** -30, 0
    halves = [reference_rows(x[:, :dim]), reference_rows(x[:, dim:])]
    k, u = (reference_values(h, dim) for h in halves)
    value, slope, off, slope_off = formula(k, f)
    dd = d.double()
    kept = torch.cat(halves, 1).to(cuda_device)
    got = ops.activation_grad(d.to(cuda_device), halves[0].to(cuda_device), f)
    assert got.isfinite().all()
    check(got, dd * slope, dd.abs() * slope_off + 3 * U32 * (dd * slope).abs(), dtype)
    got = ops.activation_grad(d.to(cuda_device), kept, f, gated=True)
    ref = torch.cat((dd * slope * u, dd * value), 1)
    bound = torch.cat((dd.abs() * slope_off * u.abs(), dd.abs() * off), 1)
    assert got.isfinite().all()
    check(got, ref, bound + 3 * U32 * ref.abs(), dtype)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_silu_far_below_zero(cuda_device, dtype):
    """Where exp(-v) leaves fp32's range the value, v exp(v), is still in it."""
    v = torch.linspace(-100, -80, 2001).to(dtype)[:, None]
    y, kept = ops.activation(v.to(cuda_device), "silu")
    # exp(v) to 2 units and half of fp32's smallest number, 1 + e, a reciprocal to 2 units, two
    # products; 16-bit types take the exponential whose error grows by a unit for 0.86 of v
    units = 12 * U32 if dtype == torch.float32 else 2 * (8 + 1.2 * 100) * U32
    least = 2.0 ** -149

    def check_at(got, v, ref):
        assert got.dtype == dtype
        assert_within(got, ref, units * ref.abs() + (2 + v.abs()) * least
                      + 1.01 * rounding(ref, dtype))
    x = v.double()
    check_at(y, x, x * torch.sigmoid(x))
    assert (y[v > -95] != 0).all()
    k = reference_values(reference_rows(v), 1)
    got = ops.activation_grad(torch.ones(len(v), 1, dtype=dtype, device=cuda_device), kept, "silu")
    p = torch.sigmoid(k)
    check_at(got, k, p * (1 + k * torch.sigmoid(-k)))


@pytest.mark.gpu
def test_silu_slope_far_above_zero(cuda_device):
    """1 + v exp(-v): what is left of 1 - p is not a difference of numbers next to one."""
    v = torch.linspace(4, 60, 3001)[:, None]
    _, kept = ops.activation(v.to(cuda_device), "silu")
    k = reference_values(reference_rows(v), 1)
    got = ops.activation_grad(torch.ones(len(v), 1, device=cuda_device), kept, "silu")
    p, q = torch.sigmoid(k), torch.sigmoid(-k)
    # p and q to 4 units each, v q <= 0.08, a product, a sum, a product, a rounding
    assert_within(got, p * (1 + k * q), U32 * (2 * 4 + 2 * 5 * k * q + 4))
