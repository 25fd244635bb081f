"""8-bit rows, their product and its gradients (include/agnes_ops.h) against the
format's definition, in 64 bits."""
import math

import pytest
import torch

from ops_support import FLOATS, U32, assert_within, gen, rounding
from paper_2601_01473_gb300 import AgnesError, Graph, ops


def row_bytes(dim):
    return -(-(dim + 4) // 16) * 16


def _f32(x):
    return x.to(torch.float32).double()


def reference_rows(x):
    """The bytes of x's 8-bit rows: the scale's bits are counted up, the quotients are taken
    in 64 bits and rounded to 32."""
    rows, dim = x.shape
    x = x.double()
    top = x.abs().amax(1)
    fine = torch.isfinite(top)
    some = fine & (top >= 2.0 ** -100)
    bits = _f32(torch.where(some, top, 1.0) / 127).float().view(torch.int32)
    scale = torch.where(bits % 65536 == 0, bits, (bits // 65536 + 1) * 65536).view(torch.float32)
    q = torch.round(_f32(x * _f32(1 / scale.double())[:, None]))
    q = torch.where(some[:, None], q, 0.0)
    scale = torch.where(some, scale, torch.where(fine, 0.0, math.nan))
    out = torch.zeros(rows, row_bytes(dim), dtype=torch.uint8)
    out[:, :dim] = q.to(torch.int8).view(torch.uint8)
    # the bytes of the NaN are the kernel's choice
    out[:, -4:] = torch.where(scale.isnan(), 0x7fffffff, scale.view(torch.int32))[:, None] \
        .contiguous().view(torch.uint8)
    return out


def reference_values(packed, dim):
    scale = packed[:, -4:].contiguous().view(torch.float32).double()
    return packed[:, :dim].contiguous().view(torch.int8).double() * scale


def values(rows, dim, seed):
    g = gen(seed)
    x = torch.randn(rows, dim, generator=g) * torch.exp2(3 * torch.randn(rows, 1, generator=g))
    return torch.where(torch.rand(rows, dim, generator=g) < 0.02, 20 * x, x)


# ---- without a GPU --------------------------------------------------------------------

def test_row_bytes_and_refusals():
    from paper_2601_01473_gb300 import build
    build.build()
    for dim in (1, 11, 12, 13, 16, 128, 301, 4096, 1 << 17):
        assert ops.int8_row_bytes(dim) == row_bytes(dim)
    assert ops.int8_row_bytes(128) == 144 and ops.int8_row_bytes(12) == 16
    with pytest.raises(AgnesError, match="EINVAL"):
        ops.int8_row_bytes(0)
    with pytest.raises(AgnesError, match="ERANGE"):
        ops.int8_row_bytes((1 << 17) + 1)
    with pytest.raises(ValueError, match="CUDA device"):
        ops.int8_quantize(torch.zeros(2, 8))
    rows8 = torch.zeros(2, 144, dtype=torch.uint8)
    with pytest.raises(ValueError, match="CUDA device"):
        ops.int8_linear(rows8, rows8, 128)
    for call in (lambda: ops.int8_linear(rows8, rows8, 160), lambda: ops.int8_dequantize(rows8, 99),
                 lambda: ops.int8_linear_grad_input(torch.zeros(3, 2), rows8, 64)):
        with pytest.raises(ValueError, match="bytes|CUDA"):
            call()
    with pytest.raises(TypeError, match="2-D"):
        ops.int8_quantize(torch.zeros(2, 8, dtype=torch.int32))
    with pytest.raises(TypeError, match="8-bit"):
        ops.int8_linear(rows8.to(torch.int32), rows8, 128)


def test_the_c_entries_refuse():
    L = ops.lib()
    linear = [None, 144, 4, None, 144, 5, 128, None, None, 0, 5, None, 0, None, None]
    assert L.agnes_int8_linear(*linear) == 1 and b"NULL" in L.agnes_last_error(None)
    for at, value, status in ((1, 128, 1), (1, 152, 1), (2, -1, 1), (4, 72, 1), (5, -1, 1),
                              (6, 0, 1), (9, 3, 1), (10, 4, 1), (2, 1 << 31, 2),
                              (6, 1 << 18, 2)):
        bad = list(linear)
        bad[at] = value
        assert L.agnes_int8_linear(*bad) == status, (at, value)
    linear[2] = 0
    assert L.agnes_int8_linear(*linear) == 0
    weight = [None, 0, 5, 4, 5, None, 144, 128, None, 0, 128, None, None, 0, None, None]
    assert L.agnes_int8_linear_grad_weight(*weight) == 1
    for at, value, status in ((1, 7, 1), (2, 4, 1), (3, -1, 1), (6, 100, 1), (9, 3, 1),
                              (10, 127, 1), (3, 1 << 31, 2), (7, 1 << 18, 2)):
        bad = list(weight)
        bad[at] = value
        assert L.agnes_int8_linear_grad_weight(*bad) == status, (at, value)
    given = [None, 0, 5, 4, 5, None, 144, 128, None, 0, 128, None, 0, None, None]
    assert L.agnes_int8_linear_grad_input(*given) == 1
    for at, value, status in ((1, 7, 1), (2, 4, 1), (3, -1, 1), (6, 100, 1), (9, 3, 1),
                              (10, 127, 1), (4, 1 << 31, 2), (7, 1 << 18, 2)):
        bad = list(given)
        bad[at] = value
        assert L.agnes_int8_linear_grad_input(*bad) == status, (at, value)
    quantize = [None, 0, 8, 4, 8, None, 16, None]
    assert L.agnes_int8_quantize(*quantize) == 1
    for at, value in ((1, 3), (2, 7), (3, -1), (4, 0), (6, 8), (6, 24)):
        bad = list(quantize)
        bad[at] = value
        assert L.agnes_int8_quantize(*bad) == 1, (at, value)


def test_the_reference_rounds_as_the_format_says():
    # a scale of 1: whole numbers, ties to even
    x = torch.tensor([[127.0, -127.0, 0.5, 1.5, 2.5, -0.5, -1.5, 0.49, 0.0]])
    packed = reference_rows(x)
    assert reference_values(packed, 9).tolist() == [[127, -127, 0, 2, 2, 0, -2, 0, 0]]
    # rounded up to eight significant bits, and never more than 127
    x = values(50, 40, 1)
    packed = reference_rows(x)
    scale = packed[:, -4:].contiguous().view(torch.float32)[:, 0].double()
    least = x.double().abs().amax(1) / 127
    assert (scale >= least * (1 - 2.0 ** -24)).all() and (scale <= least * (1 + 2.0 ** -7)).all()
    assert int(packed[:, :40].contiguous().view(torch.int8).abs().max()) <= 127
    off = (reference_values(packed, 40) - x.double()).abs()
    assert (off <= scale[:, None] * (0.5 + 1e-4)).all()


# ---- rounding --------------------------------------------------------------------------

@pytest.mark.gpu
@pytest.mark.parametrize("dtype", FLOATS)
@pytest.mark.parametrize("rows,dim", [(1, 1), (3, 7), (5, 12), (4, 13), (7, 16), (100, 64),
                                      (33, 128), (9, 301), (17, 602), (2, 4096), (3, 8192),
                                      (2, 8193), (3, 8200), (1, 100_001), (2, 131_072),
                                      (1500, 8)])
def test_quantize_and_back(cuda_device, dtype, rows, dim):
    x = values(rows, dim, rows + dim).to(dtype)
    packed = ops.int8_quantize(x.to(cuda_device))
    ref = reference_rows(x)
    assert torch.equal(packed.cpu(), ref)
    for out in FLOATS:
        got = ops.int8_dequantize(packed, dim, out_dtype=out).cpu()
        most = torch.finfo(out).max
        assert torch.equal(got, reference_values(ref, dim).clamp(-most, most).to(out))


@pytest.mark.gpu
def test_ties_ranges_and_special_values(cuda_device):
    rows = []
    halves = torch.arange(0, 255).float() / 2
    for power in (0, -100, -106, -107, -126, -149, 100, 120):  # below 2^-100 a row is zeros
        rows += [halves * 2.0 ** power, -halves * 2.0 ** power]
    rows += [torch.full((255,), 3.4e38), torch.full((255,), 65504.0), torch.zeros(255),
             -torch.zeros(255)]
    one = torch.ones(255)
    for special in (math.inf, -math.inf, math.nan):
        r = one.clone()
        r[5] = special
        rows.append(r)
    x = torch.stack(rows)
    ref = reference_rows(x)
    for dim in (255, 248):  # single elements and vectors
        packed = ops.int8_quantize(x[:, :dim].contiguous().to(cuda_device)).cpu()
        assert torch.equal(packed, reference_rows(x[:, :dim]))
        for out in FLOATS:
            back = ops.int8_dequantize(packed.to(cuda_device), dim, out_dtype=out).cpu()
            assert back[-3:].isnan().all() and back[:-3].isfinite().all()
    assert (ref[-5:-3, :-4] == 0).all()


@pytest.mark.gpu
def test_strides(cuda_device):
    dim, n = 104, row_bytes(104)
    x = values(20, dim, 3)
    wide = torch.zeros(20, 200, device=cuda_device)
    for first in (0, 3, 4, 8):
        wide[:, first:first + dim] = x.to(cuda_device)
        out = torch.full((20, n + 48), 7, dtype=torch.uint8, device=cuda_device)
        got = ops.int8_quantize(wide[:, first:first + dim], out=out[:, 16:16 + n])
        assert torch.equal(got.cpu(), reference_rows(x))
        assert (out[:, :16] == 7).all() and (out[:, 16 + n:] == 7).all()
        back = torch.full((20, 120), 7.0, device=cuda_device)
        ops.int8_dequantize(got, dim, out=back[:, first:first + dim])
        assert torch.equal(back[:, first:first + dim].cpu(),
                           reference_values(reference_rows(x), dim).float())
        assert (back[:, :first] == 7).all() and (back[:, first + dim:] == 7).all()
    assert ops.int8_quantize(wide[:0]).shape == (0, row_bytes(200))
    assert ops.int8_dequantize(out[:0, :n], dim).shape == (0, dim)


# ---- product -----------------------------------------------------------------------------

def _exact_product(x, w, dim, dev):
    xv, wv = (reference_values(v, dim).to(dev) for v in (x, w))
    return xv @ wv.t(), xv.abs() @ wv.abs().t()


def _product_bound(ref, size, dim, out):
    # an fp32 sum of up to dim exact terms, each step off by a unit of 2^-23 of the sum of
    # magnitudes at most; two products with the scales, the bias, one rounding
    return (dim + 4) * 2 * U32 * size + 1.01 * rounding(ref, out) + 1e-30


def _product_check(dev, rows, width, dim, out, bias, seed=0):
    x = reference_rows(values(rows, dim, seed + 1))
    w = reference_rows(values(width, dim, seed + 2))
    b = torch.randn(width, generator=gen(seed)).to(dev) if bias else None
    got = ops.int8_linear(x.to(dev), w.to(dev), dim, b, out_dtype=out)
    ref, size = _exact_product(x, w, dim, dev)
    if bias:
        ref, size = ref + b.double(), size + b.double().abs()
    assert got.dtype == out
    assert_within(got, ref, _product_bound(ref, size, dim, out))
    ops.check()


@pytest.mark.gpu
@pytest.mark.parametrize("out", FLOATS)
@pytest.mark.parametrize("rows", [1, 2, 3, 5, 8])
@pytest.mark.parametrize("width,dim", [(1, 1), (7, 20), (33, 128), (257, 301), (100, 2048)])
def test_product_of_few_rows(cuda_device, out, rows, width, dim):
    _product_check(cuda_device, rows, width, dim, out, rows % 2 == 0)


@pytest.mark.gpu
@pytest.mark.parametrize("rows", [9, 16, 17, 31, 32, 33, 64])
@pytest.mark.parametrize("width,dim", [(1, 1), (70, 301), (257, 2048)])
def test_product_of_some_rows(cuda_device, rows, width, dim):
    _product_check(cuda_device, rows, width, dim, FLOATS[rows % 3], rows % 2 == 0)


SIZES = [(9, 8, 32), (128, 128, 64), (128, 256, 128), (16, 1, 1), (129, 130, 33), (200, 96, 128),
         (1000, 257, 301), (130, 300, 1024), (64, 500, 4096), (40_000, 256, 128), (300, 17, 12),
         (257, 513, 80), (5000, 64, 520), (700, 1000, 2000)]


@pytest.mark.gpu
@pytest.mark.parametrize("rows,width,dim", SIZES)
@pytest.mark.parametrize("out", FLOATS)
def test_product(cuda_device, out, rows, width, dim):
    _product_check(cuda_device, rows, width, dim, out, width % 2 == 0)


# more tiles than there are pairs of CTAs, ragged ones among them
MANY = [(20_000, 600, 520), (9000, 900, 640), (19_900, 500, 1100), (5001, 2000, 515)]


@pytest.mark.gpu
@pytest.mark.parametrize("rows,width,dim", MANY)
@pytest.mark.parametrize("out", FLOATS)
def test_product_of_many_tiles(cuda_device, out, rows, width, dim):
    _product_check(cuda_device, rows, width, dim, out, width % 4 == 0)


@pytest.mark.gpu
@pytest.mark.parametrize("rows", [3, 40])
def test_product_of_the_longest_rows(cuda_device, rows):
    _product_check(cuda_device, rows, 5, 131_072, torch.float32, True)


@pytest.mark.gpu
@pytest.mark.parametrize("rows", [2, 40])
@pytest.mark.parametrize("dim", [1040, 131_072])
def test_product_of_the_largest_whole_numbers(cuda_device, rows, dim):
    """Sums of 127^2: exact up to 2^24, and for few rows beyond."""
    x = torch.full((rows, dim), 127.0)
    w = torch.full((3, dim), 127.0)
    w[1] *= -1
    w[2, ::2] *= -1
    got = ops.int8_linear(*(ops.int8_quantize(v.to(cuda_device)) for v in (x, w)), dim)
    want = (x.double() @ w.double().t()).to(cuda_device)
    if dim == 1040 or rows == 2:
        assert torch.equal(got, want.float())
    else:
        assert_within(got, want, 2 * U32 * 127.0 ** 2 * dim * dim * torch.ones_like(want))


@pytest.mark.gpu
@pytest.mark.parametrize("rows", [3, 140])
def test_product_strides_and_what_lies_past_the_ends(cuda_device, rows):
    """Rows apart, and bytes around them, and a row's padding, that must not be looked at."""
    for dim, width in ((96, 70), (90, 72)):
        x, w = reference_rows(values(rows, dim, 1)), reference_rows(values(width, dim, 2))
        ref = ops.int8_linear(x.to(cuda_device), w.to(cuda_device), dim)
        n = row_bytes(dim)
        xw = torch.full((rows + 2, n + 48), 127, dtype=torch.uint8, device=cuda_device)
        ww = torch.full((width + 2, n + 16), 127, dtype=torch.uint8, device=cuda_device)
        xw[1:-1, 16:16 + n] = x.to(cuda_device)
        ww[1:-1, :n] = w.to(cuda_device)
        xw[1:-1, 16 + dim:16 + n - 4] = 127
        ww[1:-1, dim:n - 4] = 127
        for first in (0, 1, 4):
            out = torch.full((rows, width + 10), 7.0, device=cuda_device)
            got = ops.int8_linear(xw[1:-1, 16:16 + n], ww[1:-1, :n], dim,
                                  out=out[:, first:first + width])
            assert torch.equal(got, ref)
            assert (out[:, :first] == 7).all() and (out[:, first + width:] == 7).all()
    ops.check()


@pytest.mark.gpu
@pytest.mark.parametrize("rows", [2, 150])
def test_product_of_nan_and_far_apart_scales(cuda_device, rows):
    dim = 160
    xv, wv = torch.ones(rows, dim), torch.ones(10, dim)
    xv[0, 40] = math.nan
    wv[3, 100] = math.inf
    wv[4] = 0
    wv[5] *= 2.0 ** -90
    xv[1] *= 2.0 ** 100
    wv[6, 1:] = 0
    wv[6] *= 2.0 ** 20
    x, w = ops.int8_quantize(xv.to(cuda_device)), ops.int8_quantize(wv.to(cuda_device))
    got = ops.int8_linear(x, w, dim).cpu()
    assert got[0].isnan().all() and got[:, 3].isnan().all()
    ok = [j for j in range(10) if j != 3]
    ref, size = _exact_product(x.cpu(), w.cpu(), dim, "cpu")
    assert (ref[1:, ok].abs() < 3e38).all()
    assert_within(got[1:, ok], ref[1:, ok],
                  _product_bound(ref, size, dim, torch.float32)[1:, ok])


@pytest.mark.gpu
def test_products_of_nothing(cuda_device):
    x = torch.zeros(0, 144, dtype=torch.uint8, device=cuda_device)
    w = torch.zeros(5, 144, dtype=torch.uint8, device=cuda_device)
    assert ops.int8_linear(x, w, 128).shape == (0, 5)
    assert ops.int8_linear(w, x, 128).shape == (5, 0)
    r = ops.int8_linear_grad_weight(torch.zeros(0, 7, device=cuda_device), x, 128)
    assert r.weight.shape == (7, 128) and not r.weight.any() and not r.bias.any()
    r = ops.int8_linear_grad_weight(torch.zeros(5, 0, device=cuda_device), w, 128)
    assert r.weight.shape == (0, 128) and r.bias.shape == (0,)
    assert ops.int8_linear_grad_input(torch.zeros(0, 5, device=cuda_device), w, 128).shape == \
        (0, 128)
    got = ops.int8_linear_grad_input(torch.zeros(3, 0, device=cuda_device), x, 128)
    assert got.shape == (3, 128) and not got.any()


# ---- gradients ---------------------------------------------------------------------------

def _grad_inputs(rows, width, dim, dtype, seed=0):
    x = reference_rows(values(rows, dim, seed + 1))
    w = reference_rows(values(width, dim, seed + 2))
    return values(rows, width, seed + 3).to(dtype), x, w


def _grad_check(dev, rows, width, dim, dtype, out):
    d, x, w = _grad_inputs(rows, width, dim, dtype)
    got = ops.int8_linear_grad_weight(d.to(dev), x.to(dev), dim, out_dtype=out)
    dx = ops.int8_linear_grad_input(d.to(dev), w.to(dev), dim, out_dtype=out)
    assert got.weight.dtype == out and dx.dtype == out and got.bias.dtype == torch.float32
    dd = d.double().to(dev)
    xv, wv = (reference_values(v, dim).to(dev) for v in (x, w))
    # products to 2^-23, an fp32 sum whose steps are off by a unit of 2^-23 at most
    for y, a, b, n in ((got.weight, dd.t(), xv, rows), (dx, dd, wv, width),
                       (got.bias[:, None], dd.t(), torch.ones_like(dd[:, :1]), rows)):
        ref, size = a @ b, a.abs() @ b.abs()
        # a gradient past fp16's largest number is infinite, and so is all that it enters
        fine = torch.isfinite(ref)
        assert not y[~fine].isfinite().any()
        bound = (n + 8) * 2 * U32 * size + 1.01 * rounding(ref, y.dtype) + 1e-30
        assert_within(y[fine], ref[fine], bound[fine])
    ops.check()


@pytest.mark.gpu
@pytest.mark.parametrize("rows,width,dim", [(1, 1, 1), (3, 5, 7)] + SIZES)
@pytest.mark.parametrize("dtype", FLOATS)
def test_gradients(cuda_device, dtype, rows, width, dim):
    _grad_check(cuda_device, rows, width, dim, dtype, FLOATS[(rows + dim) % 3])


@pytest.mark.gpu
@pytest.mark.parametrize("rows,width,dim", [(m, k, n) for m, n, k in MANY])
@pytest.mark.parametrize("dtype,out", [(torch.bfloat16, torch.bfloat16),
                                       (torch.float16, torch.float16),
                                       (torch.float32, torch.bfloat16),
                                       (torch.bfloat16, torch.float32)])
def test_gradients_of_many_tiles(cuda_device, dtype, out, rows, width, dim):
    _grad_check(cuda_device, rows, width, dim, dtype, out)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", FLOATS)
@pytest.mark.parametrize("out", FLOATS)
def test_gradients_of_each_type(cuda_device, dtype, out):
    _grad_check(cuda_device, 300, 100, 140, dtype, out)


@pytest.mark.gpu
def test_gradients_are_those_of_differences(cuda_device):
    """Of the product in 64 bits of the same values: a linear function, so a difference over a
    whole step is the gradient."""
    rows, width, dim = 30, 20, 40
    d, x, w = _grad_inputs(rows, width, dim, torch.float32)
    xv, wv, dd = reference_values(x, dim), reference_values(w, dim), d.double()
    got = ops.int8_linear_grad_weight(d.to(cuda_device), x.to(cuda_device), dim).weight.cpu()
    dx = ops.int8_linear_grad_input(d.to(cuda_device), w.to(cuda_device), dim).cpu()
    loss = lambda a, b: ((a @ b.t()) * dd).sum()  # noqa: E731
    for j, i in ((0, 0), (7, 39), (19, 5)):
        step = torch.zeros_like(wv)
        step[j, i] = 1
        want = (loss(xv, wv + step) - loss(xv, wv - step)) / 2
        size = (dd[:, j] * xv[:, i]).abs().sum() + 1e-9 * loss(xv.abs(), wv.abs()).abs()
        assert abs(float(got[j, i] - want)) <= 80 * U32 * float(size)
    for r, i in ((0, 0), (29, 39), (5, 17)):
        step = torch.zeros_like(xv)
        step[r, i] = 1
        want = (loss(xv + step, wv) - loss(xv - step, wv)) / 2
        size = (dd[r] * wv[:, i]).abs().sum() + 1e-9 * loss(xv.abs(), wv.abs()).abs()
        assert abs(float(dx[r, i] - want)) <= 80 * U32 * float(size)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", FLOATS)
def test_gradient_strides_and_what_lies_past_the_ends(cuda_device, dtype):
    for rows, width, dim in ((140, 72, 96), (150, 70, 90)):
        d, x, w = _grad_inputs(rows, width, dim, dtype)
        d = d.to(cuda_device)
        want = ops.int8_linear_grad_weight(d, x.to(cuda_device), dim)
        want_dx = ops.int8_linear_grad_input(d, w.to(cuda_device), dim)
        n = row_bytes(dim)
        xw = torch.full((rows + 2, n + 48), 127, dtype=torch.uint8, device=cuda_device)
        ww = torch.full((width + 2, n + 16), 127, dtype=torch.uint8, device=cuda_device)
        xw[1:-1, 16:16 + n] = x.to(cuda_device)
        ww[1:-1, :n] = w.to(cuda_device)
        xw[1:-1, 16 + dim:16 + n - 4] = 127
        ww[1:-1, dim:n - 4] = 127
        for first in (0, 1, 8):
            dw = torch.full((rows + 2, width + 24), math.nan, dtype=dtype, device=cuda_device)
            dw[1:-1, first:first + width] = d
            out = torch.full((width, dim + 10), 7.0, device=cuda_device)
            got = ops.int8_linear_grad_weight(dw[1:-1, first:first + width], xw[1:-1, 16:16 + n],
                                              dim, out=out[:, first:first + dim])
            assert torch.equal(got.weight, want.weight) and torch.equal(got.bias, want.bias)
            assert (out[:, :first] == 7).all() and (out[:, first + dim:] == 7).all()
            out = torch.full((rows, dim + 10), 7.0, dtype=dtype, device=cuda_device)
            got = ops.int8_linear_grad_input(dw[1:-1, first:first + width], ww[1:-1, :n], dim,
                                             out=out[:, first:first + dim])
            assert torch.equal(got, want_dx)
            assert (out[:, :first] == 7).all() and (out[:, first + dim:] == 7).all()
    ops.check()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", FLOATS)
def test_gradients_of_infinities_and_nan(cuda_device, dtype):
    """What is not finite stays where the formula has it."""
    rows, width, dim = 200, 70, 50
    d, x, w = _grad_inputs(rows, width, dim, dtype)
    xv = values(rows, dim, 5)
    xv[7, 3] = math.nan
    x, w = ops.int8_quantize(xv.to(cuda_device)), w.to(cuda_device)
    d[9, 4], d[11, 5], d[12, 6], d[13, 6] = math.nan, math.inf, math.inf, -math.inf
    d = d.to(cuda_device)
    got = ops.int8_linear_grad_weight(d, x, dim)
    # the row that stands for NaN is in every sum
    assert got.weight.isnan().all()
    bias = got.bias.cpu()
    assert bias[4].isnan() and bias[5] == math.inf and bias[6].isnan()
    assert bias[7:].isfinite().all() and bias[:4].isfinite().all()
    xv[7, 3] = 1.0
    got = ops.int8_linear_grad_weight(d, ops.int8_quantize(xv.to(cuda_device)), dim).weight.cpu()
    assert not got[4:7].isfinite().any() and got[7:].isfinite().all() and got[:4].isfinite().all()
    dx = ops.int8_linear_grad_input(d, w, dim, out_dtype=torch.float32).cpu()
    bad = torch.tensor([9, 11, 12, 13])
    assert not dx[bad].isfinite().any() and dx[:9].isfinite().all() and dx[14:].isfinite().all()


@pytest.mark.gpu
@pytest.mark.parametrize("rows,width", [(4200, 2000), (4200, 2100), (700, 300)])
def test_a_row_that_is_no_number_and_the_others(cuda_device, rows, width):
    """Over a slice's end and the last rows, in all variants of the gradient to the weights."""
    dim = 150
    d, x, _ = _grad_inputs(rows, width, dim, torch.bfloat16)
    clean = ops.int8_linear_grad_weight(d.to(cuda_device), x.to(cuda_device), dim)
    assert clean.weight.isfinite().all() and clean.bias.isfinite().all()
    d[rows - 1, 7] = math.inf
    got = ops.int8_linear_grad_weight(d.to(cuda_device), x.to(cuda_device), dim)
    assert not got.weight[7].isfinite().any() and not got.bias[7].isfinite()
    got.weight[7], got.bias[7] = clean.weight[7], clean.bias[7]
    assert torch.equal(got.weight, clean.weight) and torch.equal(got.bias, clean.bias)
    # a row of x that stands for NaN enters all sums over the rows, the bias' not
    d[rows - 1, 7] = 0
    x[rows - 1, -4:] = torch.tensor([0xff, 0xff, 0xff, 0x7f], dtype=torch.uint8)
    got = ops.int8_linear_grad_weight(d.to(cuda_device), x.to(cuda_device), dim)
    assert got.weight.isnan().all() and got.bias.isfinite().all()


@pytest.mark.gpu
def test_gradients_are_the_same_each_time(cuda_device):
    d, x, w = _grad_inputs(30_000, 200, 150, torch.bfloat16)
    d, x, w = d.to(cuda_device), x.to(cuda_device), w.to(cuda_device)
    first = ops.int8_linear_grad_weight(d, x, 150)
    first_dx = ops.int8_linear_grad_input(d, w, 150)
    for _ in range(20):
        got = ops.int8_linear_grad_weight(d, x, 150)
        assert torch.equal(got.weight, first.weight) and torch.equal(got.bias, first.bias)
        assert torch.equal(ops.int8_linear_grad_input(d, w, 150), first_dx)


@pytest.mark.gpu
@pytest.mark.parametrize("rows,width,dim,dtype", [(40_000, 256, 128, torch.bfloat16),
                                                  (9000, 640, 700, torch.bfloat16),
                                                  (4000, 120, 300, torch.float32),
                                                  (12, 300, 400, torch.float16)])
def test_a_thousand_calls_give_the_same(cuda_device, rows, width, dim, dtype):
    """What a race between a kernel's warps, or of a pair's two halves, would change now and then."""
    d, x, w = (t.to(cuda_device) for t in _grad_inputs(rows, width, dim, dtype))
    x8 = torch.randn(rows, dim, generator=gen(5)).to(cuda_device)

    def run():
        r = ops.int8_linear_grad_weight(d, x, dim)
        return [ops.int8_linear(x, w, dim), r.weight, r.bias, ops.int8_linear_grad_input(d, w, dim),
                ops.int8_quantize(x8)]
    first = run()
    changed = torch.zeros((), dtype=torch.int64, device=cuda_device)
    for _ in range(1000):
        for got, want in zip(run(), first):
            changed += (got.view(torch.uint8) != want.view(torch.uint8)).sum()
    assert int(changed) == 0
    ops.check()


# at and beside the sizes where a call takes another variant
@pytest.mark.gpu
@pytest.mark.parametrize("rows,width,dim", [
    (16, 130, 260), (17, 130, 260), (128, 128, 128), (129, 129, 129), (50_000, 257, 511),
    (50_000, 256, 512), (20_000, 384, 128), (20_000, 385, 128), (300, 64, 2048), (300, 64, 2049),
    (64, 2048, 512), (700, 300, 129), (4101, 1921, 130), (4096, 2060, 200), (4095, 1921, 72)])
@pytest.mark.parametrize("dtype", FLOATS)
def test_where_variants_meet(cuda_device, rows, width, dim, dtype):
    _product_check(cuda_device, rows, width, dim, dtype, True)
    _grad_check(cuda_device, rows, width, dim, dtype, dtype)


@pytest.mark.gpu
def test_refusals_on_a_device(cuda_device):
    flat = torch.zeros(64 * 144 + 16, dtype=torch.uint8, device=cuda_device)
    apart = torch.zeros(4, 152, dtype=torch.uint8, device=cuda_device)[:, :144]  # 152 bytes apart
    good = flat[:64 * 144].view(64, 144)
    off = flat[8:8 + 64 * 144].view(64, 144)
    d = torch.zeros(64, 64, device=cuda_device)
    for x, w in ((off, good), (good, off), (apart, good), (good, apart)):
        with pytest.raises(AgnesError, match="aligned|multiple of 16"):
            ops.int8_linear(x, w, 128)
    for bad in (off, apart):
        n = bad.shape[0]
        with pytest.raises(AgnesError, match="aligned|multiple of 16"):
            ops.int8_linear_grad_weight(d[:n], bad, 128)
        with pytest.raises(AgnesError, match="aligned|multiple of 16"):
            ops.int8_linear_grad_input(d[:, :n], bad, 128)
        with pytest.raises(AgnesError, match="aligned|multiple of 16"):
            ops.int8_dequantize(bad, 128)
        with pytest.raises(AgnesError, match="aligned|multiple of 16"):
            ops.activation_grad(d[:n].repeat(1, 2), bad, "silu")
        with pytest.raises(AgnesError, match="aligned|multiple of 16"):
            ops.int8_quantize(torch.zeros(n, 128, device=cuda_device), out=bad)


@pytest.mark.gpu
def test_sums_over_many_rows(cuda_device):
    """A hyperbatch's rows, all of one sign: what a single fp32 sum would lose step by step."""
    rows, width, dim = 700_001, 24, 40
    g = torch.Generator(device=cuda_device).manual_seed(1)
    x = ops.int8_quantize(torch.rand(rows, dim, generator=g, device=cuda_device) + 0.5)
    for dtype in FLOATS:
        d = (torch.rand(rows, width, generator=g, device=cuda_device) + 0.5).to(dtype)
        got = ops.int8_linear_grad_weight(d, x, dim)
        ref = d.double().t() @ ops.int8_dequantize(x, dim).double()
        # sums of at most 2^14 rows each in fp32, each step off by a unit of 2^-23 of it at most
        # (half of that on average)
        assert_within(got.weight, ref, 2.0 ** 14 * 2 * U32 * ref)
        off = ((got.weight.double() - ref) / ref).abs().max()
        assert off < 1e-5, float(off)
        ref = d.double().sum(0)
        assert ((got.bias.double() - ref) / ref).abs().max() < 1e-5


# ---- how they are called --------------------------------------------------------------------

def _calls(dev, rows, width, dim):
    d, x, w = (t.to(dev) for t in _grad_inputs(rows, width, dim, torch.bfloat16))

    def run(**stream):
        r = ops.int8_linear_grad_weight(d, x, dim, **stream)
        return [ops.int8_linear(x, w, dim, **stream), r.weight, r.bias,
                ops.int8_linear_grad_input(d, w, dim, **stream)]
    return run


@pytest.mark.gpu
def test_streams_and_graphs(cuda_device):
    run = _calls(cuda_device, 3000, 200, 128)
    ref = run()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = run(stream=side)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, ref))
    graphs = []
    for _ in range(2):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            got = run()
        graphs.append((graph, got))
    for _ in range(3):
        for graph, _ in graphs:
            graph.replay()
    torch.cuda.synchronize()
    for _, got in graphs:
        assert all(torch.equal(a, b) for a, b in zip(got, ref))
    ops.check()


@pytest.mark.gpu
def test_calls_on_two_streams_at_once(cuda_device):
    """Kernels that each want an SM's tensor memory, side by side, with workspaces of their own."""
    cases = [(run, run(), torch.cuda.Stream())
             for run in (_calls(cuda_device, 40_000, 256, 128), _calls(cuda_device, 9000, 500, 640))]
    torch.cuda.synchronize()
    got = [[run(stream=stream) for run, _, stream in cases] for _ in range(20)]
    torch.cuda.synchronize()
    for outs in got:
        for out, (_, ref, _) in zip(outs, cases):
            assert all(torch.equal(a, b) for a, b in zip(out, ref))
    ops.check()


@pytest.mark.gpu
def test_a_graph_gathers_8bit_rows_unchanged(cuda_device):
    from agnes_inputs import synth
    n, dim = 3000, 128
    off, ind = synth.rmat_csr(n, 8, 0.57, 0.19, 0.19, seed=5, offsets_dtype=torch.int64)
    packed = ops.int8_quantize(values(n, dim, 4).to(cuda_device))
    w = ops.int8_quantize(values(64, dim, 6).to(cuda_device))
    whole = ops.int8_linear(packed, w, dim)
    with Graph(off.to(cuda_device), ind.to(cuda_device), packed.view(torch.float16)) as g:
        g.prepare(torch.arange(40, dtype=torch.int32, device=cuda_device).view(1, 40), [5, 3], 7)
        mb = g.fetch(0)
        assert torch.equal(mb.feats.view(torch.uint8), packed[mb.nodes.long()])
        assert torch.equal(ops.int8_linear(mb.feats, w, dim), whole[mb.nodes.long()])
        d = torch.ones(mb.nodes.numel(), 64, device=cuda_device)
        a = ops.int8_linear_grad_weight(d, mb.feats, dim)
        b = ops.int8_linear_grad_weight(d, packed[mb.nodes.long()], dim)
        assert torch.equal(a.weight, b.weight)
    ops.check()


@pytest.mark.gpu
def test_offsets_past_32_bits(cuda_device):
    rows, width, dim = 9_000_000, 256, 16  # 2.3e9 values of the output
    part = reference_rows(values(7, dim, 3))
    x = torch.zeros(rows, row_bytes(dim), dtype=torch.uint8, device=cuda_device)
    at = torch.tensor([0, 1, 8_388_607, 8_388_608, 8_388_609, rows - 2, rows - 1],
                      device=cuda_device)
    x[at] = part.to(cuda_device)
    w = reference_rows(values(width, dim, 4))
    y = ops.int8_linear(x, w.to(cuda_device), dim, out_dtype=torch.float16)
    ref, size = _exact_product(part, w, dim, cuda_device)
    assert_within(y[at], ref, _product_bound(ref, size, dim, y.dtype))
    assert int((y != 0).any(1).sum()) <= 7
    y.zero_()
    y[at] = ref.half()
    got = ops.int8_linear_grad_weight(y, x, dim)
    part = part.to(cuda_device)
    want = ops.int8_linear_grad_weight(y[at], part, dim)
    xv = reference_values(part.cpu(), dim).to(cuda_device)
    size = y[at].double().abs().t() @ xv.abs()
    assert_within(got.weight, want.weight.double(), 100 * U32 * size)
    dx = ops.int8_linear_grad_input(y, w.to(cuda_device), dim)
    wv = reference_values(w, dim).to(cuda_device)
    ref, size = y[at].double() @ wv, y[at].double().abs() @ wv.abs()
    assert_within(dx[at], ref, _product_bound(ref, size, width, dx.dtype))
    assert int((dx != 0).any(1).sum()) <= 7
    ops.check()


# ---- the largest numbers of a type -----------------------------------------------------------

def _with_the_largest(rows, dim, dtype, seed):
    """8-bit rows, of which row 5 and the last have their type's lowest number (the usual mask) and
    its largest beside ordinary values.  They stand for finite numbers that round to infinity in
    bfloat16."""
    x = values(rows, dim, seed).to(dtype)
    x[5, 7], x[rows - 1, 3] = torch.finfo(dtype).min, torch.finfo(dtype).max
    packed = reference_rows(x)
    most = reference_values(packed, dim).abs().amax(1)[[5, rows - 1]]
    assert (most < 2.0 ** 128).all() and most.float().bfloat16().isinf().all()
    return packed


# a CTA to a tile, pairs, pairs with the scaled whole numbers made before
@pytest.mark.gpu
@pytest.mark.parametrize("rows,width", [(90, 70), (700, 300), (4200, 2000)])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("grad", FLOATS)
def test_gradient_to_the_weights_of_rows_with_the_largest_numbers(cuda_device, rows, width, dtype,
                                                                  grad):
    dim = 150
    x = _with_the_largest(rows, dim, dtype, 1)
    xv = reference_values(x, dim).to(cuda_device)
    d = (values(rows, width, 3) / 64).to(grad)
    assert d.isfinite().all()
    for weight in (0.0, 2.0 ** -20, 1.0):
        d[5], d[rows - 1] = 0, 0
        d[5, 2], d[rows - 1, 4] = weight, -weight
        got = ops.int8_linear_grad_weight(d.to(cuda_device), x.to(cuda_device), dim).weight
        dd = d.double().to(cuda_device)
        ref, size = dd.t() @ xv, dd.abs().t() @ xv.abs()
        assert got.isfinite().all()
        assert_within(got, ref, (rows + 8) * 2 * U32 * size + 1.01 * rounding(ref, got.dtype))
    ops.check()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("grad", FLOATS)
def test_gradient_to_the_input_of_weights_with_the_largest_numbers(cuda_device, dtype, grad):
    rows, width, dim = 130, 200, 150
    w = _with_the_largest(width, dim, dtype, 2)
    wv = reference_values(w, dim).to(cuda_device)
    d = (values(rows, width, 3) / 64).to(grad)
    assert d.isfinite().all()
    for weight in (0.0, 2.0 ** -20, 1.0):
        d[:, 5], d[:, width - 1] = 0, 0
        d[2, 5], d[4, width - 1] = weight, -weight
        got = ops.int8_linear_grad_input(d.to(cuda_device), w.to(cuda_device), dim,
                                         out_dtype=torch.float32)
        dd = d.double().to(cuda_device)
        ref, size = dd @ wv, dd.abs() @ wv.abs()
        assert got.isfinite().all()
        assert_within(got, ref, (width + 8) * 2 * U32 * size + 1.01 * rounding(ref, got.dtype))
    ops.check()


# ---- rows that another program wrote ---------------------------------------------------------

def _other_rows(rows, dim, seed):
    """8-bit rows whose scales are fp32 numbers of 24 bits, one of them negative."""
    x = values(rows, dim, seed)
    scale = x.abs().amax(1, keepdim=True) / 127
    scale[rows // 2] *= -1
    assert (scale.view(torch.int32) % 65536 != 0).float().mean() > 0.9 or rows == 1
    packed = torch.zeros(rows, row_bytes(dim), dtype=torch.uint8)
    packed[:, :dim] = torch.round(x / scale).clamp(-127, 127).to(torch.int8).view(torch.uint8)
    packed[:, -4:] = scale.contiguous().view(torch.uint8)
    return packed


@pytest.mark.gpu
@pytest.mark.parametrize("rows,width,dim", [(90, 70, 40), (700, 300, 150), (4200, 2000, 150)])
@pytest.mark.parametrize("dtype", FLOATS)
def test_scales_of_more_than_eight_bits(cuda_device, rows, width, dim, dtype):
    """A scale is any fp32 number: values of 31 bits then, which the products' operands keep
    the leading 16 bits of."""
    x, w = _other_rows(rows, dim, 1), _other_rows(width, dim, 2)
    d = (values(rows, width, 3) / 64).to(dtype)
    assert d.isfinite().all()
    x_dev, w_dev, d_dev = x.to(cuda_device), w.to(cuda_device), d.to(cuda_device)
    back = ops.int8_dequantize(x_dev, dim)
    ref = reference_values(x, dim)
    assert_within(back, ref, rounding(ref, torch.float32))
    ref, size = _exact_product(x, w, dim, cuda_device)
    assert_within(ops.int8_linear(x_dev, w_dev, dim), ref,
                  _product_bound(ref, size, dim, torch.float32))
    got = ops.int8_linear_grad_weight(d_dev, x_dev, dim).weight
    dx = ops.int8_linear_grad_input(d_dev, w_dev, dim, out_dtype=torch.float32)
    dd = d_dev.double()
    xv, wv = (reference_values(v, dim).to(cuda_device) for v in (x, w))
    for y, a, b, n in ((got, dd.t(), xv, rows), (dx, dd, wv, width)):
        ref, size = a @ b, a.abs() @ b.abs()
        # the second term is rounded to 8 bits, 2^-9 of what is at most 2^-7 of the value; the sum
        assert_within(y, ref, (2.0 ** -16 + (n + 8) * 2 * U32) * size)
        # and on average far less than the 2^-9 that one rounding of the scales would lose
        assert float((y - ref).norm() / ref.norm()) < 2.0 ** -15
    ops.check()


# ---- long contractions -----------------------------------------------------------------------

# Tensor memory's sums are cut off instead of rounded: a product of 16 aligns these and the sum with
# the largest of them, cuts each off two bits below its unit (2^-23 of it at most) and the result at
# the unit: 17 eighths and a half of a unit on average, 2.6.  Over a sum of values of one sign a
# partial sum's unit is 0.375 of the result's 2^-23 on average at most (m - 2/3 over m^2 for a result
# of m, 1 <= m < 2), so that a product loses 2^-23 of the result.  How many products one such sum may
# have, of the product and of the gradient to the input:
CHAIN = {torch.float32: 64, torch.float16: 512, torch.bfloat16: 2048}
GRAD_CHAIN = {torch.float32: 24, torch.float16: 128, torch.bfloat16: 128}


def _one_sign_check(got, ref, products, chains):
    """`got` of sums of positive numbers whose rows differ in size, `products` to an accumulator,
    `chains` of those added up in fp32."""
    loss = products * 2 * U32 + (chains + 4) * U32
    assert_within(got, ref, loss * ref + 1.01 * rounding(ref, got.dtype))
    # The mean, relative to 64 bits rounded once.  A loss takes a value to its neighbour, a unit
    # away, as often as it is a part of a unit; rows alone count as independent.
    off = ((got.double() - ref.to(got.dtype).double()) / ref).mean()
    unit = 2 * float((rounding(ref, got.dtype) / ref).max())
    assert abs(float(off)) <= loss + 4 * math.sqrt(unit * loss / got.shape[0])


def _of_one_sign(dev, rows, dim, seed, scale=1.0):
    """Between 0.5 and 1.5, times a number of the row's own between 1 and 2."""
    g = torch.Generator(device=dev).manual_seed(seed)
    x = torch.rand(rows, dim, generator=g, device=dev) + 0.5
    return x * torch.exp2(torch.rand(rows, 1, generator=g, device=dev)) * scale


# beside each limit and the longest rows
@pytest.mark.gpu
@pytest.mark.parametrize("out,dim", [(torch.float16, 8192), (torch.float16, 8193),
                                     (torch.float16, 32_768), (torch.float16, 32_769),
                                     (torch.bfloat16, 32_768), (torch.bfloat16, 32_769),
                                     (torch.float16, 131_072), (torch.bfloat16, 131_072),
                                     (torch.float32, 32_768)])
def test_product_of_long_rows_of_one_sign(cuda_device, out, dim):
    x = ops.int8_quantize(_of_one_sign(cuda_device, 1000, dim, 1))
    w = ops.int8_quantize(_of_one_sign(cuda_device, 130, dim, 2, 2.0 ** -8))
    got = ops.int8_linear(x, w, dim, out_dtype=out)
    ref, _ = _exact_product(x, w, dim, cuda_device)
    _one_sign_check(got, ref, min(CHAIN[out], -(-dim // 16)), dim / 1024)


# widths beside the limits of each gradient's number of terms
@pytest.mark.gpu
@pytest.mark.parametrize("grad", FLOATS)
@pytest.mark.parametrize("out", FLOATS)
@pytest.mark.parametrize("width", [384, 385, 512, 513, 1024, 1025, 2048, 4097, 6592, 8193, 16_384,
                                   16_385])
def test_gradient_to_the_input_of_wide_layers_of_one_sign(cuda_device, grad, out, width):
    rows, dim = 2000, 140
    d = _of_one_sign(cuda_device, rows, width, width).to(grad)
    w = ops.int8_quantize(_of_one_sign(cuda_device, width, dim, 3, 2.0 ** -8))
    got = ops.int8_linear_grad_input(d, w, dim, out_dtype=out)
    ref = d.double() @ reference_values(w, dim)
    # products of 16 for each two terms: of bfloat16, fp16 and fp32
    terms = {torch.bfloat16: 2, torch.float16: 4, torch.float32: 5}[grad]
    _one_sign_check(got, ref, min(GRAD_CHAIN[out], -(-width // 16) * terms), width / 64)


@pytest.mark.gpu
@pytest.mark.parametrize("rows", [40, 300])
@pytest.mark.parametrize("dim", [1040, 2048, 2049, 131_072])
def test_product_of_the_largest_whole_numbers_in_chains(cuda_device, rows, dim):
    """1024 columns' sum of 127^2 is exact; beyond 2048 columns those are added up in fp32."""
    x = torch.full((rows, dim), 127.0)
    w = torch.full((3, dim), 127.0)
    w[1] *= -1
    w[2, ::2] *= -1
    got = ops.int8_linear(*(ops.int8_quantize(v.to(cuda_device)) for v in (x, w)), dim)
    want = (x.double() @ w.double().t()).to(cuda_device)
    # undrained: each product past 2^24 is cut off by 2 at most, or by 4 past 2^25
    off = dim / 1024 * U32 * 127.0 ** 2 * dim if dim > 2048 else 0 if dim <= 1040 else \
        4 * (dim - 1040) / 16
    assert_within(got, want, off * torch.ones_like(want) + U32 * want.abs())


@pytest.mark.gpu
@pytest.mark.parametrize("out", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("grad", FLOATS)
def test_long_contractions_of_both_signs(cuda_device, grad, out):
    """The variants that add up chains for 16-bit results, ragged on each side."""
    _product_check(cuda_device, 139, 261, 33_001, out, True)
    d, _, w = _grad_inputs(139, 16_501, 261, grad)
    got = ops.int8_linear_grad_input(d.to(cuda_device), w.to(cuda_device), 261, out_dtype=out)
    dd, wv = d.double().to(cuda_device), reference_values(w, 261).to(cuda_device)
    fine = torch.isfinite(dd).all(1)  # values past fp16's largest number
    ref, size = dd[fine] @ wv, dd[fine].abs() @ wv.abs()
    # 128 products to an accumulator, up to 259 of those
    bound = (2 * 128 + 259 + 8) * U32 * size + 1.01 * rounding(ref, out)
    assert_within(got[fine], ref, bound)
    assert not got[~fine].isfinite().any()
    ops.check()
