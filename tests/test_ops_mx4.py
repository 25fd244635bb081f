"""Microscaled 4-bit rows and their product (include/agnes_ops.h) against the
format's definition, in 64 bits."""
import math

import pytest
import torch

from ops_support import FLOATS, U32, assert_within, gen, rounding
from paper_2601_01473_gb300 import AgnesError, Graph, ops

GRID = [0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0]


def row_bytes(dim):
    blocks = -(-dim // 32)
    return -(-blocks * 17 // 16) * 16


def reference_rows(x):
    """The bytes of x's 4-bit rows, block by block: the nearest grid magnitude by
    distance, the even code of two as near."""
    rows, dim = x.shape
    blocks = -(-dim // 32)
    v = torch.zeros(rows, blocks * 32, dtype=torch.float64)
    v[:, :dim] = x.double()
    v = v.view(rows, blocks, 32)
    fine = torch.isfinite(v).all(2)
    v = torch.where(fine[:, :, None], v, 0.0)
    top = v.abs().amax(2)
    exponent = torch.frexp(top)[1].double() - 3  # floor(log2(top)) - 2
    exponent = torch.where(top > 0, exponent, -127.0).clamp(min=-127)
    size = (v.abs() * torch.exp2(-exponent)[:, :, None])
    grid = torch.tensor(GRID, dtype=torch.float64)
    far = (size[..., None] - grid).abs()
    # an even code wins a tie: odd codes are pushed away by less than any other distance
    far = far + torch.tensor([0, 1, 0, 1, 0, 1, 0, 1]) * 1e-12
    code = far.argmin(-1) + 8 * torch.signbit(v).long()
    code = torch.where(fine[:, :, None], code, 0).view(rows, blocks * 16, 2)
    out = torch.zeros(rows, row_bytes(dim), dtype=torch.uint8)
    out[:, :blocks * 16] = (code[:, :, 0] + 16 * code[:, :, 1]).to(torch.uint8)
    out[:, blocks * 16:blocks * 17] = torch.where(fine, exponent + 127, 255.0).to(torch.uint8)
    return out


def reference_values(packed, dim):
    blocks = -(-dim // 32)
    grid = torch.tensor(GRID + [-g for g in GRID], dtype=torch.float64)
    codes = packed[:, :blocks * 16]
    v = torch.stack((grid[(codes & 15).long()], grid[(codes >> 4).long()]), 2)
    byte = packed[:, blocks * 16:blocks * 17].double()
    scale = torch.where(byte == 255, math.nan, torch.exp2(byte - 127))
    v = v.view(packed.shape[0], blocks, 32) * scale[:, :, None]
    return v.view(packed.shape[0], blocks * 32)[:, :dim]


def _values(rows, dim, seed):
    g = gen(seed)
    x = torch.randn(rows, dim, generator=g) * torch.exp2(3 * torch.randn(rows, 1, generator=g))
    return torch.where(torch.rand(rows, dim, generator=g) < 0.02, 20 * x, x)


# ---- without a GPU --------------------------------------------------------------------

def test_row_bytes_and_refusals():
    from paper_2601_01473_gb300 import build
    build.build()
    for dim in (1, 31, 32, 33, 128, 301, 512, 4096):
        assert ops.mx4_row_bytes(dim) == row_bytes(dim)
    assert ops.mx4_row_bytes(128) == 80
    with pytest.raises(AgnesError, match="EINVAL"):
        ops.mx4_row_bytes(0)
    with pytest.raises(AgnesError, match="ERANGE"):
        ops.mx4_row_bytes((1 << 26) + 1)
    with pytest.raises(ValueError, match="CUDA device"):
        ops.mx4_quantize(torch.zeros(2, 8))
    with pytest.raises(ValueError, match="bytes"):
        ops.mx4_linear(torch.zeros(2, 32, dtype=torch.uint8), torch.zeros(2, 32, dtype=torch.uint8),
                       128)
    L = ops.lib()
    args = [None, 80, 4, None, 80, 5, 128, None, None, 0, 5, None, None]
    assert L.agnes_mx4_linear(*args) == 1 and b"NULL" in L.agnes_last_error(None)
    for at, value, status in ((1, 64, 1), (1, 88, 1), (2, -1, 1), (4, 72, 1), (5, -1, 1),
                              (6, 0, 1), (9, 9, 1), (10, 4, 1), (2, 1 << 31, 2), (6, 1 << 27, 2)):
        bad = list(args)
        bad[at] = value
        assert L.agnes_mx4_linear(*bad) == status, (at, value)
    args[2] = 0
    assert L.agnes_mx4_linear(*args) == 0


def test_the_reference_rounds_as_the_format_says():
    x = torch.tensor([[0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 6.0, 7.9, -0.26, 4.0, -0.0]])
    got = reference_values(reference_rows(x), 12)
    assert got.tolist() == [[0.0, 1.0, 1.0, 2.0, 2.0, 4.0, 4.0, 6.0, 6.0, -0.5, 4.0, 0.0]]


# ---- rounding --------------------------------------------------------------------------

@pytest.mark.gpu
@pytest.mark.parametrize("dtype", FLOATS)
@pytest.mark.parametrize("rows,dim", [(1, 1), (3, 7), (5, 31), (4, 32), (7, 33), (100, 64),
                                      (33, 128), (9, 301), (17, 602), (2, 4096), (1, 100_001),
                                      (1500, 8)])
def test_quantize_and_back(cuda_device, dtype, rows, dim):
    x = _values(rows, dim, rows + dim).to(dtype)
    packed = ops.mx4_quantize(x.to(cuda_device))
    ref = reference_rows(x)
    assert torch.equal(packed.cpu(), ref)
    for out in FLOATS:
        got = ops.mx4_dequantize(packed, dim, out_dtype=out).cpu()
        # a code times a power of two: only the output's range can round it
        assert torch.equal(got, reference_values(ref, dim).to(out))


@pytest.mark.gpu
def test_ties_ranges_and_special_values(cuda_device):
    rows = []
    halves = torch.arange(0, 32).float() / 4  # every tie of the grid, and beyond 6
    rows.append(halves)
    rows.append(-halves)
    rows.append(halves * 2.0 ** -126)      # subnormal steps, the scale at its least
    rows.append(halves * 2.0 ** -149)
    rows.append(halves * 2.0 ** 125)       # the largest scales
    rows.append(torch.full((32,), 3.4e38))
    rows.append(torch.zeros(32))
    rows.append(-torch.zeros(32))
    one = torch.ones(32)
    for special in (math.inf, -math.inf, math.nan):
        r = one.clone()
        r[5] = special
        rows.append(r)
    x = torch.stack(rows)
    packed = ops.mx4_quantize(x.to(cuda_device)).cpu()
    assert torch.equal(packed, reference_rows(x))
    assert packed[-3:, 16].tolist() == [255] * 3 and packed[6, 16] == 0
    back = ops.mx4_dequantize(packed.to(cuda_device), 32).cpu()
    assert back[-3:].isnan().all() and (back[6:8] == 0).all()
    ref = reference_values(packed, 32)[:-3].float()
    assert torch.equal(back[:-3], ref)


@pytest.mark.gpu
def test_strides(cuda_device):
    x = _values(20, 100, 3)
    wide = torch.zeros(20, 200, device=cuda_device)
    for first in (0, 3, 4, 8):
        wide[:, first:first + 100] = x.to(cuda_device)
        out = torch.full((20, 160), 7, dtype=torch.uint8, device=cuda_device)
        got = ops.mx4_quantize(wide[:, first:first + 100], out=out[:, 16:96])
        assert torch.equal(got.cpu(), reference_rows(x))
        assert (out[:, :16] == 7).all() and (out[:, 96:] == 7).all()
        back = torch.full((20, 120), 7.0, device=cuda_device)
        ops.mx4_dequantize(got, 100, out=back[:, first:first + 100])
        assert torch.equal(back[:, first:first + 100].cpu(),
                           reference_values(reference_rows(x), 100).float())
        assert (back[:, :first] == 7).all() and (back[:, first + 100:] == 7).all()
    assert ops.mx4_quantize(wide[:0]).shape == (0, ops.mx4_row_bytes(200))


# ---- product -----------------------------------------------------------------------------

def _product_check(dev, rows, width, dim, out, bias, seed=0):
    x = reference_rows(_values(rows, dim, seed + 1))
    w = reference_rows(_values(width, dim, seed + 2))
    b = torch.randn(width, generator=gen(seed)) if bias else None
    got = ops.mx4_linear(x.to(dev), w.to(dev), dim, b.to(dev) if bias else None, out_dtype=out)
    xv, wv = reference_values(x, dim), reference_values(w, dim)
    ref, size = xv @ wv.t(), xv.abs() @ wv.abs().t()
    if bias:
        ref, size = ref + b.double(), size + b.double().abs()
    assert got.dtype == out
    # exact products; an fp32 sum of up to dim terms, each step off by a unit of 2^-23 of the
    # sum of magnitudes at most
    assert_within(got, ref, (dim + 2) * 2 * U32 * size + 1.01 * rounding(ref, out) + 1e-30)
    ops.check()


@pytest.mark.gpu
@pytest.mark.parametrize("out", FLOATS)
@pytest.mark.parametrize("rows", [1, 2, 3, 5, 8])
@pytest.mark.parametrize("width,dim", [(1, 1), (7, 20), (33, 128), (257, 301), (100, 2048)])
def test_product_of_few_rows(cuda_device, out, rows, width, dim):
    _product_check(cuda_device, rows, width, dim, out, rows % 2 == 0)


@pytest.mark.gpu
@pytest.mark.parametrize("rows,width,dim", [
    (9, 8, 32), (128, 128, 64), (128, 128, 256), (16, 1, 1), (129, 130, 33), (200, 96, 128),
    (1000, 257, 301), (130, 300, 1024), (64, 500, 4096), (40_000, 256, 128)])
@pytest.mark.parametrize("out", FLOATS)
def test_product(cuda_device, out, rows, width, dim):
    _product_check(cuda_device, rows, width, dim, out, width % 2 == 0)


@pytest.mark.gpu
def test_product_of_rows_too_long_for_shared_memory(cuda_device):
    _product_check(cuda_device, 2, 3, 100_000, torch.float32, True)


@pytest.mark.gpu
@pytest.mark.parametrize("rows", [3, 140])
def test_product_strides_and_what_lies_past_the_ends(cuda_device, rows):
    """Rows apart, and bytes around them that would be NaN if they were read."""
    dim, width = 96, 70
    x, w = reference_rows(_values(rows, dim, 1)), reference_rows(_values(width, dim, 2))
    ref = ops.mx4_linear(x.to(cuda_device), w.to(cuda_device), dim)
    n = row_bytes(dim)
    xw = torch.full((rows + 2, n + 48), 255, dtype=torch.uint8, device=cuda_device)
    ww = torch.full((width + 2, n + 16), 255, dtype=torch.uint8, device=cuda_device)
    xw[1:-1, 16:16 + n] = x.to(cuda_device)
    ww[1:-1, :n] = w.to(cuda_device)
    xw[1:-1, 16 + 51:16 + n] = 255  # the padding of a row is not looked at either
    for first in (0, 1, 4):
        out = torch.full((rows, width + 10), 7.0, device=cuda_device)
        got = ops.mx4_linear(xw[1:-1, 16:16 + n], ww[1:-1, :n], dim,
                             out=out[:, first:first + width])
        assert torch.equal(got, ref)
        assert (out[:, :first] == 7).all() and (out[:, first + width:] == 7).all()
    ops.check()


@pytest.mark.gpu
@pytest.mark.parametrize("rows", [2, 150])
def test_product_of_nan_and_extreme_scales(cuda_device, rows):
    dim = 160
    xv, wv = torch.ones(rows, dim), torch.ones(10, dim)
    xv[0, 40] = math.nan
    wv[3, 100] = math.inf
    wv[5] *= 2.0 ** -100
    xv[1] *= 2.0 ** 60
    x, w = ops.mx4_quantize(xv.to(cuda_device)), ops.mx4_quantize(wv.to(cuda_device))
    got = ops.mx4_linear(x, w, dim).cpu()
    assert got[0].isnan().all() and got[:, 3].isnan().all()
    ok = [j for j in range(10) if j != 3]
    ref = reference_values(x.cpu(), dim) @ reference_values(w.cpu(), dim).t()
    assert torch.equal(got[1:][:, ok], ref[1:][:, ok].float())


@pytest.mark.gpu
def test_product_of_nothing(cuda_device):
    x = torch.zeros(0, 80, dtype=torch.uint8, device=cuda_device)
    w = torch.zeros(5, 80, dtype=torch.uint8, device=cuda_device)
    assert ops.mx4_linear(x, w, 128).shape == (0, 5)
    assert ops.mx4_linear(w, x, 128).shape == (5, 0)


@pytest.mark.gpu
def test_product_streams_and_graphs(cuda_device):
    x = ops.mx4_quantize(_values(300, 128, 1).to(cuda_device))
    w = ops.mx4_quantize(_values(200, 128, 2).to(cuda_device))
    ref = ops.mx4_linear(x, w, 128)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = ops.mx4_linear(x, w, 128, stream=side)
    torch.cuda.synchronize()
    assert torch.equal(got, ref)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = ops.mx4_linear(x, w, 128)
    graph.replay()
    assert torch.equal(got, ref)
    ops.check()


@pytest.mark.gpu
def test_a_graph_gathers_4bit_rows_unchanged(cuda_device):
    from agnes_inputs import synth
    n, dim = 3000, 128
    off, ind = synth.rmat_csr(n, 8, 0.57, 0.19, 0.19, seed=5, offsets_dtype=torch.int64)
    packed = ops.mx4_quantize(_values(n, dim, 4).to(cuda_device))
    w = ops.mx4_quantize(_values(64, dim, 6).to(cuda_device))
    whole = ops.mx4_linear(packed, w, dim)
    with Graph(off.to(cuda_device), ind.to(cuda_device), packed.view(torch.float16)) as g:
        g.prepare(torch.arange(40, dtype=torch.int32, device=cuda_device).view(1, 40), [5, 3], 7)
        mb = g.fetch(0)
        assert torch.equal(mb.feats.view(torch.uint8), packed[mb.nodes.long()])
        assert torch.equal(ops.mx4_linear(mb.feats, w, dim), whole[mb.nodes.long()])
    ops.check()


@pytest.mark.gpu
@pytest.mark.parametrize("out", FLOATS)
def test_product_of_a_ragged_last_tile_each_time(cuda_device, out):
    """The CTA that ends with a tile of fewer rows stores the whole of the one before:
    the warps without rows in the last tile leave their buffers alone."""
    rows, width, dim = 40_000, 256, 128
    x = ops.mx4_quantize(_values(rows, dim, 1).to(cuda_device))
    w = ops.mx4_quantize(_values(width, dim, 2).to(cuda_device))
    b = torch.ones(width, device=cuda_device)
    got = torch.empty(rows, width, dtype=out, device=cuda_device)
    ops.mx4_linear(x, w, dim, b, out=got)
    first = got.clone()
    differ = torch.zeros((), dtype=torch.int64, device=cuda_device)
    for _ in range(2000):
        got.zero_()
        ops.mx4_linear(x, w, dim, b, out=got)
        differ += (got != first).sum()
    assert int(differ) == 0


@pytest.mark.gpu
def test_products_on_two_streams_at_once(cuda_device):
    """Kernels that each want all of an SM's tensor memory, side by side."""
    cases = []
    for seed, (rows, width, dim) in enumerate([(40_000, 256, 128), (9000, 500, 640)]):
        x = ops.mx4_quantize(_values(rows, dim, seed).to(cuda_device))
        w = ops.mx4_quantize(_values(width, dim, seed + 9).to(cuda_device))
        cases.append((x, w, dim, ops.mx4_linear(x, w, dim), torch.cuda.Stream()))
    torch.cuda.synchronize()
    got = [[ops.mx4_linear(x, w, dim, stream=stream) for x, w, dim, _, stream in cases]
           for _ in range(20)]
    torch.cuda.synchronize()
    for outs in got:
        for out, (_, _, _, ref, _) in zip(outs, cases):
            assert torch.equal(out, ref)
    ops.check()


@pytest.mark.gpu
def test_product_offsets_past_32_bits(cuda_device):
    rows, width, dim = 9_000_000, 256, 32  # 2.3e9 values of the output
    part = reference_rows(_values(7, dim, 3))
    x = torch.zeros(rows, row_bytes(dim), dtype=torch.uint8, device=cuda_device)
    at = torch.tensor([0, 1, 8_388_607, 8_388_608, 8_388_609, rows - 2, rows - 1],
                      device=cuda_device)
    x[at] = part.to(cuda_device)
    w = reference_rows(_values(width, dim, 4))
    y = ops.mx4_linear(x, w.to(cuda_device), dim, out_dtype=torch.float16)
    xv, wv = reference_values(part, dim), reference_values(w, dim)
    ref, size = xv @ wv.t(), xv.abs() @ wv.abs().t()
    assert_within(y[at], ref, (dim + 2) * 2 * U32 * size + 1.01 * rounding(ref, y.dtype) + 1e-30)
    assert int((y != 0).any(1).sum()) <= 7
    ops.check()


@pytest.mark.gpu
@pytest.mark.parametrize("dim", [8, 9, 15, 31, 33, 39, 63, 301, 8191, 8193, 12_345])
@pytest.mark.parametrize("out", FLOATS)
def test_back_from_rows_that_are_not_whole_eights(cuda_device, dim, out):
    for rows in (1, 2, 3 + 30_000 // dim):
        packed = reference_rows(_values(rows, dim, rows))
        got = ops.mx4_dequantize(packed.to(cuda_device), dim, out_dtype=out).cpu()
        assert torch.equal(got, reference_values(packed, dim).to(out))


def _product_of_values(dev, xv, wv, out=torch.float32):
    """(product, its value in 64 bits, the bound of the difference) of xv and wv in 4 bits."""
    dim = xv.shape[1]
    x, w = reference_rows(xv), reference_rows(wv)
    xv, wv = reference_values(x, dim), reference_values(w, dim)
    ref, size = xv @ wv.t(), xv.abs() @ wv.abs().t()
    got = ops.mx4_linear(x.to(dev), w.to(dev), dim, out_dtype=out)
    return got, ref, (dim + 2) * 2 * U32 * size + 1.01 * rounding(ref, out) + 1e-30


@pytest.mark.gpu
@pytest.mark.parametrize("rows", [1, 2, 4, 8, 9, 150])
@pytest.mark.parametrize("large,small,used", [(2.0 ** 126, 2.0 ** -20, 96), (3.4e38, 0.1, 8),
                                              (2.0 ** 120, 2.0 ** -120, 96)])
def test_a_finite_product_of_far_apart_scales_is_finite(cuda_device, rows, large, small, used):
    """Whichever side has the large values, and where blocks cancel one another.  The sum of the
    magnitudes is in fp32's range, and so is every partial sum."""
    g = gen(rows)
    dim, width = 96, 20
    column = torch.arange(dim)
    sign = torch.where(column < 32, 1.0, -1.0)
    sign[(column < 32 - used // 2) | (column >= 32 + used // 2)] = 0
    for x_scale, w_scale in ((large, small), (small, large)):
        xv = (torch.rand(rows, dim, generator=g) / 2 + 0.5) * x_scale * sign
        wv = (torch.rand(width, dim, generator=g) / 2 + 0.5) * w_scale
        wv[1] *= -1
        assert xv.abs().max() * wv.abs().max() * used < 3e38
        got, ref, bound = _product_of_values(cuda_device, xv, wv)
        assert got.isfinite().all()
        assert_within(got, ref, bound)
    ops.check()


@pytest.mark.gpu
@pytest.mark.parametrize("rows", [2, 150])
def test_a_product_past_fp32_is_infinite(cuda_device, rows):
    xv = torch.full((rows, 64), 2.0 ** 100)
    wv = torch.full((3, 64), 2.0 ** 100)
    wv[1] *= -1
    wv[2] = 0
    got = ops.mx4_linear(*(ops.mx4_quantize(v.to(cuda_device)) for v in (xv, wv)), 64).cpu()
    assert (got[:, 0] == math.inf).all() and (got[:, 1] == -math.inf).all()
    assert (got[:, 2] == 0).all()


@pytest.mark.gpu
@pytest.mark.parametrize("out", FLOATS)
@pytest.mark.parametrize("rows,width,dim", [(20_000, 600, 500), (9000, 900, 640),
                                            (9000, 900, 1024), (20_000, 500, 1100)])
def test_product_of_several_tiles_a_cta(cuda_device, out, rows, width, dim):
    """Rows of two stages and more, odd and even, over more tiles than there are CTAs."""
    x = ops.mx4_quantize(_values(rows, dim, 1).to(cuda_device))
    w = ops.mx4_quantize(_values(width, dim, 2).to(cuda_device))
    b = torch.randn(width, generator=gen(3))
    got = ops.mx4_linear(x, w, dim, b.to(cuda_device), out_dtype=out)
    xv, wv = (reference_values(v.cpu(), dim).to(cuda_device) for v in (x, w))
    ref, size = xv @ wv.t() + b.to(cuda_device).double(), xv.abs() @ wv.abs().t()
    size += b.to(cuda_device).double().abs()
    assert_within(got, ref, (dim + 2) * 2 * U32 * size + 1.01 * rounding(ref, out) + 1e-30)
    ops.check()


@pytest.mark.gpu
@pytest.mark.parametrize("out", FLOATS)
@pytest.mark.parametrize("dim", [9, 33, 301])
def test_back_from_strided_rows_that_are_not_whole_eights(cuda_device, out, dim):
    """Rows apart, and bytes between them that would be NaN if they were read as scales."""
    rows, n = 700, row_bytes(dim)
    packed = reference_rows(_values(rows, dim, dim))
    wide = torch.full((rows, n + 48), 255, dtype=torch.uint8, device=cuda_device)
    wide[:, 16:16 + n] = packed.to(cuda_device)
    got = ops.mx4_dequantize(wide[:, 16:16 + n], dim, out_dtype=out).cpu()
    assert torch.equal(got, reference_values(packed, dim).to(out))
