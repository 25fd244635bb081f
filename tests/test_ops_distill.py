"""Distillation from a teacher's top logits (include/agnes_ops.h) against its
formula in 64 bits."""
import math

import pytest
import torch

from ops_support import FLOATS, U32, assert_within, gen, rounding
from paper_2601_01473_gb300 import AgnesError, ops

INF = math.inf


def _reference(x, t, at, temperature, weight):
    """(loss, gradient, bound of loss, bound of gradient before its rounding)."""
    T = temperature
    x, t, at = x.double(), t.double(), at.long()
    R, V = x.shape
    here = (at >= 0) & (at < V)
    t = torch.where(here, t, -INF)
    some = (t.amax(1) > -INF if t.shape[1] else torch.zeros(R, dtype=torch.bool)) & \
        (x.amax(1) > -INF)
    at = torch.where(here, at, 0)
    t = torch.where(some[:, None], t, 0.0)
    p = torch.softmax(t / T, 1) * some[:, None]
    x0 = torch.where(some[:, None], x, 0.0)
    log_q = torch.log_softmax(x0 / T, 1)
    q = log_q.exp() * some[:, None]
    lp, lq = torch.log_softmax(t / T, 1), log_q.gather(1, at)
    loss = T * T * torch.where(p > 0, p * (lp - lq), 0.0).sum(1)
    grad = q.scatter_add(1, at, -p) * (weight.double() * T)[:, None]
    # in fp32: exponentials to 2^-22 and their arguments' rounding (weighted by e^-a a < 0.4),
    # sums of V / 64 terms in a row at most and of the top entries
    rel = 2.0 ** -19 + (V / 64 + t.shape[1]) * U32
    far = (x0.amax(1, keepdim=True) - x0) / T
    size = torch.where(p > 0, p * (1 + lp.abs() + lq.abs() + far.gather(1, at)), 0.0).sum(1)
    mass = torch.zeros_like(q).scatter_add(1, at, p)
    far = torch.where(q > 0, far, 0.0)
    return (loss, grad, T * T * rel * size + 1e-30,
            (q * (rel + 4 * U32 * far) + mass * rel) * (weight.double() * T)[:, None] + 1e-30)


def _case(R, V, K, dtype, tdtype, seed, index=torch.int32):
    g = gen(seed)
    x = (torch.randn(R, V, generator=g) * 3).to(dtype)
    t = (torch.randn(R, K, generator=g) * 3).to(tdtype)
    at = torch.rand(R, V, generator=g).argsort(1)[:, :K] if V < 2000 else \
        (torch.randint(0, V, (R, 1), generator=g) + torch.arange(K) * (V // K)) % V
    at = at.to(index)
    at[torch.rand(R, K, generator=g) < 0.2] = -1
    if R > 2:
        at[2] = -1  # a row without a teacher
    return x, t, at, torch.rand(R, generator=g) + 0.1


def _run(dev, x, t, at, weight, T, out_dtype=None):
    x, t, at, weight = (v.to(dev) for v in (x, t, at, weight))
    loss, stats = ops.distill_loss(x, t, at, T)
    grad = ops.distill_grad(x, t, at, stats, weight, T, out_dtype=out_dtype)
    loss2, grad2 = ops.distill_loss_grad(x, t, at, weight, T, out_dtype=out_dtype)
    return loss, grad, loss2, grad2


def _check(dev, x, t, at, weight, T, out_dtype=None):
    ref_loss, ref_grad, loss_bound, grad_bound = _reference(x, t, at, T, weight)
    loss, grad, loss2, grad2 = _run(dev, x, t, at, weight, T, out_dtype)
    for got in (loss, loss2):
        assert_within(got, ref_loss, loss_bound)
    bound = grad_bound + 1.01 * rounding(ref_grad.abs() + grad_bound, out_dtype or x.dtype)
    for got in (grad, grad2):
        assert got.dtype == (out_dtype or x.dtype)
        assert_within(got, ref_grad, bound)


# ---- refusals (no GPU needed) -----------------------------------------------------------

def test_arguments_are_checked_before_any_device_is_used():
    x, t, at = torch.zeros(2, 5), torch.zeros(2, 1), torch.zeros(2, 1, dtype=torch.int64)
    with pytest.raises(ValueError, match="CUDA device"):
        ops.distill_loss(x, t, at)
    with pytest.raises(TypeError, match="2-D"):
        ops.distill_loss(x[0], t, at)


def test_the_c_entries_refuse_bad_arguments_without_a_device():
    from paper_2601_01473_gb300 import build
    build.build()
    L = ops.lib()
    args = [None, 0, 5, 2, 5, None, 0, None, 32, 1, 1.0, None, None, None, None]
    assert L.agnes_distill_loss(*args) == 1 and b"logits is NULL" in L.agnes_last_error(None)
    for at, value, status in ((1, 3, 1), (3, -1, 1), (4, 0, 1), (2, 4, 1), (6, -1, 1), (8, 8, 1),
                              (9, -1, 1), (9, 513, 2), (10, 0.0, 1), (10, -1.0, 1),
                              (10, math.nan, 1), (10, INF, 1), (4, (1 << 30) + 1, 2),
                              (3, 1 << 31, 2)):
        bad = list(args)
        bad[at] = value
        assert L.agnes_distill_loss(*bad) == status, (at, value)
    args[3] = 0
    assert L.agnes_distill_loss(*args) == 0


# ---- values ------------------------------------------------------------------------------

SIZES = [(1, 1, 1), (3, 2, 2), (5, 7, 3), (4, 31, 5), (9, 172, 5), (3, 1024, 16), (2, 4097, 64),
         (3, 10007, 33), (1, 50_001, 100), (2, 131_072, 512)]


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", FLOATS)
@pytest.mark.parametrize("R,V,K", SIZES)
def test_loss_and_gradient(cuda_device, dtype, R, V, K):
    for T in (1.0, 2.5):
        _check(cuda_device, *_case(R, V, K, dtype, dtype, R + V), T)
    ops.check()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", FLOATS)
@pytest.mark.parametrize("tdtype", FLOATS)
@pytest.mark.parametrize("out", FLOATS)
@pytest.mark.parametrize("index", [torch.int32, torch.int64])
def test_types(cuda_device, dtype, tdtype, out, index):
    _check(cuda_device, *_case(6, 333, 9, dtype, tdtype, 3, index), 0.7, out)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", FLOATS)
@pytest.mark.parametrize("V", [513, 4001, 8192, 8193, 16_385])
def test_many_rows_of_more_classes(cuda_device, dtype, V):
    _check(cuda_device, *_case(1300, V, 7, dtype, torch.float32, V), 1.5)


@pytest.mark.gpu
def test_many_rows_of_many_classes(cuda_device):
    """Rows that are a warp's for the loss alone, at both ends of what is, checked against the
    same rows taken a few at a time."""
    for V in (65_536, 65_537):
        g = torch.Generator(device=cuda_device).manual_seed(V)
        x = torch.randn(1300, V, generator=g, device=cuda_device).half()
        t = torch.randn(1300, 5, generator=g, device=cuda_device)
        at = torch.randint(0, V, (1300, 5), generator=g, device=cuda_device)
        loss, stats = ops.distill_loss(x, t, at, 2.0)
        for part in (slice(0, 4), slice(1296, 1300)):
            ref, _, bound, _ = _reference(x[part].cpu(), t[part].cpu(), at[part].cpu(), 2.0,
                                          torch.ones(4))
            assert_within(loss[part], ref, bound)
            few, few_stats = ops.distill_loss(x[part], t[part], at[part], 2.0)
            assert_within(few, ref, bound)
            assert torch.equal(stats[part, 0], few_stats[:, 0])


@pytest.mark.gpu
@pytest.mark.parametrize("rows", [200, 2000, 70_000])
def test_many_rows(cuda_device, rows):
    _check(cuda_device, *_case(rows, 40, 4, torch.float16, torch.float32, 8), 2.0)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", FLOATS)
def test_rows_past_shared_memory(cuda_device, dtype):
    """A slice of an eighth of the row is more than a CTA keeps."""
    _check(cuda_device, *_case(2, 1_000_003, 7, dtype, dtype, 12), 3.0)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", FLOATS)
@pytest.mark.parametrize("V", [350_003, 409_088, 409_217, 818_688])
def test_rows_that_fill_shared_memory(cuda_device, dtype, V):
    """Slices up to the most that a CTA keeps, and just past it."""
    _check(cuda_device, *_case(2, V, 9, dtype, dtype, V), 2.0)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", FLOATS)
def test_strides_and_alignments(cuda_device, dtype):
    R, V, K = 4, 1000, 6
    x, t, at, w = _case(R, V, K, dtype, torch.float32, 21)
    ref = _run(cuda_device, x, t, at, w, 2.0)
    for first in range(0, 8):
        for out_first in (0, 1, 3):
            wide = torch.full((R, V + 21), 77.0, dtype=dtype, device=cuda_device)
            wide[:, first:first + V] = x.to(cuda_device)
            out = torch.full((R, V + 33), 77.0, dtype=dtype, device=cuda_device)
            got = ops.distill_loss_grad(wide[:, first:first + V], t.to(cuda_device),
                                        at.to(cuda_device), w.to(cuda_device), 2.0,
                                        out=out[:, out_first:out_first + V])
            # what is added to what follows the alignment: a few roundings of fp32
            assert torch.allclose(got[0], ref[2], rtol=2e-5, atol=1e-6)
            assert (got[1].float() - ref[3].float()).abs().max() <= \
                2 * rounding(ref[3].float().abs().max(), dtype)
            assert (out[:, :out_first] == 77).all() and (out[:, out_first + V:] == 77).all()


@pytest.mark.gpu
@pytest.mark.parametrize("V", [50, 3000, 40_000, 500_001])
def test_in_place(cuda_device, V):
    x, t, at, w = (v.to(cuda_device) for v in _case(3, V, 5, torch.float32, torch.float32, V))
    loss, grad = ops.distill_loss_grad(x, t, at, w, 2.0)
    _, stats = ops.distill_loss(x, t, at, 2.0)
    apart = ops.distill_grad(x, t, at, stats, w, 2.0)
    y = x.clone()
    loss2, got = ops.distill_loss_grad(y, t, at, w, 2.0, out=y)
    assert got.data_ptr() == y.data_ptr()
    assert torch.equal(loss, loss2) and torch.equal(grad, y)
    y = x.clone()
    ops.distill_grad(y, t, at, stats, w, 2.0, out=y)
    assert torch.equal(apart, y)


@pytest.mark.gpu
def test_entries_that_name_the_same_class(cuda_device):
    x, t, at, w = _case(3, 500, 8, torch.float32, torch.float32, 4)
    at[0] = 7
    at[1] = torch.tensor([3, 4, 3, -1, 4, 3, 499, 0], dtype=at.dtype)
    _check(cuda_device, x, t, at, w, 1.3)


@pytest.mark.gpu
def test_masked_classes_and_rows(cuda_device):
    for V in (6, 5000, 60_000):
        for dtype in FLOATS:
            x, t, at, w = _case(6, V, 4, dtype, torch.float32, V)
            at[:] = torch.tensor([1, 2, 0, -1], dtype=at.dtype)
            lowest = torch.finfo(dtype).min
            x[0, 3:] = -INF                 # masked classes
            x[1, 3:] = lowest               # masked by the type's lowest value
            x[2] = -INF                     # nothing left: no loss, no gradient
            x[3] = lowest                   # uniform
            x[4, 1] = -INF                  # the teacher's class is masked: loss +inf
            t[5] = -INF                     # no teacher
            for T in (0.5, 1.0):
                loss, grad, loss2, grad2 = _run(cuda_device, x, t, at, w, T)
                ref_loss, ref_grad, lb, gb = _reference(x, t, at, T, w)
                for got in (loss.cpu(), loss2.cpu()):
                    assert got[2] == 0 and got[5] == 0 and got[4] == INF
                    keep = [0, 1, 3]
                    assert_within(got[keep], ref_loss[keep], lb[keep])
                for got in (grad, grad2):
                    assert (got[2] == 0).all() and (got[5] == 0).all()
                    bound = gb + 1.01 * rounding(ref_grad.abs() + gb, dtype)
                    assert_within(got, ref_grad, bound)


@pytest.mark.gpu
def test_infinities_and_nan(cuda_device):
    for V in (9, 30_000):
        x, t, at, w = _case(6, V, 4, torch.float32, torch.float32, V)
        at[:] = torch.tensor([1, 2, 0, -1], dtype=at.dtype)
        x[0, 5] = math.nan
        x[1, 5] = INF
        t[2, 1] = math.nan
        t[3, 1] = INF
        t[4, 3] = math.nan                  # an absent entry's value is not looked at
        x[5] = -INF
        x[5, 4] = math.nan
        for got_loss, got_grad in (_run(cuda_device, x, t, at, w, 2.0)[:2],
                                   _run(cuda_device, x, t, at, w, 2.0)[2:]):
            assert got_loss.isnan().tolist() == [True, True, True, True, False, True]
            assert got_grad.isnan().all(1).tolist() == [True, True, True, True, False, True]


@pytest.mark.gpu
def test_a_label_is_the_top_entry_alone(cuda_device):
    g = gen(6)
    x = torch.randn(20, 40, generator=g)
    label = torch.randint(0, 40, (20, 1), generator=g)
    label[3] = -1
    loss, grad = ops.distill_loss_grad(x.to(cuda_device), torch.zeros(20, 1, device=cuda_device),
                                       label.to(cuda_device), 1 / 20)
    y = x.double().requires_grad_()
    ref = torch.nn.functional.cross_entropy(y, label[:, 0], ignore_index=-1, reduction="none")
    (ref.sum() / 20).backward()
    assert_within(loss, ref.detach(), 2.0 ** -18 * (1 + ref.detach()))
    assert_within(grad, y.grad, torch.full_like(y.grad, 2.0 ** -18 / 20))


@pytest.mark.gpu
def test_an_index_past_the_end_is_left_out_and_reported(cuda_device):
    x, t, at, w = _case(2, 20, 3, torch.float32, torch.float32, 1, torch.int64)
    at[0] = torch.tensor([4, 20, 2 ** 40])
    at[1] = torch.tensor([19, -7, 0])
    got = _run(cuda_device, x, t, at, w, 1.0)
    with pytest.raises(AgnesError, match="past the end"):
        ops.check()
    ref = _reference(x, t, at, 1.0, w)
    assert_within(got[0], ref[0], ref[2])
    assert_within(got[3], ref[1], ref[3] + 1.01 * rounding(ref[1], x.dtype))


@pytest.mark.gpu
def test_nothing(cuda_device):
    at = torch.zeros(0, 3, dtype=torch.int32, device=cuda_device)
    x, t = torch.zeros(0, 7, device=cuda_device), torch.zeros(0, 3, device=cuda_device)
    loss, grad = ops.distill_loss_grad(x, t, at)
    assert loss.shape == (0,) and grad.shape == (0, 7)
    x = torch.randn(4, 7, device=cuda_device)
    loss, grad = ops.distill_loss_grad(x, t.new_zeros(4, 0), at.new_zeros(4, 0))
    assert (loss == 0).all() and (grad == 0).all()


@pytest.mark.gpu
def test_gradient_against_differences(cuda_device):
    R, V, K, T = 3, 12, 4, 1.7
    x, t, at, w = (v.to(cuda_device) for v in _case(R, V, K, torch.float32, torch.float32, 5))
    _, grad = ops.distill_loss_grad(x, t, at, w, T)
    h = 2.0 ** -6
    for v in range(V):
        up, down = x.clone(), x.clone()
        up[:, v] += h
        down[:, v] -= h
        step = (up[:, v] - down[:, v]).double()
        slope = (ops.distill_loss(up, t, at, T)[0].double()
                 - ops.distill_loss(down, t, at, T)[0].double()) * w / step
        # h^2 / 6 times the third derivative (below 1 / T at these values) and the losses'
        # roundings (about 1e-6 of 20) over the step
        assert ((slope - grad[:, v].double()).abs() <= w * (h * h / 6 + 2 * 2e-5 / (2 * h))).all()


@pytest.mark.gpu
def test_streams_and_graphs(cuda_device):
    x, t, at, w = (v.to(cuda_device) for v in _case(64, 9000, 8, torch.float16, torch.float32, 2))
    loss, grad = ops.distill_loss_grad(x, t, at, w, 2.0)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    loss2, grad2 = ops.distill_loss_grad(x, t, at, w, 2.0, stream=side)
    torch.cuda.synchronize()
    assert torch.equal(loss, loss2) and torch.equal(grad, grad2)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        loss3, grad3 = ops.distill_loss_grad(x, t, at, w, 2.0)
    graph.replay()
    assert torch.equal(loss, loss3) and torch.equal(grad, grad3)


@pytest.mark.gpu
def test_refusals_on_the_device(cuda_device):
    x = torch.zeros(2, 5, device=cuda_device)
    t = torch.zeros(2, 3, device=cuda_device)
    at = torch.zeros(2, 3, dtype=torch.int32, device=cuda_device)
    with pytest.raises(ValueError, match="top"):
        ops.distill_loss(x, t[:1], at[:1])
    with pytest.raises(ValueError, match="top"):
        ops.distill_loss(x, t, at[:, :2].contiguous())
    with pytest.raises(AgnesError, match="temperature"):
        ops.distill_loss(x, t, at, 0.0)
    with pytest.raises(AgnesError, match="ERANGE"):
        ops.distill_loss(x, t.new_zeros(2, 513), at.new_zeros(2, 513))
    with pytest.raises(TypeError, match="weight"):
        ops.distill_loss_grad(x, t, at, torch.ones(3, device=cuda_device))
    with pytest.raises(TypeError, match="stats"):
        ops.distill_grad(x, t, at, torch.zeros(2, device=cuda_device))
    with pytest.raises(TypeError, match="out"):
        ops.distill_loss_grad(x, t, at, out=torch.zeros(2, 5, device=cuda_device),
                              out_dtype=torch.float16)


@pytest.mark.gpu
def test_offsets_past_32_bits(cuda_device):
    R, V, K = 60_000, 50_000, 4  # 3e9 logits
    x = torch.zeros(R, V, dtype=torch.float16, device=cuda_device)
    part, t, at, w = _case(5, V, K, torch.float16, torch.float32, 31)
    rows = torch.tensor([0, 1, 42_949, 42_950, R - 1], device=cuda_device)
    x[rows] = part.to(cuda_device)
    teacher = torch.zeros(R, K, device=cuda_device)
    index = torch.full((R, K), -1, dtype=torch.int32, device=cuda_device)
    weight = torch.ones(R, device=cuda_device)
    teacher[rows], index[rows], weight[rows] = (v.to(cuda_device) for v in (t, at, w))
    ref_loss, ref_grad, loss_bound, grad_bound = _reference(part, t, at, 2.0, w)
    bound = grad_bound + 1.01 * rounding(ref_grad.abs() + grad_bound, x.dtype)
    _, stats = ops.distill_loss(x, teacher, index, 2.0)
    grad = ops.distill_grad(x, teacher, index, stats, weight, 2.0)
    assert_within(grad[rows], ref_grad, bound)
    del grad
    loss, grad = ops.distill_loss_grad(x, teacher, index, weight, 2.0, out=x)  # in place
    assert_within(loss[rows], ref_loss, loss_bound)
    assert_within(grad[rows], ref_grad, bound)
    assert (loss.sum() - loss[rows].sum()).abs() == 0


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", FLOATS)
@pytest.mark.parametrize("V", [6, 5000, 60_000])
@pytest.mark.parametrize("T", [0.25, 0.5, 2.0])
def test_a_teacher_of_classes_masked_by_the_lowest_value(cuda_device, dtype, V, T):
    """The loss is large and finite wherever the formula's is: differences of logits beyond the
    type's range, over T, and T^2 of it do not leave fp32 on the way."""
    x, t, at, w = _case(4, V, 4, dtype, torch.float32, V)
    at[:] = torch.tensor([1, 2, 4, 5], dtype=at.dtype)
    lowest, most = torch.finfo(dtype).min, torch.finfo(dtype).max
    x[:, 3:] = lowest                # two of the teacher's classes
    x[1, 0] = most / 4               # and the others are far below the largest
    x[2, 0] = most
    t[3, 2:] = t[3, :2].max() - 40 * T  # almost nothing on the masked ones
    _check(cuda_device, x, t, at, w, T)
    ref = _reference(x, t, at, T, w)[0]
    got = ops.distill_loss(*(v.to(cuda_device) for v in (x, t, at)), T)[0].cpu()
    assert got.isfinite()[ref < 3e38].all()
