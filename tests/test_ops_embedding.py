"""Embedding lookup and its gradient (include/agnes_ops.h) against their
formulas in 64 bits."""
import pytest
import torch

from ops_support import FLOATS, U32, assert_within, gen, rounding
from paper_2601_01473_gb300 import AgnesError, ops


def _lookup_ref(table, ids, scale):
    ids = ids.reshape(-1).long()
    ref = torch.zeros((ids.numel(), table.shape[1]), dtype=torch.float64)
    real = (ids >= 0) & (ids < table.shape[0])
    ref[real] = table[ids[real]].double() * scale
    return ref


def _grad_ref(grad, ids, rows, scale):
    """(d, sum of magnitudes, tokens) of every row of the table."""
    ids = ids.reshape(-1).long()
    real = (ids >= 0) & (ids < rows)
    d = torch.zeros((rows, grad.shape[1]), dtype=torch.float64)
    size = torch.zeros_like(d)
    d.index_add_(0, ids[real], grad[real].double() * scale)
    size.index_add_(0, ids[real], grad[real].double().abs() * abs(scale))
    return d, size, torch.bincount(ids[real], minlength=rows).double()[:, None]


def _grad_bound(d, size, tokens, dtype):
    # a sum of m terms in fp32, in any order, the scale's rounding and the product's
    return (tokens + 3) * U32 * size * 1.01 + rounding(d, dtype) * 1.01


# ---- refusals (no GPU needed) ---------------------------------------------------------

def test_arguments_are_checked_before_any_device_is_used():
    table, ids = torch.zeros(4, 8), torch.zeros(3, dtype=torch.int32)
    with pytest.raises(ValueError, match="CUDA device"):
        ops.embedding_lookup(table, ids)
    with pytest.raises(TypeError, match="2-D"):
        ops.embedding_lookup(table[0], ids)
    with pytest.raises(TypeError, match="2-D"):
        ops.embedding_lookup(table.double(), ids)
    with pytest.raises(TypeError, match="2-D"):
        ops.embedding_grad(torch.zeros(3, dtype=torch.int8), ids, 4)


def test_the_c_entries_refuse_bad_arguments_without_a_device():
    import ctypes

    from paper_2601_01473_gb300 import build
    build.build()
    L = ops.lib()
    need = ctypes.c_int64()
    assert L.agnes_embedding_grad_workspace(10, 0, ctypes.byref(need)) == 1
    assert L.agnes_embedding_grad_workspace(10, 4, None) == 1
    assert L.agnes_embedding_grad_workspace(1 << 31, 4, ctypes.byref(need)) == 2
    assert L.agnes_embedding_grad_workspace(1000, 4, ctypes.byref(need)) == 0
    assert need.value >= 16 * 1000
    args = [None, 0, 10, 8, 8, None, 32, 3, 1.0, None, 0, 8, None, None]
    assert L.agnes_embedding_lookup(*args) == 1
    assert b"NULL" in L.agnes_last_error(None)
    for at, value, status in ((1, 7, 1), (10, -1, 1), (6, 16, 1), (4, 0, 1), (2, -1, 1), (7, -1, 1),
                              (3, 7, 1), (11, 7, 1), (2, 1 << 31, 2), (7, 1 << 31, 2)):
        bad = list(args)
        bad[at] = value
        assert L.agnes_embedding_lookup(*bad) == status, (at, value)
    args[7] = 0  # nothing to do
    assert L.agnes_embedding_lookup(*args) == 0


# ---- lookup --------------------------------------------------------------------------

@pytest.mark.gpu
@pytest.mark.parametrize("tin", FLOATS)
@pytest.mark.parametrize("tout", FLOATS)
@pytest.mark.parametrize("n,rows,dim", [(1, 1, 1), (5, 3, 7), (1000, 77, 128), (333, 1000, 130),
                                        (9, 5, 1000), (3, 4, 5001), (2048, 10, 2)])
def test_lookup(cuda_device, tin, tout, n, rows, dim):
    g = gen(n + dim)
    table = torch.randn(rows, dim, generator=g).to(tin)
    ids = torch.randint(-1, rows, (n,), generator=g, dtype=torch.int64)
    for scale in (1.0, 11.25):
        got = ops.embedding_lookup(table.to(cuda_device), ids.to(cuda_device), scale,
                                   out_dtype=tout)
        ref = _lookup_ref(table, ids, scale)
        assert got.dtype == tout
        # both scales are exact in fp32: the product's rounding, then the output's
        assert_within(got, ref, ref.abs() * U32 + rounding(ref, tout) * 1.01)
    ops.check()


@pytest.mark.gpu
@pytest.mark.parametrize("index", [torch.int32, torch.int64])
def test_lookup_strides_shapes_and_views(cuda_device, index):
    g = gen(3)
    wide = torch.randn(50, 3 * 40 + 1, generator=g)
    ids = torch.randint(-1, 50, (4, 6), generator=g, dtype=index)
    for first in (0, 1, 3):  # alignments of the rows' starts
        table = wide.to(cuda_device)[:, first:first + 40]
        out = torch.full((24, 100), 7.0, device=cuda_device)
        got = ops.embedding_lookup(table, ids.to(cuda_device), 2.0, out=out[:, 5:45])
        assert got.data_ptr() == out[:, 5:45].data_ptr()
        assert torch.equal(out[:, 5:45].cpu(), _lookup_ref(table.cpu(), ids, 2.0).float())
        assert (out[:, :5] == 7).all() and (out[:, 45:] == 7).all()
        assert ops.embedding_lookup(table, ids.to(cuda_device)).shape == (4, 6, 40)
    ops.check()


@pytest.mark.gpu
def test_lookup_special_values_and_empty(cuda_device):
    table = torch.tensor([[float("inf"), float("nan"), -0.0, 65504.0]], device=cuda_device)
    ids = torch.tensor([0, -1, -5], device=cuda_device)
    got = ops.embedding_lookup(table, ids, 2.0, out_dtype=torch.float16).cpu()
    assert got[0, 0] == float("inf") and got[0, 1].isnan() and got[0, 3] == float("inf")
    assert torch.equal(got[1:], torch.zeros(2, 4, dtype=torch.float16))
    assert ops.embedding_lookup(table, ids[:0]).shape == (0, 4)
    assert (ops.embedding_lookup(table[:0], ids[1:]) == 0).all()
    ops.check()


@pytest.mark.gpu
def test_lookup_past_the_end_is_reported(cuda_device):
    table = torch.ones(10, 16, device=cuda_device)
    for bad in (10, 2 ** 31 - 1):
        ids = torch.tensor([3, bad, 9], device=cuda_device)
        status = torch.zeros(1, dtype=torch.int32, device=cuda_device)
        got = ops.embedding_lookup(table, ids, status=status)
        assert got.sum(1).tolist() == [16, 0, 16]
        assert int(status) == ops.BAD_INDEX
        ops.embedding_lookup(table, ids)
        with pytest.raises(AgnesError, match="past the end"):
            ops.check()
        ops.check()  # cleared
    huge = torch.tensor([2 ** 40], device=cuda_device)
    assert (ops.embedding_lookup(table, huge) == 0).all()
    with pytest.raises(AgnesError):
        ops.check()


@pytest.mark.gpu
def test_lookup_offsets_past_32_bits(cuda_device):
    rows, dim = 40_000_000, 128  # 5.1e9 elements
    table = torch.empty(rows, dim, dtype=torch.float16, device=cuda_device)
    ids = torch.tensor([0, 1, 16_777_216, 33_554_432, rows - 1], device=cuda_device)
    want = torch.randn(5, dim, generator=gen(5)).half().to(cuda_device)
    table[ids] = want
    assert torch.equal(ops.embedding_lookup(table, ids), want)


# ---- gradient --------------------------------------------------------------------------

def _case(n, rows, dim, tin, skew, seed, index=torch.int32, padding=True):
    g = gen(seed)
    grad = torch.randn(n, dim, generator=g).to(tin)
    u = torch.rand(n, generator=g, dtype=torch.float64)
    ids = ((u ** skew) * rows).long().clamp(max=rows - 1) * 7919 % rows
    if padding:
        ids[torch.rand(n, generator=g) < 0.05] = -1
    return grad, ids.to(index)


@pytest.mark.gpu
@pytest.mark.parametrize("tin", FLOATS)
@pytest.mark.parametrize("tout", FLOATS)
@pytest.mark.parametrize("n,rows,dim,skew", [
    (1, 1, 1, 1), (2, 5, 3, 1), (31, 7, 130, 1), (33, 1000, 16, 1), (64, 1, 33, 1),
    (4096, 50, 24, 2), (4097, 5000, 8, 1), (9000, 3, 130, 1), (20000, 40000, 65, 3),
    (100_000, 100, 9, 4)])
def test_gradient(cuda_device, tin, tout, n, rows, dim, skew):
    scale = 1.5
    grad, ids = _case(n, rows, dim, tin, skew, n + dim)
    d, size, tokens = _grad_ref(grad, ids, rows, scale)
    bound = _grad_bound(d, size, tokens, tout)
    dense = ops.embedding_grad(grad.to(cuda_device), ids.to(cuda_device), rows, scale,
                               out_dtype=tout)
    assert dense.dtype == tout
    assert_within(dense, d, bound)
    r = ops.embedding_grad_rows(grad.to(cuda_device), ids.to(cuda_device), rows, scale,
                                out_dtype=tout)
    hit = torch.nonzero(tokens[:, 0])[:, 0]
    c = hit.numel()
    assert r.count.tolist() == [c]
    assert torch.equal(r.ids[:c].cpu().long(), hit) and (r.ids[c:] == -1).all()
    assert torch.equal(r.rows[:c].cpu(), dense.cpu()[hit])  # the same sums, bit by bit
    assert (r.rows[c:] == 0).all()
    ops.check()


@pytest.mark.gpu
def test_gradient_of_a_large_table_and_wide_ids(cuda_device):
    for rows in (2 ** 31 - 1, 10_000_000):
        grad, ids = _case(30_000, rows, 12, torch.float32, 2, 5, torch.int64)
        ids[17] = rows - 1
        r = ops.embedding_grad_rows(grad.to(cuda_device), ids.to(cuda_device), rows)
        real = ids >= 0
        node, where = torch.unique(ids[real], return_inverse=True)
        c = node.numel()
        assert r.count.tolist() == [c] and torch.equal(r.ids[:c].cpu().long(), node)
        d = torch.zeros((c, 12), dtype=torch.float64)
        size = torch.zeros_like(d)
        d.index_add_(0, where, grad[real].double())
        size.index_add_(0, where, grad[real].double().abs())
        tokens = torch.bincount(where).double()[:, None]
        assert_within(r.rows[:c], d, _grad_bound(d, size, tokens, torch.float32))
    ops.check()


@pytest.mark.gpu
@pytest.mark.parametrize("n", [1, 5000, 50_000])
def test_gradient_without_any_real_id(cuda_device, n):
    grad = torch.full((n, 10), float("nan"), device=cuda_device)
    ids = torch.full((n,), -1, dtype=torch.int32, device=cuda_device)
    assert (ops.embedding_grad(grad, ids, 20) == 0).all()
    r = ops.embedding_grad_rows(grad, ids, 20)
    assert r.count.tolist() == [0] and (r.ids == -1).all() and (r.rows == 0).all()
    ops.check()


@pytest.mark.gpu
def test_gradient_of_nothing(cuda_device):
    grad = torch.zeros(0, 10, device=cuda_device)
    ids = torch.zeros(0, dtype=torch.int64, device=cuda_device)
    assert (ops.embedding_grad(grad, ids, 20) == 0).all()
    r = ops.embedding_grad_rows(grad, ids, 20)
    assert r.count.tolist() == [0] and r.rows.shape == (0, 10)
    assert ops.embedding_grad(grad, ids, 0).shape == (0, 10)


@pytest.mark.gpu
def test_gradient_past_the_end_is_left_out_and_reported(cuda_device):
    for n in (6, 6000):
        grad = torch.ones(n, 4, device=cuda_device)
        ids = torch.full((n,), 3, device=cuda_device)
        ids[1], ids[4] = 10, 2 ** 35
        got = ops.embedding_grad(grad, ids, 10)
        with pytest.raises(AgnesError, match="past the end"):
            ops.check()
        assert got[3].tolist() == [n - 2.0] * 4 and got.sum() == 4 * (n - 2)


@pytest.mark.gpu
def test_gradient_is_the_same_each_time_and_on_any_stream(cuda_device):
    grad, ids = _case(200_000, 1000, 40, torch.float16, 4, 9)
    grad, ids = grad.to(cuda_device), ids.to(cuda_device)
    first = ops.embedding_grad(grad, ids, 1000, out_dtype=torch.float32)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    for stream in (None, side):
        again = ops.embedding_grad(grad, ids, 1000, out_dtype=torch.float32, stream=stream)
        torch.cuda.synchronize()
        assert torch.equal(first, again)


@pytest.mark.gpu
def test_gradient_in_a_cuda_graph(cuda_device):
    grad, ids = _case(10_000, 500, 32, torch.float32, 2, 11)
    grad, ids = grad.to(cuda_device), ids.to(cuda_device)
    ops.embedding_grad(grad, ids, 500)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = ops.embedding_grad(grad, ids, 500)
    grad.mul_(-2)
    graph.replay()
    assert torch.equal(got, ops.embedding_grad(grad, ids, 500))


@pytest.mark.gpu
def test_gradient_against_differences(cuda_device):
    """d(sum of g * lookup) / d table[v], by central differences in the table."""
    rows, dim = 6, 5
    g = gen(2)
    table = torch.randn(rows, dim, generator=g)
    ids = torch.tensor([0, 3, 3, -1, 5, 3, 0], dtype=torch.int32)
    out_grad = torch.randn(7, dim, generator=g)
    scale, h = 3.0, 0.5  # linear in the table: the step only scales the rounding
    got = ops.embedding_grad(out_grad.to(cuda_device), ids.to(cuda_device), rows, scale).cpu()

    def value(t):
        y = ops.embedding_lookup(t.to(cuda_device), ids.to(cuda_device), scale).cpu()
        return (y.double() * out_grad.double()).sum()

    for v in range(rows):
        for c in range(dim):
            up, down = table.clone(), table.clone()
            up[v, c] += h
            down[v, c] -= h
            step = float(up[v, c].double() - down[v, c].double())
            slope = float(value(up) - value(down)) / step
            # the lookups round to fp32: 21 products of about 10, over the step
            assert abs(slope - float(got[v, c])) <= 21 * 10 * 2 * U32 * 4 / step + 1e-5


@pytest.mark.gpu
def test_refusals_on_the_device(cuda_device):
    table = torch.zeros(10, 8, device=cuda_device)
    ids = torch.zeros(4, dtype=torch.int32, device=cuda_device)
    with pytest.raises(TypeError):
        ops.embedding_lookup(table, ids.float())
    with pytest.raises(TypeError):
        ops.embedding_lookup(table, ids, out_dtype=torch.float64)
    with pytest.raises(ValueError, match="contiguous"):
        ops.embedding_lookup(table, torch.zeros(8, dtype=torch.int32, device=cuda_device)[::2])
    with pytest.raises(ValueError, match="adjacent"):
        ops.embedding_lookup(table.t(), ids)
    with pytest.raises(ValueError, match="CUDA device"):
        ops.embedding_lookup(table, ids.cpu())
    with pytest.raises(ValueError, match="must be"):
        ops.embedding_lookup(table, ids, out=torch.zeros(5, 8, device=cuda_device))
    with pytest.raises(ValueError, match="rows of grad"):
        ops.embedding_grad(torch.zeros(3, 8, device=cuda_device), ids, 10)
    with pytest.raises(RuntimeError):  # a negative number of rows
        ops.embedding_grad(torch.zeros(4, 8, device=cuda_device), ids, -1)
    with pytest.raises(ValueError, match="contiguous"):
        ops.embedding_grad(torch.zeros(4, 8, device=cuda_device), ids, 10,
                           out=torch.zeros(10, 16, device=cuda_device)[:, :8])


@pytest.mark.gpu
def test_gradient_offsets_past_32_bits(cuda_device):
    rows, dim, n = 20_000_000, 128, 40_000  # 2.6e9 values of the dense gradient
    grad, ids = _case(n, rows, dim, torch.float16, 1, 6)
    ids[:3] = torch.tensor([0, rows - 1, 16_777_217])
    d = ops.embedding_grad(grad.to(cuda_device), ids.to(cuda_device), rows)
    r = ops.embedding_grad_rows(grad.to(cuda_device), ids.to(cuda_device), rows)
    c = int(r.count)
    assert torch.equal(d[r.ids[:c].long()], r.rows[:c])
    assert int((d != 0).any(1).sum()) == c
    where = int((r.ids[:c] == rows - 1).nonzero())
    mine = grad[ids == rows - 1].double().sum(0)
    assert_within(r.rows[where], mine, rounding(mine, torch.float16) + n * U32)


@pytest.mark.gpu
def test_a_gradient_with_more_rows_than_an_index_of_elements(cuda_device):
    n, dim = 18_000_000, 128  # 2.3e9 values of the tokens' gradients
    grad = torch.zeros(n, dim, dtype=torch.float16, device=cuda_device)
    grad[-1], grad[0], grad[16_777_216] = 3, 5, 7
    ids = torch.zeros(n, dtype=torch.int32, device=cuda_device)
    ids[n // 2:] = 9
    d = ops.embedding_grad(grad, ids, 10, out_dtype=torch.float32)
    want = torch.zeros(10, dim)
    want[0], want[9] = 5, 10
    assert torch.equal(d.cpu(), want)


@pytest.mark.gpu
@pytest.mark.parametrize("n", [7, 8, 9, 255, 1023, 1024, 1025, 2047, 2048, 2049, 4095, 4096, 4097,
                               4128, 8191, 8192, 8193])
@pytest.mark.parametrize("rows", [1, 3, 200, 2 ** 20])
def test_gradient_at_the_ends_of_its_chunks(cuda_device, n, rows):
    grad, ids = _case(n, rows, 20, torch.float32, 2, n)
    d, size, tokens = _grad_ref(grad, ids, rows, 1.0)
    r = ops.embedding_grad_rows(grad.to(cuda_device), ids.to(cuda_device), rows)
    hit = torch.nonzero(tokens[:, 0])[:, 0]
    c = hit.numel()
    assert r.count.tolist() == [c]
    assert torch.equal(r.ids[:c].cpu().long(), hit) and (r.ids[c:] == -1).all()
    assert_within(r.rows[:c], d[hit], _grad_bound(d, size, tokens, torch.float32)[hit])
    assert (r.rows[c:] == 0).all()
    ops.check()


@pytest.mark.gpu
@pytest.mark.parametrize("n", [5000, 130 * 32, 200_000])
def test_gradient_of_one_row_from_any_token_to_the_next_row(cuda_device, n):
    """A row that fills runs of chunks, beginning and ending within, at and past their ends."""
    for first, last in ((0, n), (1, n - 1), (31, n - 32), (32, n - 31), (64 * 32, n), (0, 64 * 32),
                        (63, 129 * 32 + 5)):
        last = min(last, n)
        ids = torch.zeros(n, dtype=torch.int32)
        ids[first:last], ids[last:] = 1, 2
        grad = torch.ones(n, 6)
        d = ops.embedding_grad(grad.to(cuda_device), ids.to(cuda_device), 3)
        assert d[:, 0].tolist() == [first, last - first, n - last] and (d == d[:, :1]).all()


@pytest.mark.gpu
@pytest.mark.parametrize("dim", [8, 9, 11, 31, 301, 1023, 8191, 8192, 8193, 20_011])
@pytest.mark.parametrize("tin,tout", [(torch.float16, torch.float16),
                                      (torch.float32, torch.float32),
                                      (torch.bfloat16, torch.float32),
                                      (torch.float32, torch.float16)])
def test_lookup_of_rows_that_no_vector_divides(cuda_device, dim, tin, tout):
    g = gen(dim)
    table = torch.randn(50, dim, generator=g).to(tin)
    for n in (1, 3, 2 + 40_000 // dim):
        ids = torch.randint(-2, 53, (n,), generator=g, dtype=torch.int32)
        status = torch.zeros(1, dtype=torch.int32, device=cuda_device)
        got = ops.embedding_lookup(table.to(cuda_device), ids.to(cuda_device), 2.0, out_dtype=tout,
                                   status=status)
        ref = _lookup_ref(table, ids, 2.0)
        assert_within(got, ref, rounding(ref, tout) * 1.01)
        assert int(status) == (ops.BAD_INDEX if (ids >= 50).any() else 0)
    empty = ops.embedding_lookup(table[:0].to(cuda_device),
                                 torch.tensor([-1, -1], device=cuda_device))
    assert (empty == 0).all()


@pytest.mark.gpu
def test_a_status_that_is_not_aligned_is_refused(cuda_device):
    """By every C entry that takes one, on the host."""
    z = torch.zeros(4096, dtype=torch.uint8, device=cuda_device)
    p, L = z.data_ptr(), ops.lib()
    for off in (1, 2, 3):
        bad = p + 2048 + off
        for call in (
                lambda: L.agnes_embedding_lookup(p, 0, 4, 8, 8, p, 32, 3, 1.0, p + 512, 0, 8, bad,
                                                 None),
                lambda: L.agnes_embedding_grad(p, 0, 8, p, 32, 3, 4, 8, 1.0, p + 512, 0, p + 1024,
                                               1024, bad, None),
                lambda: L.agnes_embedding_grad_rows(p, 0, 8, p, 32, 3, 4, 8, 1.0, p + 512, p + 768,
                                                    0, p + 896, p + 1024, 1024, bad, None),
                lambda: L.agnes_distill_loss(p, 0, 5, 2, 5, p, 0, p, 32, 1, 1.0, p + 512, p + 768,
                                             bad, None),
                lambda: L.agnes_distill_grad(p, 0, 5, 2, 5, p, 0, p, 32, 1, 1.0, p + 512, None, 1.0,
                                             p + 768, 0, 5, bad, None),
                lambda: L.agnes_distill_loss_grad(p, 0, 5, 2, 5, p, 0, p, 32, 1, 1.0, None, 1.0,
                                                  p + 512, p + 768, 0, 5, bad, None),
                lambda: L.agnes_mx4_linear(p, 32, 3, p, 32, 4, 32, None, p + 512, 0, 4, bad, None)):
            assert call() == 1
            assert b"status is not aligned" in L.agnes_last_error(None)
    torch.cuda.synchronize()
    assert (z == 0).all()


@pytest.mark.gpu
def test_a_first_call_in_inference_mode_leaves_a_status_that_can_be_cleared(cuda_device,
                                                                            monkeypatch):
    monkeypatch.setattr(ops, "_status", {})
    table, ids = torch.ones(10, 16, device=cuda_device), torch.tensor([10], device=cuda_device)
    with torch.inference_mode():
        ops.embedding_lookup(table, ids)
    with pytest.raises(AgnesError, match="past the end"):
        ops.check()
    ops.check()  # cleared


@pytest.mark.gpu
@pytest.mark.parametrize("index", [torch.int32, torch.int64])
def test_gradient_of_a_table_without_rows_reports_ids(cuda_device, index):
    for n in (1, 300, 70_000):
        grad = torch.ones(n, 4, device=cuda_device)
        ids = torch.full((n,), -1, dtype=index, device=cuda_device)
        status = torch.zeros(1, dtype=torch.int32, device=cuda_device)
        assert ops.embedding_grad(grad, ids, 0, status=status).shape == (0, 4)
        assert int(status) == 0
        ids[n - 1] = 0
        ops.embedding_grad(grad, ids, 0, status=status)
        assert int(status) == ops.BAD_INDEX
        ops.embedding_grad(grad, ids, 0)
        with pytest.raises(AgnesError, match="past the end"):
            ops.check()
    # by the C entry: ids and the status alone, and without a status nothing
    L, ids = ops.lib(), torch.zeros(8, dtype=index, device=cuda_device)
    bits, p = 8 * ids.element_size(), status.data_ptr()
    for at, rc in ((p, 0), (None, 0), (p + 2, 1)):
        assert L.agnes_embedding_grad(None, 0, 4, ids.data_ptr(), bits, 8, 0, 4, 1.0, None, 0, None,
                                      0, at, None) == rc
    assert L.agnes_embedding_grad(None, 0, 4, None, bits, 8, 0, 4, 1.0, None, 0, None, 0, p,
                                  None) == 1


# The widest vector that divides the rows, and how many of them a lane and a column tile take,
# follow from dim: every kernel of the sums, and grids of one and of several column tiles.
_DIMS = {8: [256, 512, 768, 1024, 1296], 4: [128, 256, 300, 384, 516, 640],
         2: [66, 130, 302, 322, 642], 1: [33, 65, 161, 301, 321, 643]}
_SUMS = [(tin, tout, dim) for tin, tout in
         [(torch.float16, torch.float16), (torch.bfloat16, torch.bfloat16),
          (torch.float32, torch.float32), (torch.bfloat16, torch.float32)]
         for vec, dims in _DIMS.items() for dim in dims
         if vec <= 16 // max(tin.itemsize, tout.itemsize)]


@pytest.mark.gpu
@pytest.mark.parametrize("tin,tout,dim", _SUMS)
def test_gradient_of_longer_rows(cuda_device, tin, tout, dim):
    for n, rows, skew in ((600, 40, 2), (9000, 60, 4)):  # rows within, across and over chunks
        grad, ids = _case(n, rows, dim, tin, skew, n + dim)
        d, size, tokens = _grad_ref(grad, ids, rows, 1.5)
        hit = torch.nonzero(tokens[:, 0])[:, 0]
        c = hit.numel()
        wide = torch.full((n, dim + 24), float("nan"), dtype=tin, device=cuda_device)
        wide[:, 8:8 + dim] = grad.to(cuda_device)
        odd = torch.full((n, dim + 3), float("nan"), dtype=tin, device=cuda_device)
        odd[:, 1:1 + dim] = grad.to(cuda_device)
        for x in (grad.to(cuda_device), wide[:, 8:8 + dim], odd[:, 1:1 + dim]):
            dense = ops.embedding_grad(x, ids.to(cuda_device), rows, 1.5, out_dtype=tout)
            assert_within(dense, d, _grad_bound(d, size, tokens, tout))
            r = ops.embedding_grad_rows(x, ids.to(cuda_device), rows, 1.5, out_dtype=tout)
            assert r.count.tolist() == [c]
            assert torch.equal(r.ids[:c].cpu().long(), hit) and (r.ids[c:] == -1).all()
            assert torch.equal(r.rows[:c].cpu(), dense.cpu()[hit])
            assert (r.rows[c:] == 0).all()
    ops.check()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", FLOATS)
@pytest.mark.parametrize("dim", [9, 41, 301])
def test_lookup_of_strided_rows_that_no_vector_divides(cuda_device, dtype, dim):
    g = gen(dim)
    wide = torch.randn(50, dim + 7, generator=g).to(dtype)
    for first in (0, 1, 6):
        ids = torch.randint(-1, 50, (2 + 30_000 // dim,), generator=g, dtype=torch.int32)
        got = ops.embedding_lookup(wide.to(cuda_device)[:, first:first + dim],
                                   ids.to(cuda_device), 2.0)
        ref = _lookup_ref(wide[:, first:first + dim], ids, 2.0)
        assert_within(got, ref, rounding(ref, dtype) * 1.01)
    ops.check()
