"""The norms around a residual block and their gradients (include/agnes_ops.h) against
their formulas in 64 bits, within bounds that a running error analysis of the fp32
arithmetic gives."""
import itertools
import math

import pytest
import torch

from ops_support import FLOATS, U32, assert_within, gen, rounding
from paper_2601_01473_gb300 import AgnesError, ops
from test_ops_int8 import reference_rows, row_bytes

EPS = 1e-5
# x's and branch's types
TYPES = [(a, a) for a in FLOATS] + [(torch.float32, a) for a in FLOATS[1:]]
# A row's sums: a thread's 8 values in turn, then a tree of at most 10 steps, with every
# product rounded on the way
DEPTH = 20


class Num:
    """Values in 64 bits with a bound of how far fp32 arithmetic may be off them."""

    def __init__(self, v, err=None):
        self.v = v
        self.err = torch.zeros_like(v) if err is None else err

    def __add__(self, o):
        o = o if isinstance(o, Num) else Num(torch.as_tensor(o, dtype=torch.float64))
        v = self.v + o.v
        return Num(v, self.err + o.err + U32 * v.abs())

    def __mul__(self, o):
        o = o if isinstance(o, Num) else Num(torch.as_tensor(o, dtype=torch.float64))
        v = self.v * o.v
        return Num(v, self.v.abs() * o.err + o.v.abs() * self.err + self.err * o.err
                   + U32 * v.abs())

    def __sub__(self, o):
        return self + o * Num(torch.tensor(-1.0, dtype=torch.float64))

    def mean(self):
        """Of a row: sum and product with 1 / dim (rounded itself)."""
        v = self.v.mean(1, keepdim=True)
        return Num(v, (self.err + (DEPTH + 2) * U32 * self.v.abs()).mean(1, keepdim=True))

    def rsqrt(self):
        v = self.v.rsqrt()
        return Num(v, v * (0.6 * self.err / self.v + 3 * U32))

    def sum(self):
        """Over the rows, in any order."""
        n = self.v.shape[0]
        return Num(self.v.sum(0), (self.err + n * U32 * self.v.abs()).sum(0))


def standard(v, kind, eps=EPS):
    if kind == "layer":
        v = v - v.mean()
    inv = ((v * v).mean() + eps).rsqrt()
    return v * inv, inv


def through(d, n, inv, kind):
    along = (d * n).mean()
    out = d - n * along
    if kind == "layer":
        out = out - d.mean()
    return out * inv


def num(t):
    return None if t is None else Num(t.double().cpu())


def forward(c):
    """(sum before its rounding, next from a given sum) of a case."""
    b = num(c["branch"])
    u = b
    if c["after"] is not None:
        u = standard(b, c["kind"])[0] * num(c["after"])
        if c["after_bias"] is not None:
            u = u + num(c["after_bias"])
    if c["gate"] is not None:
        u = u * num(c["gate"])
    return num(c["x"]) + u * c["scale"]


def following(total, c):
    n = standard(num(total), c["kind"])[0] * num(c["before"])
    return n if c["before_bias"] is None else n + num(c["before_bias"])


def backward(c, total, d_next, d_sum):
    out = {}
    d = num(d_sum) if d_sum is not None else Num(torch.zeros(total.shape, dtype=torch.float64))
    if c["before"] is not None:
        n, inv = standard(num(total), c["kind"])
        g = num(d_next)
        out["before"] = (g * n).sum()
        if c["before_bias"] is not None:
            out["before_bias"] = g.sum()
        d = d + through(g * num(c["before"]), n, inv, c["kind"])
    out["x"] = d
    if c["branch"] is None:
        return out
    b = num(c["branch"])
    u = b
    if c["after"] is not None:
        n, inv = standard(b, c["kind"])
        u = n * num(c["after"])
        if c["after_bias"] is not None:
            u = u + num(c["after_bias"])
    d = d * c["scale"]
    if c["gate"] is not None:
        g = d * u
        out["gate"] = g.sum() if c["gate"].ndim == 1 else g
        d = d * num(c["gate"])
    if c["after"] is not None:
        out["after"] = (d * n).sum()
        if c["after_bias"] is not None:
            out["after_bias"] = d.sum()
        d = through(d * num(c["after"]), n, inv, c["kind"])
    out["branch"] = d
    return out


def make(rows, dim, types, kind, after, gate, bias, scale=0.75, seed=0, before=True):
    g = gen(seed)
    x_type, b_type = types

    def normal(*shape):
        return torch.randn(shape, generator=g)

    c = {"x": (normal(rows, dim) * 2).to(x_type), "branch": (normal(rows, dim) + 0.5).to(b_type),
         "after": 1 + 0.3 * normal(dim) if after else None,
         "after_bias": normal(dim) if after and bias else None,
         "before": 1 + 0.3 * normal(dim) if before else None,
         "before_bias": normal(dim) if before and bias else None,
         "gate": None if gate == "none" else normal(dim) if gate == "columns" else
         normal(rows, dim).to(b_type), "scale": torch.tensor(scale).item(), "kind": kind}
    d_next = normal(rows, dim).to(b_type) if before else None
    return c, d_next, normal(rows, dim).to(x_type)


def on(dev, c):
    return {k: v.to(dev) if isinstance(v, torch.Tensor) else v for k, v in c.items()}


def check_forward(dev, c, rows8=False):
    x_type, b_type = c["x"].dtype, c["branch"].dtype
    total, n = ops.residual_norm(**on(dev, c), rows8=rows8)
    ref = forward(c)
    assert total.dtype == x_type
    assert_within(total, ref.v, ref.err + 1.01 * rounding(ref.v, x_type))
    if c["before"] is None:
        assert n is None
        return total, n
    ref = following(total.cpu(), c)
    if rows8:
        back = ops.int8_dequantize(n, c["x"].shape[1])
        step = ref.v.abs().amax(1, keepdim=True) / 127 * 1.01
        assert ((back.double().cpu() - ref.v).abs() <= 0.502 * step + ref.err).all()
    else:
        assert n.dtype == b_type
        assert_within(n, ref.v, ref.err + 1.01 * rounding(ref.v, b_type))
    return total, n


def check_backward(dev, c, total, d_next, d_sum):
    args = on(dev, c)
    del args["x"]
    to = lambda t: None if t is None else t.to(dev)  # noqa: E731
    got = ops.residual_norm_grad(to(d_next), to(d_sum), to(total), **args)
    ref = backward(c, total.cpu(), d_next, d_sum)
    for name, y in got._asdict().items():
        assert (y is not None) == (name in ref), name
        if y is not None:
            want = ref[name]
            assert y.shape == want.v.shape
            assert_within(y, want.v, want.err + 1.01 * rounding(want.v, y.dtype) + 1e-30)
    return got


# ---- without a GPU --------------------------------------------------------------------

def test_refusals():
    from paper_2601_01473_gb300 import build
    build.build()
    x = torch.zeros(2, 8)
    with pytest.raises(ValueError, match="CUDA device"):
        ops.residual_norm(x, x)
    L = ops.lib()
    f = [None, 0, 8, 1, 0, 8, 4, 8, None, 0, 0, 1.0, None, None, 1, None, 0, 1e-5, None, 8, None,
         0, 8, None]
    assert L.agnes_residual_norm(*f) == 1 and b"NULL" in L.agnes_last_error(None)
    # types, sizes, a gate, biases without norms, a kind, eps, next's type and stride
    for at, value, status in ((1, 1, 1), (1, 5, 1), (4, 3, 1), (6, -1, 1), (7, 0, 1), (7, 8193, 2),
                              (6, 1 << 31, 2), (9, 3, 1), (13, 1, 1), (16, 2, 1), (17, -1.0, 1),
                              (17, math.nan, 1), (21, 1, 1), (21, 3, 1)):
        bad = list(f)
        bad[at] = value
        assert L.agnes_residual_norm(*bad) == status, (at, value)
    bad = list(f)
    bad[3] = bad[14] = None  # neither a branch nor a norm
    assert L.agnes_residual_norm(*bad) == 1
    bad[14], bad[12] = 1, 1  # a norm of no branch
    assert L.agnes_residual_norm(*bad) == 1
    f[6] = 0
    assert L.agnes_residual_norm(*f) == 0
    g = [None, 8, None, 8, None, 0, 8, 1, 0, 8, 4, 8, None, 0, 0, 1.0, None, None, 1, 0, 1e-5, None,
         8, None, 8, None, 8, None, None, None, None, None, 0, None]
    assert L.agnes_residual_norm_grad(*g) == 1
    for at, value in ((5, 2), (8, 7), (10, -1), (11, 0), (13, 9), (17, 1), (19, 5), (20, -1.0),
                      (27, 1), (28, 1)):
        bad = list(g)
        bad[at] = value
        assert L.agnes_residual_norm_grad(*bad) == 1, (at, value)
    with pytest.raises(AgnesError, match="ERANGE"):
        ops._workspace_bytes("agnes_residual_norm_grad_workspace", 5, 8193)


@pytest.mark.parametrize("kind", ["rms", "layer"])
def test_the_formulas_gradients_are_autograds(kind):
    c, d_next, d_sum = make(5, 24, TYPES[0], kind, True, "columns", True)
    leaves = {k: c[k].double().requires_grad_() for k in
              ("x", "branch", "gate", "after", "after_bias", "before", "before_bias")}

    def norm(v):
        if kind == "layer":
            v = v - v.mean(1, keepdim=True)
        return v * (v.square().mean(1, keepdim=True) + EPS).rsqrt()

    u = norm(leaves["branch"]) * leaves["after"] + leaves["after_bias"]
    total = leaves["x"] + c["scale"] * leaves["gate"] * u
    n = norm(total) * leaves["before"] + leaves["before_bias"]
    assert torch.allclose(forward(c).v, total)
    ((n * d_next).sum() + (total * d_sum).sum()).backward()
    got = backward(c, total.detach(), d_next, d_sum)
    for k, leaf in leaves.items():
        assert torch.allclose(got[k].v, leaf.grad, rtol=1e-9, atol=1e-10), k


# ---- on a GPU ----------------------------------------------------------------------------

@pytest.mark.gpu
@pytest.mark.parametrize("types", TYPES)
@pytest.mark.parametrize("rows,dim", [(1, 1), (1, 8), (3, 7), (70, 16), (33, 128), (9, 301),
                                      (300, 64), (5, 1000), (40, 1024), (3, 2056), (7, 4096),
                                      (2, 4100), (3, 8192), (2, 8191)])
@pytest.mark.parametrize("kind", ["rms", "layer"])
def test_forward_and_backward(cuda_device, types, rows, dim, kind):
    gate = ["none", "columns", "rows"][(rows + dim) % 3]
    c, d_next, d_sum = make(rows, dim, types, kind, True, gate, kind == "layer")
    total, _ = check_forward(cuda_device, c)
    check_backward(cuda_device, c, total, d_next, d_sum)


@pytest.mark.gpu
@pytest.mark.parametrize("kind,after,gate,bias,before", [
    v for v in itertools.product(["rms", "layer"], [True, False], ["none", "columns", "rows"],
                                 [True, False], [True, False])])
def test_every_combination(cuda_device, kind, after, gate, bias, before):
    for dim in (72, 75):
        c, d_next, d_sum = make(50, dim, TYPES[4], kind, after, gate, bias, before=before)
        total, _ = check_forward(cuda_device, c)
        check_backward(cuda_device, c, total, d_next, d_sum)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", FLOATS)
@pytest.mark.parametrize("kind", ["rms", "layer"])
def test_the_first_norm_of_a_network(cuda_device, dtype, kind):
    """Without a branch: the norm of x itself, of its type or another."""
    for next_type in {dtype, torch.bfloat16 if dtype == torch.float32 else dtype}:
        c, d_next, d_sum = make(20, 96, (dtype, next_type), kind, False, "none", True)
        x = c["x"].to(cuda_device)
        vectors = {"before": c["before"].to(cuda_device),
                   "before_bias": c["before_bias"].to(cuda_device), "kind": kind}
        total, n = ops.residual_norm(x, next_dtype=next_type, **vectors)
        assert total is x and n.dtype == next_type
        ref = following(c["x"], c)
        assert_within(n, ref.v, ref.err + 1.01 * rounding(ref.v, next_type))
        c["branch"] = None
        check_backward(cuda_device, c, c["x"], d_next, d_sum)
        check_backward(cuda_device, c, c["x"], d_next, None)
    with pytest.raises(AgnesError, match="nothing to compute"):
        ops.residual_norm(x)
    with pytest.raises(ValueError, match="out"):
        ops.residual_norm(x, before=vectors["before"], out=x)


@pytest.mark.gpu
@pytest.mark.parametrize("types", TYPES)
def test_next_in_8_bits(cuda_device, types):
    for rows, dim in ((1, 1), (40, 128), (9, 301), (3, 8192), (5, 8000)):
        c, _, _ = make(rows, dim, types, "layer", True, "columns", True)
        total, n8 = check_forward(cuda_device, c, rows8=True)
        assert n8.shape == (rows, row_bytes(dim))
        if types[1] == torch.float32:  # the same bytes as of next, which has not been rounded
            plain = ops.residual_norm(**on(cuda_device, c)).next
            assert torch.equal(n8.cpu(), reference_rows(plain.cpu()))


@pytest.mark.gpu
@pytest.mark.parametrize("rows,dim", [(20_000, 64), (3000, 301), (2500, 1024)])
@pytest.mark.parametrize("gate", ["columns", "rows"])
def test_sums_over_many_rows(cuda_device, rows, dim, gate):
    """More rows than the device takes at a time; the same each time."""
    c, d_next, d_sum = make(rows, dim, TYPES[0], "layer", True, gate, True)
    total, _ = check_forward(cuda_device, c)
    got = check_backward(cuda_device, c, total, d_next, d_sum)
    for _ in range(5):
        again = check_backward(cuda_device, c, total, d_next, d_sum)
        assert all(torch.equal(a, b) for a, b in zip(got, again))


@pytest.mark.gpu
def test_strides_and_in_place(cuda_device):
    rows, dim = 30, 104
    c, d_next, d_sum = make(rows, dim, TYPES[1], "layer", True, "rows", True)
    c = on(cuda_device, c)
    d_next, d_sum = d_next.to(cuda_device), d_sum.to(cuda_device)
    want = ops.residual_norm(**c)
    args = {k: v for k, v in c.items() if k != "x"}
    want_grad = ops.residual_norm_grad(d_next, d_sum, want.sum, **args)

    def apart(t, first):
        wide = torch.full((rows + 2, dim + 24), math.nan, dtype=t.dtype, device=cuda_device)
        wide[1:-1, first:first + dim] = t
        return wide[1:-1, first:first + dim]

    for first in (0, 1, 8):
        moved = dict(c, x=apart(c["x"], first), branch=apart(c["branch"], first),
                     gate=apart(c["gate"], first))
        out = torch.full((rows, dim + 16), 7.0, dtype=torch.float16, device=cuda_device)
        got = ops.residual_norm(**moved, out=out[:, first:first + dim])
        # another way of spreading a row over threads sums in another order
        close = dict(rtol=0, atol=0) if first != 1 else dict(rtol=2e-3, atol=2e-3)
        torch.testing.assert_close(got.sum, want.sum, **close)
        torch.testing.assert_close(got.next, want.next, **close)
        assert (out[:, :first] == 7).all() and (out[:, first + dim:] == 7).all()
        moved.pop("x")
        grad = ops.residual_norm_grad(apart(d_next, first), apart(d_sum, first),
                                      apart(want.sum, first), **moved)
        for a, b in zip(grad, want_grad):
            torch.testing.assert_close(a, b, **close)
        x = c["x"].clone()
        got = ops.residual_norm(**dict(c, x=x), out=x)
        assert got.sum is x and torch.equal(x, want.sum) and torch.equal(got.next, want.next)


@pytest.mark.gpu
@pytest.mark.parametrize("rows,dim,types", [(20_011, 301, 1), (30_003, 100, 1), (6001, 350, 4),
                                            (1301, 500, 2), (17, 8191, 4), (700, 7, 2)])
def test_runs_of_odd_rows_from_any_element_on(cuda_device, rows, dim, types):
    """Rows that no vector divides, several batches to a CTA and an empty end, next to what others own."""
    c, d_next, d_sum = make(rows, dim, TYPES[types], "layer", True, "rows", True)
    want, want_next = check_forward(cuda_device, c)
    grads = check_backward(cuda_device, c, want, d_next, d_sum)
    want8 = check_forward(cuda_device, c, rows8=True)[1]
    c = on(cuda_device, c)

    def run(t, first):
        flat = torch.full((rows * dim + 32,), 7.0, dtype=t.dtype, device=cuda_device)
        v = flat[first:first + rows * dim].view(rows, dim)
        v.copy_(t)
        return flat, v

    for first in (1, 5):
        _, x = run(c["x"], first)
        moved = dict(c, x=x, branch=run(c["branch"], first + 2)[1], gate=run(c["gate"], 3)[1])
        flat, out = run(c["x"], first + 1)
        got = ops.residual_norm(**moved, out=out)
        assert torch.equal(got.sum, want) and torch.equal(got.next, want_next)
        assert (flat[:first + 1] == 7).all() and (flat[first + 1 + rows * dim:] == 7).all()
        assert torch.equal(ops.residual_norm(**moved, rows8=True).next, want8)
        rest = {k: v for k, v in moved.items() if k != "x"}
        got = ops.residual_norm_grad(run(d_next, first)[1], run(d_sum, first + 4)[1],
                                     run(want, 2)[1], **rest)
        assert all(torch.equal(a, b) for a, b in zip(got, grads))
        got = ops.residual_norm(**moved, out=x)  # in place
        assert got.sum is x and torch.equal(x, want) and torch.equal(got.next, want_next)


@pytest.mark.gpu
def test_rows_of_zeros_of_one_value_and_of_what_is_not_finite(cuda_device):
    c, d_next, d_sum = make(6, 64, TYPES[0], "layer", True, "columns", True)
    c["branch"][1] = 0
    c["branch"][2] = 5.0  # no variance: N is exactly zero
    c["branch"][3, 7] = math.nan
    c["branch"][4, 9] = math.inf
    c = on(cuda_device, c)
    total, n = ops.residual_norm(**c)
    fine = torch.tensor([0, 1, 2, 5])
    assert total.cpu()[fine].isfinite().all() and n.cpu()[fine].isfinite().all()
    assert total.cpu()[3:5].isnan().all() and n.cpu()[3:5].isnan().all()
    shift = c["scale"] * c["gate"] * c["after_bias"]
    for r in (1, 2):
        assert (total[r] - (c["x"][r] + shift)).abs().max() <= 4 * U32 * 16
    _, n8 = ops.residual_norm(**c, rows8=True)
    back = ops.int8_dequantize(n8, 64).cpu()
    assert back[3:5].isnan().all() and back[fine].isfinite().all()
    args = {k: v for k, v in c.items() if k != "x"}
    g = ops.residual_norm_grad(d_next.to(cuda_device), d_sum.to(cuda_device), total, **args)
    assert g.branch.cpu()[fine].isfinite().all() and g.x.cpu()[fine].isfinite().all()
    assert not g.branch.cpu()[3:5].isfinite().any()
    # eps of 0: a row of zeros has no norm, the others have theirs, and so have their sums
    x = torch.randn(9, 40, generator=gen(4)).to(cuda_device)
    w = torch.ones(40, device=cuda_device)
    n = ops.residual_norm(x, before=w, eps=0.0).next
    ref = x.double() * x.double().square().mean(1, keepdim=True).rsqrt()
    assert ((n - ref).abs() <= 30 * U32 * ref.abs()).all()
    g = ops.residual_norm_grad(x, None, x, before=w, eps=0.0)
    assert g.before.isfinite().all() and g.x.isfinite().all()


@pytest.mark.gpu
def test_a_large_mean_is_not_lost(cuda_device):
    """Values of 1000 +- 1: a variance from the squares' difference would have two digits."""
    c, _, _ = make(16, 512, TYPES[0], "layer", False, "none", False)
    c["x"] = c["x"] * 0.25 + 1000
    c["branch"] = c["branch"] * 0
    check_forward(cuda_device, c)


@pytest.mark.gpu
def test_of_no_rows(cuda_device):
    c, d_next, d_sum = make(0, 32, TYPES[0], "layer", True, "columns", True)
    c = on(cuda_device, c)
    out = ops.residual_norm(**c)
    assert out.sum.shape == (0, 32) and out.next.shape == (0, 32)
    c.pop("x")
    g = ops.residual_norm_grad(d_next.to(cuda_device), d_sum.to(cuda_device), out.sum, **c)
    assert g.x.shape == (0, 32)
    for v in (g.gate, g.after, g.after_bias, g.before, g.before_bias):
        assert v.shape == (32,) and not v.any()


@pytest.mark.gpu
def test_gradients_are_those_of_differences(cuda_device):
    """Of the formula in 64 bits, over small steps of single values."""
    c, d_next, d_sum = make(4, 24, TYPES[0], "layer", True, "columns", True)

    def loss(**changed):
        v = dict({k: t.double() if isinstance(t, torch.Tensor) else t for k, t in c.items()},
                 **changed)
        total = forward(v).v
        return float((following(total, v).v * d_next).sum() + (total * d_sum).sum())

    total = forward(c).v.float()
    args = on(cuda_device, c)
    args.pop("x")
    got = ops.residual_norm_grad(d_next.to(cuda_device), d_sum.to(cuda_device),
                                 total.to(cuda_device), **args)
    h = 1e-5
    for name, g in got._asdict().items():
        base = c[name].double()
        for at in (0, base.numel() // 2, base.numel() - 1):
            step = torch.zeros_like(base).view(-1)
            step[at] = h
            step = step.view_as(base)
            want = (loss(**{name: base + step}) - loss(**{name: base - step})) / (2 * h)
            # the difference's own error is h^2 and 1e-16 / h of a loss of some hundreds
            assert abs(float(g.view(-1)[at]) - want) <= 2e-5 * max(1, abs(want)), (name, at)


@pytest.mark.gpu
def test_python_refusals(cuda_device):
    x = torch.zeros(4, 8, device=cuda_device)
    w = torch.ones(8, device=cuda_device)
    h = x.half()
    for kind, call in (
            (TypeError, lambda: ops.residual_norm(x, x, before=w[:7])),
            (TypeError, lambda: ops.residual_norm(x, x, before=w.half())),
            (ValueError, lambda: ops.residual_norm(x, x[:3], before=w)),
            (ValueError, lambda: ops.residual_norm(x, x, gate=x[:3])),
            (ValueError, lambda: ops.residual_norm(x, h, gate=x)),
            (TypeError, lambda: ops.residual_norm(x, x, gate=w[:5])),
            (ValueError, lambda: ops.residual_norm(x, x, kind="batch")),
            (AgnesError, lambda: ops.residual_norm(h, x)),
            (AgnesError, lambda: ops.residual_norm(x, x, after_bias=w)),
            (AgnesError, lambda: ops.residual_norm(x, before=w, gate=w)),
            (ValueError, lambda: ops.residual_norm(x, x, before=w.cpu())),
            (TypeError, lambda: ops.residual_norm(x, x, next_dtype=torch.float16)),
            (ValueError, lambda: ops.residual_norm_grad(x, x, x, x)),
            (ValueError, lambda: ops.residual_norm_grad(None, x, x, x, before=w)),
            (ValueError, lambda: ops.residual_norm_grad(x[:2], x, x, x, before=w)),
            (ValueError, lambda: ops.residual_norm_grad(x, h, x, x, before=w))):
        with pytest.raises(kind):
            call()


@pytest.mark.gpu
def test_streams_and_graphs(cuda_device):
    c, d_next, d_sum = make(2000, 256, TYPES[4], "rms", True, "columns", False)
    c, d_next, d_sum = on(cuda_device, c), d_next.to(cuda_device), d_sum.to(cuda_device)
    args = {k: v for k, v in c.items() if k != "x"}

    def run(**stream):
        total, n = ops.residual_norm(**c, **stream)
        g = ops.residual_norm_grad(d_next, d_sum, total, **args, **stream)
        return [total, n] + [v for v in g if v is not None]
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


@pytest.mark.gpu
def test_offsets_past_32_bits(cuda_device):
    rows, dim = 1_100_000, 2048  # 2.3e9 values
    c, d_next, d_sum = make(3, dim, TYPES[1], "rms", True, "columns", False)
    at = [0, 1_048_577, rows - 1]

    def spread(t):
        big = torch.ones(rows, dim, dtype=t.dtype, device=cuda_device)
        big[at] = t.to(cuda_device)
        return big

    c, d_next, d_sum = on(cuda_device, c), d_next.to(cuda_device), d_sum.to(cuda_device)
    want = ops.residual_norm(**c)
    args = {k: v for k, v in c.items() if k != "x"}
    want_grad = ops.residual_norm_grad(d_next, d_sum, want.sum, **args)
    big = dict(c, x=spread(c["x"]), branch=spread(c["branch"]))
    got = ops.residual_norm(**big)
    assert torch.equal(got.sum[at], want.sum) and torch.equal(got.next[at], want.next)
    big.pop("x")
    d_next, d_sum = spread(d_next), spread(d_sum)
    g = ops.residual_norm_grad(d_next, d_sum, got.sum, **big)
    assert torch.equal(g.x[at], want_grad.x) and torch.equal(g.branch[at], want_grad.branch)


@pytest.mark.gpu
@pytest.mark.parametrize("types", [(torch.float32, torch.bfloat16), (torch.float16, torch.float16)])
def test_the_longest_rows_from_any_element_on(cuda_device, types):
    """What takes most shared memory: 8192 columns that no vector's alignment suits, a full gate."""
    rows, dim = 3, 8192
    c, _, _ = make(rows, dim, types, "layer", True, "rows", True)
    flat = torch.zeros(rows * dim + 1, dtype=types[0], device=cuda_device)
    moved = on(cuda_device, c)
    moved["x"] = flat[1:].view(rows, dim).copy_(c["x"])
    got = ops.residual_norm(**moved)
    ref = forward(c)
    assert_within(got.sum, ref.v, ref.err + 1.01 * rounding(ref.v, types[0]))
    ref = following(got.sum.cpu(), c)
    assert_within(got.next, ref.v, ref.err + 1.01 * rounding(ref.v, types[1]))
    got8 = ops.residual_norm(**moved, rows8=True)
    assert torch.equal(got8.sum, got.sum)
    back = ops.int8_dequantize(got8.next, dim).double().cpu()
    step = ref.v.abs().amax(1, keepdim=True) / 127 * 1.01
    assert ((back - ref.v).abs() <= 0.502 * step + ref.err).all()
