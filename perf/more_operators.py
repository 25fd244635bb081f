"""The operators of a deeper student whose layers are trained on prepared
hyperbatches with their activations kept in 8 bits, as a user's program calls
them, and the plain form of each.

Four kinds of pass:

  "norm"        the step between two blocks of a residual network: the block's
                output normalised, gated, scaled and added to the residual, and the
                sum normalised for the next block: "forward", or "grad" (the gradient
                to everything that entered);
  "linear"      8-bit rows times 8-bit weights, with a scale for each row and each
                column of the output; the rows come in 8 bits (gathered features, an
                earlier layer's activations) or are rounded in the call;
  "linear_grad" that layer's backward pass from what it keeps in 8 bits: the gradient
                to the weights and the bias from the kept rows, and to the input from
                the weights;
  "activation"  a nonlinearity, gated or not: "forward" (serving), or "step" (forward,
                its input kept in 8 bits, and backward from that).

Norm: with N(v) = (v - mean v) / sqrt(var v + eps) ("layer") or v / sqrt(mean v^2 +
eps) ("rms"), row by row,
    u = N(branch) * after + after_bias, or branch where there is no `after`
    sum = x + scale * gate * u, rounded to x's type
    next = N(sum) * before + before_bias, of the rounded sum
gate is absent, a vector over the columns or a matrix.

8-bit rows: a row's scale is s = its largest magnitude / 127 in fp32, rounded up to a
bfloat16 value; a value is round(v * (1 / s)) (the inverse and the product in fp32, ties
to even) times s.  A row whose largest magnitude is below 2^-100 is zeros (scale 0), one
with an infinity or NaN stands for NaN (scale NaN).  A row's bytes are its values, zeros,
and the scale as fp32 in the last four of a multiple of 16 bytes.

Linear: out[r][j] = s_r s_j sum_i x[r][i] w[j][i] + bias[j].

Activation: y = f(x), or f(x[:, :dim]) * x[:, dim:] where gated; f is relu, silu
(v / (1 + exp -v)) or gelu (v Phi(v)).  The backward pass takes f' and f of the kept
values; of a gated row the two halves are kept as rows of their own.
"""
import math

import torch

own = False

DTYPES = {"f16": torch.float16, "bf16": torch.bfloat16, "f32": torch.float32}
SIZE = {"f16": 2, "bf16": 2, "f32": 4}
EPS = 1e-5


def listed():
    return [
        # an online request: the states of a few nodes between two blocks; latency only
        {"name": "norm_request", "kind": "norm", "form": "forward", "rows": 4, "dim": 1024,
         "x": "bf16", "branch": "bf16", "norm": "rms", "after": True, "gate": "none",
         "bias": False, "scale": 1.0, "out": "bf16"},
        # all nodes of a hyperbatch between two layers, with layer norms and a learned scale
        # per column
        {"name": "norm_hyperbatch", "kind": "norm", "form": "forward", "rows": 786_432,
         "dim": 128, "x": "f16", "branch": "f16", "norm": "layer", "after": True,
         "gate": "columns", "bias": True, "scale": 0.5, "out": "f16"},
        # the backward pass of one small minibatch, odd rows, a gate per node and column
        {"name": "norm_grad_minibatch", "kind": "norm", "form": "grad", "rows": 1500, "dim": 301,
         "x": "f32", "branch": "f32", "norm": "layer", "after": True, "gate": "full",
         "bias": True, "scale": 0.25, "out": "f32"},
        # the backward pass over long rows, the residual in fp32
        {"name": "norm_grad_long", "kind": "norm", "form": "grad", "rows": 16_384, "dim": 4096,
         "x": "f32", "branch": "bf16", "norm": "rms", "after": True, "gate": "columns",
         "bias": False, "scale": 1.0, "out": "bf16"},
        # an online request: a few nodes, a wide layer; latency and the weights' bytes count
        {"name": "linear_request", "kind": "linear", "rows": 4, "dim": 1024, "width": 4096,
         "x": "i8", "out": "f16", "bias": True},
        # the first layer over the gathered 8-bit rows of a hyperbatch
        {"name": "linear_hyperbatch", "kind": "linear", "rows": 786_432, "dim": 128, "width": 256,
         "x": "i8", "out": "f16", "bias": True},
        # a wide layer over states that are rounded on the way in
        {"name": "linear_wide", "kind": "linear", "rows": 16_384, "dim": 4096, "width": 4096,
         "x": "bf16", "out": "bf16", "bias": False},
        # the backward pass of a minibatch's first layer: raw features of odd length, the
        # classes of a papers graph; latency only
        {"name": "linear_grad_minibatch", "kind": "linear_grad", "rows": 1500, "dim": 301,
         "width": 172, "grad": "f32"},
        # the backward pass of the first layer over a hyperbatch: a long sum for the weights
        {"name": "linear_grad_hyperbatch", "kind": "linear_grad", "rows": 786_432, "dim": 128,
         "width": 256, "grad": "bf16"},
        # the backward pass of a wide layer
        {"name": "linear_grad_wide", "kind": "linear_grad", "rows": 8192, "dim": 2048,
         "width": 4096, "grad": "bf16"},
        # a minibatch's activation, odd rows, forward and backward; latency only
        {"name": "activation_minibatch", "kind": "activation", "form": "step", "rows": 1000,
         "dim": 301, "f": "gelu", "gated": False, "x": "f32", "out": "f32"},
        # the gated activation of a wide block over a hyperbatch's nodes
        {"name": "activation_hyperbatch", "kind": "activation", "form": "step", "rows": 131_072,
         "dim": 1024, "f": "silu", "gated": True, "x": "bf16", "out": "bf16"},
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["norm", "norm", "linear", "linear", "linear_grad", "linear_grad",
                       "activation"])
    float_type = lambda: rng.choice(["f16", "bf16", "f32"])  # noqa: E731
    if kind == "norm":
        dim = rng.choice([_log(rng, 8, 8192), rng.randint(8, 80) * 8, rng.randint(8, 64) * 128])
        form, branch = rng.choice(["forward", "grad"]), float_type()
        norm = rng.choice(["rms", "layer"])
        i8 = form == "forward" and branch != "f32" and rng.random() < 0.3
        most = 16_384 * 4096 * (1 if form == "grad" else 2) // dim
        return {"kind": kind, "form": form, "rows": _log(rng, 1, min(most, 786_432)), "dim": dim,
                "x": rng.choice([branch, "f32"]), "branch": branch, "norm": norm,
                "after": rng.random() < 0.7, "gate": rng.choice(["none", "columns", "full"]),
                "bias": norm == "layer", "scale": rng.choice([1.0, round(rng.uniform(0.1, 2), 3)]),
                "out": "i8" if i8 else branch}
    if kind == "linear":
        dim, width = _log(rng, 16, 4096), _log(rng, 8, 4096)
        x, out = rng.choice(["i8", "i8", "f16", "bf16", "f32"]), float_type()
        most = min(16_384 * 4096 * 4096 // (dim * width), 786_432 * 512 // (width * SIZE[out]),
                   786_432 * 512 // (dim * SIZE.get(x, 1)))
        return {"kind": kind, "rows": _log(rng, 1, max(1, min(most, 786_432))), "dim": dim,
                "width": width, "x": x, "out": out, "bias": rng.random() < 0.5}
    if kind == "linear_grad":
        dim, width = _log(rng, 16, 4096), _log(rng, 8, 4096)
        grad = rng.choice(["bf16", "bf16", "f16", "f32"])
        most = min(8192 * 2048 * 4096 * (1 if grad == "bf16" else 0.5) // (dim * width),
                   786_432 * 512 // (max(width, dim) * SIZE[grad]))
        return {"kind": kind, "rows": _log(rng, 1, max(1, min(int(most), 786_432))), "dim": dim,
                "width": width, "grad": grad}
    dim, x, gated = _log(rng, 2, 8192), float_type(), rng.random() < 0.5
    most = 131_072 * 4096 // (dim * SIZE[x] * (2 if gated else 1))
    form = rng.choice(["forward", "step", "step"])
    out = "i8" if x != "f32" and rng.random() < 0.3 else x
    return {"kind": kind, "form": form, "rows": _log(rng, 1, min(most, 786_432)), "dim": dim,
            "f": rng.choice(["relu", "silu", "gelu"]), "gated": gated, "x": x, "out": out}


# ---- inputs -------------------------------------------------------------------------------

def _normal(g, shape, dtype, scale=1.0):
    return (torch.randn(shape, generator=g, device="cuda") * scale).to(dtype)


def _features(g, rows, dim):
    """Rows of differing magnitude, a few large values among them."""
    x = torch.randn((rows, dim), generator=g, device="cuda")
    x *= torch.exp2(torch.randn((rows, 1), generator=g, device="cuda"))
    return torch.where(torch.rand((rows, dim), generator=g, device="cuda") < 0.01, 6 * x, x)


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    c = dict(case)
    if c["kind"] == "norm":
        rows, dim, to, branch = c["rows"], c["dim"], DTYPES[c["x"]], DTYPES[c["branch"]]
        c["stream"] = _features(g, rows, dim).to(to)
        c["b"] = (_features(g, rows, dim) + 0.3).to(branch)
        c["g"] = None if c["gate"] == "none" else \
            _normal(g, (dim,), torch.float32, 0.5) if c["gate"] == "columns" else \
            torch.sigmoid(torch.randn((rows, dim), generator=g, device="cuda")).to(branch)
        c["w1"] = 1 + _normal(g, (dim,), torch.float32, 0.2) if c["after"] else None
        c["w2"] = 1 + _normal(g, (dim,), torch.float32, 0.2)
        c["b1"] = _normal(g, (dim,), torch.float32, 0.2) if c["bias"] and c["after"] else None
        c["b2"] = _normal(g, (dim,), torch.float32, 0.2) if c["bias"] else None
        if c["form"] == "grad":  # `stream` is the sum that the forward pass returned
            c["d_next"] = _normal(g, (rows, dim), branch, 0.1)
            c["d_sum"] = _normal(g, (rows, dim), to, 0.1)
    elif c["kind"] == "linear":
        x = _features(g, c["rows"], c["dim"])
        c["a"] = _pack(x) if c["x"] == "i8" else x.to(DTYPES[c["x"]])
        c["w"] = _pack(torch.randn((c["width"], c["dim"]), generator=g, device="cuda")
                       / math.sqrt(c["dim"]))
        c["b"] = torch.randn(c["width"], generator=g, device="cuda") if c["bias"] else None
    elif c["kind"] == "linear_grad":
        c["a"] = _pack(_features(g, c["rows"], c["dim"]))
        c["w"] = _pack(torch.randn((c["width"], c["dim"]), generator=g, device="cuda")
                       / math.sqrt(c["dim"]))
        c["d"] = _normal(g, (c["rows"], c["width"]), DTYPES[c["grad"]], 0.1)
    else:
        c["a"] = _features(g, c["rows"], c["dim"] * (2 if c["gated"] else 1)).to(DTYPES[c["x"]])
        if c["form"] == "step":
            c["d"] = _normal(g, (c["rows"], c["dim"]), DTYPES[c["x"]], 0.1)
    return c


# ---- the plain forms ----------------------------------------------------------------------

def _round(x):
    """(whole values, scales [rows, 1]) of x's 8-bit rows, in 32 bits; what the format rounds
    to 32 bits is computed in 64 and rounded there."""
    x = x.float()
    top = x.abs().amax(1, keepdim=True)
    fine = torch.isfinite(top)
    some = fine & (top >= 2.0 ** -100)
    scale = (torch.where(some, top, 1.0).double() / 127).float()
    scale = ((scale.view(torch.int32) + 0xffff) & -0x10000).view(torch.float32)
    inverse = (1 / scale.double()).float()
    q = torch.where(some, torch.round((x.double() * inverse.double()).float()), 0.0)
    return q, torch.where(some, scale, torch.where(fine, 0.0, math.nan))


def _pack(x):
    """[rows, dim] to the bytes of 8-bit rows."""
    rows, dim = x.shape
    q, scale = _round(x)
    n = (dim + 4 + 15) // 16 * 16
    packed = torch.zeros((rows, n), dtype=torch.uint8, device=x.device)
    packed[:, :dim] = q.to(torch.int8).view(torch.uint8)
    packed[:, n - 4:] = scale.contiguous().view(torch.uint8)
    return packed


def _unpack(packed, dim):
    """(whole values, scales [rows, 1]) of 8-bit rows, in 32 bits."""
    scale = packed[:, -4:].contiguous().view(torch.float32)
    return packed[:, :dim].contiguous().view(torch.int8).float(), scale


def _standard(v, norm):
    """(N(v), 1 / the root), row by row."""
    if norm == "layer":
        v = v - v.mean(1, keepdim=True)
    inverse = 1 / torch.sqrt(v.square().mean(1, keepdim=True) + EPS)
    return v * inverse, inverse


def _norm(s):
    b = s["b"].float()
    u = b if s["w1"] is None else _standard(b, s["norm"])[0] * s["w1"]
    u = u if s["b1"] is None else u + s["b1"]
    u = u if s["g"] is None else u * s["g"].float()
    total = (s["stream"].float() + s["scale"] * u).to(DTYPES[s["x"]])
    n = _standard(total.float(), s["norm"])[0] * s["w2"]
    n = n if s["b2"] is None else n + s["b2"]
    if s["out"] == "i8":
        q, scale = _round(n)
        return {"sum": total, "next": (q * scale).to(DTYPES[s["branch"]])}
    return {"sum": total, "next": n.to(DTYPES[s["branch"]])}


def _through(d, standard, inverse, norm):
    """The gradient to v of a gradient d to N(v)."""
    d = d - standard * (d * standard).mean(1, keepdim=True)
    if norm == "layer":
        d = d - d.mean(1, keepdim=True)
    return d * inverse


def _columns(x):
    return x.double().sum(0).float()


def _norm_grad(s):
    d_next, scale = s["d_next"].float(), s["scale"]
    standard, inverse = _standard(s["stream"].float(), s["norm"])
    out = {"before": _columns(d_next * standard)}
    if s["b2"] is not None:
        out["before_bias"] = _columns(d_next)
    d = s["d_sum"].float() + _through(d_next * s["w2"], standard, inverse, s["norm"])
    out["x"] = d.to(DTYPES[s["x"]])
    b = s["b"].float()
    u = b
    if s["w1"] is not None:
        standard, inverse = _standard(b, s["norm"])
        u = standard * s["w1"]
        u = u if s["b1"] is None else u + s["b1"]
    if s["g"] is None:
        d = scale * d
    else:
        d_gate = scale * d * u
        out["gate"] = _columns(d_gate) if s["gate"] == "columns" else \
            d_gate.to(DTYPES[s["branch"]])
        d = scale * s["g"].float() * d
    if s["w1"] is not None:
        out["after"] = _columns(d * standard)
        if s["b1"] is not None:
            out["after_bias"] = _columns(d)
        d = _through(d * s["w1"], standard, inverse, s["norm"])
    out["branch"] = d.to(DTYPES[s["branch"]])
    return out


def _linear(s):
    x, sx = _unpack(s["a"], s["dim"]) if s["x"] == "i8" else _round(s["a"])
    w, sw = _unpack(s["w"], s["dim"])
    y = (x @ w.t()) * (sx * sw.t())
    if s["b"] is not None:
        y = y + s["b"]
    return y.to(DTYPES[s["out"]])


def _linear_grad(s):
    x, sx = _unpack(s["a"], s["dim"])
    w, sw = _unpack(s["w"], s["dim"])
    d = s["d"].float()
    # the sum over all rows in parts, each in 32 bits
    rows, part = d.shape[0], 4096
    pad = -rows % part if rows > part else 0
    xs, ds = (torch.nn.functional.pad(t, (0, 0, 0, pad)) for t in (x * sx, d))
    parts = -(-rows // part)
    weight = torch.bmm(ds.view(parts, -1, s["width"]).transpose(1, 2),
                       xs.view(parts, -1, s["dim"]))
    return {"weight": weight.double().sum(0).float() if parts > 1 else weight[0],
            "bias": _columns(d), "x": (d @ (w * sw)).to(DTYPES[s["grad"]])}


def _f(v, f):
    """f(v) and f'(v)."""
    if f == "relu":
        return v.clamp(min=0), (v > 0).float()
    if f == "silu":
        p = 1 / (1 + torch.exp(-v))
        return v * p, p * (1 + v * (1 - p))
    # Phi(v), as 1 - Phi(-v) loses the tail
    p = 0.5 * torch.erfc(v * -math.sqrt(0.5))
    return v * p, p + v * torch.exp(-0.5 * v * v) * (1 / math.sqrt(2 * math.pi))


def _activation(s):
    x, dim = s["a"].float(), s["dim"]
    y = _f(x[:, :dim], s["f"])[0]
    y = y * x[:, dim:] if s["gated"] else y
    if s["out"] == "i8":
        q, scale = _round(y)
        y = q * scale
    y = y.to(DTYPES[s["x"]])
    if s["form"] == "forward":
        return {"y": y}
    q, scale = _round(x[:, :dim])
    value, slope = _f(q * scale, s["f"])
    d = s["d"].float()
    if s["gated"]:
        q, scale = _round(x[:, dim:])
        grad = torch.cat((d * slope * (q * scale), d * value), 1)
    else:
        grad = d * slope
    return {"y": y, "x": grad.to(DTYPES[s["x"]])}


# ---- one pass -------------------------------------------------------------------------------

def run(s):
    kind = s["kind"]
    if own:
        from paper_2601_01473_gb300 import ops
        if kind == "norm":
            arguments = {"gate": s["g"], "scale": s["scale"], "after": s["w1"],
                         "after_bias": s["b1"], "before": s["w2"], "before_bias": s["b2"],
                         "kind": s["norm"], "eps": EPS}
            if s["form"] == "forward":
                total, n = ops.residual_norm(s["stream"], s["b"], rows8=s["out"] == "i8",
                                             **arguments)
                if s["out"] == "i8":
                    n = ops.int8_dequantize(n, s["dim"], out_dtype=DTYPES[s["branch"]])
                return {"sum": total, "next": n}
            r = ops.residual_norm_grad(s["d_next"], s["d_sum"], s["stream"], s["b"], **arguments)
            return {k: v for k, v in r._asdict().items() if v is not None}
        if kind == "linear":
            x = s["a"] if s["x"] == "i8" else ops.int8_quantize(s["a"])
            return ops.int8_linear(x, s["w"], s["dim"], s["b"], out_dtype=DTYPES[s["out"]])
        if kind == "linear_grad":
            weight, bias = ops.int8_linear_grad_weight(s["d"], s["a"], s["dim"])
            return {"weight": weight, "bias": bias,
                    "x": ops.int8_linear_grad_input(s["d"], s["w"], s["dim"])}
        y, kept = ops.activation(s["a"], s["f"], gated=s["gated"], keep=s["form"] == "step",
                                 rows8=s["out"] == "i8")
        if s["out"] == "i8":
            y = ops.int8_dequantize(y, s["dim"], out_dtype=DTYPES[s["x"]])
        if s["form"] == "forward":
            return {"y": y}
        return {"y": y, "x": ops.activation_grad(s["d"], kept, s["f"], gated=s["gated"])}
    if kind == "norm":
        return _norm(s) if s["form"] == "forward" else _norm_grad(s)
    if kind == "linear":
        return _linear(s)
    if kind == "linear_grad":
        return _linear_grad(s)
    return _activation(s)


def _row_bytes(dim):
    return (dim + 4 + 15) // 16 * 16


def work(case):
    c = case
    if c["kind"] == "norm":
        cells, x, branch = c["rows"] * c["dim"], SIZE[c["x"]], SIZE[c["branch"]]
        full = branch if c["gate"] == "full" else 0
        vectors = 4 * c["dim"] * (1 + c["after"] + (c["gate"] == "columns")
                                  + c["bias"] * (1 + c["after"]))
        if c["form"] == "forward":
            out = c["rows"] * _row_bytes(c["dim"]) if c["out"] == "i8" else cells * branch
            return {"bytes": cells * (2 * x + branch + full) + out + vectors, "flops": 12 * cells}
        return {"bytes": cells * (3 * x + 3 * branch + 2 * full) + 2 * vectors,
                "flops": 30 * cells}
    if c["kind"] == "linear":
        row = _row_bytes(c["dim"]) if c["x"] == "i8" else c["dim"] * SIZE[c["x"]]
        return {"bytes": c["rows"] * row + c["width"] * _row_bytes(c["dim"])
                + c["rows"] * c["width"] * SIZE[c["out"]] + (4 * c["width"] if c["bias"] else 0),
                "flops": 2 * c["rows"] * c["dim"] * c["width"]}
    if c["kind"] == "linear_grad":
        return {"bytes": (c["rows"] + c["width"]) * _row_bytes(c["dim"])
                + (c["rows"] * (c["width"] + c["dim"])) * SIZE[c["grad"]]
                + 4 * c["width"] * (c["dim"] + 1),
                "flops": 4 * c["rows"] * c["dim"] * c["width"]}
    cells, n = c["rows"] * c["dim"], 2 if c["gated"] else 1
    kept = c["rows"] * _row_bytes(c["dim"])
    out = kept if c["out"] == "i8" else cells * SIZE[c["out"]]
    if c["form"] == "forward":
        return {"bytes": cells * n * SIZE[c["x"]] + out, "flops": 8 * cells}
    return {"bytes": cells * (2 * n + 1) * SIZE[c["x"]] + out + 2 * n * kept, "flops": 24 * cells}


# ---- the definitions in 64 bits ---------------------------------------------------------------

def _exact_rows(x):
    """The values of x's 8-bit rows, in 64 bits: a row at a time's scale by its definition."""
    x = x.double()
    top = x.abs().max(1).values[:, None]
    fp32 = lambda v: v.to(torch.float32).to(torch.float64)  # noqa: E731
    quotient = fp32(top / 127)
    # up to eight significant bits
    size = torch.exp2(torch.floor(torch.log2(quotient)) - 7)
    size = torch.where(quotient / size >= 256, size * 2, torch.where(quotient / size < 128,
                                                                     size / 2, size))
    scale = torch.ceil(quotient / size) * size
    values = torch.round(fp32(x * fp32(1 / scale))) * scale
    values = torch.where(top < 2.0 ** -100, 0.0, values)
    return torch.where(torch.isfinite(top), values, math.nan)


def _exact_values(packed, dim):
    scale = packed[:, -4:].clone().view(torch.float32).double()
    whole = packed[:, :dim].double()
    return torch.where(whole > 127, whole - 256, whole) * scale


def _layer_or_rms(v, w, bias, norm):
    """N(v) * w + bias as torch.autograd sees it."""
    if norm == "layer":
        y = (v - v.mean(1, keepdim=True)) / (v.var(1, unbiased=False, keepdim=True) + EPS).sqrt()
    else:
        y = v / ((v * v).sum(1, keepdim=True) / v.shape[1] + EPS).sqrt()
    y = y * w
    return y if bias is None else y + bias


def _exact_norm(s):
    double = lambda t: None if t is None else t.double()  # noqa: E731
    with torch.no_grad():
        u = s["b"].double()
        if s["w1"] is not None:
            u = _layer_or_rms(u, double(s["w1"]), double(s["b1"]), s["norm"])
        if s["g"] is not None:
            u = u * s["g"].double()
        total = s["stream"].double() + s["scale"] * u
        n = _layer_or_rms(total.to(DTYPES[s["x"]]).double(), double(s["w2"]), double(s["b2"]),
                          s["norm"])
        return {"sum": total, "next": _exact_rows(n) if s["out"] == "i8" else n}


def _exact_norm_grad(s):
    leaf = lambda t: None if t is None else t.double().requires_grad_()  # noqa: E731
    names = {"x": "stream", "branch": "b", "gate": "g", "after": "w1", "after_bias": "b1",
             "before": "w2", "before_bias": "b2"}
    v = {k: leaf(s[n]) for k, n in names.items()}
    # the sum is given: what led to it enters by its own derivative
    u = v["branch"]
    if v["after"] is not None:
        u = _layer_or_rms(u, v["after"], v["after_bias"], s["norm"])
    if v["gate"] is not None:
        u = u * v["gate"]
    u = u * s["scale"]
    total = v["x"] + (u - u.detach())
    n = _layer_or_rms(total, v["before"], v["before_bias"], s["norm"])
    keys = [k for k in names if v[k] is not None]
    grads = torch.autograd.grad((n * s["d_next"].double()).sum()
                                + (total * s["d_sum"].double()).sum(), [v[k] for k in keys])
    return dict(zip(keys, grads))


def _exact_f(v, f):
    if f == "relu":
        return torch.where(v > 0, v, 0.0), torch.where(v > 0, 1.0, 0.0).double()
    if f == "silu":
        p = torch.sigmoid(v)
        return v * p, p + v * p * torch.sigmoid(-v)
    p = 0.5 * torch.special.erfc(-v / math.sqrt(2))
    return v * p, p + v * torch.exp(-v * v / 2) / math.sqrt(2 * math.pi)


def exact(case, seed):
    s = prepare(case, seed)
    kind = s["kind"]
    if kind == "norm":
        return _exact_norm(s) if s["form"] == "forward" else _exact_norm_grad(s)
    if kind == "linear":
        x = _exact_values(s["a"], s["dim"]) if s["x"] == "i8" else _exact_rows(s["a"])
        y = x @ _exact_values(s["w"], s["dim"]).t()
        return y if s["b"] is None else y + s["b"].double()
    if kind == "linear_grad":
        x, w = _exact_values(s["a"], s["dim"]), _exact_values(s["w"], s["dim"])
        d = s["d"].double()
        return {"weight": d.t() @ x, "bias": d.sum(0), "x": d @ w}
    x, dim = s["a"].double(), s["dim"]
    y, _ = _exact_f(x[:, :dim], s["f"])
    if s["gated"]:
        y = y * x[:, dim:]
    if s["out"] == "i8":
        y = _exact_rows(y)
    if s["form"] == "forward":
        return {"y": y}
    value, slope = _exact_f(_exact_rows(s["a"][:, :dim]), s["f"])
    d = s["d"].double()
    if not s["gated"]:
        return {"y": y, "x": d * slope}
    return {"y": y, "x": torch.cat((d * slope * _exact_rows(s["a"][:, dim:]), d * value), 1)}
