"""The operators of a student model that is trained on prepared hyperbatches,
as a user's program calls them, and the plain form of each.

Five kinds of pass:

  "lookup"    rows of a learned table of node embeddings, scaled, for the nodes
              of a minibatch or a hyperbatch;
  "gradient"  that lookup's gradient, the tokens' gradients summed by node:
              "dense" (a row for every row of the table) or "rows" (a row for
              every distinct node, ascending, padded to the number of tokens);
  "distill"   the loss against a teacher's top logits and its gradient to the
              student's logits: "pair" (a forward and then a backward call) or
              "step" (both in one call, as a training step has them);
  "quantize"  feature rows to microscaled 4-bit rows and back;
  "product"   4-bit rows times 4-bit weights, as the first layer over gathered
              rows.

Embedding: out[t] = scale * table[ids[t]]; a negative id selects no row: zeros,
and no gradient.

Distillation: of row r's teacher entries those with a negative index are
absent.  p = softmax(teacher / T) over the others, q = softmax(logits / T) over
all classes, loss = T^2 sum_k p_k (log p_k - log q_k), and the gradient is
weight * T * (q sum_k p_k - sum_{k: index k = v} p_k).  A row without a teacher
entry, or whose logits are all -inf, has loss 0 and gradient 0.

4-bit rows: blocks of 32 values share a scale 2^(byte - 127), byte - 127 =
floor(log2(largest magnitude)) - 2, at least -127, and byte 255 where a value
is not finite; a value is the nearest of 0, 0.5, 1, 1.5, 2, 3, 4, 6 times the
scale, ties to the even code, with a sign in bit 3.  A row holds the codes of
its blocks (16 bytes each, the even element in the low half of a byte), then the
blocks' scale bytes, then zeros up to a multiple of 16 bytes; values past the
row's end are zeros.
"""
import math

import torch

own = False

DTYPES = {"f16": torch.float16, "bf16": torch.bfloat16, "f32": torch.float32}
SIZE = {"f16": 2, "bf16": 2, "f32": 4}


def listed():
    return [
        # an online request: the embeddings of one small minibatch's nodes; latency only
        {"name": "lookup_request", "kind": "lookup", "tokens": 200, "rows": 100_000, "dim": 128,
         "table": "f32", "out": "f32", "scale": 1.0, "index": "i32"},
        # all nodes of a hyperbatch, repeats and padding among them, from a table of 10M nodes
        {"name": "lookup_hyperbatch", "kind": "lookup", "tokens": 1_310_720, "rows": 10_000_000,
         "dim": 128, "table": "f16", "out": "f16", "scale": 11.3137085, "index": "i32"},
        # the backward pass of one small minibatch on a small graph; latency only
        {"name": "gradient_minibatch", "kind": "gradient", "form": "rows", "tokens": 1500,
         "rows": 100_000, "dim": 128, "grad": "f32", "out": "f32", "scale": 1.0, "index": "i32",
         "skew": 2.0},
        # a table small enough for a dense gradient: categories of nodes, rows of odd length,
        # hot rows with thousands of tokens
        {"name": "gradient_dense", "kind": "gradient", "form": "dense", "tokens": 300_001,
         "rows": 50_000, "dim": 301, "grad": "bf16", "out": "f32", "scale": 17.3493515,
         "index": "i64", "skew": 4.0},
        # the backward pass of a hyperbatch on a graph of 10M nodes
        {"name": "gradient_hyperbatch", "kind": "gradient", "form": "rows", "tokens": 1_000_003,
         "rows": 10_000_000, "dim": 128, "grad": "f16", "out": "f16", "scale": 11.3137085,
         "index": "i32", "skew": 3.0},
        # the targets of a small minibatch, the classes of a papers graph; latency only
        {"name": "distill_nodes", "kind": "distill", "form": "step", "rows": 300, "classes": 172,
         "top": 5, "logits": "f32", "out": "f32", "teacher": "f32", "temperature": 2.0,
         "index": "i32"},
        # few rows over a long axis (entities as classes), forward and backward apart
        {"name": "distill_entities", "kind": "distill", "form": "pair", "rows": 6,
         "classes": 250_001, "top": 100, "logits": "f16", "out": "f16", "teacher": "f16",
         "temperature": 1.0, "index": "i64"},
        # the targets of eight minibatches over a large vocabulary, in one training step
        {"name": "distill_step", "kind": "distill", "form": "step", "rows": 8192,
         "classes": 50_000, "top": 64, "logits": "bf16", "out": "bf16", "teacher": "f32",
         "temperature": 4.0, "index": "i32"},
        # a minibatch's raw features on their way into a 4-bit table, rows of odd length
        {"name": "quantize_minibatch", "kind": "quantize", "rows": 1000, "dim": 301,
         "values": "f32", "out": "f32"},
        # a table of features, as it is loaded
        {"name": "quantize_table", "kind": "quantize", "rows": 2_000_000, "dim": 128,
         "values": "f16", "out": "f16"},
        # an online request: a few nodes, a wide layer; latency and the weights' bytes count
        {"name": "product_request", "kind": "product", "rows": 4, "dim": 1024, "width": 4096,
         "out": "f16", "bias": True},
        # the first layer over the gathered rows of a hyperbatch
        {"name": "product_hyperbatch", "kind": "product", "rows": 786_432, "dim": 128,
         "width": 256, "out": "f16", "bias": True},
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["lookup", "gradient", "gradient", "distill", "distill", "quantize",
                       "product", "product"])
    float_type = lambda: rng.choice(["f16", "bf16", "f32"])  # noqa: E731
    index = rng.choice(["i32", "i64"])
    if kind == "lookup":
        dim = rng.choice([rng.randint(1, 64), rng.randint(8, 80) * 8, rng.randint(65, 700), 128])
        table, out = float_type(), float_type()
        most = 1_310_720 * 512 // (dim * (SIZE[table] + SIZE[out]))
        return {"kind": kind, "tokens": _log(rng, 1, min(most, 1_310_720)),
                "rows": _log(rng, 10, min(10_000_000, 2_500_000_000 // (dim * SIZE[table]))),
                "dim": dim, "table": table, "out": out, "index": index,
                "scale": round(rng.uniform(0.05, 20.0), 4)}
    if kind == "gradient":
        dim = rng.choice([rng.randint(1, 64), rng.randint(8, 80) * 8, rng.randint(65, 700), 128])
        form, grad = rng.choice(["dense", "rows"]), float_type()
        most = 1_000_003 * 256 // (dim * SIZE[grad])
        return {"kind": kind, "form": form, "tokens": _log(rng, 1, min(most, 1_000_003)),
                "rows": _log(rng, 10, min(10_000_000, 100_000_000 // dim) if form == "dense"
                             else 10_000_000),
                "dim": dim, "grad": grad, "out": rng.choice([grad, "f32"]), "index": index,
                "scale": round(rng.uniform(0.05, 20.0), 4), "skew": rng.choice([1.0, 2.0, 4.0])}
    if kind == "distill":
        classes = _log(rng, 2, 262_144)
        logits = float_type()
        most = 8192 * 50_000 * 2 // (classes * SIZE[logits])
        return {"kind": kind, "form": rng.choice(["pair", "step"]),
                "rows": _log(rng, 1, min(most, 16384)), "classes": classes,
                "top": min(classes, _log(rng, 1, 256)), "logits": logits, "out": logits,
                "teacher": rng.choice([logits, "f32"]), "index": index,
                "temperature": rng.choice([1.0, 2.0, round(rng.uniform(0.5, 8.0), 3)])}
    if kind == "quantize":
        dim, values = _log(rng, 1, 2048), float_type()
        most = 2_000_000 * 256 // (dim * SIZE[values])
        return {"kind": kind, "rows": _log(rng, 1, min(most, 2_000_000)), "dim": dim,
                "values": values, "out": values}
    dim, width, out = _log(rng, 16, 4096), _log(rng, 8, 4096), float_type()
    most = min(786_432 * 128 * 256 // (dim * width), 786_432 * 512 // (width * SIZE[out]),
               786_432 * 128 // dim)
    return {"kind": kind, "rows": _log(rng, 1, max(1, min(most, 786_432))), "dim": dim,
            "width": width, "out": out, "bias": rng.random() < 0.5}


# ---- inputs -------------------------------------------------------------------------------

def _ids(g, tokens, rows, skew, dtype):
    """Node ids with hubs: id rank u^skew, spread over the table; one in 50 is padding."""
    u = torch.rand(tokens, generator=g, device="cuda", dtype=torch.float64)
    rank = (u ** skew * rows).long().clamp_(max=rows - 1)
    step = next(p for p in (7919, 104729, 1299709, 15485863) if rows % p)
    ids = (rank * step) % rows
    pad = torch.rand(tokens, generator=g, device="cuda") < 0.02
    return torch.where(pad, -1, ids).to(torch.int32 if dtype == "i32" else torch.int64)


def _normal(g, shape, dtype, scale=1.0):
    return (torch.randn(shape, generator=g, device="cuda") * scale).to(dtype)


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    c = dict(case)
    if c["kind"] == "lookup":
        c["x"] = _normal(g, (c["rows"], c["dim"]), DTYPES[c["table"]], 0.1)
        c["ids"] = _ids(g, c["tokens"], c["rows"], 2.0, c["index"])
    elif c["kind"] == "gradient":
        c["x"] = _normal(g, (c["tokens"], c["dim"]), DTYPES[c["grad"]], 0.1)
        c["ids"] = _ids(g, c["tokens"], c["rows"], c["skew"], c["index"])
    elif c["kind"] == "distill":
        R, V, K = c["rows"], c["classes"], c["top"]
        first = torch.randint(0, V, (R, 1), generator=g, device="cuda")
        step = torch.randint(1, max(V // K, 1) + 1, (R, 1), generator=g, device="cuda")
        at = (first + step * torch.arange(K, device="cuda")) % V  # K distinct classes
        t = 8.0 - torch.rand((R, K), generator=g, device="cuda").mul_(4.0).cumsum(1).mul_(4.0 / K)
        t = t + torch.randn((R, K), generator=g, device="cuda").mul_(0.3)
        x = torch.randn((R, V), generator=g, device="cuda").mul_(1.5)
        x.scatter_add_(1, at, 0.6 * t + torch.randn((R, K), generator=g, device="cuda"))
        # a teacher that keeps fewer than K, and one row in 16 without a teacher at all
        keep = torch.randint(max(K // 2, 1), K + 1, (R, 1), generator=g, device="cuda")
        keep[5::16] = 0
        at = torch.where(torch.arange(K, device="cuda") < keep, at, -1)
        c["x"] = x.to(DTYPES[c["logits"]])
        c["t"] = t.to(DTYPES[c["teacher"]])
        c["at"] = at.to(torch.int32 if c["index"] == "i32" else torch.int64)
        c["weight"] = torch.rand(R, generator=g, device="cuda").add_(0.5).div_(R)
    elif c["kind"] == "quantize":
        c["x"] = _features(g, c["rows"], c["dim"]).to(DTYPES[c["values"]])
    else:
        c["x"] = _pack(_features(g, c["rows"], c["dim"]))
        c["w"] = _pack(torch.randn((c["width"], c["dim"]), generator=g, device="cuda")
                       / math.sqrt(c["dim"]))
        c["b"] = torch.randn(c["width"], generator=g, device="cuda") if c["bias"] else None
    return c


def _features(g, rows, dim):
    """Rows of differing magnitude, a few large values among them."""
    x = torch.randn((rows, dim), generator=g, device="cuda")
    x *= torch.exp2(torch.randn((rows, 1), generator=g, device="cuda"))
    return torch.where(torch.rand((rows, dim), generator=g, device="cuda") < 0.01, 6 * x, x)


# ---- the plain forms ----------------------------------------------------------------------

def _lookup(s):
    ids = s["ids"].long()
    x = s["x"][ids.clamp(min=0)].float() * s["scale"]
    return torch.where((ids >= 0)[:, None], x, 0.0).to(DTYPES[s["out"]])


def _gradient_dense(s):
    ids = s["ids"].long()
    rows, dim = s["rows"], s["dim"]
    total = torch.zeros((rows + 1, dim), device="cuda")
    total.index_add_(0, torch.where(ids < 0, rows, ids), s["x"].float())
    return (total[:rows] * s["scale"]).to(DTYPES[s["out"]])


def _gradient_rows(s):
    ids = s["ids"].long()
    T, rows = ids.numel(), s["rows"]
    key, token = torch.where(ids < 0, rows, ids).sort(stable=True)
    head = torch.ones(T, dtype=torch.bool, device="cuda")
    head[1:] = key[1:] != key[:-1]
    slot = torch.where(key < rows, head.long().cumsum(0) - 1, T)  # the last slot is padding's
    total = torch.zeros((T + 1, s["dim"]), device="cuda")
    total.index_add_(0, slot, s["x"][token].float())
    node = torch.full((T + 1,), -1, dtype=torch.int32, device="cuda")
    node.scatter_(0, slot, key.to(torch.int32))
    total[T] = 0
    count = (head & (key < rows)).sum(dtype=torch.int32).reshape(1)
    return {"ids": node[:T], "rows": (total[:T] * s["scale"]).to(DTYPES[s["out"]]), "count": count}


def _distill(s):
    T = s["temperature"]
    x = s["x"].float()
    top = x.amax(1, keepdim=True)
    alive = torch.isfinite(top)
    e = torch.exp((x - torch.where(alive, top, 0.0)) / T)
    total = e.sum(1, keepdim=True)
    at = s["at"].long()
    here = at >= 0
    t = torch.where(here, s["t"].float(), -math.inf)
    t_top = t.amax(1, keepdim=True)
    some = torch.isfinite(t_top) & alive
    t_e = torch.exp((t - torch.where(some, t_top, 0.0)) / T) * some
    t_total = torch.where(some, t_e.sum(1, keepdim=True), 1.0)
    p = t_e / t_total
    log_p = (t - t_top) / T - torch.log(t_total)
    log_q = (x.gather(1, at.clamp(min=0)) - top) / T - torch.log(total)
    loss = T * T * torch.where(p > 0, p * (log_p - log_q), 0.0).sum(1)
    grad = torch.where(some, e / total, 0.0)
    grad = grad.scatter_add(1, at.clamp(min=0), -p)
    grad = grad * (s["weight"] * T)[:, None]
    return loss, grad.to(DTYPES[s["out"]])


def _pack(x):
    """[rows, dim] to 4-bit rows."""
    rows, dim = x.shape
    blocks = (dim + 31) // 32
    v = torch.nn.functional.pad(x.float(), (0, blocks * 32 - dim)).view(rows, blocks, 32)
    top = v.abs().amax(2)
    fine = torch.isfinite(v).all(2)
    exponent = (torch.frexp(torch.where(fine, top, 0.0))[1] - 3).clamp(min=-127)
    exponent = torch.where(top > 0, exponent, -127)
    inverse = ((127 - exponent).to(torch.int32) << 23).view(torch.float32)
    v = torch.where(fine[:, :, None], v, 0.0)
    a = v.abs() * inverse[:, :, None]
    # the code is the number of midpoints passed; a tie goes to the even code
    code = ((a > 0.25).to(torch.uint8) + (a >= 0.75) + (a > 1.25) + (a >= 1.75) + (a > 2.5)
            + (a >= 3.5) + (a > 5.0))
    code = code + 8 * torch.signbit(v).to(torch.uint8)
    scale = torch.where(fine, exponent + 127, 255).to(torch.uint8)
    code = code.view(rows, blocks * 16, 2)
    packed = torch.zeros((rows, (blocks * 17 + 15) // 16 * 16), dtype=torch.uint8, device=x.device)
    packed[:, :blocks * 16] = code[:, :, 0] + 16 * code[:, :, 1]
    packed[:, blocks * 16:blocks * 17] = scale
    return packed


def _unpack(packed, dim):
    """4-bit rows to [rows, dim] in 32 bits."""
    rows, blocks = packed.shape[0], (dim + 31) // 32
    code = packed[:, :blocks * 16]
    code = torch.stack((code & 15, code >> 4), 2).view(rows, blocks, 32)
    values = torch.tensor([0, 0.5, 1, 1.5, 2, 3, 4, 6], device=packed.device)
    values = torch.cat((values, -values))
    byte = packed[:, blocks * 16:blocks * 17]
    # 2^(byte - 127) as a product of two powers, as 2^-127 has no normal form
    half = byte.to(torch.int32) >> 1
    scale = ((half + 64) << 23).view(torch.float32) * \
        ((byte.to(torch.int32) - half + 63) << 23).view(torch.float32)
    scale = torch.where(byte == 255, math.nan, scale)
    return (values[code.int()] * scale[:, :, None]).view(rows, blocks * 32)[:, :dim]


def _product(s):
    y = _unpack(s["x"], s["dim"]) @ _unpack(s["w"], s["dim"]).t()
    if s["b"] is not None:
        y = y + s["b"]
    return y.to(DTYPES[s["out"]])


# ---- one pass -------------------------------------------------------------------------------

def run(s):
    kind = s["kind"]
    if own:
        from paper_2601_01473_gb300 import ops
        if kind == "lookup":
            return ops.embedding_lookup(s["x"], s["ids"], s["scale"], out_dtype=DTYPES[s["out"]])
        if kind == "gradient":
            if s["form"] == "dense":
                return ops.embedding_grad(s["x"], s["ids"], s["rows"], s["scale"],
                                          out_dtype=DTYPES[s["out"]])
            r = ops.embedding_grad_rows(s["x"], s["ids"], s["rows"], s["scale"],
                                        out_dtype=DTYPES[s["out"]])
            return {"ids": r.ids, "rows": r.rows, "count": r.count}
        if kind == "distill":
            if s["form"] == "step":
                return ops.distill_loss_grad(s["x"], s["t"], s["at"], s["weight"],
                                             s["temperature"], out_dtype=DTYPES[s["out"]])
            loss, stats = ops.distill_loss(s["x"], s["t"], s["at"], s["temperature"])
            return loss, ops.distill_grad(s["x"], s["t"], s["at"], stats, s["weight"],
                                          s["temperature"], out_dtype=DTYPES[s["out"]])
        if kind == "quantize":
            packed = ops.mx4_quantize(s["x"])
            return ops.mx4_dequantize(packed, s["dim"], out_dtype=DTYPES[s["out"]])
        return ops.mx4_linear(s["x"], s["w"], s["dim"], s["b"], out_dtype=DTYPES[s["out"]])
    if kind == "lookup":
        return _lookup(s)
    if kind == "gradient":
        return _gradient_dense(s) if s["form"] == "dense" else _gradient_rows(s)
    if kind == "distill":
        return _distill(s)
    if kind == "quantize":
        return _unpack(_pack(s["x"]), s["dim"]).to(DTYPES[s["out"]])
    return _product(s)


def work(case):
    c = case
    if c["kind"] == "lookup":
        # distinct rows of the table are what has to be read; repeats are few in a large one
        read = min(c["tokens"], c["rows"]) * c["dim"] * SIZE[c["table"]]
        return {"bytes": read + c["tokens"] * (c["dim"] * SIZE[c["out"]] + _index_size(c)),
                "flops": c["tokens"] * c["dim"]}
    if c["kind"] == "gradient":
        out_rows = c["rows"] if c["form"] == "dense" else c["tokens"]
        extra = 4 * (c["tokens"] + 1) if c["form"] == "rows" else 0
        return {"bytes": c["tokens"] * (c["dim"] * SIZE[c["grad"]] + _index_size(c))
                + out_rows * c["dim"] * SIZE[c["out"]] + extra,
                "flops": c["tokens"] * c["dim"]}
    if c["kind"] == "distill":
        cells = c["rows"] * c["classes"]
        top = c["rows"] * c["top"] * (SIZE[c["teacher"]] + _index_size(c))
        if c["form"] == "step":  # the logits are read once
            return {"bytes": cells * (SIZE[c["logits"]] + SIZE[c["out"]]) + top + 8 * c["rows"],
                    "flops": 8 * cells}
        return {"bytes": cells * (2 * SIZE[c["logits"]] + SIZE[c["out"]]) + 2 * top
                + 24 * c["rows"], "flops": 10 * cells}
    if c["kind"] == "quantize":
        cells = c["rows"] * c["dim"]
        return {"bytes": cells * (SIZE[c["values"]] + SIZE[c["out"]])
                + 2 * c["rows"] * _row_bytes(c["dim"]), "flops": 4 * cells}
    return {"bytes": (c["rows"] + c["width"]) * _row_bytes(c["dim"])
            + c["rows"] * c["width"] * SIZE[c["out"]] + (4 * c["width"] if c["bias"] else 0),
            "flops": 2 * c["rows"] * c["dim"] * c["width"]}


def _index_size(c):
    return 4 if c["index"] == "i32" else 8


def _row_bytes(dim):
    return ((dim + 31) // 32 * 17 + 15) // 16 * 16


# ---- the definitions in 64 bits ---------------------------------------------------------------

_E2M1 = [0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0]


def _power(exponent):
    """2^exponent in 64 bits, by its bits."""
    return ((exponent.long() + 1023) << 52).view(torch.float64)


def _exact_values(packed, dim):
    """The values that 4-bit rows stand for, byte by byte."""
    blocks = (dim + 31) // 32
    out = torch.empty((packed.shape[0], blocks * 32), dtype=torch.float64, device=packed.device)
    sign_and_size = torch.tensor(_E2M1 + [-v for v in _E2M1], dtype=torch.float64,
                                 device=packed.device)
    out[:, 0::2] = sign_and_size[(packed[:, :blocks * 16] % 16).long()]
    out[:, 1::2] = sign_and_size[(packed[:, :blocks * 16] // 16).long()]
    exponent = packed[:, blocks * 16:blocks * 17].double() - 127
    scale = torch.where(exponent == 128, math.nan, _power(exponent))
    return (out * scale.repeat_interleave(32, 1))[:, :dim]


def _exact_rounded(x):
    """x with each block of 32 rounded to its 4-bit form: the nearest value of the grid, found by
    comparing distances, the even code first where two are as near."""
    rows, dim = x.shape
    x = x.double()
    out = torch.empty_like(x)
    grid = torch.tensor([_E2M1[i] for i in (0, 2, 4, 6, 1, 3, 5, 7)], dtype=torch.float64,
                        device=x.device)
    for b in range(0, dim, 32):
        v = x[:, b:b + 32]
        top = v.abs().amax(1, keepdim=True)
        exponent = torch.floor(torch.log2(top)).clamp(min=-1000, max=1000)  # may be one off
        exponent += (_power(exponent + 1) <= top).double() - (_power(exponent) > top).double()
        scale = _power(torch.clamp(exponent - 2, min=-127))
        size, best, value = v.abs() / scale, None, None
        for q in grid:
            far = (size - q).abs()
            if best is None:
                best, value = far, torch.zeros_like(far) + q
            else:
                value = torch.where(far < best, q, value)
                best = torch.minimum(far, best)
        out[:, b:b + 32] = torch.where(torch.isfinite(top), torch.copysign(value * scale, v),
                                       math.nan)
    return out


def exact(case, seed):
    s = prepare(case, seed)
    kind = s["kind"]
    if kind == "lookup":
        out = torch.zeros((s["tokens"], s["dim"]), dtype=torch.float64, device="cuda")
        real = s["ids"] >= 0
        out[real] = s["x"][s["ids"][real].long()].double() * s["scale"]
        return out
    if kind == "gradient":
        real = s["ids"] >= 0
        node, where = torch.unique(s["ids"][real], return_inverse=True)
        total = torch.zeros((node.numel(), s["dim"]), dtype=torch.float64, device="cuda")
        total.index_add_(0, where, s["x"][real].double() * s["scale"])
        if s["form"] == "dense":
            out = torch.zeros((s["rows"], s["dim"]), dtype=torch.float64, device="cuda")
            out[node.long()] = total
            return out
        out = torch.zeros((s["tokens"], s["dim"]), dtype=torch.float64, device="cuda")
        out[:node.numel()] = total
        ids = torch.full((s["tokens"],), -1, dtype=torch.int32, device="cuda")
        ids[:node.numel()] = node.to(torch.int32)
        return {"ids": ids, "rows": out,
                "count": torch.tensor([node.numel()], dtype=torch.int32, device="cuda")}
    if kind == "distill":
        loss = torch.zeros(s["rows"], dtype=torch.float64, device="cuda")
        grad = torch.zeros((s["rows"], s["classes"]), dtype=torch.float64, device="cuda")
        T = s["temperature"]
        for a in range(0, s["rows"], 512):
            part = slice(a, min(a + 512, s["rows"]))
            log_q = torch.log_softmax(s["x"][part].double() / T, 1)
            at = s["at"][part].long()
            t = s["t"][part].double().masked_fill(at < 0, -math.inf) / T
            some = (at >= 0).any(1)
            t[~some] = 0.0
            log_p = torch.log_softmax(t, 1)
            p = log_p.exp()
            p[~some] = 0.0
            at = at.clamp(min=0)
            loss[part] = T * T * torch.where(p > 0, p * (log_p - log_q.gather(1, at)), 0.0).sum(1)
            d = log_q.exp() * some[:, None]
            d.scatter_add_(1, at, -p)
            grad[part] = d * (T * s["weight"][part].double()[:, None])
        return loss, grad
    if kind == "quantize":
        return _exact_rounded(s["x"])
    y = _exact_values(s["x"], s["dim"]) @ _exact_values(s["w"], s["dim"]).t()
    return y if s["b"] is None else y + s["b"].double()
