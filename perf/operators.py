"""The dense operators beside the mini-batch path, as cases that can be timed.

What a vertex model does with gathered feature rows: it normalises them (rms_norm, in the type or
in 8 bits with scales), multiplies them by weights (linear, with bias, activation and residual in
one pass), and learns from the top logits that a teacher left for each vertex (distill).

A case is a dict of plain values.  "op" is the operator, "dir" the direction:
  norm     forward | backward     rows, dim, dtype; out "same" or "e4m3"; residual; ids (rows taken
                                  from a table of "nodes" rows by vertex ID)
  linear   forward | backward     m rows, k columns in, n out, dtype ("e4m3": 8-bit operands with
                                  scales, "out" the result's type); act, bias, residual; pre (the
                                  values before the activation are kept for the backward pass)
  distill  loss | step            rows, classes, top entries a row, dtype, temperature; step gives the
                                  loss and the gradient

`run` with `own` false is the plain form: elementary torch operations in 32 bits, rounded once at the
end.  With `own` true it calls the library.  `exact` is the definition in 64 bits.
"""
import math

import torch

own = False

DTYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16,
          "e4m3": torch.float8_e4m3fn}
SIZES = {"f32": 4, "f16": 2, "bf16": 2, "e4m3": 1}
EPS = 1e-6
E4M3_MAX = 448.0
TINY = 2.0 ** -126


def listed():
    return [
        # serving one vertex (or one token): the norm before an 8-bit product; latency is all
        {"name": "norm one row 8 bits", "op": "norm", "dir": "forward", "rows": 1, "dim": 1024,
         "dtype": "bf16", "out": "e4m3", "residual": True, "nodes": 0},
        # the input rows of a mini-batch, taken from a node type's float table by vertex ID and
        # written in 8 bits: the academic graph's papers, 128 floats a row
        {"name": "norm gathered rows 8 bits", "op": "norm", "dir": "forward", "rows": 150_001,
         "dim": 128, "dtype": "f32", "out": "e4m3", "residual": False, "nodes": 736_000},
        # a layer's norm in training: the residual stream is added, kept and normalised
        {"name": "norm residual", "op": "norm", "dir": "forward", "rows": 65_537, "dim": 1024,
         "dtype": "bf16", "out": "same", "residual": True, "nodes": 0},
        # its backward pass, with the residual stream's own gradient
        {"name": "norm backward", "op": "norm", "dir": "backward", "rows": 16_385, "dim": 4096,
         "dtype": "bf16", "out": "same", "residual": True, "nodes": 0},
        # serving one vertex in 8 bits: the weights are read once, and that is the time
        {"name": "linear one row 8 bits", "op": "linear", "dir": "forward", "m": 1, "k": 2048,
         "n": 8192, "dtype": "e4m3", "out": "bf16", "act": "silu", "bias": True,
         "residual": False, "pre": False},
        # offline inference in 8 bits: a large square product with the residual added
        {"name": "linear batch 8 bits", "op": "linear", "dir": "forward", "m": 16_384, "k": 4096,
         "n": 4096, "dtype": "e4m3", "out": "bf16", "act": "none", "bias": True,
         "residual": True, "pre": False},
        # a training layer on float rows of the academic graph: short rows, many of them
        {"name": "linear float rows", "op": "linear", "dir": "forward", "m": 150_001, "k": 128,
         "n": 256, "dtype": "f32", "out": "f32", "act": "relu", "bias": True, "residual": False,
         "pre": False},
        # a training layer on wide 16-bit features, activation and residual fused, the values
        # before the activation kept
        {"name": "linear wide features", "op": "linear", "dir": "forward", "m": 65_537, "k": 512,
         "n": 1024, "dtype": "bf16", "out": "bf16", "act": "gelu", "bias": True,
         "residual": True, "pre": True},
        # a hidden layer's backward pass: three results from one gradient
        {"name": "linear backward", "op": "linear", "dir": "backward", "m": 16_385, "k": 1024,
         "n": 4096, "dtype": "bf16", "out": "bf16", "act": "gelu", "bias": True,
         "residual": False, "pre": True},
        # vertex classification: a batch of seeds, some hundred classes
        {"name": "distill classes", "op": "distill", "dir": "step", "rows": 4096, "classes": 153,
         "top": 10, "dtype": "f32", "temperature": 2.0},
        # a vocabulary for classes (text on the vertices): loss and gradient of a training step
        {"name": "distill vocabulary step", "op": "distill", "dir": "step", "rows": 8193,
         "classes": 50_001, "top": 64, "dtype": "bf16", "temperature": 1.0},
        # evaluation over the longest rows: the loss alone
        {"name": "distill wide loss", "op": "distill", "dir": "loss", "rows": 2048,
         "classes": 131_072, "top": 16, "dtype": "f16", "temperature": 1.5},
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _width(rng, lo, hi):
    """A row's width: usually a multiple of 16 as models choose them, one in four any number."""
    d = _log_int(rng, lo, hi)
    d = d if rng.random() < 0.25 else max(16, d // 16 * 16)
    return d if d != 3072 else d - 16


def draw(rng):
    op = rng.choice(["norm", "linear", "linear", "distill"])
    dtype = rng.choice(["f32", "f16", "bf16", "bf16"])
    if op == "norm":
        back = rng.random() < 0.4
        case = {"op": "norm", "dir": "backward" if back else "forward",
                "rows": _log_int(rng, 1, 200_000), "dim": _width(rng, 16, 8192), "dtype": dtype,
                "out": "same" if back else rng.choice(["same", "e4m3"]),
                "residual": rng.random() < 0.6, "nodes": 0}
        if not back and rng.random() < 0.3:
            case["nodes"], case["dim"] = case["rows"] * rng.choice([1, 2, 5]) + 64, _width(rng, 16, 768)
        shrink = "rows"
    elif op == "linear":
        back = rng.random() < 0.35
        if not back and rng.random() < 0.4:
            dtype = "e4m3"
        m = _log_int(rng, 1, 150_000)
        case = {"op": "linear", "dir": "backward" if back else "forward", "m": m,
                "k": _width(rng, 16, 8192), "n": _width(rng, 16, 8192), "dtype": dtype,
                "out": rng.choice(["bf16", "f16", "f32"]) if dtype == "e4m3" else dtype,
                "act": rng.choice(["none", "relu", "gelu", "silu"]), "bias": rng.random() < 0.7,
                "residual": not back and rng.random() < 0.4, "pre": False}
        case["pre"] = case["act"] != "none" and (back or (dtype != "e4m3" and rng.random() < 0.5))
        shrink = "m"
    else:
        classes = _log_int(rng, 16, 131_072)
        case = {"op": "distill", "dir": rng.choice(["loss", "step"]),
                "rows": _log_int(rng, 1, 16_384), "classes": classes,
                "top": min(classes, _log_int(rng, 1, 128)), "dtype": dtype,
                "temperature": rng.choice([1.0, 1.5, 2.0, 4.0])}
        shrink = "rows"
    while _cost(case) > 1.6e9 and case[shrink] > 1:
        case[shrink] //= 2
    while _cost(case) > 1.6e9:
        case["n"] //= 2
    return case


def _cost(case):
    """Bytes, with a float operation of a product counted by what it takes in the plain form."""
    w = work(case)
    return max(w["bytes"], w["flops"] / 350)


def work(case):
    if case["op"] == "norm":
        s, M, D = SIZES[case["dtype"]], case["rows"], case["dim"]
        if case["dir"] == "backward":  # dy, the rows and (with a residual) its gradient in; dx out
            return {"bytes": float(M * D * s * (3 + case["residual"]) + 8 * D), "flops": 10.0 * M * D}
        b = M * D * s * (1 + 2 * case["residual"]) + 4 * D  # x; residual in and sum out
        b += M * D + 4 * M if case["out"] == "e4m3" else M * D * s
        return {"bytes": float(b + (8 * M if case["nodes"] else 0)), "flops": 6.0 * M * D}
    if case["op"] == "linear":
        m, k, n = case["m"], case["k"], case["n"]
        s, o = SIZES[case["dtype"]], SIZES[case["out"]]
        if case["dir"] == "backward":  # dy, x, w (and the values before the activation) in
            b = s * (m * n * (1 + case["pre"]) + 2 * m * k + 2 * n * k) + 4 * n * case["bias"]
            return {"bytes": float(b), "flops": 4.0 * m * k * n}
        b = s * (m * k + n * k) + o * m * n * (1 + case["residual"] + case["pre"])
        b += 4 * n * case["bias"] + (4 * (m + n) if case["dtype"] == "e4m3" else 0)
        return {"bytes": float(b), "flops": 2.0 * m * k * n}
    M, V, K, s = case["rows"], case["classes"], case["top"], SIZES[case["dtype"]]
    step = case["dir"] == "step"
    return {"bytes": float(M * V * s * (1 + step) + M * K * (8 + s) + 8 * M),
            "flops": 5.0 * M * V * (1 + step)}


def _normal(gen, *shape, dtype="f32", scale=1.0):
    x = torch.empty(shape, dtype=torch.float32, device="cuda").normal_(generator=gen)
    return x.mul_(scale).to(DTYPES[dtype])


def _to_8_bits(x):
    """Rows in 8 bits with a scale each, as weights are kept."""
    c = torch.clamp(x.abs().amax(1) / E4M3_MAX, min=TINY)
    return (x / c[:, None]).to(torch.float8_e4m3fn), c


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    dt = case["dtype"]
    st = {"case": case}
    if case["op"] == "norm":
        M, D = case["rows"], case["dim"]
        st["weight"] = 1 + _normal(gen, D, scale=0.1)  # kept in 32 bits, as an optimiser does
        # rows of unlike sizes, as hidden states are
        size = 1 + 3 * torch.rand((max(case["nodes"], M), 1), generator=gen, device="cuda")
        st["x"] = (_normal(gen, max(case["nodes"], M), D) * size).to(DTYPES[dt])
        st["ids"] = None
        if case["nodes"]:
            st["ids"] = torch.randperm(case["nodes"], generator=gen, device="cuda")[:M].contiguous()
        if case["dir"] == "backward":
            st["dy"] = _normal(gen, M, D, dtype=dt, scale=0.5)
            st["dsum"] = _normal(gen, M, D, dtype=dt, scale=0.5) if case["residual"] else None
        else:
            st["residual"] = _normal(gen, M, D, dtype=dt) if case["residual"] else None
        return st
    if case["op"] == "linear":
        m, k, n = case["m"], case["k"], case["n"]
        x, w = _normal(gen, m, k), _normal(gen, n, k, scale=k ** -0.5)
        st["x_scale"] = st["w_scale"] = None
        if dt == "e4m3":
            (st["x"], st["x_scale"]), (st["w"], st["w_scale"]) = _to_8_bits(x), _to_8_bits(w)
        else:
            st["x"], st["w"] = x.to(DTYPES[dt]), w.to(DTYPES[dt])
        st["bias"] = _normal(gen, n, scale=0.3) if case["bias"] else None
        if case["dir"] == "backward":
            st["dy"] = _normal(gen, m, n, dtype=dt)
            st["pre"] = _normal(gen, m, n, dtype=dt, scale=1.5) if case["pre"] else None
        else:
            st["residual"] = _normal(gen, m, n, dtype=case["out"]) if case["residual"] else None
        return st
    M, V, K = case["rows"], case["classes"], case["top"]
    st["logits"] = _normal(gen, M, V, dtype=dt, scale=2.0)
    # distinct classes per row, the teacher's logits in descending order
    start = torch.randint(V, (M, 1), generator=gen, device="cuda")
    st["ids"] = (start + torch.arange(K, device="cuda") * (V // K)) % V
    t = torch.sort(_normal(gen, M, K, scale=2.0) + 6, 1, descending=True)[0]
    # lists of unlike lengths: every 7th row keeps half of its entries, every 31st none
    row = torch.arange(M, device="cuda")[:, None]
    kept = torch.where(row % 31 == 30, 0, torch.where(row % 7 == 6, (K + 1) // 2, K))
    st["ids"] = torch.where(torch.arange(K, device="cuda") < kept, st["ids"], -1)
    st["teacher"] = t.to(DTYPES[dt])
    # the loss is a mean over the rows; one row in 13 has no part in it
    st["row_weight"] = torch.where(row[:, 0] % 13 == 12, 0.0, 1.0 / M).to(torch.float32)
    return st


# ---- the plain forms -----------------------------------------------------------------------


def _act(z, act):
    if act == "relu":
        return torch.where(z > 0, z, torch.zeros_like(z))
    if act == "gelu":
        return 0.5 * z * (1 + torch.tanh(math.sqrt(2 / math.pi) * (z + 0.044715 * z * z * z)))
    if act == "silu":
        return z / (1 + torch.exp(-z))
    return z


def _act_grad(z, act):
    if act == "relu":
        return (z > 0).to(z.dtype)
    if act == "gelu":
        t = torch.tanh(math.sqrt(2 / math.pi) * (z + 0.044715 * z * z * z))
        return (0.5 * (1 + t)
                + 0.5 * z * (1 - t * t) * math.sqrt(2 / math.pi) * (1 + 3 * 0.044715 * z * z))
    if act == "silu":
        s = 1 / (1 + torch.exp(-z))
        return s * (1 + z * (1 - s))
    return torch.ones_like(z)


def _plain_norm(st):
    case = st["case"]
    x = (st["x"] if st["ids"] is None else st["x"][st["ids"]]).float()
    h = x + st["residual"].float() if st["residual"] is not None else x
    y = h * (1 / torch.sqrt((h * h).mean(1, keepdim=True) + EPS)) * st["weight"]
    out = {}
    if case["out"] == "e4m3":
        out["y"], out["scale"] = _to_8_bits(y)
    else:
        out["y"] = y.to(st["x"].dtype)
    if st["residual"] is not None:
        out["sum"] = h.to(st["x"].dtype)
    return out


def _plain_norm_grad(st):
    h, dy, w = st["x"].float(), st["dy"].float(), st["weight"]
    s = 1 / torch.sqrt((h * h).mean(1, keepdim=True) + EPS)
    g = dy * w
    dx = s * (g - h * (s * s) * (g * h).mean(1, keepdim=True))
    if st["dsum"] is not None:
        dx = dx + st["dsum"].float()
    return {"dx": dx.to(st["x"].dtype), "dweight": (dy * (h * s)).sum(0)}


def _plain_linear(st):
    case = st["case"]
    z = st["x"].float() @ st["w"].float().t()
    if st["x_scale"] is not None:
        z = z * st["x_scale"][:, None] * st["w_scale"]
    if st["bias"] is not None:
        z = z + st["bias"]
    y = _act(z, case["act"])
    if st["residual"] is not None:
        y = y + st["residual"].float()
    out = {"y": y.to(DTYPES[case["out"]])}
    if case["pre"]:
        out["pre"] = z.to(DTYPES[case["out"]])
    return out


def _plain_linear_grad(st):
    case = st["case"]
    dz = st["dy"].float()
    if st["pre"] is not None:
        dz = dz * _act_grad(st["pre"].float(), case["act"])
    out = {"dx": (dz @ st["w"].float()).to(st["x"].dtype),
           "dw": (dz.t() @ st["x"].float()).to(st["w"].dtype)}
    if case["bias"]:
        out["dbias"] = dz.sum(0)
    return out


def _plain_distill(st):
    case = st["case"]
    T = case["temperature"]
    ids, a = st["ids"], st["row_weight"]
    valid = ids >= 0
    some = valid.any(1)
    t = torch.where(valid, st["teacher"].float() / T, -math.inf)
    e = torch.where(valid, torch.exp(t - torch.where(some, t.amax(1), 0.0)[:, None]), 0.0)
    p = e / torch.where(some, e.sum(1), 1.0)[:, None]
    z = st["logits"].float() / T
    top = z.amax(1, keepdim=True)
    e = torch.exp(z - top)
    total = e.sum(1, keepdim=True)
    at = torch.where(valid, ids, 0)
    log_q = z.gather(1, at) - top - torch.log(total)
    loss = torch.where(p > 0, p * (torch.log(torch.where(p > 0, p, 1.0)) - log_q), 0.0).sum(1)
    out = {"loss": loss}
    if case["dir"] == "step":
        g = e / total
        g.scatter_add_(1, at, -p)
        g = g * torch.where(some, a / T, 0.0)[:, None]
        out["grad"] = g.to(st["logits"].dtype)
    return out


# ---- one pass ------------------------------------------------------------------------------


def run(st):
    case = st["case"]
    kind = (case["op"], case["dir"])
    if not own:
        return {("norm", "forward"): _plain_norm, ("norm", "backward"): _plain_norm_grad,
                ("linear", "forward"): _plain_linear, ("linear", "backward"): _plain_linear_grad,
                ("distill", "loss"): _plain_distill, ("distill", "step"): _plain_distill}[kind](st)
    import paper_2112_15345_amd as hg
    if kind == ("norm", "forward"):
        y, h, scale = hg.rms_norm(st["x"], st["weight"], residual=st["residual"], ids=st["ids"],
                                  eps=EPS, out_dtype=torch.float8_e4m3fn
                                  if case["out"] == "e4m3" else None)
        out = {"y": y, "sum": h, "scale": scale}
    elif kind == ("norm", "backward"):
        dx, dw = hg.rms_norm_grad(st["dy"], st["x"], st["weight"], dsum=st["dsum"], eps=EPS)
        out = {"dx": dx, "dweight": dw}
    elif kind == ("linear", "forward"):
        y, pre = hg.linear(st["x"], st["w"], bias=st["bias"], act=case["act"],
                           residual=st["residual"], x_scale=st["x_scale"], w_scale=st["w_scale"],
                           out_dtype=DTYPES[case["out"]], keep_pre=case["pre"])
        out = {"y": y, "pre": pre}
    elif kind == ("linear", "backward"):
        dx, dw, db = hg.linear_grad(st["dy"], st["x"], st["w"], pre=st["pre"], act=case["act"],
                                    want_dbias=case["bias"])
        out = {"dx": dx, "dw": dw, "dbias": db}
    else:
        loss, grad = hg.distill(st["logits"], st["ids"], st["teacher"],
                                temperature=case["temperature"], row_weight=st["row_weight"],
                                want_grad=case["dir"] == "step")
        out = {"loss": loss, "grad": grad}
    return {k: v for k, v in out.items() if v is not None}


# ---- the definitions in 64 bits ------------------------------------------------------------


def _sigmoid64(z):
    return torch.sigmoid(z)


def _slope64(z, act):
    """Derivative of the activation, by its parts: gelu is z sigmoid(2 u(z)), silu z sigmoid(z)."""
    if act == "none":
        return torch.ones_like(z)
    if act == "relu":
        return torch.heaviside(z, torch.zeros((), dtype=z.dtype, device=z.device))
    if act == "silu":
        u, du = z, 1.0
    else:
        c = math.sqrt(8 / math.pi)
        u, du = c * (z + 0.044715 * z ** 3), c * (1 + 0.134145 * z ** 2)
    s = _sigmoid64(u)
    return s + z * s * (1 - s) * du


def _value64(z, act):
    if act == "none":
        return z
    if act == "relu":
        return z.clamp(min=0)
    return z * _sigmoid64(z if act == "silu" else math.sqrt(8 / math.pi) * (z + 0.044715 * z ** 3))


def exact(case, seed):
    st = prepare(case, seed)
    kind = (case["op"], case["dir"])
    if kind == ("norm", "forward"):
        h = st["x"].double()
        if st["ids"] is not None:
            h = h.index_select(0, st["ids"])
        if st["residual"] is not None:
            h = h + st["residual"].double()
        y = h / ((h.square().sum(1) / case["dim"] + EPS).sqrt()[:, None]) * st["weight"].double()
        out = {"y": y}
        if case["out"] == "e4m3":  # before its rounding to 8 bits
            out["scale"] = (y.abs().max(1)[0] / E4M3_MAX).clamp(min=TINY)
            out["y"] = y / out["scale"][:, None]
        if st["residual"] is not None:
            out["sum"] = h
        return out
    if kind == ("norm", "backward"):
        h, dy, w = st["x"].double(), st["dy"].double(), st["weight"].double()
        r = (h.square().sum(1) / case["dim"] + EPS).rsqrt()[:, None]
        n = h * r
        g = dy * w
        dx = r * (g - n * ((g * n).sum(1) / case["dim"])[:, None])
        dx = dx if st["dsum"] is None else dx + st["dsum"].double()
        return {"dx": dx, "dweight": torch.einsum("md,md->d", dy, n)}
    if kind == ("linear", "forward"):
        x, w = st["x"].double(), st["w"].double()
        if st["x_scale"] is not None:
            x, w = x * st["x_scale"].double()[:, None], w * st["w_scale"].double()[:, None]
        z = torch.matmul(x, w.T)
        if st["bias"] is not None:
            z += st["bias"].double()
        y = _value64(z, case["act"])
        if st["residual"] is not None:
            y = y + st["residual"].double()
        return {"y": y, "pre": z} if case["pre"] else {"y": y}
    if kind == ("linear", "backward"):
        dz = st["dy"].double()
        if st["pre"] is not None:
            dz = dz * _slope64(st["pre"].double(), case["act"])
        out = {"dx": torch.matmul(dz, st["w"].double()), "dw": torch.matmul(dz.T, st["x"].double())}
        if case["bias"]:
            out["dbias"] = dz.sum(0)
        return out
    T = case["temperature"]
    off = st["ids"] < 0
    empty = off.all(1)
    log_p = torch.log_softmax((st["teacher"].double() / T).masked_fill(off, -math.inf), 1)
    p = log_p.exp().masked_fill(off, 0.0)
    log_q = torch.log_softmax(st["logits"].double() / T, 1)
    at = st["ids"].clamp(min=0)
    each = p * (log_p - log_q.gather(1, at))
    out = {"loss": each.masked_fill(off, 0.0).sum(1)}
    if case["dir"] == "step":
        g = log_q.exp().scatter_add(1, at, -p)
        g *= (st["row_weight"].double() / T)[:, None]
        out["grad"] = g.masked_fill(empty[:, None], 0.0)
    return out
