"""Cases of the operators that turn hidden states into the features a partition reads, for measuring them through the
package's public entry points.

A data set of texts comes as hidden states of a language model: rows of the residual stream, one per sample.  Between
them and ``rcd_partition``'s features lie a root-mean-square norm (with the residual's addition, and int8 or 16-bit
output) and a projection (a matrix product with bias, activation and residual), and, where the projection is trained,
their backward passes.

  norm         ``Context.rcd_rms_norm``: h = x + r; y = h * w / sqrt(mean(h^2) + eps), as 16 or 32 bits, as int8 with a
               scale per row, or as int8 with one given scale; without the norm, ``Context.rcd_quantize_rows``
  norm_back    ``Context.rcd_rms_norm_backward``: gradients of x (the same as r's) and w
  linear       ``Context.rcd_linear``: act(x w^T + b) + r for bf16, fp16, and int8 with scales of rows and columns
  linear_back  ``Context.rcd_linear_backward``: gradients of x, w and b

Sizes are those of the package's workloads (rows 400 to 50 000, feature widths 64, 512, 2048), and hidden sizes up to
8192 around them.  Hidden states have a few columns that are much larger than the others, as residual streams do.

int8 outputs are returned as the integers themselves, beside their scales in fp32.  Their arithmetic is laid down step by
step (one fp32 operation each), so that two implementations give the same integers.
"""
import math

import torch

own = False
_context = None

_TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32, "int8": torch.int8}
_SIZE = {"bf16": 2, "fp16": 2, "fp32": 4, "int8": 1}


def listed():
    return [
        # One sample's hidden state, normalised on arrival: launches and latency.
        dict(name="norm_row", op="norm", rows=1, d=2048, dtype="bf16", out="bf16", residual=True, weight=True, pad=0),
        # The data set's hidden states (fifty thousand rows of 2048) to int8 with a scale per row, for the int8 projection;
        # the sum goes on as the residual stream.
        dict(name="norm_int8", op="norm", rows=50000, d=2048, dtype="bf16", out="int8", residual=True, weight=True, pad=0),
        # Projected features of the ten-class data set, fp32, to int8 of one scale: what the exact partition reads.
        dict(name="norm_features", op="norm", rows=50000, d=512, dtype="fp32", out="features", residual=False, weight=False,
             pad=0),
        # A training batch's backward pass through the norm, hidden size 4096, the residual stream's gradient joined.
        dict(name="norm_back", op="norm_back", rows=16384, d=4096, dtype="bf16", residual=True, weight=True, pad=0),
        # The same at an odd width, in fp16, rows with a stride of their own.
        dict(name="norm_back_odd", op="norm_back", rows=1300, d=1001, dtype="fp16", residual=False, weight=True, pad=7),
        # One sample through the projection: every weight is read for one row.
        dict(name="linear_row", op="linear", rows=1, n=2048, k=2048, dtype="bf16", out="bf16", act="silu", residual=False,
             bias=True, pre=False, pad=0),
        # A few samples through a wide int8 projection.
        dict(name="linear_few", op="linear", rows=32, n=4096, k=4096, dtype="int8", out="bf16", act="none", residual=True,
             bias=True, pre=False, pad=0),
        # One class (5000 samples) projected from 2048 to 512 columns in training: the values before the activation are kept.
        dict(name="linear_class", op="linear", rows=5000, n=512, k=2048, dtype="bf16", out="bf16", act="gelu", residual=False,
             bias=True, pre=True, pad=0),
        # The whole data set through an int8 projection of the hidden size: the largest.
        dict(name="linear_int8", op="linear", rows=50000, n=2048, k=2048, dtype="int8", out="bf16", act="none", residual=True,
             bias=True, pre=False, pad=0),
        # Odd sizes in fp16: rows that do not start on 16 bytes, edges inside every tile.
        dict(name="linear_odd", op="linear", rows=1300, n=333, k=777, dtype="fp16", out="fp16", act="relu", residual=True,
             bias=True, pre=False, pad=0),
        # A class's backward pass through the projection from 2048 to 512 columns.
        dict(name="linear_back_class", op="linear_back", rows=5000, n=512, k=2048, dtype="bf16", dw="bf16", act="gelu",
             bias=True, pad=0),
        # A training batch's backward pass at hidden size 4096, weight gradients in fp32.
        dict(name="linear_back", op="linear_back", rows=8192, n=4096, k=4096, dtype="bf16", dw="fp32", act="none", bias=True,
             pad=0),
    ]


def _log(rng, lo, hi):
    return int(round(lo * (max(lo, hi) / lo) ** rng.random()))


def _width(rng, lo, hi):
    """Mostly multiples of 64, as hidden sizes are, and any others."""
    d = _log(rng, lo, hi)
    return max(lo, d // 64 * 64) if d >= 64 and rng.random() < 0.7 else d


def draw(rng):
    op = rng.choice(["norm", "norm", "norm_back", "linear", "linear", "linear", "linear_back"])
    pad = rng.choice([0, 0, 0, rng.randint(1, 64)])
    if op in ("norm", "norm_back"):
        d = _width(rng, 32, 8192)
        rows = _log(rng, 1, min(50000, int(1.0e8 if op == "norm" else 6.5e7) // d))
        if op == "norm":
            return dict(op=op, rows=rows, d=d, dtype=rng.choice(["bf16", "fp16", "fp32"]),
                        out=rng.choice(["same", "bf16", "int8", "int8", "features", "quantize"]),
                        residual=rng.random() < 0.5, weight=rng.random() < 0.7, pad=pad)
        return dict(op=op, rows=rows, d=d, dtype=rng.choice(["bf16", "fp16", "fp32"]), residual=rng.random() < 0.5,
                    weight=rng.random() < 0.8, pad=pad)
    k, n = _width(rng, 32, 8192), _width(rng, 16, 8192)
    most = 2.0e11 if op == "linear" else 1.3e11
    rows = _log(rng, 1, min(50000, int(most / (n * k))))
    act = rng.choice(["none", "relu", "gelu", "gelu_tanh", "silu"])
    if op == "linear":
        dtype = rng.choice(["bf16", "fp16", "int8"])
        out = "bf16" if dtype == "int8" else dtype
        return dict(op=op, rows=rows, n=n, k=k, dtype=dtype, out=rng.choice([out, out, "fp32"]), act=act,
                    residual=rng.random() < 0.5, bias=rng.random() < 0.8, pre=act != "none" and rng.random() < 0.3, pad=pad)
    dtype = rng.choice(["bf16", "fp16"])
    # (gradients of the weights are kept in fp32 where no activation's derivative is rounded on the way to them)
    return dict(op=op, rows=rows, n=n, k=k, dtype=dtype, dw=rng.choice([dtype, "fp32"]) if act == "none" else dtype, act=act,
                bias=rng.random() < 0.8, pad=pad)


def _hidden(g, rows, d, dtype, pad, spread=True):
    """Rows of a residual stream: normal values, one column in 64 ten times as large, rows of unequal length.  With `pad` the
    rows lie that many elements further apart than they are long."""
    x = torch.randn(rows, d + pad, generator=g, device="cuda")
    if spread:
        big = torch.rand(d + pad, generator=g, device="cuda") < 1.0 / 64
        x *= torch.where(big, 10.0, 1.0) * (0.5 + torch.rand(rows, 1, generator=g, device="cuda"))
    return x.to(dtype)[:, :d]


def _plain(g, rows, d, dtype, pad, size=1.0):
    return (torch.randn(rows, d + pad, generator=g, device="cuda") * size).to(dtype)[:, :d]


#: The one scale of int8 features: rows of root mean square 1, cut off at four times that.
_SCALE = 4.0 / 127.0
_EPS = 1e-6


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed) * 7919 + 13)
    s = dict(case)
    t, pad, rows = _TYPES[case["dtype"]], case["pad"], case["rows"]
    if case["op"] == "norm":
        d = case["d"]
        s["x"] = _hidden(g, rows, d, t, pad)
        s["r"] = _plain(g, rows, d, t, pad) if case["residual"] else None
        s["w"] = (1.0 + 0.2 * torch.randn(d, generator=g, device="cuda")).to(t) if case["weight"] else None
    elif case["op"] == "norm_back":
        d = case["d"]
        s["h"] = _hidden(g, rows, d, t, pad)
        s["dy"] = _plain(g, rows, d, t, 0)
        s["dsum"] = _plain(g, rows, d, t, 0) if case["residual"] else None
        s["w"] = (1.0 + 0.2 * torch.randn(d, generator=g, device="cuda")).to(t) if case["weight"] else None
    else:
        n, k = case["n"], case["k"]
        if case["dtype"] == "int8":
            s["x"] = torch.randint(-127, 128, (rows, k + pad), generator=g, device="cuda", dtype=torch.int8)[:, :k]
            s["w"] = torch.randint(-127, 128, (n, k), generator=g, device="cuda", dtype=torch.int8)
            s["sx"] = (0.5 + torch.rand(rows, generator=g, device="cuda")) / 73.0
            s["sw"] = (0.5 + torch.rand(n, generator=g, device="cuda")) / (73.0 * math.sqrt(k))
        else:
            s["x"] = _hidden(g, rows, k, t, pad, spread=False)
            s["w"] = _plain(g, n, k, t, 0, 1.0 / math.sqrt(k))
            s["sx"] = s["sw"] = None
        s["b"] = 0.2 * torch.randn(n, generator=g, device="cuda") if case["bias"] else None
        if case["op"] == "linear":
            s["r"] = _plain(g, rows, n, _TYPES[case["out"]], 0) if case["residual"] else None
        else:
            s["dy"] = _plain(g, rows, n, t, 0)
            s["pre"] = _plain(g, rows, n, t, 0) if case["act"] != "none" else None
    return s


def _handle():
    """A program's context, made once."""
    global _context
    from paper_2211_00839_b200 import binding as rcd
    if _context is None:
        _context = rcd.Context(0)
    return rcd, _context


def _run_own(s):
    rcd, ctx = _handle()
    op = s["op"]
    if op == "norm":
        if s["out"] == "quantize":
            q, scales = ctx.rcd_quantize_rows(s["x"])
            return {"q": q, "scales": scales}
        kind = _TYPES["int8"] if s["out"] in ("int8", "features") else s["x"].dtype if s["out"] == "same" else _TYPES[s["out"]]
        y, scales, total = ctx.rcd_rms_norm(s["x"], residual=s["r"], weight=s["w"], eps=_EPS, out_dtype=kind,
                                            scale=_SCALE if s["out"] == "features" else None, want_sum=s["residual"])
        return {"y": y, "scales": scales, "sum": total}
    if op == "norm_back":
        dx, dw = ctx.rcd_rms_norm_backward(s["dy"], s["h"], weight=s["w"], eps=_EPS, dsum=s["dsum"])
        return {"dx": dx, "dw": dw}
    act = {"none": rcd.RCD_ACT_NONE, "relu": rcd.RCD_ACT_RELU, "gelu": rcd.RCD_ACT_GELU, "gelu_tanh": rcd.RCD_ACT_GELU_TANH,
           "silu": rcd.RCD_ACT_SILU}[s["act"]]
    if op == "linear":
        y, pre = ctx.rcd_linear(s["x"], s["w"], bias=s["b"], residual=s["r"], activation=act, x_scales=s["sx"],
                                w_scales=s["sw"], out_dtype=_TYPES[s["out"]], want_preact=s["pre"])
        return {"y": y, "pre": pre}
    dx, dw, db = ctx.rcd_linear_backward(s["dy"], s["x"], s["w"], preact=s["pre"], activation=act, dw_dtype=_TYPES[s["dw"]],
                                         want_dbias=s["bias"])
    return {"dx": dx, "dw": dw, "db": db}


def _int8_rows(t, rstd):
    """q = rint(t * (127 / a)), a the row's largest |t|; scale = rstd * a / 127.  Every step is one fp32 operation (tensors
    divide tensors: a division by a number would be a product with its reciprocal)."""
    a = t.abs().amax(1, keepdim=True)
    top = torch.full_like(a, 127.0)
    inv = torch.where(a > 0, torch.div(top, a), torch.zeros_like(a)).clamp(max=torch.finfo(torch.float32).max)
    return torch.round(t * inv).to(torch.int8), torch.div(rstd * a, top)[:, 0]


def _run_norm(s):
    h = s["x"].float()
    if s["out"] == "quantize":
        q, scales = _int8_rows(h, torch.ones(h.shape[0], 1, device=h.device))
        return {"q": q, "scales": scales}
    if s["r"] is not None:
        h = h + s["r"].float()
    t = h * s["w"].float() if s["w"] is not None else h
    # (in 64 bits for features: a value next to a border between two integers has to fall on the same side every time)
    ms = (h.double().square().mean(1, keepdim=True) if s["out"] == "features" else h.square().mean(1, keepdim=True)) + _EPS
    rstd = (1.0 / torch.sqrt(ms)).float()
    scales = None
    if s["out"] == "int8":
        y, scales = _int8_rows(t, rstd)
    elif s["out"] == "features":
        inv = torch.div(torch.ones((), device="cuda"), torch.tensor(_SCALE, dtype=torch.float32, device="cuda"))
        y = torch.round((t * rstd) * inv).clamp(-127, 127).to(torch.int8)
    else:
        y = (t * rstd).to(s["x"].dtype if s["out"] == "same" else _TYPES[s["out"]])
    return {"y": y, "scales": scales, "sum": h.to(s["x"].dtype) if s["residual"] else None}


def _run_norm_back(s):
    dy, h = s["dy"].float(), s["h"].float()
    rstd = 1.0 / torch.sqrt(h.square().mean(1, keepdim=True) + _EPS)
    g = dy * s["w"].float() if s["w"] is not None else dy
    dx = rstd * (g - h * (rstd.square() * (g * h).mean(1, keepdim=True)))
    if s["dsum"] is not None:
        dx = dx + s["dsum"].float()
    return {"dx": dx.to(s["h"].dtype), "dw": (dy * h * rstd).sum(0) if s["w"] is not None else None}


_R2, _R2PI, _K0, _K1 = math.sqrt(0.5), 1.0 / math.sqrt(2.0 * math.pi), math.sqrt(2.0 / math.pi), 0.044715


def _act(z, kind):
    if kind == "relu":
        return z.clamp(min=0)
    if kind == "gelu":
        return 0.5 * z * (1.0 + torch.erf(z * _R2))
    if kind == "gelu_tanh":
        return 0.5 * z * (1.0 + torch.tanh(_K0 * (z + _K1 * z * z * z)))
    if kind == "silu":
        return z / (1.0 + torch.exp(-z))
    return z


def _slope(z, kind):
    if kind == "relu":
        return (z > 0).to(z.dtype)
    if kind == "gelu":
        return 0.5 * (1.0 + torch.erf(z * _R2)) + z * torch.exp(-0.5 * z * z) * _R2PI
    if kind == "gelu_tanh":
        t = torch.tanh(_K0 * (z + _K1 * z * z * z))
        return 0.5 * (1.0 + t) + 0.5 * z * (1.0 - t * t) * _K0 * (1.0 + 3.0 * _K1 * z * z)
    if kind == "silu":
        p = 1.0 / (1.0 + torch.exp(-z))
        return p * (1.0 + z * (1.0 - p))
    return torch.ones_like(z)


def _run_linear(s):
    if s["sx"] is not None:          # (sums of up to k products of 127 * 127 pass 24 bits: exact in 64)
        z = (s["x"].double() @ s["w"].double().t()).float() * s["sx"][:, None] * s["sw"][None, :]
    else:
        z = s["x"].float() @ s["w"].float().t()
    if s["b"] is not None:
        z = z + s["b"]
    y = _act(z, s["act"])
    if s["r"] is not None:
        y = y + s["r"].float()
    out = _TYPES[s["out"]]
    return {"y": y.to(out), "pre": z.to(out) if s["pre"] else None}


def _run_linear_back(s):
    dz = s["dy"].float()
    if s["pre"] is not None:
        dz = dz * _slope(s["pre"].float(), s["act"])
    t = s["x"].dtype
    return {"dx": (dz @ s["w"].float()).to(t), "dw": (dz.t() @ s["x"].float()).to(_TYPES[s["dw"]]),
            "db": dz.sum(0) if s["bias"] else None}


def run(state):
    if own:
        return _run_own(state)
    return {"norm": _run_norm, "norm_back": _run_norm_back, "linear": _run_linear, "linear_back": _run_linear_back}[state["op"]](state)


def work(case):
    e, rows = _SIZE[case["dtype"]], case["rows"]
    if case["op"] == "norm":
        d = case["d"]
        o = {"same": e, "bf16": 2}.get(case["out"], 1)
        streams = 1 if case["out"] == "quantize" or not case["residual"] else 3          # x; x, r and the sum
        return {"bytes": rows * d * (streams * e + o), "flops": 6 * rows * d}
    if case["op"] == "norm_back":
        d = case["d"]
        return {"bytes": rows * d * e * (4 if case["residual"] else 3) + 4 * d, "flops": 12 * rows * d}
    n, k = case["n"], case["k"]
    if case["op"] == "linear":
        o = _SIZE[case["out"]]
        return {"bytes": (rows + n) * k * e + rows * n * o * (1 + case["residual"] + case["pre"]), "flops": 2 * rows * n * k}
    kept = 0 if case["act"] == "none" else 1
    return {"bytes": (2 * rows * k + n * k + (1 + kept) * rows * n) * e + n * k * _SIZE[case["dw"]], "flops": 4 * rows * n * k}


def exact(case, seed):
    """From the definitions, in 64 bits.  int8 outputs have no such value (each is a choice between two integers), their
    scales do."""
    s = prepare(case, seed)
    D = torch.float64
    if case["op"] == "norm":
        if case["out"] == "quantize":
            return {"q": None, "scales": s["x"].to(D).abs().max(dim=1).values / 127}
        h = s["x"].to(D)
        h = h if s["r"] is None else h + s["r"].to(D)
        if case["out"] == "features" and not case["residual"]:
            return None
        norm = torch.linalg.vector_norm(h, dim=1) / math.sqrt(case["d"])
        y = h / torch.sqrt(norm ** 2 + _EPS).unsqueeze(1)
        y = y if s["w"] is None else y * s["w"].to(D)
        return {"y": None if case["out"] in ("int8", "features") else y,
                "scales": torch.linalg.vector_norm(y, ord=math.inf, dim=1) / 127 if case["out"] == "int8" else None,
                "sum": h if case["residual"] else None}
    if case["op"] == "norm_back":
        # through the unit vectors: y = c u * w with u = h / |h|, c = |h| / sqrt(mean(h^2) + eps)
        h, dy = s["h"].to(D), s["dy"].to(D)
        g = dy if s["w"] is None else dy * s["w"].to(D)
        v = h.pow(2).sum(1, keepdim=True) / case["d"] + _EPS
        dx = g / v.sqrt() - h * torch.einsum("rc,rc->r", g, h).unsqueeze(1) / (case["d"] * v.pow(1.5))
        dx = dx if s["dsum"] is None else dx + s["dsum"].to(D)
        return {"dx": dx, "dw": None if s["w"] is None else torch.einsum("rc,rc->c", dy, h / v.sqrt())}
    x, w = s["x"].to(D), s["w"].to(D)
    if case["op"] == "linear":
        if s["sx"] is not None:
            x, w = x * s["sx"].to(D).unsqueeze(1), w * s["sw"].to(D).unsqueeze(1)
        z = torch.einsum("mk,nk->mn", x, w)
        z = z if s["b"] is None else z + s["b"].to(D)
        y = _act64(z, case["act"])[0]
        return {"y": y if s["r"] is None else y + s["r"].to(D), "pre": z if case["pre"] else None}
    dz = s["dy"].to(D)
    dz = dz if s["pre"] is None else dz * _act64(s["pre"].to(D), case["act"])[1]
    return {"dx": torch.einsum("mn,nk->mk", dz, w), "dw": torch.einsum("mn,mk->nk", dz, x),
            "db": torch.einsum("mn->n", dz) if case["bias"] else None}


def _act64(z, kind):
    """An activation and its derivative, written apart from the plain forms: through the normal distribution and the
    logistic function (tanh(u) = 2 / (1 + exp(-2u)) - 1)."""
    if kind == "none":
        return z, torch.ones_like(z)
    if kind == "relu":
        on = torch.heaviside(z, torch.zeros((), dtype=z.dtype, device=z.device))
        return z * on, on
    if kind == "gelu":
        p = torch.special.ndtr(z)
        return z * p, p + z * torch.exp(-z * z / 2) / math.sqrt(2 * math.pi)
    if kind == "silu":
        p = torch.sigmoid(z)
        return z * p, p + z * p * torch.sigmoid(-z)
    u = 2 * math.sqrt(2 / math.pi) * (z + 0.044715 * z ** 3)
    p, du = torch.sigmoid(u), 2 * math.sqrt(2 / math.pi) * (1 + 3 * 0.044715 * z ** 2)
    return z * p, p + z * p * torch.sigmoid(-u) * du
