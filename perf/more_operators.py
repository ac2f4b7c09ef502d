"""Cases of the operators that train a head or a projection, for measuring them through the package's public entry points.

Where the projection of hidden states is trained on the samples' labels (a handful of classes, or the entries of a
vocabulary), three operators stand between ``rcd_linear`` and the next weights:

  loss         ``Context.rcd_linear_cross_entropy``: z = x w^T + b; lse = log(sum(exp(z))); loss = lse - z[label], without
               the logits z in memory; rows whose label is negative are passed over
  loss_back    ``Context.rcd_linear_cross_entropy_backward``: gradients of x, w and b from those of loss and lse
  orthogonal   ``Context.rcd_orthogonalize``: a weight gradient on its way to the update, its singular values brought near
               one by Newton-Schulz products (X = G / |G|; X <- a X + (b A + c A^2) X with A = X X^T, five times)

Sizes are those of the package's workloads (10 and 1000 classes, rows 1300 to 50 000, widths 512 and 2048), and vocabularies and
hidden sizes around them.  Hidden rows lean towards their label's weights, as they do once training is under way; weight
gradients are noise with a few strong directions.
"""
import math

import torch

own = False
_context = None

_TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
_SIZE = {"bf16": 2, "fp16": 2, "fp32": 4}
_QUINTIC = (3.4445, -4.7750, 2.0315)
_STEPS = 5
_EPS = 1e-7


def listed():
    return [
        # One sample's loss over a vocabulary: every weight is read for one row.
        dict(name="loss_row", op="loss", rows=1, n=32000, k=2048, dtype="bf16", bias=False, ignored=False, pad=0),
        # The ten-class data set's loss from its features: few classes, many rows.
        dict(name="loss_classes", op="loss", rows=50000, n=10, k=512, dtype="bf16", bias=True, ignored=False, pad=0),
        # A batch of tokens over a vocabulary: the largest.
        dict(name="loss_vocab", op="loss", rows=8192, n=65536, k=4096, dtype="bf16", bias=False, ignored=True, pad=0),
        # Odd sizes in fp16: rows that do not start on 16 bytes, a vocabulary that ends inside a tile.
        dict(name="loss_odd", op="loss", rows=1300, n=5003, k=777, dtype="fp16", bias=True, ignored=True, pad=7),
        # A few samples through a small head: launches and latency.
        dict(name="back_few", op="loss_back", rows=32, n=1000, k=512, dtype="bf16", bias=True, dlse=False,
             ignored=False, pad=0),
        # A class-sized batch of the thousand-class data set.
        dict(name="back_classes", op="loss_back", rows=5000, n=1000, k=2048, dtype="bf16", bias=True, dlse=False,
             ignored=False, pad=0),
        # A training batch over a vocabulary.
        dict(name="back_vocab", op="loss_back", rows=8192, n=32768, k=4096, dtype="bf16", bias=False, dlse=True,
             ignored=True, pad=0),
        # Odd sizes in fp16, whose range the gradients of many a logit leave.
        dict(name="back_odd", op="loss_back", rows=1300, n=5003, k=1001, dtype="fp16", bias=True, dlse=True,
             ignored=True, pad=7),
        # The update of one projection from 2048 to 512 columns: fifteen products that wait for one another.
        dict(name="orthogonal_one", op="orthogonal", batch=1, rows=512, cols=2048, dtype="bf16", pad=0),
        # The projections of several heads, stacked.
        dict(name="orthogonal_stack", op="orthogonal", batch=8, rows=1024, cols=2048, dtype="bf16", pad=0),
        # A large square weight, its gradient in fp32.
        dict(name="orthogonal_large", op="orthogonal", batch=1, rows=4096, cols=4096, dtype="fp32", pad=0),
        # A tall one of odd sizes.
        dict(name="orthogonal_odd", op="orthogonal", batch=3, rows=1001, cols=333, dtype="fp16", pad=5),
    ]


def _log(rng, lo, hi):
    return int(round(lo * (max(lo, hi) / lo) ** rng.random()))


def _width(rng, lo, hi):
    """Mostly multiples of 64, as hidden sizes are, and any others."""
    d = _log(rng, lo, hi)
    return max(lo, d // 64 * 64) if d >= 64 and rng.random() < 0.7 else d


def draw(rng):
    op = rng.choice(["loss", "loss", "loss_back", "loss_back", "orthogonal"])
    pad = rng.choice([0, 0, 0, rng.randint(1, 64)])
    if op == "orthogonal":
        rows, cols = _width(rng, 16, 4096), _width(rng, 16, 4096)
        small, large = min(rows, cols), max(rows, cols)
        each = small * small * (3 * large + small)
        batch = max(1, min(rng.choice([1, 1, 2, 3, 8, 16]), int(4 * 4096 ** 3 / each)))
        return dict(op=op, batch=batch, rows=rows, cols=cols, dtype=rng.choice(["bf16", "bf16", "fp16", "fp32"]), pad=pad)
    k, n = _width(rng, 32, 8192), _width(rng, 2, 131072)
    most = 8192 * 65536 * 4096 if op == "loss" else 8192 * 32768 * 4096
    rows = _log(rng, 1, max(1, min(50000, int(5.0e8 / n), int(most / (n * k)))))
    dtype = rng.choice(["bf16", "bf16", "fp16"])
    case = dict(op=op, rows=rows, n=n, k=k, dtype=dtype, bias=rng.random() < 0.5, ignored=rng.random() < 0.5, pad=pad)
    if op == "loss_back":
        case.update(dlse=rng.random() < 0.5)
    return case


def _rows(g, rows, d, pad):
    return torch.randn(rows, d + pad, generator=g, device="cuda")


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed) * 7919 + 29)
    s = dict(case)
    t, pad, rows = _TYPES[case["dtype"]], case["pad"], case["rows"]
    if case["op"] == "orthogonal":
        batch, cols = case["batch"], case["cols"]
        x = torch.randn(batch, rows, cols + pad, generator=g, device="cuda")
        strong = torch.randn(batch, rows, 4, generator=g, device="cuda") @ torch.randn(batch, 4, cols + pad, generator=g, device="cuda")
        s["g"] = ((x + 2.0 * strong) * 1e-3).to(t)[:, :, :cols]
        return s
    n, k = case["n"], case["k"]
    w = torch.randn(n, k, generator=g, device="cuda") * (2.0 / math.sqrt(k))
    labels = torch.randint(0, n, (rows,), generator=g, device="cuda", dtype=torch.int32)
    x = _rows(g, rows, k, pad)
    x[:, :k] += 1.5 * w[labels.long()]
    if case["ignored"]:
        labels[torch.rand(rows, generator=g, device="cuda") < 0.1] = -100
    s["x"], s["w"], s["labels"] = x.to(t)[:, :k], w.to(t), labels
    s["b"] = 0.5 * torch.randn(n, generator=g, device="cuda") if case["bias"] else None
    if case["op"] == "loss_back":
        # (what the forward pass has handed over, and the gradients of a mean with weights and of lse^2's mean; in fp16 the
        # loss is scaled, as programs do that train in it)
        s["lse"] = _run_loss(s)["lse"]
        scale = (1024.0 if case["dtype"] == "fp16" else 1.0) / rows
        s["dloss"] = (0.5 + torch.rand(rows, generator=g, device="cuda")) * scale
        s["dlse"] = s["lse"] * (2e-2 * scale) if case["dlse"] else None
    return s


def _handle():
    """A program's context, made once."""
    global _context
    from paper_2211_00839_b200 import binding as rcd
    if _context is None:
        _context = rcd.Context(0)
    return _context


def _run_own(s):
    ctx = _handle()
    if s["op"] == "loss":
        loss, lse = ctx.rcd_linear_cross_entropy(s["x"], s["w"], s["labels"], bias=s["b"])
        return {"loss": loss, "lse": lse}
    if s["op"] == "loss_back":
        dx, dw, db = ctx.rcd_linear_cross_entropy_backward(s["x"], s["w"], s["labels"], s["lse"], bias=s["b"], dloss=s["dloss"],
                                                           dlse=s["dlse"], want_dbias=s["bias"])
        return {"dx": dx, "dw": dw, "db": db}
    return {"o": ctx.rcd_orthogonalize(s["g"], steps=_STEPS, coefficients=_QUINTIC, eps=_EPS)}


def _logits(s):
    z = s["x"].float() @ s["w"].float().t()
    return z if s["b"] is None else z + s["b"]


def _run_loss(s):
    z = _logits(s)
    top = z.amax(1, keepdim=True)
    lse = (top + torch.log(torch.exp(z - top).sum(1, keepdim=True)))[:, 0]
    labels = s["labels"].long()
    at = z[torch.arange(z.shape[0], device=z.device), labels.clamp(min=0)]
    return {"loss": torch.where(labels < 0, torch.zeros_like(lse), lse - at), "lse": lse}


def _run_loss_back(s):
    p = torch.exp(_logits(s) - s["lse"][:, None])
    labels = s["labels"].long()
    g = torch.where(labels < 0, torch.zeros_like(s["dloss"]), s["dloss"])
    dz = p * (g if s["dlse"] is None else g + s["dlse"])[:, None]
    dz[torch.arange(dz.shape[0], device=dz.device), labels.clamp(min=0)] -= g
    return {"dx": (dz @ s["w"].float()).to(s["x"].dtype), "dw": (dz.t() @ s["x"].float()).to(s["x"].dtype),
            "db": dz.sum(0) if s["bias"] else None}


def _run_orthogonal(s):
    x = s["g"].float()
    x = x / (torch.sqrt(x.square().sum((1, 2), keepdim=True)) + _EPS)
    tall = x.shape[1] > x.shape[2]
    if tall:
        x = x.transpose(1, 2)
    a, b, c = _QUINTIC
    for _ in range(_STEPS):
        m = x @ x.transpose(1, 2)
        x = a * x + (b * m + c * (m @ m)) @ x
    return {"o": (x.transpose(1, 2) if tall else x).to(torch.bfloat16)}


def run(state):
    if own:
        return _run_own(state)
    return {"loss": _run_loss, "loss_back": _run_loss_back, "orthogonal": _run_orthogonal}[state["op"]](state)


def work(case):
    e, rows = _SIZE[case["dtype"]], case["rows"]
    if case["op"] == "orthogonal":
        # (X X^T and A^2 are symmetric: half of their products)
        cols, batch = case["cols"], case["batch"]
        small, large = min(rows, cols), max(rows, cols)
        return {"bytes": batch * rows * cols * (e + 2),
                "flops": _STEPS * batch * (small * (small + 1) * (large + small) + 2 * small * small * large)}
    n, k = case["n"], case["k"]
    if case["op"] == "loss":
        return {"bytes": (rows + n) * k * e + 12 * rows + 4 * n * case["bias"], "flops": 2 * rows * n * k}
    return {"bytes": 2 * (rows + n) * k * e + (12 + 4 * case["dlse"]) * rows + 8 * n * case["bias"],
            "flops": 6 * rows * n * k}


def exact(case, seed):
    """From the definitions, in 64 bits."""
    s = prepare(case, seed)
    D = torch.float64
    if case["op"] == "orthogonal":
        # through the smaller Gram matrix alone: o = q x with q the product of the steps' polynomials of m = x x^T, m <- p m p
        x = s["g"].to(D)
        x = x / (torch.linalg.vector_norm(x, dim=(1, 2), keepdim=True) + _EPS)
        x = x.mT if case["rows"] > case["cols"] else x
        m = torch.einsum("bik,bjk->bij", x, x)
        one = torch.eye(m.shape[1], dtype=D, device=m.device)
        q = one.expand_as(m)
        a, b, c = _QUINTIC
        for _ in range(_STEPS):
            p = a * one + torch.einsum("bij,bjk->bik", m, b * one + c * m)
            q = torch.einsum("bij,bjk->bik", p, q)
            m = torch.einsum("bij,bjk,bkl->bil", p, m, p)
        o = torch.einsum("bij,bjk->bik", q, x)
        return {"o": o.mT if case["rows"] > case["cols"] else o}
    z = torch.einsum("rk,nk->rn", s["x"].to(D), s["w"].to(D))
    if s["b"] is not None:
        z += s["b"].to(D)
    labels = s["labels"].long()
    valid = labels >= 0
    picked = torch.zeros(z.shape[0], dtype=D, device=z.device)
    r = valid.nonzero()[:, 0]
    if case["op"] == "loss":
        picked[r] = z[r, labels[r]]
        lse = torch.logsumexp(z, dim=1)
        return {"loss": torch.where(valid, lse - picked, picked), "lse": lse}
    z -= s["lse"].to(D).unsqueeze(1)
    dz = z.exp_()
    dloss = s["dloss"].to(D) * valid
    dz *= (dloss if s["dlse"] is None else dloss + s["dlse"].to(D)).unsqueeze(1)
    dz[r, labels[r]] -= dloss[r]
    return {"dx": torch.einsum("rn,nk->rk", dz, s["w"].to(D)), "dw": torch.einsum("rn,rk->nk", dz, s["x"].to(D)),
            "db": dz.sum(0) if case["bias"] else None}
