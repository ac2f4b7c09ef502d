"""Softmax cross entropy of a linear head without its logits in memory, and its gradients, against 64 bits.

Most inputs are small multiples of a power of two, so that the logits are exact in fp32 whatever the order of their sums: what is measured
then is the softmax's own arithmetic."""
import math

import pytest

from test_gpu_norm import ctx, half_step, kind, rcd, rows, seeded  # noqa: F401  (fixtures)

pytestmark = pytest.mark.gpu
U = 2.0 ** -24


def grid(g, n, d, dtype, pad=0, shift=0, most=4, step=2.0 ** -3):
    """Multiples of `step` up to `most` of them, laid out like rows()."""
    import torch
    x = (torch.randint(-most, most + 1, (n * (d + pad) + shift,), generator=g, device="cuda").double() * step).to(dtype)
    return x[shift:].view(n, d + pad)[:, :d]


def head(g, m, n, k, dtype, pad=0, shift=0, bias=True, spread=None):
    """x, w, bias and labels with exact logits of a few units; a tenth of the rows passed over."""
    import torch
    x = grid(g, m, k, dtype, pad, shift)
    w = grid(g, n, k, dtype, pad, 0, step=2.0 ** -(3 + int(math.log2(max(k, 4)) / 2)) if spread is None else spread)
    b = torch.randint(-32, 33, (n,), generator=g, device="cuda").float() / 16 if bias else None
    y = torch.randint(0, n, (m,), generator=g, device="cuda", dtype=torch.int32)
    y[torch.rand(m, generator=g, device="cuda") < 0.1] = -1
    return x, w, b, y


def logits64(x, w, b):
    z = x.double() @ w.double().t()
    return z if b is None else z + b.double()


def loss_bound(z, lse, n):
    """Of lse: each term's exponential 2 units and the argument's roundings (their mean is the entropy, log n at most); up to 4 + n / 32
    / 32 + 32 times a partial sum is brought to another reference (an exponential, two products, an addition); the logarithm."""
    joins = 4 + n / 1024 + 34
    return joins * 2.0 ** -21 + math.log(n + 1) * 2.0 ** -21 + 2.0 ** -20 + lse.abs() * 2.0 ** -22


def check_loss(ctx, x, w, b, y, z_slack=0.0):
    import torch
    loss, lse = ctx.rcd_linear_cross_entropy(x, w, y, bias=b)
    z = logits64(x, w, b)
    want = torch.logsumexp(z, 1)
    n = w.shape[0]
    bound = loss_bound(z, want, n) + z_slack
    assert loss.dtype == lse.dtype == torch.float32 and loss.shape == lse.shape == y.shape
    assert float(((lse.double() - want).abs() - bound).max()) <= 0
    at = z.gather(1, y.long().clamp(min=0)[:, None])[:, 0]
    wl = torch.where(y < 0, torch.zeros_like(want), want - at)
    assert float(((loss.double() - wl).abs() - bound - z_slack - (want.abs() + at.abs()) * 2 * U).max()) <= 0
    assert not loss[y < 0].any()
    return loss, lse


# rows and classes around the tiles' sizes, widths around a slab's and beyond a chunk of sums
SIZES = [(1, 1, 1), (1, 2, 64), (1, 5003, 64), (2, 32, 8), (3, 33, 72), (5, 1000, 520), (31, 63, 65), (32, 1000, 512), (33, 10, 128), (65, 300, 256), (127, 129, 64),
         (128, 256, 128), (129, 257, 65), (200, 64, 2048), (256, 512, 256), (300, 1, 33), (333, 777, 1001), (500, 2100, 192), (1300, 1000, 512), (700, 31, 777),
         (64, 40, 4608), (5000, 10, 512), (20000, 7, 64), (40, 33000, 64), (2100, 4100, 72)]


@pytest.mark.parametrize("m,n,k", SIZES)
@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("pad,shift,bias", [(0, 0, True), (3, 1, False)])
def test_loss(rcd, ctx, m, n, k, dtype, pad, shift, bias):
    g = seeded("loss", m, n, k, dtype, pad)
    x, w, b, y = head(g, m, n, k, kind(dtype), pad, shift, bias)
    check_loss(ctx, x, w, b, y)
    ctx.sync_status()


@pytest.mark.parametrize("m,n,k", [(1, 700, 300), (300, 1000, 2048), (260, 5003, 777), (70, 400, 8192)])
@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
def test_loss_of_real_values(rcd, ctx, m, n, k, dtype):
    """Logits are off by what a sum of products loses: within 512 k (1024 without a chunk) a unit each of the sum of their sizes, and half a unit per chunk."""
    import torch
    g = seeded("real", m, n, k, dtype)
    x, w = rows(g, m, k, kind(dtype)), rows(g, n, k, kind(dtype), size=2 * k ** -0.5)
    y = torch.randint(0, n, (m,), generator=g, device="cuda", dtype=torch.int32)
    size = float((x.double().abs() @ w.double().abs().t()).max())
    check_loss(ctx, x, w, None, y, z_slack=2 * size * 2 * U * (min(k, 1024) + k / 512))
    ctx.sync_status()


def gradients64(x, w, b, y, lse, dloss, dlse):
    import torch
    z = logits64(x, w, b)
    n = w.shape[0]
    valid = (y >= 0) & (y < n)
    g = torch.where(valid, torch.ones_like(lse).double() if dloss is None else dloss.double(), torch.zeros_like(lse).double())
    gl = torch.zeros_like(g) if dlse is None else dlse.double()
    none = torch.isneginf(lse)[:, None]
    d = torch.where(none, torch.full_like(z, -math.inf), z - lse.double()[:, None])
    p = torch.exp(d)
    dz = torch.where(((g + gl) == 0)[:, None], torch.zeros_like(p), p * (g + gl)[:, None])
    mark = torch.zeros_like(dz)
    mark[torch.arange(len(y), device=y.device), y.long().clamp(0, n - 1)] = g
    dz = dz - mark
    # fp32 steps: the difference and its product with log2(e) three halves of a unit each of the exponent, the exponential 2 units, two
    # products, the subtraction at the label
    slack = p * (g.abs() + gl.abs())[:, None] * (d.abs().clamp(max=200) * 4 * U + 8 * U) + 2 * U * (mark.abs() + dz.abs()) + 2.0 ** -126
    most = float((g.abs() + gl.abs()).max())
    return dz, slack, most


def check_back(ctx, x, w, b, y, lse, dloss, dlse, got, dtype, dw_dtype=None, pieces=1):
    import torch
    dx, dw, db = got
    dz, slack, most = gradients64(x, w, b, y, lse, dloss, dlse)
    # dz as the products take it: rounded to the type; fp16's smallest step is 2^-24, with the largest gradient at 2^13 or more
    half = dz.abs() * half_step(dtype) + slack * (1 + half_step(dtype)) + (most * 2.0 ** -38 if dtype == torch.float16 else 0)
    m, n = dz.shape

    def near(out, want, bound, sizes, terms, out_type):
        # sums lose a unit a term at most within 4096 (they cut off), half a unit per chunk of 512 or piece beyond
        bound = bound + sizes * 2 * U * (min(terms, 4096) + terms / 512 + 2 * pieces)
        bound = bound * (1 + half_step(out_type)) + want.abs() * half_step(out_type) + torch.finfo(out_type).tiny * half_step(out_type) * 2
        worst = float(((out.double() - want).abs() - bound).max())
        assert worst <= 0, worst
    if dx is not None:
        aw = w.double().abs()
        near(dx, dz @ w.double(), half @ aw, (dz.abs() + half) @ aw, n, dtype)
    if dw is not None:
        ax = x.double().abs()
        near(dw, dz.t() @ x.double(), half.t() @ ax, (dz.abs() + half).t() @ ax, m, dtype if dw_dtype is None else dw_dtype)
    if db is not None:
        assert db.dtype == torch.float32
        # (32 rows by halves, then a tree over the groups: under 32 + m / 32 roundings)
        bound = slack.sum(0) + dz.abs().sum(0) * U * (8 + m / 1024 + 40) + dz.sum(0).abs() * U + 2.0 ** -126
        assert float(((db.double() - dz.sum(0)).abs() - bound).max()) <= 0


@pytest.mark.parametrize("m,n,k", SIZES)
@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("pad,shift,bias,given", [(0, 0, True, "both"), (3, 1, False, "loss"), (8, 0, True, "none")])
def test_gradients(rcd, ctx, m, n, k, dtype, pad, shift, bias, given):
    import torch
    t, g = kind(dtype), seeded("back", m, n, k, dtype, pad)
    x, w, b, y = head(g, m, n, k, t, pad, shift, bias)
    _, lse = ctx.rcd_linear_cross_entropy(x, w, y, bias=b)
    dloss = (0.5 + torch.rand(m, generator=g, device="cuda")) / m if given != "none" else None
    dlse = torch.randn(m, generator=g, device="cuda") * 0.1 / m if given == "both" else None
    got = ctx.rcd_linear_cross_entropy_backward(x, w, y, lse, bias=b, dloss=dloss, dlse=dlse)
    ctx.sync_status()
    assert got[0].dtype == got[1].dtype == t and got[0].shape == x.shape and got[1].shape == w.shape
    check_back(ctx, x, w, b, y, lse, dloss, dlse, got, t)
    # each alone, and fp32 weight gradients
    dx, none, none2 = ctx.rcd_linear_cross_entropy_backward(x, w, y, lse, bias=b, dloss=dloss, dlse=dlse, want_dw=False, want_dbias=False)
    assert none is None and none2 is None and torch.equal(dx, got[0])
    _, dw, _ = ctx.rcd_linear_cross_entropy_backward(x, w, y, lse, bias=b, dloss=dloss, dlse=dlse, want_dx=False, want_dbias=False)
    assert torch.equal(dw, got[1])
    _, dw, db = ctx.rcd_linear_cross_entropy_backward(x, w, y, lse, bias=b, dloss=dloss, dlse=dlse, want_dx=False, dw_dtype=torch.float32)
    assert torch.equal(db, got[2])
    check_back(ctx, x, w, b, y, lse, dloss, dlse, (None, dw, db), t, torch.float32)
    ctx.sync_status()


@pytest.mark.parametrize("m,n,k,piece", [(50, 1000, 128, 64), (300, 777, 257, 256), (1, 300, 64, 100), (129, 200, 72, 199), (700, 2100, 512, 512), (64, 65, 33, 64), (33, 64, 64, 1)])
@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
def test_pieces_of_the_classes(rcd, ctx, m, n, k, piece, dtype):
    """Several pieces: dx adds up over them, and every class's gradients come from its own."""
    import torch
    t, g = kind(dtype), seeded("pieces", m, n, k, dtype)
    x, w, b, y = head(g, m, n, k, t)
    _, lse = ctx.rcd_linear_cross_entropy(x, w, y, bias=b)
    dloss = torch.randn(m, generator=g, device="cuda") / m
    dlse = torch.randn(m, generator=g, device="cuda") / m
    got = ctx.rcd_linear_cross_entropy_backward(x, w, y, lse, bias=b, dloss=dloss, dlse=dlse, piece=piece)
    ctx.sync_status()
    check_back(ctx, x, w, b, y, lse, dloss, dlse, got, t, pieces=-(-n // max(64, piece // 64 * 64)))
    whole = ctx.rcd_linear_cross_entropy_backward(x, w, y, lse, bias=b, dloss=dloss, dlse=dlse)
    assert torch.equal(whole[2], got[2])                      # (a class's sum over the rows does not depend on its piece)


def test_small_gradients_in_fp16(rcd, ctx):
    """dloss of 2^-30: gradients of logits far below fp16's range, whose products are right all the same where the output's type holds them."""
    import torch
    g = seeded("small")
    x, w, b, y = head(g, 200, 300, 128, torch.float16)
    _, lse = ctx.rcd_linear_cross_entropy(x, w, y, bias=b)
    dloss = torch.full((200,), 2.0 ** -30, device="cuda")
    _, dw, db = ctx.rcd_linear_cross_entropy_backward(x, w, y, lse, bias=b, dloss=dloss, want_dx=False, dw_dtype=torch.float32)
    check_back(ctx, x, w, b, y, lse, dloss, None, (None, dw, db), torch.float16, torch.float32)
    assert dw.abs().max() > 0
    # nothing to pass back
    dx, dw, db = ctx.rcd_linear_cross_entropy_backward(x, w, y, lse, bias=b, dloss=torch.zeros_like(dloss))
    assert not dx.any() and not dw.any() and not db.any()
    ctx.sync_status()


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("n", [5, 300, 2100])
def test_closed_classes_and_rows_without_any(rcd, ctx, n, dtype):
    """Biases of -inf and of the type's lowest value close classes; a label among them has an infinite loss and finite gradients; where none
    is open lse is -inf, and p 0."""
    import torch
    t, g = kind(dtype), seeded("closed", n, dtype)
    m, k = 70, 64
    for low in (-math.inf, -3.4028234663852886e38):
        x, w, b, y = head(g, m, n, k, t)
        b[::2] = low
        y[0], y[1] = 0, 1
        loss, lse = ctx.rcd_linear_cross_entropy(x, w, y, bias=b)
        z = logits64(x, w, b)
        want = torch.logsumexp(z, 1)
        assert float(((lse.double() - want).abs() - loss_bound(z, want, n)).max()) <= 0
        assert float(loss[0]) == math.inf if low == -math.inf else float(loss[0]) > 3e38
        assert torch.isfinite(loss[1])
        dx, dw, db = ctx.rcd_linear_cross_entropy_backward(x, w, y, lse, bias=b)
        check_back(ctx, x, w, b, y, lse, None, None, (dx, dw, db), t)
        ctx.sync_status()
    b[:] = -math.inf
    y[:3] = torch.tensor([0, -1, 1], device="cuda", dtype=torch.int32)
    loss, lse = ctx.rcd_linear_cross_entropy(x, w, y, bias=b)
    assert bool((lse == -math.inf).all()) and math.isnan(float(loss[0])) and float(loss[1]) == 0.0
    dx, dw, db = ctx.rcd_linear_cross_entropy_backward(x, w, y, lse, bias=b)
    check_back(ctx, x, w, b, y, lse, None, None, (dx, dw, db), t)
    ctx.sync_status()


def test_infinities_and_nan_stay_in_their_rows(rcd, ctx):
    import torch
    g = seeded("inf")
    x, w, b, y = head(g, 150, 400, 64, torch.bfloat16)
    y = y.clamp(min=0)
    clean, clean_lse = ctx.rcd_linear_cross_entropy(x, w, y, bias=b)
    xn = x.clone()
    xn[7] = float("nan")
    xn[140, 3] = float("inf")
    loss, lse = ctx.rcd_linear_cross_entropy(xn, w, y, bias=b)
    others = torch.ones(150, dtype=torch.bool, device="cuda")
    others[[7, 140]] = False
    assert torch.equal(loss[others], clean[others]) and torch.equal(lse[others], clean_lse[others])
    assert math.isnan(float(loss[7])) and math.isnan(float(lse[7])) and not math.isfinite(float(lse[140]))
    # +inf in the bias of one class: lse is +inf for every row
    b2 = b.clone()
    b2[5] = float("inf")
    _, lse = ctx.rcd_linear_cross_entropy(x, w, y, bias=b2)
    assert bool((lse == math.inf).all())
    # large logits: 2^13 apart and around 2^20, the differences are what counts
    b3 = torch.full_like(b, 2.0 ** 20)
    check_loss(ctx, x, w, b3, y)
    ctx.sync_status()


def test_labels_out_of_range_are_reported(rcd, ctx):
    import torch
    g = seeded("labels")
    x, w, b, y = head(g, 300, 500, 64, torch.bfloat16)
    loss0, lse0 = ctx.rcd_linear_cross_entropy(x, w, y, bias=b)
    ctx.sync_status()
    bad = y.clone()
    bad[17], bad[299] = 500, 2 ** 31 - 1
    loss, lse = ctx.rcd_linear_cross_entropy(x, w, bad, bias=b)
    with pytest.raises(rcd.RcdError) as e:
        ctx.sync_status()
    assert e.value.status == 1 and "label" in str(e.value)
    ctx.sync_status()
    assert torch.isnan(loss[[17, 299]]).all() and torch.equal(lse, lse0)
    keep = torch.ones(300, dtype=torch.bool, device="cuda")
    keep[[17, 299]] = False
    assert torch.equal(loss[keep], loss0[keep])
    got = ctx.rcd_linear_cross_entropy_backward(x, w, bad, lse, bias=b, piece=128)
    with pytest.raises(rcd.RcdError):
        ctx.sync_status()
    skipped = y.clone()
    skipped[[17, 299]] = -5
    want = ctx.rcd_linear_cross_entropy_backward(x, w, skipped, lse, bias=b, piece=128)
    ctx.sync_status()
    assert all(torch.equal(p, q) for p, q in zip(got, want))


@pytest.mark.parametrize("dtype,m,n,k", [("bf16", 40, 90, 64), ("fp16", 300, 1000, 128)])
def test_gradients_against_differences(rcd, ctx, dtype, m, n, k):
    """(f(x + e v) - f(x - e v)) / 2e of the summed loss, with x +- e v held exactly: off by e^2 / 6 times the third derivative along v, at most the third
    power of the logits' range along v, and by the loss's own error over e."""
    import torch
    t, g = kind(dtype), seeded("differences", dtype)
    x, w, b, y = head(g, m, n, k, t)
    e = 2.0 ** -5
    v = torch.randint(-1, 2, (m, k), generator=g, device="cuda").double()
    plus, minus = (x.double() + e * v).to(t), (x.double() - e * v).to(t)
    assert torch.equal(plus.double() - minus.double(), 2 * e * v)
    _, lse = ctx.rcd_linear_cross_entropy(x, w, y, bias=b)
    dx, _, _ = ctx.rcd_linear_cross_entropy_backward(x, w, y, lse, bias=b)
    up, lse_up = ctx.rcd_linear_cross_entropy(plus, w, y, bias=b)
    down, _ = ctx.rcd_linear_cross_entropy(minus, w, y, bias=b)
    along = (dx.double() * v).sum(1)
    u = v @ w.double().t()
    span = u.max(1).values - u.min(1).values
    z = logits64(plus, w, b)
    bound = e * e / 6 * span ** 3 + 2 * (loss_bound(z, lse_up.double(), n) + lse_up.double().abs() * 4 * U) / (2 * e)
    # (dx: half a step of the output and of dz each, whose sizes along a row of w are p and the label)
    wide = w.double().abs().max()
    bound = bound + half_step(t) * (2 * wide + dx.double().abs().max(1).values) * k * 2
    slope = (up.double() - down.double()) / (2 * e)
    assert float(((slope - along).abs() - bound).max()) <= 0
    assert float((slope - along).abs().mean()) < 0.05 * float(slope.abs().mean())
    ctx.sync_status()


def test_leading_dimensions_strides_and_empty_batches(rcd, ctx):
    import torch
    g = seeded("shapes")
    x, w, b, y = head(g, 60, 100, 64, torch.bfloat16)
    loss, lse = ctx.rcd_linear_cross_entropy(x, w, y, bias=b)
    l3, s3 = ctx.rcd_linear_cross_entropy(x.view(5, 12, 64), w, y.view(5, 12), bias=b)
    assert l3.shape == (5, 12) and torch.equal(l3.flatten(), loss) and torch.equal(s3.flatten(), lse)
    dx, dw, db = ctx.rcd_linear_cross_entropy_backward(x, w, y, lse, bias=b)
    dx3, dw3, db3 = ctx.rcd_linear_cross_entropy_backward(x.view(5, 12, 64), w, y.view(5, 12), s3, bias=b)
    assert torch.equal(dx3.view(60, 64), dx) and torch.equal(dw3, dw) and torch.equal(db3, db)
    # one row, columns first, every second label
    one, _ = ctx.rcd_linear_cross_entropy(x[3], w, y[3], bias=b)
    assert one.shape == () and math.isclose(float(one), float(loss[3]), rel_tol=1e-4, abs_tol=1e-4)
    lt, _ = ctx.rcd_linear_cross_entropy(x.t().contiguous().t(), w.t().contiguous().t(), torch.stack([y, y], 1)[:, 0], bias=b)
    assert torch.equal(lt, loss)
    # no rows
    empty, s0 = ctx.rcd_linear_cross_entropy(x[:0], w, y[:0], bias=b)
    assert empty.shape == (0,) and s0.shape == (0,)
    dx, dw, db = ctx.rcd_linear_cross_entropy_backward(x[:0], w, y[:0], s0, bias=b)
    assert dx.shape == (0, 64) and not dw.any() and not db.any()
    ctx.sync_status()


def test_same_bits_every_time_captured_and_on_other_streams(rcd, ctx):
    """Two graphs of both calls, replayed in turn with new inputs in place, and the same on a stream of its own."""
    import torch
    g = seeded("graph")
    x, w, b, y = head(g, 200, 700, 128, torch.float16)
    dloss = torch.rand(200, generator=g, device="cuda")

    def step(p=0):
        loss, lse = ctx.rcd_linear_cross_entropy(x, w, y, bias=b)
        return (loss, lse, *ctx.rcd_linear_cross_entropy_backward(x, w, y, lse, bias=b, dloss=dloss, piece=p))
    want, want_pieces = step(), step(128)
    graphs = []
    for p in (0, 128):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            out = step(p)
        graphs.append((graph, out))
    for _ in range(2):
        for graph, out in graphs:
            graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(p, q) for p, q in zip(graphs[0][1], want)) and all(torch.equal(p, q) for p, q in zip(graphs[1][1], want_pieces))
    x2 = grid(g, 200, 128, torch.float16)
    x.copy_(x2)
    for graph, _ in graphs:
        graph.replay()
    torch.cuda.synchronize()
    again = step()
    assert all(torch.equal(p, q) for p, q in zip(graphs[0][1], again))
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        other = step()
    s.synchronize()
    assert all(torch.equal(p, q) for p, q in zip(other, again))
    ctx.sync_status()


def test_nothing_is_written_beside_the_outputs(rcd, ctx):
    """Through the C structs: dx and dw inside wider rows, marks around them and behind loss and lse."""
    import ctypes as C
    import torch
    g = seeded("marks")
    for m, n, k in ((70, 130, 65), (33, 300, 127), (1, 64, 8)):
        for dtype in (torch.bfloat16, torch.float16):
            x, w, b, y = head(g, m, n, k, dtype)
            f = rcd.RcdCrossEntropyArgs(rows=m, n=n, k=k, type=rcd._elem(dtype, "x"), x=x.data_ptr(), ldx=x.stride(0), w=w.data_ptr(), ldw=w.stride(0), bias=b.data_ptr(),
                                        labels=y.data_ptr())
            out = torch.full((2, m + 16), 7.0, device="cuda")
            f.loss, f.lse = out[0, 8:].data_ptr(), out[1, 8:].data_ptr()
            need = C.c_size_t()
            assert rcd.lib.rcd_linear_cross_entropy_workspace_bytes(ctx._h, C.byref(f), C.byref(need)) == 0
            ws = torch.full((need.value + 512,), 0x5a, dtype=torch.uint8, device="cuda")
            assert rcd.lib.rcd_linear_cross_entropy(ctx._h, C.byref(f), ws.data_ptr(), need.value, ctx._stream()) == 0
            ctx.sync_status()
            assert bool((ws[need.value:] == 0x5a).all()) and bool((out[:, :8] == 7).all()) and bool((out[:, m + 8:] == 7).all())
            loss, lse = ctx.rcd_linear_cross_entropy(x, w, y, bias=b)
            assert torch.equal(out[0, 8:m + 8], loss) and torch.equal(out[1, 8:m + 8], lse)
            for piece in (0, 64):
                dx = torch.full((m + 2, k + 9), 7.0, device="cuda", dtype=dtype)
                dw = torch.full((n + 2, k + 9), 7.0, device="cuda", dtype=dtype)
                db = torch.full((n + 16,), 7.0, device="cuda")
                a = rcd.RcdCrossEntropyBackArgs(rows=m, n=n, k=k, type=f.type, x=f.x, ldx=f.ldx, w=f.w, ldw=f.ldw, bias=f.bias, labels=f.labels, lse=lse.data_ptr(), piece=piece,
                                                dx=dx[1, 3:].data_ptr(), ld_dx=k + 9, dw_type=f.type, dw=dw[1, 5:].data_ptr(), ld_dw=k + 9, dbias=db[8:].data_ptr())
                assert rcd.lib.rcd_linear_cross_entropy_backward_workspace_bytes(ctx._h, C.byref(a), C.byref(need)) == 0
                ws = torch.full((need.value + 512,), 0x5a, dtype=torch.uint8, device="cuda")
                assert rcd.lib.rcd_linear_cross_entropy_backward(ctx._h, C.byref(a), ws.data_ptr(), need.value, ctx._stream()) == 0
                ctx.sync_status()
                assert bool((ws[need.value:] == 0x5a).all())
                want = ctx.rcd_linear_cross_entropy_backward(x, w, y, lse, bias=b, piece=piece)
                assert torch.equal(dx[1:-1, 3:k + 3], want[0]) and torch.equal(dw[1:-1, 5:k + 5], want[1]) and torch.equal(db[8:n + 8], want[2])
                dx[1:-1, 3:k + 3] = 7
                dw[1:-1, 5:k + 5] = 7
                db[8:n + 8] = 7
                assert bool((dx == 7).all()) and bool((dw == 7).all()) and bool((db == 7).all())


def test_refusals(rcd, ctx):
    import ctypes as C
    import torch
    g = seeded("refusals")
    x, w, b, y = head(g, 20, 600, 64, torch.bfloat16)             # (more classes than one tile takes: the call has a workspace)
    _, lse = ctx.rcd_linear_cross_entropy(x, w, y, bias=b)
    for call in (lambda **kw: ctx.rcd_linear_cross_entropy(**{**dict(x=x, w=w, labels=y, bias=b), **kw}),
                 lambda **kw: ctx.rcd_linear_cross_entropy_backward(**{**dict(x=x, w=w, labels=y, lse=lse, bias=b), **kw})):
        with pytest.raises(TypeError):
            call(labels=y.long())
        with pytest.raises(ValueError):
            call(labels=y[:5])
        with pytest.raises(TypeError):
            call(w=w.half())
        with pytest.raises(ValueError):
            call(w=w[:, :32])
        with pytest.raises(ValueError):
            call(x=x.cpu())
        with pytest.raises(TypeError):
            call(bias=b.double())
        with pytest.raises(ValueError):
            call(bias=b[:4])
        with pytest.raises(rcd.RcdError):
            call(x=x.float(), w=w.float())
        with pytest.raises(rcd.RcdError):
            call(w=w[:0], bias=None)
    with pytest.raises(TypeError):
        ctx.rcd_linear_cross_entropy_backward(x, w, y, lse.double(), bias=b)
    with pytest.raises(ValueError):
        ctx.rcd_linear_cross_entropy_backward(x, w, y, lse, bias=b, dloss=torch.ones(3, device="cuda"))
    with pytest.raises(rcd.RcdError):
        ctx.rcd_linear_cross_entropy_backward(x, w, y, lse, bias=b, piece=-1)
    with pytest.raises(rcd.RcdError):
        ctx.rcd_linear_cross_entropy_backward(x, w, y, lse, bias=b, dw_dtype=torch.float16)
    loss = torch.empty(20, device="cuda")
    ok = dict(rows=20, n=600, k=64, type=1, x=x.data_ptr(), ldx=64, w=w.data_ptr(), ldw=64, bias=b.data_ptr(), labels=y.data_ptr(), loss=loss.data_ptr(), lse=lse.data_ptr())
    need = C.c_size_t()

    def refused(status, ws=None, size=0, **change):
        a = rcd.RcdCrossEntropyArgs(**{**ok, **change})
        got = rcd.lib.rcd_linear_cross_entropy_workspace_bytes(ctx._h, C.byref(a), C.byref(need)) if ws is None else rcd.lib.rcd_linear_cross_entropy(ctx._h, C.byref(a), ws, size, None)
        assert got == status, got
    refused(0)
    big = torch.empty(need.value + 256, dtype=torch.uint8, device="cuda")
    for change in (dict(x=None), dict(w=None), dict(labels=None), dict(loss=None), dict(ldx=63), dict(ldw=1), dict(rows=-1), dict(k=0), dict(n=0), dict(type=3), dict(type=0),
                   dict(x=x.data_ptr() + 1), dict(labels=y.data_ptr() + 2), dict(bias=b.data_ptr() + 1), dict(lse=lse.data_ptr() + 3)):
        refused(1, **change)
    refused(2, rows=1 << 30, n=1 << 30, ldx=64)
    refused(3, ws=big.data_ptr(), size=need.value - 1)
    refused(1, ws=big.data_ptr() + 8, size=need.value)
    refused(1, ws=big.data_ptr(), size=need.value, loss=lse.data_ptr())
    refused(1, ws=big.data_ptr(), size=need.value, loss=x.data_ptr())
    ctx.sync_status()
