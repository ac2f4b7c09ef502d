"""Matrix product with bias, activation and residual (bf16, fp16, int8 with scales) and its gradients, against 64 bits.

Most inputs are small integers: their products' sums are exact in fp32 whatever the order, so that a product without an activation has
to be right bit for bit, its one rounding included."""
import pytest

from test_gpu_norm import ctx, half_step, kind, rcd, rows, seeded  # noqa: F401  (fixtures)

pytestmark = pytest.mark.gpu

ACTS = ["none", "relu", "gelu", "gelu_tanh", "silu"]
U = 2.0 ** -24


def code(rcd, act):
    return {"none": rcd.RCD_ACT_NONE, "relu": rcd.RCD_ACT_RELU, "gelu": rcd.RCD_ACT_GELU, "gelu_tanh": rcd.RCD_ACT_GELU_TANH,
            "silu": rcd.RCD_ACT_SILU}[act]


def act64(z, act):
    """Activation and slope in 64 bits."""
    import math
    import torch
    one = torch.ones_like(z)
    if act == "none":
        return z, one
    if act == "relu":
        return z.clamp(min=0), (z > 0).double()
    if act == "gelu":
        p = 0.5 * (1 + torch.erf(z / math.sqrt(2)))
        return z * p, p + z * torch.exp(-z * z / 2) / math.sqrt(2 * math.pi)
    if act == "silu":
        p = torch.sigmoid(z)
        return z * p, p + z * p * (1 - p)
    c = math.sqrt(2 / math.pi)
    t = torch.tanh(c * (z + 0.044715 * z ** 3))
    return 0.5 * z * (1 + t), 0.5 * (1 + t) + 0.5 * z * (1 - t * t) * c * (1 + 3 * 0.044715 * z * z)


def whole(g, n, d, dtype, pad=0, shift=0, most=4):
    """Integers from -most to most, laid out like rows()."""
    import torch
    x = torch.randint(-most, most + 1, (n * (d + pad) + shift,), generator=g, device="cuda", dtype=torch.int32).to(dtype)
    return x[shift:].view(n, d + pad)[:, :d]


def near(got, want, dtype, slack):
    """Half a step of the type, and `slack` for what comes before the rounding."""
    import torch
    got, want = got.double(), want.double()
    bound = (want.abs() + slack) * half_step(dtype) + slack + torch.finfo(dtype).tiny * half_step(dtype) * 2
    worst = (got - want).abs() - bound
    assert worst.numel() == 0 or float(worst.max()) <= 0, float(worst.max())


def rounded(z, dtype):
    """An exact result rounded once (through fp32, which holds the integers and quarters of these tests exactly)."""
    return z.float().to(dtype)


# rows 1 to past several tiles, widths and depths around 8, 16, 32, 64, 128 and 256, odd ones among them
SIZES = [(1, 1, 1), (1, 2048, 2048), (1, 16, 8), (1, 333, 77), (2, 64, 64), (3, 130, 72), (5, 1000, 520), (8, 512, 1024), (9, 256, 64), (16, 48, 4096), (17, 512, 200),
         (31, 129, 65), (32, 1024, 512), (64, 320, 640), (65, 256, 128), (100, 8, 16), (127, 127, 127), (128, 128, 64), (129, 257, 65), (200, 64, 64),
         (256, 512, 256), (300, 1, 33), (333, 777, 1001), (500, 520, 2048), (1300, 333, 777), (700, 2048, 512), (2100, 1300, 192), (5000, 64, 512),
         (20000, 512, 256), (12000, 1288, 72), (32, 8200, 2048), (16, 8256, 4096)]


@pytest.mark.parametrize("m,n,k", SIZES)
@pytest.mark.parametrize("dtype", ["bf16", "fp16", "int8"])
@pytest.mark.parametrize("pad,shift", [(0, 0), (16, 0), (3, 1)])
def test_exact_products(rcd, ctx, m, n, k, dtype, pad, shift):
    import torch
    t, g = kind(dtype), seeded(m, n, k, dtype, pad)
    most = 4 if dtype != "int8" else 127
    x, w = whole(g, m, k, t, pad, shift, most), whole(g, n, k, t, pad, 0, most)
    z = x.double() @ w.double().t()
    outs = [torch.float32, torch.bfloat16 if dtype != "fp16" else torch.float16]
    for out in outs:
        y, pre = ctx.rcd_linear(x, w, out_dtype=out)
        assert pre is None and y.shape == (m, n) and torch.equal(y, rounded(z, out))
        if dtype == "int8":
            # scales that are powers of two: still exact
            sx = 2.0 ** torch.randint(-6, 3, (m,), generator=g, device="cuda").float()
            sw = 2.0 ** torch.randint(-6, 3, (n,), generator=g, device="cuda").float()
            y, _ = ctx.rcd_linear(x, w, x_scales=sx, w_scales=sw, out_dtype=out)
            assert torch.equal(y, rounded(z * sx.double()[:, None] * sw.double(), out))
            y, _ = ctx.rcd_linear(x, w, w_scales=sw, out_dtype=out)
            assert torch.equal(y, rounded(z * sw.double(), out))
        else:
            b = torch.randint(-64, 65, (n,), generator=g, device="cuda").float() / 4
            r = whole(g, m, n, out, pad, shift)
            y, pre = ctx.rcd_linear(x, w, bias=b, residual=r, activation=rcd.RCD_ACT_RELU, out_dtype=out, want_preact=True)
            zb = z + b.double()
            assert torch.equal(pre, rounded(zb, out)) and torch.equal(y, rounded(zb.clamp(min=0) + r.double(), out))
            y, pre = ctx.rcd_linear(x, w, bias=b, residual=r, activation=rcd.RCD_ACT_RELU, out_dtype=out)
            assert pre is None and torch.equal(y, rounded(zb.clamp(min=0) + r.double(), out))
            y, pre = ctx.rcd_linear(x, w, bias=b, out_dtype=out, want_preact=True)
            assert torch.equal(pre, rounded(zb, out)) and torch.equal(y, pre)
    ctx.sync_status()


@pytest.mark.parametrize("m,n,k", [(1, 512, 2048), (4, 777, 300), (40, 260, 512), (300, 333, 1001), (600, 512, 2048), (1000, 256, 96)])
@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("dtype,out", [("bf16", "bf16"), ("fp16", "fp32"), ("int8", "bf16"), ("int8", "fp32")])
def test_epilogue(rcd, ctx, m, n, k, act, dtype, out):
    """Real values.  A sum of k products is off by k units at most of the sum of their sizes (an addition that cuts off instead of
    rounding loses a whole one); the epilogue's handful of fp32 steps by a unit each of what they work on, and the exponential
    by 2 + 1.16 |z| more; slopes stay below 1.13."""
    import torch
    t, o, g = kind(dtype), kind(out), seeded(m, n, k, act, dtype)
    if dtype == "int8":
        x, w = whole(g, m, k, t, most=127), whole(g, n, k, t, most=127)
        sx, sw = torch.rand(m, generator=g, device="cuda") / 60, torch.rand(n, generator=g, device="cuda") / (60 * k ** 0.5)
        z = (x.double() @ w.double().t()) * sx.double()[:, None] * sw.double()
        size = z.abs() * 4
    else:
        x, w, sx, sw = rows(g, m, k, t), rows(g, n, k, t, size=k ** -0.5), None, None
        z = x.double() @ w.double().t()
        size = (x.double().abs() @ w.double().abs().t()) * k * 2
    b = torch.randn(n, generator=g, device="cuda")
    r = rows(g, m, n, o)
    zb = z + b.double()
    slack = U * (2 * size + 4 * zb.abs() + 4 * b.double().abs())
    y, pre = ctx.rcd_linear(x, w, bias=b, residual=r, activation=code(rcd, act), x_scales=sx, w_scales=sw, out_dtype=o, want_preact=True)
    ctx.sync_status()
    near(pre, zb, o, slack)
    want = act64(zb, act)[0] + r.double()
    near(y, want, o, 1.13 * slack + U * ((16 + 4 * zb.abs()) * zb.abs() + 2 * r.double().abs()))


@pytest.mark.parametrize("act", ACTS)
def test_activations_over_their_range(rcd, ctx, act):
    """Values from far below to far above zero, infinities and NaN, through a product with the identity."""
    import torch
    z = torch.cat([torch.linspace(-120, 120, 4001), torch.tensor([0.0, -0.0, 1e-30, -1e-30, 3e4, -3e4, float("inf"), float("-inf"), float("nan")])]).to(torch.bfloat16)
    x = z.cuda().reshape(-1, 1).contiguous()
    y, _ = ctx.rcd_linear(x, torch.ones(1, 1, device="cuda", dtype=torch.bfloat16), activation=code(rcd, act), out_dtype=torch.float32)
    zz = z.double().cuda()
    fine = torch.isfinite(zz)
    near(y[:, 0][fine], act64(zz[fine], act)[0], torch.float32, U * (16 + 4 * zz[fine].abs()) * zz[fine].abs())
    assert torch.isnan(y[-1, 0]) and float(y[-3, 0]) == float("inf")
    low = float(y[-2, 0])                                  # at minus infinity: 0, or the formula's -inf * 0
    assert low == (float("-inf") if act == "none" else 0.0) or (act not in ("none", "relu") and low != low)


@pytest.mark.parametrize("m,n,k", [(1, 512, 256), (4, 64, 64), (100, 320, 72), (1300, 333, 777)])
@pytest.mark.parametrize("dtype", ["bf16", "fp16", "int8"])
def test_nan_and_infinity_stay_in_their_rows(ctx, m, n, k, dtype):
    """A NaN in x reaches its row alone, one in w its column alone; the zeros that fill a tile's edge reach nothing."""
    import torch
    t, g = kind(dtype), seeded(m, n, k, "nan")
    x, w = whole(g, m, k, t), whole(g, n, k, t)
    b = torch.zeros(n, device="cuda")
    if dtype == "int8":
        b[n // 2] = float("nan")
        y, _ = ctx.rcd_linear(x, w, bias=b, out_dtype=torch.float32)
        bad = torch.zeros(m, n, dtype=torch.bool, device="cuda")
        bad[:, n // 2] = True
    else:
        x[m // 2, k - 1] = float("nan")
        w[n - 1, k // 2] = float("nan")
        y, _ = ctx.rcd_linear(x, w, out_dtype=torch.float32)
        bad = torch.zeros(m, n, dtype=torch.bool, device="cuda")
        bad[m // 2], bad[:, n - 1] = True, True
    assert torch.equal(torch.isnan(y), bad)


def test_out_and_what_lies_behind(ctx):
    import torch
    for m, n, k, pad in [(3, 64, 64, 8), (130, 257, 72, 3), (300, 512, 128, 64), (700, 256, 512, 0)]:
        g = seeded(m, n, k)
        x, w = whole(g, m, k, torch.bfloat16), whole(g, n, k, torch.bfloat16)
        want, _ = ctx.rcd_linear(x, w)
        buf = torch.full((m + 2, n + pad), 7.0, device="cuda", dtype=torch.bfloat16)
        y, _ = ctx.rcd_linear(x, w, out=buf[1:m + 1, :n])
        assert torch.equal(buf[1:m + 1, :n], want)
        buf[1:m + 1, :n] = 7
        assert bool((buf == 7).all())
    x3 = whole(seeded(1), 6, 64, torch.bfloat16)
    y, _ = ctx.rcd_linear(x3.reshape(2, 3, 64), x3)
    assert y.shape == (2, 3, 6) and torch.equal(y.reshape(6, 6), ctx.rcd_linear(x3, x3)[0])
    ctx.sync_status()


@pytest.mark.parametrize("m,n,k", SIZES)
@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("pad,shift", [(0, 0), (3, 1)])
def test_exact_gradients(ctx, m, n, k, dtype, pad, shift):
    import torch
    t, g = kind(dtype), seeded(m, n, k, dtype, "back")
    dy, x, w = whole(g, m, n, t, pad, shift), whole(g, m, k, t, pad), whole(g, n, k, t, 0, shift)
    for dwt in (t, torch.float32):
        dx, dw, db = ctx.rcd_linear_backward(dy, x, w, dw_dtype=dwt)
        ctx.sync_status()
        assert torch.equal(dx, rounded(dy.double() @ w.double(), t))
        assert torch.equal(dw, rounded(dy.double().t() @ x.double(), dwt))
        assert torch.equal(db, dy.double().sum(0).float())
    for want in (dict(want_dx=False), dict(want_dw=False), dict(want_dbias=False), dict(want_dx=False, want_dw=False)):
        got = ctx.rcd_linear_backward(dy, x, w, **want)
        for have, full, name in zip(got, ctx.rcd_linear_backward(dy, x, w), ("want_dx", "want_dw", "want_dbias")):
            assert have is None if name in want else torch.equal(have, full)


@pytest.mark.parametrize("m,n,k", [(1, 64, 128), (7, 333, 77), (300, 512, 256), (1300, 130, 520)])
@pytest.mark.parametrize("act", ACTS[1:])
@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
def test_gradients_through_activations(rcd, ctx, m, n, k, act, dtype):
    """dz is rounded to the type: half a step of every term; the rest as in test_epilogue."""
    import torch
    t, g = kind(dtype), seeded(m, n, k, act, "slope")
    dy, x, w, z = rows(g, m, n, t), rows(g, m, k, t), rows(g, n, k, t, size=n ** -0.5), rows(g, m, n, t, size=2.0)
    dx, dw, db = ctx.rcd_linear_backward(dy, x, w, preact=z, activation=code(rcd, act))
    ctx.sync_status()
    dz = dy.double() * act64(z.double(), act)[1]
    off = (half_step(t) + 2 * U) * dz.abs() + U * (16 + 4 * z.double().abs()) * dy.double().abs() + torch.finfo(t).tiny * half_step(t) * 2
    near(dx, dz @ w.double(), t, off @ w.double().abs() + 2 * U * n * (dz.abs() @ w.double().abs()))
    near(dw, dz.t() @ x.double(), t, off.t() @ x.double().abs() + 2 * U * m * (dz.abs().t() @ x.double().abs()))
    near(db, dz.sum(0), torch.float32, (off - half_step(t) * dz.abs()).sum(0) + U * m * dz.abs().sum(0))


def test_gradients_against_differences(rcd, ctx):
    """Central differences of the kernel's own forward pass in fp16 inputs and fp32 output.  The step, 2^-5, is exact in the inputs; the
    loss is sum(c y) in 64 bits; a third derivative of about 1 leaves 2^-10 / 6 of it, roundings of y 2^-24 * |y| / 2^-5, and dz's and the
    kept z's rounding to fp16 2^-11 each of the terms."""
    import torch
    g = seeded("differences")
    m, n, k = 3, 40, 24
    x, w = (torch.randint(-32, 33, (m, k), generator=g, device="cuda") / 32).half(), (torch.randint(-16, 17, (n, k), generator=g, device="cuda") / 64).half()
    b, c = torch.randn(n, generator=g, device="cuda"), torch.randn(m, n, generator=g, device="cuda").half()
    for act in ("gelu", "silu", "gelu_tanh"):
        loss = lambda xx, ww, bb: float((ctx.rcd_linear(xx, ww, bias=bb, activation=code(rcd, act), out_dtype=torch.float32)[0].double() * c.double()).sum())  # noqa: E731
        _, z = ctx.rcd_linear(x, w, bias=b, activation=code(rcd, act), want_preact=True)
        grads = ctx.rcd_linear_backward(c, x, w, preact=z, activation=code(rcd, act))
        args = [x, w, b]
        for which in range(3):
            flat = args[which].reshape(-1)
            for i in range(0, flat.numel(), 7):
                at = []
                for sign in (-1, 1):
                    moved = flat.clone()
                    moved[i] += sign * 2.0 ** -5
                    full = list(args)
                    full[which] = moved.view(args[which].shape)
                    at.append(loss(*full))
                num, got = (at[1] - at[0]) * 16, float(grads[which].reshape(-1)[i])
                assert abs(num - got) <= 1e-2 * (1 + abs(num)), (act, which, i, num, got)


def test_no_rows(ctx):
    import torch
    x, w = torch.empty(0, 64, device="cuda", dtype=torch.bfloat16), torch.ones(32, 64, device="cuda", dtype=torch.bfloat16)
    y, z = ctx.rcd_linear(x, w, want_preact=True)
    assert y.shape == (0, 32) and z.shape == (0, 32)
    dx, dw, db = ctx.rcd_linear_backward(y, x, w)
    assert dx.shape == (0, 64) and not dw.any() and not db.any() and dw.shape == (32, 64)
    y, _ = ctx.rcd_linear(w, torch.empty(0, 64, device="cuda", dtype=torch.bfloat16))
    assert y.shape == (32, 0)
    dx, dw, db = ctx.rcd_linear_backward(y, w, torch.empty(0, 64, device="cuda", dtype=torch.bfloat16))
    assert not dx.any() and dx.shape == (32, 64) and dw.shape == (0, 64) and db.shape == (0,)
    ctx.sync_status()


def test_same_bits_every_time_streams_and_graphs(rcd, ctx):
    import torch
    g = seeded("graphs")
    for m, n, k, dtype in [(1, 512, 1024, torch.bfloat16), (33, 300, 700, torch.float16), (900, 512, 2048, torch.bfloat16)]:
        x, w, b = rows(g, m, k, dtype), rows(g, n, k, dtype, size=k ** -0.5), torch.randn(n, generator=g, device="cuda")
        dy = rows(g, m, n, dtype)

        def run():
            y, z = ctx.rcd_linear(x, w, bias=b, activation=rcd.RCD_ACT_GELU, want_preact=True)
            return (y, z, *ctx.rcd_linear_backward(dy, x, w, preact=z, activation=rcd.RCD_ACT_GELU))

        first = run()
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            other = run()
        side.synchronize()
        assert all(torch.equal(p, q) for p, q in zip(first, other))
        graphs = []
        for _ in range(2):                                # two graphs, each with its own workspace
            gr = torch.cuda.CUDAGraph()
            with torch.cuda.graph(gr):
                outs = run()
            graphs.append((gr, outs))
        for _ in range(2):
            x.copy_(rows(g, m, k, dtype))
            torch.cuda.synchronize()
            streams = [torch.cuda.Stream(), torch.cuda.Stream()]
            for (gr, _), s in zip(graphs, streams):      # at the same time
                with torch.cuda.stream(s):
                    gr.replay()
            torch.cuda.synchronize()
            want = run()
            for _, outs in graphs:
                assert all(torch.equal(p, q) for p, q in zip(want, outs))
    ctx.sync_status()


def test_refusals(rcd, ctx):
    import ctypes as C
    import torch
    x, w = torch.ones(4, 64, device="cuda", dtype=torch.bfloat16), torch.ones(32, 64, device="cuda", dtype=torch.bfloat16)
    one = torch.ones(32, device="cuda")
    for args, kw in (((x, w.half()), {}), ((x, w[:, :32]), {}), ((x, w), dict(bias=one.half())), ((x, w), dict(bias=one[:31])),
                     ((x, w), dict(x_scales=torch.ones(4, device="cuda"))), ((x, w), dict(w_scales=one)), ((x, w), dict(activation=9)),
                     ((x, w), dict(activation=-1)), ((x, w), dict(out_dtype=torch.int8)), ((x, w), dict(out_dtype=torch.float64)),
                     ((x.float(), w.float()), {}), ((x, w), dict(residual=torch.ones(4, 32, device="cuda"))), ((x.cpu(), w), {}),
                     ((x, w), dict(residual=torch.ones(3, 32, device="cuda", dtype=torch.bfloat16))), ((x, w), dict(out=x)), ((x, w.reshape(-1)), {}),
                     ((x[:, :0], w[:, :0]), {}), ((torch.ones(2, 131072, device="cuda", dtype=torch.int8), torch.ones(2, 131072, device="cuda", dtype=torch.int8)), {})):
        with pytest.raises((rcd.RcdError, ValueError, TypeError)):
            ctx.rcd_linear(*args, **kw)
    sq = torch.ones(64, 64, device="cuda", dtype=torch.bfloat16)
    for over in (dict(out=sq), dict(residual=sq, out=sq)):                       # y over an argument
        with pytest.raises(rcd.RcdError):
            ctx.rcd_linear(sq, w.repeat(2, 1), **over)
    dy = torch.ones(4, 32, device="cuda", dtype=torch.bfloat16)
    for args, kw in (((dy, x, w), dict(activation=rcd.RCD_ACT_RELU)), ((dy, x, w), dict(preact=dy)), ((dy, x, w), dict(dw_dtype=torch.float16)),
                     ((dy[:3], x, w), {}), ((dy.half(), x, w), {}), ((dy.to(torch.int8), x.to(torch.int8), w.to(torch.int8)), {}),
                     ((dy.float(), x.float(), w.float()), {}), ((dy, x, w), dict(preact=dy[:, :16], activation=rcd.RCD_ACT_RELU))):
        with pytest.raises((rcd.RcdError, ValueError, TypeError)):
            ctx.rcd_linear_backward(*args, **kw)
    a = rcd.RcdLinearArgs()
    a.rows, a.n, a.k, a.type, a.y_type, a.ldx, a.ldw, a.ldy = 4, 32, 64, rcd.RCD_ELEM_BF16, rcd.RCD_ELEM_BF16, 64, 64, 32
    a.w, a.y = w.data_ptr(), dy.data_ptr()
    need = C.c_size_t()
    run = lambda: rcd.lib.rcd_linear_workspace_bytes(ctx._h, C.byref(a), C.byref(need))  # noqa: E731
    assert run() == 1                                                            # x is null
    a.x = x.data_ptr()
    assert run() == 0
    a.ldy = 31
    assert run() == 1
    a.ldy, a.k = 32, 0
    assert run() == 1
    a.k, a.rows = 64, 1 << 31
    assert run() == 1
    assert rcd.lib.rcd_linear(None, C.byref(a), None, 0, None) == 1
    ctx.sync_status()


def test_slopes_of_large_values(rcd, ctx):
    """Far from zero the slopes are 0 and 1, whatever the squares on the way to them."""
    import torch
    z = torch.tensor([[-1e30, -1e20, -200.0, 200.0, 1e20, 1e30]], device="cuda", dtype=torch.bfloat16)
    one = torch.ones_like(z)
    for act in ACTS[1:]:
        _, _, db = ctx.rcd_linear_backward(one, torch.ones(1, 8, device="cuda", dtype=torch.bfloat16), torch.ones(6, 8, device="cuda", dtype=torch.bfloat16),
                                           preact=z, activation=code(rcd, act))
        assert db.tolist() == [0, 0, 0, 1, 1, 1], act
    ctx.sync_status()


def test_offsets_beyond_32_bits(ctx):
    """An output of 2.3 billion elements: its last rows, and x's last rows behind a stride that alone passes 32 bits."""
    import torch
    g = seeded("far")
    m, n, k = 70000, 33000, 32
    x, w = whole(g, m, k, torch.bfloat16), whole(g, n, k, torch.bfloat16)
    y, _ = ctx.rcd_linear(x, w)
    at = torch.tensor([0, 1, m // 2, m - 130, m - 1], device="cuda")
    assert torch.equal(y[at], rounded(x[at].double() @ w.double().t(), torch.bfloat16))
    del y
    far = torch.zeros(5, 1 << 29, device="cuda", dtype=torch.bfloat16)[:, :k]
    far.copy_(x[:5])
    y, _ = ctx.rcd_linear(far, w)
    assert torch.equal(y, rounded(x[:5].double() @ w.double().t(), torch.bfloat16))
    far2, _ = ctx.rcd_linear(x[:400], w[:64], out=torch.empty(400, 1 << 23, device="cuda", dtype=torch.bfloat16)[:, :64])
    assert torch.equal(far2, rounded(x[:400].double() @ w[:64].double().t(), torch.bfloat16))
    ctx.sync_status()
