"""Root-mean-square norm of rows (16-, 32- and 8-bit output) and its gradients, against the formulas in 64 bits."""
import zlib

import numpy as np
import pytest

pytestmark = pytest.mark.gpu

TYPES = ["bf16", "fp16", "fp32"]
# the kernels' fp32 steps from h to y: one rounding each of h, t and y, a sum of squares of up to 32 terms per thread and
# 10 more levels, a division, a root and a reciprocal; squares halve in the root.  Fewer than 64 of half a unit.
STEPS = 64 * 2.0 ** -24


@pytest.fixture(scope="module")
def rcd():
    import torch
    if not torch.cuda.is_available():
        pytest.skip("needs a CUDA device")
    from paper_2211_00839_b200 import binding
    return binding


@pytest.fixture(scope="module")
def ctx(rcd):
    with rcd.Context(0) as c:
        yield c


def kind(name):
    import torch
    return {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32, "int8": torch.int8}[name]


def rows(g, n, d, dtype, pad=0, shift=0, size=1.0):
    """[n, d] whose rows lie d + pad elements apart and start `shift` elements into their memory."""
    import torch
    x = (torch.randn(n * (d + pad) + shift, generator=g, device="cuda") * size).to(dtype)
    return x[shift:].view(n, d + pad)[:, :d]


def seeded(*key):
    import torch
    g = torch.Generator(device="cuda")
    g.manual_seed(zlib.crc32(repr(key).encode()))
    return g


def half_step(dtype):
    import torch
    return torch.finfo(dtype).eps / 2


def check(got, want, dtype, steps=STEPS, slack=None):
    """|got - want| within half a step of the type, the fp32 steps before it, and `slack`."""
    import torch
    got, want = got.double(), want.double()
    assert torch.equal(torch.isnan(got), torch.isnan(want))
    tiny = torch.finfo(dtype).tiny * half_step(dtype) * 2
    bound = want.abs() * (half_step(dtype) * (1 + 4 * steps) + steps) + tiny
    if slack is not None:
        bound = bound + slack
    fine = torch.isfinite(want)
    assert torch.equal(got[~fine & ~torch.isnan(want)], want[~fine & ~torch.isnan(want)])
    worst = ((got - want).abs() - bound)[fine]
    assert worst.numel() == 0 or float(worst.max()) <= 0, float(worst.max())


def reference(x, r, w, eps):
    import torch
    h = x.double() if r is None else x.double() + r.double()
    v = h.square().mean(1, keepdim=True) + eps
    y = h / v.sqrt()
    return h, torch.where(v == 0, torch.zeros_like(y), y if w is None else y * w.double())


SIZES = [(1, 1), (2, 7), (5, 32), (3, 100), (1, 2048), (33, 512), (1300, 64), (7, 1001), (9, 4096), (2, 4100), (3, 9000), (2, 16384), (3, 16383), (1500, 640)]
# enough rows for the ring in shared memory: one to sixteen warps per row, rows that leave lanes without elements, a last turn not all groups have
MANY = [(7200, 64), (7105, 72), (8001, 512), (7111, 1000), (3700, 2048), (3600, 2056), (1900, 4096), (1000, 8192), (700, 16384), (650, 9000), (25000, 520), (190000, 72)]


@pytest.mark.parametrize("n,d", SIZES + MANY)
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("pad,shift,residual,weight", [(0, 0, True, "same"), (8, 0, False, "fp32"), (3, 1, True, None), (0, 1, False, "same")])
def test_norm(ctx, n, d, dtype, pad, shift, residual, weight):
    import torch
    t, g = kind(dtype), seeded(n, d, dtype, pad)
    x, r = rows(g, n, d, t, pad, shift), rows(g, n, d, t, pad) if residual else None
    w = torch.randn(d, generator=g, device="cuda").to(t if weight == "same" else torch.float32) if weight else None
    h, want = reference(x, r, w, 1e-6)
    for out in {t, torch.bfloat16, torch.float32}:
        y, scales, total = ctx.rcd_rms_norm(x, residual=r, weight=w, eps=1e-6, out_dtype=out, want_sum=True)
        ctx.sync_status()
        assert scales is None and y.dtype == out and y.shape == x.shape
        # (h is rounded once where it has a residual; in y the cancellation of x + r costs nothing: the sum's rounding is relative)
        check(y, want, out)
        check(total, h, t, 2.0 ** -23)


def steps_of(x, r, w, eps, scale=None):
    """The 8-bit forms step by step, one fp32 operation each."""
    import torch
    h = x.float() if r is None else x.float() + r.float()
    t = h if w is None else h * w.float()
    if scale is not None:
        v = h.double().square().sum(1, keepdim=True) / h.shape[1] + float(np.float32(eps))
        rstd = (1 / v.sqrt()).float()
        inv = np.float32(1) / np.float32(scale)
        return torch.round((t * rstd) * float(inv)).clamp(-127, 127).to(torch.int8)
    a = t.abs().amax(1, keepdim=True)
    inv = torch.where(a > 0, torch.full_like(a, 127.0).div(a), torch.zeros_like(a)).clamp(max=torch.finfo(torch.float32).max)
    return torch.round(t * inv).to(torch.int8), a[:, 0]


@pytest.mark.parametrize("n,d", SIZES + MANY)
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("pad,residual,weight", [(0, True, True), (5, False, False), (8, False, True)])
def test_int8(ctx, n, d, dtype, pad, residual, weight):
    """The integers are the stepwise arithmetic's, bit for bit; the scales carry rstd's few roundings."""
    import torch
    t, g = kind(dtype), seeded(n, d, dtype, pad, 8)
    x, r = rows(g, n, d, t, pad), rows(g, n, d, t) if residual else None
    w = torch.randn(d, generator=g, device="cuda").to(t) if weight else None
    want, a = steps_of(x, r, w, 1e-6)
    q, scales, _ = ctx.rcd_rms_norm(x, residual=r, weight=w, eps=1e-6, out_dtype=torch.int8)
    assert torch.equal(q, want)
    h, _ = reference(x, r, w, 1e-6)
    check(scales, a.double() / 127 / (h.square().mean(1) + 1e-6).sqrt(), torch.float32)
    q, scales, _ = ctx.rcd_rms_norm(x, residual=r, weight=w, eps=1e-6, out_dtype=torch.int8, scale=0.03)
    assert scales is None and torch.equal(q, steps_of(x, r, w, 1e-6, 0.03))
    q, scales = ctx.rcd_quantize_rows(x)
    want, a = steps_of(x, None, None, 0.0)
    assert torch.equal(q, want)
    check(scales, a.double() / 127, torch.float32, 2.0 ** -23)
    ctx.sync_status()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("d,rows_behind", [(1, 0), (48, 0), (513, 0), (2048, 0), (48, 300000), (2048, 8000)])
def test_rows_of_zeros_and_special_values(ctx, dtype, d, rows_behind):
    import torch
    t = kind(dtype)
    x = torch.ones(8 + rows_behind, d, device="cuda", dtype=t)
    x[1] = 0
    x[2, d // 2] = float("nan")
    x[3, d - 1] = float("inf")
    x[4] = -torch.finfo(t).max if dtype == "fp16" else -(2.0 ** 55)
    x[5] = torch.finfo(t).smallest_normal if dtype != "fp16" else 2.0 ** -24
    x[6] = 0
    x[6, 0] = 2.0 ** -10
    # eps 0: a row of zeros stays one; squares of the smallest fp32 and bf16 numbers are 0 in fp32, and so is their rstd
    y, _, _ = ctx.rcd_rms_norm(x, eps=0.0)
    _, want = reference(x, None, None, 0.0)
    if dtype != "fp16":
        want[5] = 0
    want[3] = torch.where(torch.isinf(x[3]), float("nan"), 0.0)        # inf * 0, and rstd is 0 for the others
    check(y, want, t)
    # with eps they shrink instead
    y, _, _ = ctx.rcd_rms_norm(x[5:6], eps=1e-6)
    check(y, reference(x[5:6], None, None, 1e-6)[1], t)
    q, s, _ = ctx.rcd_rms_norm(x, eps=0.0, out_dtype=torch.int8)
    assert torch.isnan(s[2]) and torch.isnan(s[3])
    assert not q[1].any() and float(s[1]) == 0 and not q[2].any() and not q[3].any()
    assert bool((q[4] == -127).all()) and bool((q[0] == 127).all())
    q, s = ctx.rcd_quantize_rows(x)
    assert torch.isnan(s[2]) and torch.isnan(s[3]) and not q[1:4].any() and float(s[1]) == 0
    q, s, _ = ctx.rcd_rms_norm(x, eps=0.0, out_dtype=torch.int8, scale=1e-3)
    assert not q[1].any() and not q[2].any() and not q[3].any()       # NaN: 0
    assert bool((q[0] == 127).all()) and bool((q[4] == -127).all())   # cut off at 127 scales
    # the smallest numbers: 127 / a would be infinite
    small = torch.full((1, d), torch.finfo(torch.float32).smallest_normal / 64, device="cuda")
    q, s = ctx.rcd_quantize_rows(small)
    assert bool(torch.isfinite(s).all()) and bool((q >= 0).all())
    ctx.sync_status()


def test_sum_in_place_and_rows_behind(ctx):
    """h over x or over the residual itself; what lies between the rows and behind them stays as it was."""
    import torch
    for n, d, pad in [(5, 512, 64), (3, 77, 4), (700, 96, 8)]:
        g = seeded(n, d)
        x, r = rows(g, n, d, torch.bfloat16), rows(g, n, d, torch.bfloat16)
        w = torch.ones(d, device="cuda")
        y0, _, h0 = ctx.rcd_rms_norm(x, residual=r, weight=w, want_sum=True)
        for at in ("x", "r"):
            xx, rr = x.clone(), r.clone()
            y, _, h = ctx.rcd_rms_norm(xx, residual=rr, weight=w, sum_out=xx if at == "x" else rr)
            assert torch.equal(y, y0) and torch.equal(xx if at == "x" else rr, h0)
        buf = torch.full((n + 2, d + pad), 7.0, device="cuda", dtype=torch.bfloat16)
        q = torch.full((n + 2, d + pad), 7, device="cuda", dtype=torch.int8)
        ctx.rcd_rms_norm(x, residual=r, weight=w, out=buf[1:n + 1, :d])
        ctx.rcd_rms_norm(x, residual=r, weight=w, out=q[1:n + 1, :d])
        assert torch.equal(buf[1:n + 1, :d], y0)
        for b in (buf, q):
            b[1:n + 1, :d] = 7
            assert bool((b == 7).all())
    ctx.sync_status()


def test_no_rows(ctx):
    import torch
    x = torch.empty(0, 64, device="cuda", dtype=torch.bfloat16)
    y, s, h = ctx.rcd_rms_norm(x, out_dtype=torch.int8, want_sum=True)
    assert y.shape == (0, 64) and s.shape == (0,) and h.shape == (0, 64)
    dx, dw = ctx.rcd_rms_norm_backward(x, x, weight=torch.ones(64, device="cuda"))
    assert dx.shape == (0, 64) and bool((dw == 0).all())
    y, _, _ = ctx.rcd_rms_norm(torch.ones(2, 3, 64, device="cuda"))
    assert y.shape == (2, 3, 64)
    ctx.sync_status()


def gradients(dy, h, w, eps, dsum):
    import torch
    h, dy = h.double(), dy.double()
    g = dy if w is None else dy * w.double()
    v = h.square().mean(1, keepdim=True) + eps
    rstd = torch.where(v > 0, v.rsqrt(), torch.zeros_like(v))
    dx = rstd * (g - h * rstd ** 2 * (g * h).mean(1, keepdim=True))
    return dx if dsum is None else dx + dsum.double(), (dy * h * rstd).sum(0)


@pytest.mark.parametrize("n,d", SIZES + MANY + [(3000, 2048), (2000, 1000)])
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("pad,weight,dsum", [(0, "same", True), (0, "fp32", False), (3, None, True), (16, "same", False)])
def test_backward(ctx, n, d, dtype, pad, weight, dsum):
    import torch
    t, g = kind(dtype), seeded(n, d, dtype, pad, 9)
    h, dy = rows(g, n, d, t, pad), rows(g, n, d, t)
    s = rows(g, n, d, t, pad) if dsum else None
    w = torch.randn(d, generator=g, device="cuda").to(t if weight == "same" else torch.float32) if weight else None
    dx, dw = ctx.rcd_rms_norm_backward(dy, h, weight=w, eps=1e-5, dsum=s)
    ctx.sync_status()
    want, want_dw = gradients(dy, h, w, 1e-5, s)
    # dx is a difference: what each part is rounded by counts, not the result; sum(g h) cancels among itself, too
    hd, gd = h.double(), (dy.double() if w is None else dy.double() * w.double())
    v = hd.square().mean(1, keepdim=True) + 1e-5
    parts = (gd.abs() + hd.abs() / v * (gd * hd).abs().mean(1, keepdim=True)) / v.sqrt() + (0 if s is None else s.double().abs())
    check(dx, want, t, slack=parts * STEPS)
    if weight:
        # n terms a column: at most n / 2 additions one after the other, each off by half a unit of the partial sum
        bound = (dy.double() * hd).abs().div(v.sqrt()).sum(0) * (n + 64) * 2.0 ** -24
        assert bool(((dw.double() - want_dw).abs() <= bound).all())
        dx2, dw2 = ctx.rcd_rms_norm_backward(dy, h, weight=w, eps=1e-5, dsum=s)
        assert torch.equal(dx, dx2) and torch.equal(dw, dw2)
        dx3, none = ctx.rcd_rms_norm_backward(dy, h, weight=w, eps=1e-5, dsum=s, want_dweight=False)
        assert none is None and torch.equal(dx, dx3)
    else:
        assert dw is None


def test_backward_rows_of_zeros(ctx):
    """eps 0: rstd of a row of zeros is taken as 0, and so are its gradients (but for what comes along the residual)."""
    import torch
    h = torch.zeros(3, 96, device="cuda")
    h[1] = 1
    dy, s = torch.ones_like(h), torch.full_like(h, 2.0)
    dx, dw = ctx.rcd_rms_norm_backward(dy, h, weight=torch.ones(96, device="cuda"), eps=0.0, dsum=s)
    assert torch.equal(dx[0], s[0]) and torch.equal(dx[2], s[2])
    assert torch.allclose(dw, torch.ones(96, device="cuda"), rtol=1e-6)


def test_backward_against_differences(ctx):
    """Central differences of the kernel's own forward pass, a loss of sum(c y) in 64 bits.  Steps of 2^-5 on values of about 1: the
    third derivative's part is below 2^-10 / 6 of it, the forward's roundings 2^-24 * sqrt(d) / 2^-5 below 2^-14."""
    import torch
    g = seeded("differences")
    n, d = 4, 24
    x, w, c = rows(g, n, d, torch.float32), torch.randn(d, generator=g, device="cuda"), rows(g, n, d, torch.float32)
    loss = lambda xx, ww: float((ctx.rcd_rms_norm(xx, weight=ww, eps=1e-2)[0].double() * c.double()).sum())  # noqa: E731
    dx, dw = ctx.rcd_rms_norm_backward(c, x, weight=w, eps=1e-2)
    step = 2.0 ** -5
    for at, got, mine in ((x, dx, True), (w, dw, False)):
        flat = at.reshape(-1)
        for i in range(0, flat.numel(), 5):
            lo, hi = flat.clone(), flat.clone()
            lo[i] -= step
            hi[i] += step
            num = (loss(hi.view(at.shape), w) - loss(lo.view(at.shape), w) if mine else loss(x, hi) - loss(x, lo)) / (2 * step)
            assert abs(num - float(got.reshape(-1)[i])) <= 2e-2 * (1 + abs(num)), (mine, i)


def test_streams_and_graphs(ctx):
    """Another stream than the current one of the tensors' making, and two captured graphs replayed in turn with new inputs."""
    import torch
    g = seeded("graphs")
    x, w = rows(g, 300, 256, torch.bfloat16), torch.randn(256, generator=g, device="cuda")
    dy = rows(g, 300, 256, torch.bfloat16)
    want = ctx.rcd_rms_norm(x, weight=w)[0].clone()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = ctx.rcd_rms_norm(x, weight=w)[0]
    side.synchronize()
    assert torch.equal(got, want)
    graphs = []
    for _ in range(2):
        gr = torch.cuda.CUDAGraph()
        with torch.cuda.graph(gr):
            y, _, _ = ctx.rcd_rms_norm(x, weight=w)
            dx, dw = ctx.rcd_rms_norm_backward(dy, x, weight=w)
        graphs.append((gr, y, dx, dw))
    for k in range(3):
        x.copy_(rows(g, 300, 256, torch.bfloat16))
        for gr, *_ in graphs:
            gr.replay()
        torch.cuda.synchronize()
        y, (dx, dw) = ctx.rcd_rms_norm(x, weight=w)[0], ctx.rcd_rms_norm_backward(dy, x, weight=w)
        for _, gy, gdx, gdw in graphs:
            assert torch.equal(gy, y) and torch.equal(gdx, dx) and torch.equal(gdw, dw)


def test_refusals(rcd, ctx):
    import ctypes as C
    import torch
    x = torch.ones(4, 64, device="cuda", dtype=torch.bfloat16)
    for bad in (dict(eps=-1.0), dict(eps=float("nan")), dict(eps=float("inf")), dict(out_dtype=torch.int8, scale=float("inf")),
                dict(out_dtype=torch.int8, scale=1e-45), dict(scale=0.5), dict(out=x), dict(out=x[:, :32]), dict(scale=-1.0),
                dict(weight=torch.ones(63, device="cuda")), dict(weight=torch.ones(64)), dict(residual=x[:3]), dict(residual=x.float()),
                dict(out_dtype=torch.float64), dict(weight=torch.ones(64, device="cuda", dtype=torch.float64)), dict(sum_out=x[:, :32])):
        with pytest.raises((rcd.RcdError, ValueError, TypeError)):
            ctx.rcd_rms_norm(x, **bad)
    with pytest.raises(rcd.RcdError):
        ctx.rcd_rms_norm(torch.ones(2, 16385, device="cuda"))
    with pytest.raises(rcd.RcdError):
        ctx.rcd_rms_norm(torch.ones(2, 0, device="cuda"))
    with pytest.raises(rcd.RcdError):                       # int8 in
        ctx.rcd_rms_norm(x.to(torch.int8))
    with pytest.raises(ValueError):                         # on the CPU
        ctx.rcd_rms_norm(x.cpu())
    buf = torch.ones(5, 64, device="cuda", dtype=torch.bfloat16)
    with pytest.raises(rcd.RcdError):                       # the sum one row further on than x
        ctx.rcd_rms_norm(buf[:4], sum_out=buf[1:])
    with pytest.raises(ValueError):
        ctx.rcd_rms_norm_backward(x, x[:3])
    with pytest.raises(TypeError):
        ctx.rcd_rms_norm_backward(x.float(), x)
    a = rcd.RcdNormArgs()
    a.rows, a.d, a.x_type, a.y_type, a.ldx, a.ldy, a.eps = 4, 64, rcd.RCD_ELEM_BF16, rcd.RCD_ELEM_BF16, 64, 64, 1e-6
    a.y = x.data_ptr()
    run = lambda: rcd.lib.rcd_rms_norm(ctx._h, C.byref(a), None)  # noqa: E731
    assert run() == 1                                       # x is null
    a.x, a.ldx = buf.data_ptr(), 63
    assert run() == 1
    a.ldx, a.x = 64, buf.data_ptr() + 1
    assert run() == 1
    a.x, a.x_type = buf.data_ptr(), 9
    assert run() == 1
    a.x_type, a.rows = rcd.RCD_ELEM_BF16, -1
    assert run() == 1
    b = rcd.RcdNormBackArgs()
    b.rows, b.d, b.type, b.ld_h, b.ld_dy, b.ld_dx, b.eps = 4, 64, rcd.RCD_ELEM_BF16, 64, 64, 64, 1e-6
    dx, dw = torch.empty_like(x), torch.empty(64, device="cuda")
    b.h, b.dy, b.dx, b.dweight = x.data_ptr(), buf.data_ptr(), dx.data_ptr(), dw.data_ptr()
    assert rcd.lib.rcd_rms_norm_backward(ctx._h, C.byref(b), None, 0, None) == 3        # no workspace
    b.dx = x.data_ptr()
    ws = torch.empty(1 << 20, device="cuda", dtype=torch.uint8)
    assert rcd.lib.rcd_rms_norm_backward(ctx._h, C.byref(b), C.c_void_p(ws.data_ptr()), 1 << 20, None) == 1    # dx over h
    b.dx = dx.data_ptr()
    assert rcd.lib.rcd_rms_norm_backward(ctx._h, C.byref(b), C.c_void_p(ws.data_ptr() + 8), (1 << 20) - 8, None) == 1
    assert rcd.lib.rcd_rms_norm(None, C.byref(a), None) == 1
    ctx.sync_status()


def test_offsets_beyond_32_bits(ctx):
    """2.3 billion elements: the last rows, forward and backward."""
    import torch
    n, d = 140000, 16384
    x = torch.ones(n, d, device="cuda", dtype=torch.bfloat16)
    tail = rows(seeded("far"), 300, d, torch.bfloat16)
    x[-300:] = tail
    q, s, _ = ctx.rcd_rms_norm(x, out_dtype=torch.int8)
    want, _ = steps_of(tail, None, None, 1e-6)
    assert torch.equal(q[-300:], want) and bool((q[:5] == 127).all())
    dx, _ = ctx.rcd_rms_norm_backward(x, x)
    few, _ = ctx.rcd_rms_norm_backward(tail, tail)
    parts = tail.double().abs() * 2 / tail.double().square().mean(1, keepdim=True).sqrt()
    check(dx[-300:], few.double(), torch.bfloat16, slack=parts * (STEPS + half_step(torch.bfloat16)))
    ctx.sync_status()
