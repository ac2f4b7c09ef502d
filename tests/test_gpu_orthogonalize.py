"""Weight gradients with their singular values brought near one by Newton-Schulz products, against the formula in 64 bits."""
import math

import pytest

from test_gpu_norm import ctx, half_step, kind, rcd, seeded  # noqa: F401  (fixtures)

pytestmark = pytest.mark.gpu
QUINTIC = (3.4445, -4.7750, 2.0315)
U16 = 2.0 ** -11


def newton_schulz(g, steps=5, coefficients=QUINTIC, eps=1e-7):
    """The formula in 64 bits, and a bound of the 2-norm of what fp16 between the products does to it, to first order: every rounding is half
    a step of fp16 (of X, A and B, whose 2-norms are known here), an error of A goes into B by |b| + 2 |c| |A|, one of B into X by |X|, and one of X
    through the step by the polynomial's largest slope between 0 and the largest singular value, or its largest ratio."""
    import torch
    x = g.double()
    norm = x.norm()
    x = x / (norm + eps)
    tall = x.shape[0] > x.shape[1]
    if tall:
        x = x.t()
    err = 0.0 if g.dtype != torch.float32 else U16 * float(x.norm())
    # (fp16's smallest step is 2^-24, entries stand times 2^10)
    least = math.sqrt(x.numel()) * 2.0 ** -35
    for i in range(steps):
        a, b, c = coefficients if not hasattr(coefficients[0], "__len__") else coefficients[i]
        m = x @ x.t()
        top = math.sqrt(float(torch.linalg.matrix_norm(m, 2)))
        p = b * m + c * (m @ m)
        da = U16 * float(m.norm()) + least
        dp = U16 * float(p.norm()) + least + (abs(b) + 2 * abs(c) * top * top) * da
        s = torch.linspace(0, top * 1.01, 1000, dtype=torch.float64)
        slope = float(torch.maximum((a + 3 * b * s ** 2 + 5 * c * s ** 4).abs(), (a + b * s ** 2 + c * s ** 4).abs()).max())
        x = a * x + p @ x
        err = slope * err + top * dp + U16 * float(x.norm()) + least
    return (x.t() if tall else x), err


def gradient(g, batch, rows, cols, dtype, pad=0, strong=2.0):
    import torch
    x = torch.randn(batch, rows, cols + pad, generator=g, device="cuda")
    x = x + strong * torch.randn(batch, rows, 2, generator=g, device="cuda") @ torch.randn(batch, 2, cols + pad, generator=g, device="cuda")
    return (x * 1e-3).to(dtype)[:, :, :cols]


def check(o, g, **kw):
    import torch
    assert o.dtype == torch.bfloat16 and o.shape == g.shape
    for mine, its in zip(o.reshape(-1, *o.shape[-2:]), g.reshape(-1, *g.shape[-2:])):
        want, err = newton_schulz(its, **kw)
        off = float((mine.double() - want).norm())
        assert off <= 1.05 * err + half_step(torch.bfloat16) * float(want.norm()) * 1.01, (off, err, float(want.norm()))
        # and what it comes to in practice: roundings do not add up like that.  (The steps' own amplification: 0.02 allows for ten times what was reckoned in
        # 64 bits with fp16 between the products for such gradients.)
        if min(its.shape) >= 32 and "coefficients" not in kw and "steps" not in kw:
            assert off <= 0.02 * float(want.norm()), off / float(want.norm())


SIZES = [(1, 1, 1), (1, 1, 64), (2, 3, 1), (1, 16, 16), (3, 33, 65), (1, 64, 64), (2, 64, 200), (1, 127, 129), (1, 128, 128), (5, 130, 70), (1, 200, 1000), (2, 256, 256), (1, 333, 1001),
         (3, 320, 320), (1, 512, 2048), (2, 513, 300), (1, 777, 777), (1, 1024, 1024), (1, 2048, 512), (16, 96, 160), (150, 40, 64), (2, 128, 384), (1, 100, 500), (2, 1500, 60), (1, 128, 2050), (1, 30, 4096), (2, 6100, 128), (40, 77, 300), (12, 300, 310), (20, 200, 150), (4, 300, 1000),
         (4, 1100, 290)]


@pytest.mark.parametrize("batch,rows,cols", SIZES)
@pytest.mark.parametrize("dtype", ["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("pad", [0, 3])
def test_against_the_formula(rcd, ctx, batch, rows, cols, dtype, pad):
    import torch
    g = gradient(seeded("ns", batch, rows, cols, dtype, pad), batch, rows, cols, kind(dtype), pad)
    o = ctx.rcd_orthogonalize(g)
    ctx.sync_status()
    check(o, g)
    # every matrix of a batch by itself: the same bits alone, up to the tile that a batch is gone about with, whose sums' order is the same
    if batch > 1 and rows % 32 == 0:
        alone = ctx.rcd_orthogonalize(g[1].contiguous())
        assert float((alone.double() - o[1].double()).norm()) <= 0.01 * float(o[1].double().norm())
    assert torch.equal(ctx.rcd_orthogonalize(g), o)


@pytest.mark.parametrize("batch,rows,cols,dtype", [(1, 2300, 2300, "bf16"), (1, 4200, 1100, "fp16"), (1, 600, 5000, "bf16"), (3, 1500, 1100, "fp32"), (2, 1100, 1500, "bf16"), (2, 1600, 1536, "bf16"),
                                                   (6, 900, 1000, "fp16")])
def test_large(rcd, ctx, batch, rows, cols, dtype):
    """Launches of their own: pairs of SMs, sums in chunks (more than 4096 rows or columns), blocks that end inside a matrix, matrices that the last product cannot write
    (their rows are no multiple of 32)."""
    import torch
    g = gradient(seeded("large", batch, rows, cols), batch, rows, cols, kind(dtype))
    o = ctx.rcd_orthogonalize(g)
    ctx.sync_status()
    check(o, g)
    buf = torch.full((batch, rows + 1, cols + 24), 7.0, device="cuda", dtype=torch.bfloat16)
    assert torch.equal(ctx.rcd_orthogonalize(g, out=buf[:, :-1, 8:cols + 8]), o)
    buf[:, :-1, 8:cols + 8] = 7
    assert bool((buf == 7).all())


@pytest.mark.parametrize("rows,cols", [(100, 260), (260, 100)])
def test_known_values(rcd, ctx, rows, cols):
    """Rows (columns) that are orthogonal and equally long: every singular value is 1 / sqrt(side), and the result a multiple of G by the polynomial's value
    after five steps.  One direction alone: the multiple of 1.  Zeros stay zeros."""
    import torch
    side = min(rows, cols)
    a, b, c = QUINTIC
    s = side ** -0.5
    for _ in range(5):
        s = a * s + b * s ** 3 + c * s ** 5
    g = torch.zeros(rows, cols, device="cuda", dtype=torch.bfloat16)
    perm = torch.randperm(max(rows, cols), generator=seeded("perm"), device="cuda")[:side]
    i = torch.arange(side, device="cuda")
    g[(i, perm) if rows <= cols else (perm, i)] = -3.0
    o = ctx.rcd_orthogonalize(g)
    # (one entry a row: three roundings of fp16 a step, each grown by at most 4 a step, and the output's)
    assert float((o.double() - g.double() / 3 * s).abs().max()) <= s * (half_step(torch.bfloat16) + 3 * U16 * sum(4.0 ** k for k in range(5)))
    assert not o[g == 0].any()
    s = 1.0
    for _ in range(5):
        s = a * s + b * s ** 3 + c * s ** 5
    u, v = (torch.randint(0, 2, (n,), generator=seeded(n), device="cuda").double() * 2 - 1 for n in (rows, cols))
    g = (u[:, None] * v[None, :]).to(torch.bfloat16)
    o = ctx.rcd_orthogonalize(g, eps=0.0)
    want, err = newton_schulz(g, eps=0.0)
    assert float((o.double() - want).norm()) <= 1.05 * err + half_step(torch.bfloat16) * float(want.norm()) * 1.01
    assert not ctx.rcd_orthogonalize(torch.zeros_like(g)).any() and not ctx.rcd_orthogonalize(torch.zeros_like(g), eps=0.0).any()
    ctx.sync_status()


@pytest.mark.parametrize("steps,coefficients", [(1, QUINTIC), (3, (1.5, -0.5, 0.0)), (2, [(1.875, -1.25, 0.375), (1.5, -0.5, 0.0)]), (7, (1.875, -1.25, 0.375)), (6, QUINTIC)])
@pytest.mark.parametrize("rows,cols", [(96, 200), (200, 96), (128, 128)])
def test_steps_and_coefficients(rcd, ctx, steps, coefficients, rows, cols):
    import torch
    g = gradient(seeded("steps", steps, rows), 2, rows, cols, torch.bfloat16)
    check(ctx.rcd_orthogonalize(g, steps=steps, coefficients=coefficients), g, steps=steps, coefficients=coefficients)
    ctx.sync_status()


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("size", [2.0 ** -120, 2.0 ** -60, 2.0 ** 60, 2.0 ** 110])
def test_gradients_of_any_size(rcd, ctx, dtype, size):
    """A power of two times G is the same G: bit for bit without eps."""
    import torch
    g = gradient(seeded("size"), 1, 70, 150, kind(dtype))[0]
    want = ctx.rcd_orthogonalize(g, eps=0.0)
    scaled = (g.double() * size).to(g.dtype)
    o = ctx.rcd_orthogonalize(scaled, eps=0.0)
    check(o, scaled, eps=0.0)
    if torch.equal(scaled.double(), g.double() * size):       # (not where it leaves the type's normal range)
        assert torch.equal(o, want)
    else:
        assert size == 2.0 ** -120
    # eps much larger than |G|: X stays small, and so does what the polynomial makes of it
    small = (g.double() * 2.0 ** -40).to(g.dtype)
    check(ctx.rcd_orthogonalize(small, steps=2), small, steps=2)
    ctx.sync_status()


def test_what_is_not_finite_stays_in_its_matrix(rcd, ctx):
    import torch
    g = gradient(seeded("nan"), 4, 70, 150, torch.bfloat16)
    want = ctx.rcd_orthogonalize(g)
    bad = g.clone()
    bad[1, 5, 6] = float("nan")
    bad[3, 69, 149] = float("inf")
    o = ctx.rcd_orthogonalize(bad)
    assert torch.equal(o[0], want[0]) and torch.equal(o[2], want[2])
    assert bool(torch.isnan(o[1]).all()) and bool(torch.isnan(o[3]).all())
    ctx.sync_status()


def test_layouts_out_and_what_lies_beside(rcd, ctx):
    """Leading dimensions, strides of rows and matrices, outputs inside wider buffers: direct from the last product and through a pass of their own."""
    import torch
    for batch, rows, cols in ((4, 64, 100), (4, 33, 100), (1, 70, 65), (3, 96, 64), (2, 130, 40)):
        g = gradient(seeded("layout", rows), batch, rows, cols, torch.bfloat16)
        want = ctx.rcd_orthogonalize(g)
        assert torch.equal(ctx.rcd_orthogonalize(g.view(1, batch, rows, cols))[0], want)
        assert torch.equal(ctx.rcd_orthogonalize(g.transpose(1, 2).contiguous().transpose(1, 2)), want)
        wide = torch.zeros(batch, rows + 2, cols + 11, device="cuda", dtype=torch.bfloat16)
        wide[:, 1:-1, 3:cols + 3] = g
        assert torch.equal(ctx.rcd_orthogonalize(wide[:, 1:-1, 3:cols + 3]), want)
        for off in (3, 8):
            buf = torch.full((batch, rows + 2, cols + 16), 7.0, device="cuda", dtype=torch.bfloat16)
            view = buf[:, 1:-1, off:cols + off]
            assert ctx.rcd_orthogonalize(g, out=view) is view
            assert torch.equal(view, want)
            view[:] = 7
            assert bool((buf == 7).all())
    # a slice that is only every second matrix
    g = gradient(seeded("layout"), 6, 64, 64, torch.float16)
    assert torch.equal(ctx.rcd_orthogonalize(g[::2]), ctx.rcd_orthogonalize(g[::2].contiguous()))
    for shape in ((0, 4, 4), (2, 0, 4), (4, 0)):
        e = torch.empty(shape, device="cuda", dtype=torch.bfloat16)
        assert ctx.rcd_orthogonalize(e).shape == shape
    ctx.sync_status()


def test_captured_and_on_another_stream(rcd, ctx):
    import torch
    a, b = (gradient(seeded("graph", i), 2, 96, 200, torch.bfloat16) for i in range(2))
    want = [ctx.rcd_orthogonalize(a), ctx.rcd_orthogonalize(b)]
    graphs = []
    for x in (a, b):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            o = ctx.rcd_orthogonalize(x)
        graphs.append((graph, o))
    for _ in range(3):
        for graph, _ in graphs:
            graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(o, w) for (_, o), w in zip(graphs, want))
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        o = ctx.rcd_orthogonalize(a)
    s.synchronize()
    assert torch.equal(o, want[0])
    ctx.sync_status()


def test_refusals(rcd, ctx):
    import ctypes as C
    import numpy as np
    import torch
    g = gradient(seeded("refusals"), 2, 200, 300, torch.bfloat16)        # (larger than what takes no workspace)
    for bad in (g.cpu(), g[0, 0]):
        with pytest.raises(ValueError):
            ctx.rcd_orthogonalize(bad)
    with pytest.raises(TypeError):
        ctx.rcd_orthogonalize(g.double())
    for kw in (dict(steps=0), dict(steps=65), dict(eps=-1.0), dict(eps=float("nan")), dict(eps=float("inf")), dict(coefficients=(1.0, float("nan"), 0.0)), dict(coefficients=(1e5, 0.0, 0.0))):
        with pytest.raises(rcd.RcdError):
            ctx.rcd_orthogonalize(g, **kw)
    for kw in (dict(coefficients=(1.0, 2.0)), dict(steps=3, coefficients=[QUINTIC, QUINTIC]), dict(out=g.half()), dict(out=g[:1].clone()), dict(out=torch.empty(2, 300, 200, device="cuda", dtype=torch.bfloat16).transpose(1, 2))):
        with pytest.raises(ValueError):
            ctx.rcd_orthogonalize(g, **kw)
    with pytest.raises(rcd.RcdError):
        ctx.rcd_orthogonalize(g, out=g)                       # the output is the input
    c = np.array(QUINTIC * 5, dtype=np.float32)
    o = torch.empty_like(g)
    ok = dict(batch=2, rows=200, cols=300, type=1, g=g.data_ptr(), ld_g=300, step_g=60000, steps=5, coefficients_host=c.ctypes.data, eps=0.0, o=o.data_ptr(), ld_o=300, step_o=60000)
    need = C.c_size_t()

    def refused(status, ws=None, size=0, **change):
        a = rcd.RcdOrthogonalizeArgs(**{**ok, **change})
        got = rcd.lib.rcd_orthogonalize_workspace_bytes(ctx._h, C.byref(a), C.byref(need)) if ws is None else rcd.lib.rcd_orthogonalize(ctx._h, C.byref(a), ws, size, None)
        assert got == status, (got, change)
    refused(0)
    big = torch.empty(need.value + 256, dtype=torch.uint8, device="cuda")
    for change in (dict(g=None), dict(o=None), dict(coefficients_host=None), dict(type=0), dict(type=9), dict(batch=-1), dict(rows=-3), dict(ld_g=299), dict(ld_o=2), dict(step_g=59999), dict(step_o=0),
                   dict(g=g.data_ptr() + 1), dict(o=o.data_ptr() + 1)):
        refused(1, **change)
    refused(2, rows=1 << 17)
    refused(2, batch=1 << 16)
    refused(3, ws=big.data_ptr(), size=need.value - 1)
    refused(1, ws=big.data_ptr() + 16, size=need.value)
    refused(1, ws=big.data_ptr(), size=need.value, o=big.data_ptr())
    small = dict(rows=20, cols=30)
    refused(0, **small)
    assert need.value == 0
    refused(0, ws=C.c_void_p(None), size=0, **small)
    refused(1, ws=C.c_void_p(None), size=0, **{**small, "o": g.data_ptr()})
    ctx.sync_status()
