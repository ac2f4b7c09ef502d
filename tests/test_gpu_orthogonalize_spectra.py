"""How far an update is off by the spectrum of its gradient: noise alone, and noise under a few directions ten and a hundred times as strong, which weight gradients look like.
The weak directions carry the roundings that the strong ones' entries make.  Against the formula in 64 bits, and against what the roundings that
are made come to in 64 bits: X, A and B as fp16 times 2^10 between the products, G itself in the first step's sum whatever its type, bf16 at the end."""
import pytest

from test_gpu_norm import ctx, kind, rcd, seeded  # noqa: F401  (fixtures)
from test_gpu_orthogonalize import QUINTIC
from test_gpu_orthogonalize_forms import CLUSTER, LAUNCHES, STEPS, taken

pytestmark = pytest.mark.gpu


def gradient(g, rows, cols, directions, strength):
    import torch
    x = torch.randn(rows, cols, generator=g, device="cuda")
    if directions:
        x = x + strength * torch.randn(rows, directions, generator=g, device="cuda") @ torch.randn(directions, cols, generator=g, device="cuda")
    return x


def exactly(g):
    x = g.double() / g.double().norm()
    x = x if x.shape[0] <= x.shape[1] else x.t()
    a, b, c = QUINTIC
    for _ in range(5):
        m = x @ x.t()
        x = a * x + (b * m + c * m @ m) @ x
    return x if g.shape[0] <= g.shape[1] else x.t()


def with_roundings(g):
    import math
    import torch

    def half(x):
        return (x * 1024).half().double() / 1024
    norm = float(g.double().norm())
    up = 2.0 ** -math.floor(math.log2(norm)) / 2
    factor = 1 / (norm * up)
    whole = g.double() * up
    whole = whole if g.shape[0] <= g.shape[1] else whole.t()
    x = half(whole)
    a, b, c = QUINTIC
    for i in range(5):
        f = factor if i == 0 else 1.0
        m = half(f * f * (x @ x.t()))
        p = half(b * m + c * m @ m)
        y = f * (a * (whole if i == 0 else x) + p @ x)
        x = y.to(torch.bfloat16).double() if i == 4 else half(y)
    return x if g.shape[0] <= g.shape[1] else x.t()


@pytest.mark.parametrize("rows,cols,form", [(128, 128, CLUSTER), (100, 1500, CLUSTER), (1500, 120, CLUSTER), (128, 2056, CLUSTER), (256, 512, STEPS), (512, 256, STEPS), (300, 430, STEPS),
                                            (1024, 1024, STEPS), (1500, 1100, LAUNCHES), (1100, 1500, LAUNCHES)])
@pytest.mark.parametrize("dtype", ["fp32", "bf16", "fp16"])
# (a hundred times one direction: of 64 bits' 0.5 % with the roundings; ten times sixteen: 0.8 %)
@pytest.mark.parametrize("directions,strength,bound", [(0, 0.0, 3e-3), (16, 10.0, 1e-2), (1, 100.0, 1e-2)])
def test_strong_directions(rcd, ctx, rows, cols, form, dtype, directions, strength, bound):
    g = (gradient(seeded("spectrum", rows, directions), rows, cols, directions, strength)).to(kind(dtype))
    o = ctx.rcd_orthogonalize(g, eps=0.0)
    assert taken(ctx, 5) == form
    ctx.sync_status()
    want = exactly(g)
    off, made = (float((x.double() - want).norm() / want.norm()) for x in (o, with_roundings(g)))
    # (a tenth for the sums in the tensor cores, whose last bits are below every one of these roundings)
    assert off <= 1.1 * made, (off, made)
    assert off <= bound, (off, made)


@pytest.mark.parametrize("rows,cols", [(100, 300), (300, 430), (1500, 1100)])
def test_what_an_fp32_gradient_holds_beyond_16_bits(rcd, ctx, rows, cols):
    """One step that keeps X alone (b and c zero) is a X: an fp32 G comes through it to bf16's rounding, whatever fp16 makes of it."""
    import torch
    g = gradient(seeded("beyond", rows), rows, cols, 1, 100.0)
    o = ctx.rcd_orthogonalize(g, steps=1, coefficients=(1.0, 0.0, 0.0), eps=0.0)
    want = g.double() / g.double().norm()
    # half a step of bf16; a few of fp32
    worst = float(((o.double() - want).abs() - want.abs() * (2.0 ** -8 / (1 + 2.0 ** -8) + 2.0 ** -20)).max())
    assert worst <= 0, worst
    ctx.sync_status()


@pytest.mark.parametrize("rows,cols", [(4300, 4200), (4200, 4300)])
def test_long_sums(rcd, ctx, rows, cols):
    """Sums in chunks of 2048, an fp32 gradient."""
    import torch
    g = gradient(seeded("long", rows), rows, cols, 16, 10.0)
    o = ctx.rcd_orthogonalize(g, eps=0.0)
    assert taken(ctx, 5) == LAUNCHES
    want = exactly(g)
    off, made = (float((x.double() - want).norm() / want.norm()) for x in (o, with_roundings(g)))
    assert off <= 1.1 * made and off <= 1e-2, (off, made)
    ctx.sync_status()


@pytest.mark.parametrize("batch,rows,cols", [(3, 100, 1101), (2, 300, 433), (2, 1500, 1101), (2, 1120, 1500), (1, 1101, 1503)])
def test_layouts_of_fp32_gradients(rcd, ctx, batch, rows, cols):
    import torch
    g = torch.stack([gradient(seeded("layout", rows, i), rows, cols, 1, 100.0) for i in range(batch)])
    want = ctx.rcd_orthogonalize(g)
    for one, its in zip(want, g):
        exact = exactly(its)
        assert float((one.double() - exact).norm() / exact.norm()) <= 1e-2
    wide = torch.full((batch, rows + 2, cols + 11), float("nan"), device="cuda")
    wide[:, 1:-1, 3:cols + 3] = g
    assert torch.equal(ctx.rcd_orthogonalize(wide[:, 1:-1, 3:cols + 3]), want)
    for off in (3, 8):
        buf = torch.full((batch, rows + 2, cols + 16), 7.0, device="cuda", dtype=torch.bfloat16)
        view = buf[:, 1:-1, off:cols + off]
        assert ctx.rcd_orthogonalize(g, out=view) is view
        assert torch.equal(view, want)
        view[:] = 7
        assert bool((buf == 7).all())
    ctx.sync_status()


@pytest.mark.parametrize("rows,cols", [(128, 128), (300, 430), (1500, 1100)])
@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_gradients_below_eps(rcd, ctx, rows, cols, dtype):
    """|G| a thousandth of eps: entries of X are 1e-6 and more on the mean, well above 2^-24, and the result is as good as ever."""
    import torch
    g = gradient(seeded("below", rows), rows, cols, 0, 0.0)
    g = (g / g.norm() * 1e-5).to(kind(dtype))
    o = ctx.rcd_orthogonalize(g, eps=1e-2)
    x = g.double() / (g.double().norm() + 1e-2)
    x = x if rows <= cols else x.t()
    a, b, c = QUINTIC
    for _ in range(5):
        m = x @ x.t()
        x = a * x + (b * m + c * m @ m) @ x
    want = x if rows <= cols else x.t()
    assert float((o.double() - want).norm() / want.norm()) <= 3e-3
    ctx.sync_status()
