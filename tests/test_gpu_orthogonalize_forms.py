"""Every form in which updates are computed (a cluster per matrix, all steps in one launch, launches of their own) at what the formula's tests of small
matrices reach in the first of them alone: steps and coefficients, sizes of G, what is not finite, layouts, graphs."""
import math

import pytest

from test_gpu_norm import ctx, half_step, kind, rcd, seeded  # noqa: F401  (fixtures)
from test_gpu_orthogonalize import QUINTIC, U16, check, gradient, newton_schulz

pytestmark = pytest.mark.gpu

# batch, rows, cols, form.  (320 rows or columns after padding: a tile of 128 rows reads on into the next matrix)
CLUSTER, STEPS, LAUNCHES = "a cluster per matrix", "all steps in one launch", "launches of their own"
SHAPES = [(2, 70, 150, CLUSTER), (2, 200, 330, STEPS), (2, 330, 200, STEPS), (3, 300, 450, STEPS), (1, 1500, 1100, LAUNCHES), (2, 1100, 1500, LAUNCHES), (2, 1536, 1088, LAUNCHES)]


def taken(ctx, steps):
    """The form of the last call, by its launches."""
    launches = ctx.profile()["kernel_launches"]
    return CLUSTER if launches == 1 else STEPS if launches == 3 else LAUNCHES if 2 + 3 * steps <= launches <= 3 + 3 * steps else launches


@pytest.mark.parametrize("steps,coefficients", [(1, QUINTIC), (3, (1.5, -0.5, 0.0)), (2, [(1.875, -1.25, 0.375), (1.5, -0.5, 0.0)]), (7, (1.875, -1.25, 0.375)), (6, QUINTIC),
                                                (4, [QUINTIC, (2.0, -1.5, 0.5), (1.5, -0.5, 0.0), (1.0, 0.0, 0.0)])])
@pytest.mark.parametrize("batch,rows,cols,form", SHAPES)
def test_steps_and_coefficients(rcd, ctx, steps, coefficients, batch, rows, cols, form):
    import torch
    g = gradient(seeded("steps", steps, rows), batch, rows, cols, torch.bfloat16)
    o = ctx.rcd_orthogonalize(g, steps=steps, coefficients=coefficients)
    if steps > 1:
        assert taken(ctx, steps) == form
    ctx.sync_status()
    check(o, g, steps=steps, coefficients=coefficients)


@pytest.mark.parametrize("batch,rows,cols,form", SHAPES)
def test_known_values(rcd, ctx, batch, rows, cols, form):
    """Rows (columns) that are orthogonal and equally long, in one matrix of a batch; one direction alone in another; zeros."""
    import torch
    side = min(rows, cols)
    a, b, c = QUINTIC

    def polynomial(s):
        for _ in range(5):
            s = a * s + b * s ** 3 + c * s ** 5
        return s
    first = torch.zeros(rows, cols, device="cuda", dtype=torch.bfloat16)
    perm = torch.randperm(max(rows, cols), generator=seeded("perm"), device="cuda")[:side]
    i = torch.arange(side, device="cuda")
    first[(i, perm) if rows <= cols else (perm, i)] = -3.0
    u, v = (torch.randint(0, 2, (n,), generator=seeded(n), device="cuda").double() * 2 - 1 for n in (rows, cols))
    second = (u[:, None] * v[None, :]).to(torch.bfloat16)
    s = polynomial(side ** -0.5)
    for g in [torch.stack([first, second, first])[:batch]] + [torch.stack([second, first, second])[:batch]]:
        o = ctx.rcd_orthogonalize(g, eps=0.0)
        assert taken(ctx, 5) == form
        for mine, its in zip(o, g):
            if its[0, 0] != 0 and its[0, 1] != 0:
                want, err = newton_schulz(its, eps=0.0)
                assert float((mine.double() - want).norm()) <= 1.05 * err + half_step(torch.bfloat16) * float(want.norm()) * 1.01
            else:
                # (one entry a row: three roundings of fp16 a step, each grown by at most 4 a step, and the output's)
                assert float((mine.double() - its.double() / 3 * s).abs().max()) <= s * (half_step(torch.bfloat16) + 3 * U16 * sum(4.0 ** k for k in range(5)))
                assert not mine[its == 0].any()
    none = torch.zeros(batch, rows, cols, device="cuda", dtype=torch.bfloat16)
    assert not ctx.rcd_orthogonalize(none).any() and not ctx.rcd_orthogonalize(none, eps=0.0).any()
    ctx.sync_status()


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("size", [2.0 ** -120, 2.0 ** -60, 2.0 ** 60, 2.0 ** 105])
@pytest.mark.parametrize("rows,cols,form", [(200, 330, STEPS), (330, 200, STEPS), (1500, 1100, LAUNCHES)])
def test_gradients_of_any_size(rcd, ctx, dtype, size, rows, cols, form):
    """A power of two times G is the same G: bit for bit without eps."""
    import torch
    g = gradient(seeded("size"), 1, rows, cols, kind(dtype))[0]
    want = ctx.rcd_orthogonalize(g, eps=0.0)
    assert taken(ctx, 5) == form
    scaled = (g.double() * size).to(g.dtype)
    o = ctx.rcd_orthogonalize(scaled, eps=0.0)
    check(o, scaled, eps=0.0)
    if torch.equal(scaled.double(), g.double() * size):       # (not where it leaves the type's normal range)
        assert torch.equal(o, want)
    else:
        assert size == 2.0 ** -120
    ctx.sync_status()


@pytest.mark.parametrize("rows,cols,form", [(70, 150, CLUSTER), (200, 330, STEPS), (300, 430, STEPS), (450, 300, STEPS), (1100, 1500, LAUNCHES), (1536, 1088, LAUNCHES)])
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_what_is_not_finite_stays_in_its_matrix(rcd, ctx, rows, cols, form, dtype):
    import torch
    g = gradient(seeded("nan"), 4, rows, cols, kind(dtype))
    want = ctx.rcd_orthogonalize(g)
    assert taken(ctx, 5) == form
    bad = g.clone()
    bad[1, 5, 6] = float("nan")
    bad[3, rows - 1, cols - 1] = float("inf")
    o = ctx.rcd_orthogonalize(bad)
    assert torch.equal(o[0], want[0]) and torch.equal(o[2], want[2])
    assert bool(torch.isnan(o[1]).all()) and bool(torch.isnan(o[3]).all())
    ctx.sync_status()


@pytest.mark.parametrize("batch,rows,cols,form", [(4, 160, 300, STEPS), (3, 300, 333, STEPS), (1, 257, 505, STEPS), (2, 600, 200, STEPS), (2, 1120, 1500, LAUNCHES), (2, 1500, 1101, LAUNCHES),
                                                  (1, 1501, 1103, LAUNCHES)])
def test_layouts_out_and_what_lies_beside(rcd, ctx, batch, rows, cols, form):
    """Leading dimensions, strides of rows and matrices, outputs inside wider buffers."""
    import torch
    g = gradient(seeded("layout", rows), batch, rows, cols, torch.bfloat16)
    want = ctx.rcd_orthogonalize(g)
    assert taken(ctx, 5) == form
    assert torch.equal(ctx.rcd_orthogonalize(g.view(1, batch, rows, cols))[0], want)
    assert torch.equal(ctx.rcd_orthogonalize(g.transpose(1, 2).contiguous().transpose(1, 2)), want)
    wide = torch.zeros(batch, rows + 2, cols + 11, device="cuda", dtype=torch.bfloat16)
    wide[:, 1:-1, 3:cols + 3] = g
    assert torch.equal(ctx.rcd_orthogonalize(wide[:, 1:-1, 3:cols + 3]), want)
    for off, more in ((3, 16), (8, 16 + -cols % 8), (8, 11)):
        buf = torch.full((batch, rows + 2, cols + more), 7.0, device="cuda", dtype=torch.bfloat16)
        view = buf[:, 1:-1, off:cols + off]
        assert ctx.rcd_orthogonalize(g, out=view) is view
        assert torch.equal(view, want)
        view[:] = 7
        assert bool((buf == 7).all())
    if batch > 1:
        assert torch.equal(ctx.rcd_orthogonalize(g[::batch - 1]), ctx.rcd_orthogonalize(g[::batch - 1].contiguous()))
    ctx.sync_status()


@pytest.mark.parametrize("rows,cols,form", [(96, 1500, CLUSTER), (200, 330, STEPS), (512, 1100, STEPS), (1500, 1100, LAUNCHES)])
def test_captured_and_on_another_stream(rcd, ctx, rows, cols, form):
    import torch
    a, b = (gradient(seeded("graph", i), 2, rows, cols, torch.bfloat16) for i in range(2))
    want = [ctx.rcd_orthogonalize(a), ctx.rcd_orthogonalize(b)]
    assert taken(ctx, 5) == form
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
