"""Gradients of a head's loss do not depend on what dloss holds for rows that are passed over (a label below 0, or of n or more), nor do rows on an
infinity in another row."""
import pytest

from test_gpu_cross_entropy import head
from test_gpu_norm import ctx, kind, rcd, seeded  # noqa: F401  (fixtures)

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["fp16", "bf16"])
@pytest.mark.parametrize("value", [1e30, 3e38, float("inf"), float("nan")])
@pytest.mark.parametrize("m,n,k,piece", [(300, 500, 64, 0), (40, 300, 72, 128), (2100, 100, 136, 0)])
@pytest.mark.parametrize("pull", [False, True])
def test_dloss_of_rows_passed_over(rcd, ctx, m, n, k, piece, dtype, value, pull):
    import torch
    g = seeded("passed over", m, n, k, dtype)
    x, w, b, y = head(g, m, n, k, kind(dtype))
    y[0], y[m // 2], y[m - 1] = -1, n, 2 ** 31 - 1
    none = (y < 0) | (y >= n)
    _, lse = ctx.rcd_linear_cross_entropy(x, w, y, bias=b)
    dloss = (0.5 + torch.rand(m, generator=g, device="cuda")) * 2.0 ** -18 / m
    dlse = torch.randn(m, generator=g, device="cuda") * 2.0 ** -20 / m if pull else None
    calls = []
    for there in (0.0, value):
        dloss[none] = there
        calls.append(ctx.rcd_linear_cross_entropy_backward(x, w, y, lse, bias=b, dloss=dloss, dlse=dlse, piece=piece, dw_dtype=torch.float32))
    with pytest.raises(rcd.RcdError) as e:
        ctx.sync_status()                                     # (the labels that are too large)
    assert e.value.status == 1
    # (dx in fp16 is 0 throughout: |dx| <= 2 dloss |w| <= 3 * 2^-18 / m * 2^-4, a tenth of half of that type's smallest step)
    assert bool(calls[0][1].any()) and bool(calls[0][2].any()) and (dtype == "fp16" or bool(calls[0][0].any()))
    assert all(torch.equal(p, q) for p, q in zip(*calls))


@pytest.mark.parametrize("which", ["dloss", "dlse"])
@pytest.mark.parametrize("value", [float("inf"), float("nan")])
def test_what_is_not_finite_stays_in_its_row(rcd, ctx, which, value):
    import torch
    g = seeded("row", which)
    m, n, k = 300, 500, 64
    x, w, b, y = head(g, m, n, k, torch.float16)
    y = y.clamp(min=0)
    _, lse = ctx.rcd_linear_cross_entropy(x, w, y, bias=b)
    small = {name: (0.5 + torch.rand(m, generator=g, device="cuda")) * 2.0 ** -10 / m for name in ("dloss", "dlse")}
    dx, _, _ = ctx.rcd_linear_cross_entropy_backward(x, w, y, lse, bias=b, **small)
    bad = {name: t.clone() for name, t in small.items()}
    at = int((small["dloss"] + small["dlse"]).argmin())
    bad[which][at] = value
    got, _, _ = ctx.rcd_linear_cross_entropy_backward(x, w, y, lse, bias=b, **bad)
    ctx.sync_status()
    others = torch.arange(m, device="cuda") != at
    assert torch.equal(got[others], dx[others])
    assert not torch.isfinite(got[at]).all()
