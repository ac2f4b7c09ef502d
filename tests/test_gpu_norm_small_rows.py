"""Gradients of the norm for rows whose squares lie at the lower end of fp32, without eps."""
import pytest

from test_gpu_norm import STEPS, check, ctx, gradients, kind, rcd, rows, seeded  # noqa: F401  (fixtures)

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("n,d", [(5, 512), (3, 77), (2, 8200), (2400, 1024), (180, 8192)])        # a row per group, and through the ring
@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("rms", [1e-18, 3e-20, 1e-20, 1e-21])
@pytest.mark.parametrize("weight,dsum", [(True, False), (False, True)])
def test_gradients_of_small_rows(ctx, n, d, dtype, rms, weight, dsum):
    """1 / rms is a number of fp32, its square is not.  A square below the normal range is off by 2^-150 at most, and so is the mean of
    them once more by its division: `lost` of mean(h^2), half of it in rstd and three halves in rstd^3."""
    import torch
    t, g = kind(dtype), seeded(n, d, dtype, rms)
    h, dy = rows(g, n, d, t, size=rms), rows(g, n, d, t)
    dy[n // 2] = 0                                          # mean(g h) is 0 there
    w = torch.randn(d, generator=g, device="cuda") if weight else None
    s = rows(g, n, d, t, size=1.0 / rms) if dsum else None
    dx, dw = ctx.rcd_rms_norm_backward(dy, h, weight=w, eps=0.0, dsum=s)
    ctx.sync_status()
    want, want_dw = gradients(dy, h, w, 0.0, s)
    hd, gd = h.double(), dy.double() if w is None else dy.double() * w.double()
    v = hd.square().mean(1, keepdim=True)
    lost = 2.0 ** -149 / v
    parts = (gd.abs() + hd.abs() / v * (gd * hd).abs().mean(1, keepdim=True)) / v.sqrt()
    check(dx, want, t, slack=parts * (STEPS + 2 * lost) + (0 if s is None else s.double().abs() * STEPS))
    if weight:
        terms = (dy.double() * hd).abs() / v.sqrt()
        assert bool(((dw.double() - want_dw).abs() <= (terms * ((n + 64) * 2.0 ** -24 + lost)).sum(0)).all())
