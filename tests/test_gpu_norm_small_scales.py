"""int8 with a scale per row for rows so small that 127 divided by their largest value is not a number of fp32."""
import pytest

from test_gpu_norm import ctx, kind, rcd, rows, seeded  # noqa: F401  (fixtures)

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("n,d", [(5, 512), (3, 77), (4300, 1024), (13000, 512)])          # a row per group, and through the ring
@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("size", [1e-28, 2.0 ** -100, 1e-33, 3e-37, 1e-38, 1e-40])
def test_quantized(ctx, n, d, dtype, size):
    """The integers are those of the same rows at size 1 (a row times a power of two, but for the roundings of the input at the lower end of its
    range): half a step, and the two roundings of 127 / a and its product.  A scale is off by half a unit, 2^-150 below the normal range."""
    import torch
    g = seeded(n, d, dtype, size)
    x = rows(g, n, d, kind(dtype), size=size)
    x[1] = 0
    for q, s in (ctx.rcd_quantize_rows(x), ctx.rcd_rms_norm(x, eps=1.0, out_dtype=torch.int8)[:2]):
        ctx.sync_status()
        a = x.double().abs().amax(1)
        exact = torch.where(a > 0, 127 / a, torch.zeros_like(a))[:, None] * x.double()
        assert float((q.double() - exact).abs().max()) <= 0.5 + 127 * 2.0 ** -22
        assert bool((q.abs().amax(1)[a > 0] == 127).all()) and not q[1].any() and float(s[1]) == 0
        assert bool(((s.double() - a / 127).abs() <= a / 127 * 2.0 ** -21 + 2.0 ** -150 * 2).all())
