"""A residual whose rows TMA can reach beside an output whose rows it cannot, and the other way round: both go through one place in
shared memory."""
import pytest

from test_gpu_linear import rounded, whole
from test_gpu_norm import ctx, kind, rcd, seeded  # noqa: F401  (fixtures)

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("m,n,k", [(300, 520, 72), (700, 1032, 136), (5000, 512, 256), (20000, 520, 128), (12000, 1288, 64)])
@pytest.mark.parametrize("dtype,out", [("bf16", "bf16"), ("fp16", "fp32"), ("int8", "bf16"), ("int8", "fp32")])
@pytest.mark.parametrize("y_pad,r_pad", [(3, 0), (0, 3), (3, 8), (8, 8)])
@pytest.mark.parametrize("preact", [False, True])
def test_residual_and_output_of_unlike_rows(ctx, m, n, k, dtype, out, y_pad, r_pad, preact):
    import torch
    t, o, g = kind(dtype), kind(out), seeded(m, n, k, dtype, out, y_pad, r_pad)
    x, w, r = whole(g, m, k, t), whole(g, n, k, t), whole(g, m, n, o, r_pad, most=60)
    want = x.double() @ w.double().t()
    buf = torch.full((m + 1, n + y_pad), 7.0, device="cuda", dtype=o)
    for _ in range(2):
        y, z = ctx.rcd_linear(x, w, residual=r, out=buf[:m, :n], want_preact=preact)
        ctx.sync_status()
        assert torch.equal(buf[:m, :n], rounded(want + r.double(), o))
        assert z is None if not preact else torch.equal(z, rounded(want, o))
        buf[:m, :n] = 7
        assert bool((buf == 7).all())
