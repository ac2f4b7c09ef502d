"""Column slices of one buffer, side by side: an output may be the neighbour of another argument, but share nothing with it."""
import pytest

from test_gpu_linear import whole
from test_gpu_norm import ctx, rcd, rows, seeded  # noqa: F401  (fixtures)

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("n,d,gap", [(5, 64, 0), (300, 96, 8), (9000, 512, 0), (40, 77, 0), (1, 64, 0)])
def test_norm(rcd, ctx, n, d, gap):
    import torch
    g = seeded("joint", n, d)
    joint = rows(g, n, 4 * (d + gap), torch.bfloat16)
    part = lambda k: joint[:, k * (d + gap):k * (d + gap) + d]  # noqa: E731
    w = torch.randn(d, generator=g, device="cuda")
    before = joint.clone()
    want, _, total = ctx.rcd_rms_norm(part(0).clone(), residual=part(2).clone(), weight=w, want_sum=True)
    ctx.rcd_rms_norm(part(0), residual=part(2), weight=w, out=part(1), sum_out=part(3))
    ctx.sync_status()
    assert torch.equal(part(1), want) and torch.equal(part(3), total)
    for k in (1, 3):
        part(k).copy_(before[:, k * (d + gap):k * (d + gap) + d])
    assert torch.equal(joint, before)                      # and nothing else was written
    if n > 1 and gap == 0:
        with pytest.raises(rcd.RcdError):                  # a column of x
            ctx.rcd_rms_norm(part(0), out=joint[:, d - 1:2 * d - 1])
        with pytest.raises(rcd.RcdError):                  # two outputs that share one
            ctx.rcd_rms_norm(part(0), out=part(2), sum_out=joint[:, 3 * d - 1:4 * d - 1])
        with pytest.raises(rcd.RcdError):                  # the same columns, rows further on
            ctx.rcd_rms_norm(part(0)[1:], out=part(0)[:-1])


@pytest.mark.parametrize("m,n,k", [(3, 64, 64), (300, 64, 96), (700, 260, 136), (40, 33, 77)])
def test_linear(rcd, ctx, m, n, k):
    import torch
    g = seeded("joint", m, n, k)
    joint = whole(g, m, k + 3 * n, torch.bfloat16)
    x, r, y, w = joint[:, :k], joint[:, k:k + n], joint[:, k + n:k + 2 * n], whole(g, n, k, torch.bfloat16)
    before = joint.clone()
    want = ctx.rcd_linear(x.clone(), w, residual=r.clone())[0]
    ctx.rcd_linear(x, w, residual=r, out=y)
    ctx.sync_status()
    assert torch.equal(y, want)
    y.copy_(before[:, k + n:k + 2 * n])
    assert torch.equal(joint, before)
    with pytest.raises(rcd.RcdError):
        ctx.rcd_linear(x, w, residual=r, out=joint[:, k + n - 1:k + 2 * n - 1])
    with pytest.raises(rcd.RcdError):
        ctx.rcd_linear(x, w, out=joint[:, k - 1:k + n - 1])
