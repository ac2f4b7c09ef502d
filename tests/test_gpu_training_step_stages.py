"""Every operator of a training step against 64 bits of what the one before handed it: bounds of each one's own roundings, not of the whole chain's.

A rounding to 16 bits is off by anything up to half a step, 1 / sqrt(3) = 0.58 of that on the root mean square where values stand at the foot of their binade (where a step is the
largest part of them; 0.43 over a whole one): below 0.6 of half a step.  Two independent ones: sqrt(2) times 0.58 = 0.82, below 0.83.  (The gradients of the labels' logits are nearly
-dloss, so that they may all stand there: a bound of two thirds, reckoned over whole binades, was too low for that.)"""
import pytest

from test_gpu_norm import ctx, rcd, rows, seeded  # noqa: F401  (fixtures)

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("m,d,n,classes,dtype,piece", [(300, 512, 128, 10, "bf16", 0), (257, 200, 96, 1000, "fp16", 256), (64, 1024, 256, 5003, "bf16", 0), (2000, 768, 512, 250, "fp16", 0)])
def test_stages(rcd, ctx, m, d, n, classes, dtype, piece):
    import torch
    t = {"bf16": torch.bfloat16, "fp16": torch.float16}[dtype]
    half = torch.finfo(t).eps / 2
    g = seeded("stages", m, d, n, classes)
    x, nw = rows(g, m, d, t), 1 + 0.1 * torch.randn(d, generator=g, device="cuda")
    w, v = rows(g, n, d, t, size=d ** -0.5), rows(g, classes, n, t, size=2 * n ** -0.5)
    b = 0.1 * torch.randn(classes, generator=g, device="cuda")
    y = torch.randint(0, classes, (m,), generator=g, device="cuda", dtype=torch.int32)
    y[::9] = -1
    weight = torch.full((m,), 256.0 / int((y >= 0).sum()), device="cuda")
    h, _, _ = ctx.rcd_rms_norm(x, weight=nw)
    f, pre = ctx.rcd_linear(h, w, activation=rcd.RCD_ACT_SILU, want_preact=True)
    loss, lse = ctx.rcd_linear_cross_entropy(f, v, y, bias=b)
    dlse = lse * weight * 2e-2
    df, dv, db = ctx.rcd_linear_cross_entropy_backward(f, v, y, lse, bias=b, dloss=weight, dlse=dlse, piece=piece)
    dh, dw, _ = ctx.rcd_linear_backward(df, h, w, preact=pre, activation=rcd.RCD_ACT_SILU, want_dbias=False)
    dx, dnw = ctx.rcd_rms_norm_backward(dh, x, weight=nw)
    ctx.sync_status()

    def near(name, got, want, bound):
        off = float((got.double() - want).norm() / want.norm())
        assert off <= bound, (name, off, bound)
    x64, nw64 = x.double().requires_grad_(), nw.double().requires_grad_()
    h64 = x64 / (x64.square().mean(1, keepdim=True) + 1e-6).sqrt() * nw64
    near("h", h, h64.detach(), 0.6 * half)
    z = h.double() @ w.double().t()
    near("pre", pre, z, 0.6 * half)
    near("f", f, torch.nn.functional.silu(z), 0.6 * half)
    # (fp32: what the logits' sums lose, which is below 1e-6 of the logits)
    z = f.double() @ v.double().t() + b.double()
    want = torch.logsumexp(z, 1)
    near("lse", lse, want, 2e-6)
    near("loss", loss, torch.where(y < 0, torch.zeros_like(want), want - z.gather(1, y.long().clamp(min=0)[:, None])[:, 0]), 2e-6)
    counts = torch.where(y < 0, torch.zeros_like(want), weight.double())
    dz = torch.exp(z - lse.double()[:, None]) * (counts + dlse.double())[:, None]
    dz[torch.arange(m, device="cuda"), y.long().clamp(min=0)] -= counts
    near("db", db, dz.sum(0), 5e-6)
    near("df", df, dz @ v.double(), 0.83 * half)
    near("dv", dv, dz.t() @ f.double(), 0.83 * half)
    p64 = pre.double().requires_grad_()
    torch.nn.functional.silu(p64).backward(df.double())
    near("dh", dh, p64.grad @ w.double(), 0.83 * half)
    near("dw", dw, p64.grad.t() @ h.double(), 0.83 * half)
    h64.backward(dh.double())
    near("dx", dx, x64.grad, 0.6 * half)
    near("dnw", dnw, nw64.grad, 1e-5)
