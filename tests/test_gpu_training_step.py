"""A training step of a projection and a head, as the operators are used together: norm -> projection -> cross entropy, back through all of them, and the
projection's gradient orthogonalised."""
import pytest

from test_gpu_norm import ctx, rcd, rows, seeded  # noqa: F401  (fixtures)
from test_gpu_orthogonalize import newton_schulz

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("m,d,n,classes,dtype,piece", [(300, 512, 128, 10, "bf16", 0), (257, 200, 96, 1000, "fp16", 256), (64, 1024, 256, 5003, "bf16", 0)])
def test_step(rcd, ctx, m, d, n, classes, dtype, piece):
    import torch
    t = {"bf16": torch.bfloat16, "fp16": torch.float16}[dtype]
    g = seeded("step", m, d, n, classes)
    x, nw = rows(g, m, d, t), 1 + 0.1 * torch.randn(d, generator=g, device="cuda")
    w, v = rows(g, n, d, t, size=d ** -0.5), rows(g, classes, n, t, size=2 * n ** -0.5)
    b = 0.1 * torch.randn(classes, generator=g, device="cuda")
    y = torch.randint(0, classes, (m,), generator=g, device="cuda", dtype=torch.int32)
    y[::9] = -1
    # the mean over the rows that count, and a small pull on lse
    weight = torch.full((m,), 1.0 / int((y >= 0).sum()), device="cuda")

    def step():
        h, _, _ = ctx.rcd_rms_norm(x, weight=nw)
        f, pre = ctx.rcd_linear(h, w, activation=rcd.RCD_ACT_SILU, want_preact=True)
        loss, lse = ctx.rcd_linear_cross_entropy(f, v, y, bias=b)
        df, dv, db = ctx.rcd_linear_cross_entropy_backward(f, v, y, lse, bias=b, dloss=weight * 256, dlse=lse * weight * 2e-2 * 256, piece=piece)
        dh, dw, _ = ctx.rcd_linear_backward(df, h, w, preact=pre, activation=rcd.RCD_ACT_SILU, want_dbias=False)
        dx, dnw = ctx.rcd_rms_norm_backward(dh, x, weight=nw)
        return loss, lse, dv, db, dw, dx, dnw, ctx.rcd_orthogonalize(dw)

    out = step()
    ctx.sync_status()
    loss, lse, dv, db, dw, dx, dnw, o = out
    x64, nw64, w64, v64, b64 = (p.double().requires_grad_() for p in (x, nw, w, v, b))
    f64 = torch.nn.functional.silu(x64 / (x64.square().mean(1, keepdim=True) + 1e-6).sqrt() * nw64 @ w64.t())
    z64 = f64 @ v64.t() + b64
    lse64 = torch.logsumexp(z64, 1)
    loss64 = torch.where(y < 0, torch.zeros_like(lse64), lse64 - z64.gather(1, y.long().clamp(min=0)[:, None])[:, 0])
    ((loss64 + 1e-2 * lse64.square()) * weight).sum().backward()
    # h, f, pre, dz, df, dh and the result are rounded to 16 bits (half a step each): seven of them added up without any cancelling
    half = torch.finfo(t).eps / 2
    for name, got, want in (("loss", loss, loss64.detach()), ("lse", lse, lse64.detach()), ("dv", dv, v64.grad * 256), ("db", db, b64.grad * 256), ("dw", dw, w64.grad * 256), ("dx", dx, x64.grad * 256),
                            ("dnw", dnw, nw64.grad * 256)):
        assert float((got.double() - want).norm() / want.norm()) <= 7 * half, name
    want, err = newton_schulz(dw)
    assert float((o.double() - want).norm()) <= 1.05 * err + 2.0 ** -8 * 1.01 * float(want.norm())
    # the whole step captured, and replayed with other inputs in place
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        outs = step()
    x.copy_(rows(g, m, d, t))
    graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(p, q) for p, q in zip(outs, step()))
    ctx.sync_status()


def test_logits_beyond_32_bits(rcd, ctx):
    """66 000 rows by 33 000 classes, whose gradients of logits (2.2e9) are in memory at once: the last rows and classes are right."""
    import torch
    g = seeded("large")
    m, n, k = 66000, 33000, 64
    x, w = rows(g, m, k, torch.bfloat16), rows(g, n, k, torch.bfloat16, size=0.25)
    y = torch.randint(0, n, (m,), generator=g, device="cuda", dtype=torch.int32)
    loss, lse = ctx.rcd_linear_cross_entropy(x, w, y)
    dx, dw, _ = ctx.rcd_linear_cross_entropy_backward(x, w, y, lse, dloss=torch.full((m,), 1.0, device="cuda"), want_dbias=False, piece=n)
    ctx.sync_status()
    for at in (slice(0, 40), slice(m - 40, m)):
        z = x[at].double() @ w.double().t()
        want = torch.logsumexp(z, 1)
        assert float((lse[at].double() - want).abs().max()) < 1e-4
        p = torch.exp(z - want[:, None])
        p[torch.arange(40, device="cuda"), y[at].long()] -= 1
        dx64 = p @ w.double()
        assert float((dx[at].double() - dx64).norm() / dx64.norm()) < 3 * 2.0 ** -8
    for at in (slice(0, 40), slice(n - 40, n)):
        p = torch.exp(x.double() @ w[at].double().t() - lse.double()[:, None])
        p -= (y.long()[:, None] == torch.arange(at.start, at.stop, device="cuda")).double()
        dw64 = p.t() @ x.double()
        assert float((dw[at].double() - dw64).norm() / dw64.norm()) < 3 * 2.0 ** -8


def test_launches_behind_copies_fills_and_other_streams(rcd, ctx):
    """Kernels that may overtake the end of the one before them, behind what is no kernel: copies and fills, in a captured graph and outside; and behind another stream's
    work that an event brings in."""
    import torch
    g = seeded("behind")
    m, n, k = 300, 700, 128
    x, w = rows(g, m, k, torch.bfloat16), rows(g, n, k, torch.bfloat16, size=0.2)
    y = torch.randint(0, n, (m,), generator=g, device="cuda", dtype=torch.int32)
    wide = rows(g, 96, 700, torch.bfloat16)
    want, want_lse = ctx.rcd_linear_cross_entropy(x, w, y)
    o = ctx.rcd_orthogonalize(wide)
    fx, fw, fy, fg = torch.empty_like(x), torch.empty_like(w), torch.empty_like(y), torch.empty_like(wide)
    side = torch.cuda.Stream()

    def run():
        fx.zero_()
        fx.copy_(x)
        fg.copy_(wide)
        # another stream's part
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            fw.copy_(w)
            fy.copy_(y)
            z, _ = ctx.rcd_linear(fx, fw)
        torch.cuda.current_stream().wait_stream(side)
        loss, lse = ctx.rcd_linear_cross_entropy(fx, fw, fy)
        fx.fill_(float("nan"))
        o2 = ctx.rcd_orthogonalize(fg)
        fg.zero_()
        fw.zero_()
        return z, loss, lse, o2
    z = ctx.rcd_linear(x, w)[0]
    for _ in range(3):
        assert all(torch.equal(p, q) for p, q in zip(run(), (z, want, want_lse, o)))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = run()
    for _ in range(3):
        for t in out:
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(p, q) for p, q in zip(out, (z, want, want_lse, o)))
    ctx.sync_status()


def test_two_streams_at_once(rcd, ctx):
    """Updates of the form that holds all SMs (its CTAs wait for one another), updates by clusters and products, enqueued on two streams without any order between them."""
    import torch
    g = seeded("two")
    a, b, c = (torch.randn(*s, generator=g, device="cuda").bfloat16() for s in ((512, 1100), (700, 300), (128, 1500)))
    x, w = rows(g, 2000, 512, torch.bfloat16), rows(g, 1500, 512, torch.bfloat16, size=0.05)
    y = torch.randint(0, 1500, (2000,), generator=g, device="cuda", dtype=torch.int32)

    def work():
        loss, lse = ctx.rcd_linear_cross_entropy(x, w, y)
        return [ctx.rcd_orthogonalize(a), loss, ctx.rcd_orthogonalize(b), ctx.rcd_orthogonalize(c), *ctx.rcd_linear_cross_entropy_backward(x, w, y, lse)]
    want = work()
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    got = []
    for _ in range(10):
        for s in streams:
            with torch.cuda.stream(s):
                got.append(work())
    torch.cuda.synchronize()
    ctx.sync_status()
    assert all(torch.equal(p, q) for each in got for p, q in zip(each, want))
