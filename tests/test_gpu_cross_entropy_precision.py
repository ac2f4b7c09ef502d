"""What the sums of the logits lose, where it shows: a head's dbias, whose rows nearly cancel, on real values.

Errors are parts of the norm.  Against the lse that the call is given: as good as fp32 products within a factor of two from 1000 classes on (sums of 128 k;
in sums of 512 k it would be four times as much).  Against the loss itself the forward call's lse adds its own, but for up to 256 classes, where p's sum is known."""
import pytest

from test_gpu_norm import ctx, half_step, kind, rcd, seeded  # noqa: F401  (fixtures)

pytestmark = pytest.mark.gpu


def trained(g, m, k, n, dtype):
    """Hidden rows that lean towards their label's weights."""
    import torch
    w = torch.randn(n, k, generator=g, device="cuda") * (2 / k ** 0.5)
    y = torch.randint(0, n, (m,), generator=g, device="cuda", dtype=torch.int32)
    x = torch.randn(m, k, generator=g, device="cuda") + 1.5 * w[y.long()]
    b = 0.5 * torch.randn(n, generator=g, device="cuda")
    dloss = (0.5 + torch.rand(m, generator=g, device="cuda")) / m
    return x.to(dtype), w.to(dtype), y, b, dloss


def dbias_of(z, lse, y, dloss):
    import torch
    dz = torch.exp(z - lse[:, None]) * dloss[:, None]
    dz[torch.arange(len(y), device=y.device), y.long()] -= dloss
    return dz.sum(0)


def off(got, want):
    return float((got.double() - want).norm() / want.norm())


# rows, k, classes, type; dbias from the right lse and from the call's own: what the header states and a quarter more
CASES = [(5000, 2048, 1000, "bf16", 1.25e-6, 5e-6), (1300, 1001, 5003, "fp16", 1.25e-6, 5e-6), (32, 512, 1000, "bf16", 1.25e-6, 5e-6), (50000, 1024, 1000, "bf16", 1.25e-6, 5e-6),
         (20000, 1024, 500, "bf16", 2.5e-6, 6e-6), (12237, 1914, 257, "fp16", 2.5e-6, 6e-6),
         (12237, 1914, 256, "fp16", 1.25e-6, 1.25e-6), (12237, 1914, 97, "fp16", 1.25e-6, 1.25e-6), (20000, 4096, 128, "bf16", 1.25e-6, 1.25e-6), (50000, 512, 10, "bf16", 1.25e-6, 1.25e-6),
         (20000, 2048, 10, "fp16", 1.25e-6, 1.25e-6), (300, 512, 2, "bf16", 1.25e-6, 1.25e-6), (3000, 8192, 30, "bf16", 1.25e-6, 1.25e-6), (40, 700, 200, "fp16", 1.25e-6, 1.25e-6)]


@pytest.mark.parametrize("m,k,n,dtype,given,own", CASES)
def test_dbias(rcd, ctx, m, k, n, dtype, given, own):
    import torch
    x, w, y, b, dloss = trained(seeded("precision", m, n, dtype), m, k, n, kind(dtype))
    z = x.double() @ w.double().t() + b.double()
    lse = torch.logsumexp(z, 1)
    lse32 = lse.float()
    want = dbias_of(z, lse32.double(), y, dloss.double())
    _, _, db = ctx.rcd_linear_cross_entropy_backward(x, w, y, lse32, bias=b, dloss=dloss)
    products = off(dbias_of(x.float() @ w.float().t() + b, lse32, y, dloss), want)
    assert off(db, want) <= given, (off(db, want), products)
    if n >= 1000 and m < 50000:
        assert off(db, want) <= 2 * products, (off(db, want), products)
    _, mine = ctx.rcd_linear_cross_entropy(x, w, y, bias=b)
    _, _, db = ctx.rcd_linear_cross_entropy_backward(x, w, y, mine, bias=b, dloss=dloss)
    assert off(db, dbias_of(z, lse, y, dloss.double())) <= own
    ctx.sync_status()


@pytest.mark.parametrize("m,k,n,dtype", [(700, 512, 10, "bf16"), (5000, 1024, 100, "fp16"), (40, 64, 250, "bf16"), (300, 200, 1, "bf16")])
@pytest.mark.parametrize("more", [2.0 ** -7, 0.25, 3.0, -0.5])
@pytest.mark.parametrize("bias", [True, False])
def test_lse_of_more_classes_than_these(rcd, ctx, m, k, n, dtype, more, bias):
    """An lse that takes in classes elsewhere (or any other): p stays exp(z - lse), whose sum is not one."""
    import torch
    x, w, y, b, dloss = trained(seeded("more", m, n, dtype), m, k, n, kind(dtype))
    b = b if bias else None
    z = x.double() @ w.double().t() + (0 if b is None else b.double())
    lse = (torch.logsumexp(z, 1) + more).float()
    _, _, db = ctx.rcd_linear_cross_entropy_backward(x, w, y, lse, bias=b, dloss=dloss)
    want = dbias_of(z, lse.double(), y, dloss.double())
    # (p as a whole is far from one, nothing cancels: 2e-5 of the sums of sizes is far more than sums of up to 1024 k lose, and a twentieth of the least that taking p's sum out would change)
    p = torch.exp(z - lse.double()[:, None])
    sizes = (p * dloss.double()[:, None]).sum(0) + torch.zeros(n, device="cuda", dtype=torch.float64).index_add_(0, y.long(), dloss.double())
    assert float(((db.double() - want).abs() - 2e-5 * sizes).max()) <= 0
    ctx.sync_status()


@pytest.mark.parametrize("m,k,n,dtype", [(700, 4096, 600, "fp16"), (500, 1914, 97, "bf16"), (300, 8192, 1000, "fp16")])
def test_gradients_with_and_without_dbias(rcd, ctx, m, k, n, dtype):
    """Logits are added up otherwise where dbias is wanted, so that dx and dw may round another way: each is as far off as dz's own rounding makes it, and no further."""
    import torch
    t = kind(dtype)
    x, w, y, b, dloss = trained(seeded("with", m, n, dtype), m, k, n, t)
    dloss = dloss * 256
    _, lse = ctx.rcd_linear_cross_entropy(x, w, y, bias=b)
    z = x.double() @ w.double().t() + b.double()
    dz = torch.exp(z - lse.double()[:, None]) * dloss.double()[:, None]
    dz[torch.arange(m, device="cuda"), y.long()] -= dloss.double()
    # (fp16's power of two brings the largest of dloss to 2^13..2^14)
    up = 2.0 ** (13 - int(torch.floor(torch.log2(dloss.max().double())))) if dtype == "fp16" else 1.0
    rounded = (dz * up).to(t).double() / up
    dw64, dx64 = dz.t() @ x.double(), dz @ w.double()
    for dbias in (True, False):
        dx, dw, _ = ctx.rcd_linear_cross_entropy_backward(x, w, y, lse, bias=b, dloss=dloss, want_dbias=dbias, dw_dtype=torch.float32)
        # a twentieth for logits in one sum of up to 4096 k and the products' own sums
        assert off(dw, dw64) <= 1.05 * off(rounded.t() @ x.double(), dw64)
        assert off(dx, dx64) <= 1.05 * off((rounded @ w.double()).to(t), dx64)
    ctx.sync_status()
