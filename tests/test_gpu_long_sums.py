"""Sums over a long k axis of values of one sign.  The tensor cores cut an fp32 sum off towards zero at every step of 16 k, so that one long
sum ends below the true one, by up to 6.5e-9 of it per product."""
import pytest

from test_gpu_norm import ctx, half_step, rcd, seeded  # noqa: F401  (fixtures)

pytestmark = pytest.mark.gpu


def positive(g, n, d, dtype, size=1.0):
    import torch
    return ((0.5 + torch.rand(n, d, generator=g, device="cuda", dtype=torch.float32 if n * d < 1 << 28 else dtype)) * size).to(dtype)


def chunk_error(k):
    """Chunks of 512 k: up to 33 steps of 16 products that cut off two units (2^-23 of the sum) at most, one from the sum and a sixteenth from each
    product, of a sum that grows to its whole: half of that; and one rounding for each chunk (a half unit), and a few for the pieces' and
    warps' joining."""
    return 33 * 2.0 ** -23 + (k / 512 + 32) * 2.0 ** -24


# few rows; tiles of one SM and of pairs, cut in pieces or whole
@pytest.mark.parametrize("m,n,k", [(1, 512, 16384), (16, 64, 32768), (32, 300, 8192), (40, 64, 65536), (130, 300, 32768), (300, 512, 65536), (3000, 2048, 32768), (2500, 4096, 16384)])
@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
def test_fp32_outputs(ctx, m, n, k, dtype):
    import torch
    t, g = {"bf16": torch.bfloat16, "fp16": torch.float16}[dtype], seeded(m, n, k, dtype, "long")
    x, w = positive(g, m, k, t), positive(g, n, k, t)
    at = torch.arange(0, m, max(1, m // 40), device="cuda")
    bt = torch.arange(0, n, max(1, n // 40), device="cuda")
    want = x[at].double() @ w[bt].double().t()
    y, _ = ctx.rcd_linear(x, w, out_dtype=torch.float32)
    ctx.sync_status()
    off = (y[at][:, bt].double() / want - 1).abs()
    assert float(off.max()) <= chunk_error(k), float(off.max())
    # as gradients: sums over the rows
    if dtype == "bf16":
        x, dy = positive(g, k, m, t), positive(g, k, n, t)
        _, dw, db = ctx.rcd_linear_backward(dy, x, torch.zeros(n, m, device="cuda", dtype=t), dw_dtype=torch.float32, want_dx=False)
        ctx.sync_status()
        off = (dw[bt][:, at].double() / (dy[:, bt].double().t() @ x[:, at].double()) - 1).abs()
        assert float(off.max()) <= chunk_error(k), float(off.max())


@pytest.mark.parametrize("dtype", ["fp16", "bf16"])
@pytest.mark.parametrize("n,k", [(2048, 2048), (2304, 2040), (4096, 1096)])
def test_16_bit_gradients_over_many_rows(ctx, dtype, n, k):
    """Half a step, and a twentieth of fp16's for the sums before it."""
    import torch
    t, g, rows = {"bf16": torch.bfloat16, "fp16": torch.float16}[dtype], seeded(n, k, dtype, "many"), 600000
    x, dy = positive(g, rows, k, t, 2.0 ** -6), positive(g, rows, n, t, 2.0 ** -6)
    _, dw, _ = ctx.rcd_linear_backward(dy, x, torch.zeros(n, k, device="cuda", dtype=t), want_dx=False, want_dbias=False)
    ctx.sync_status()
    at, bt = torch.arange(0, n, n // 40, device="cuda"), torch.arange(0, k, k // 40, device="cuda")
    want = dy[:, at].double().t() @ x[:, bt].double()
    got = dw[at][:, bt].double()
    assert float(((got - want).abs() / want).max()) <= half_step(t) + 2.0 ** -11 / 20


@pytest.mark.parametrize("dtype", ["fp16", "bf16"])
def test_16_bit_outputs_of_a_long_product(ctx, dtype):
    """The same forward and for dx, whose sums are over the columns."""
    import torch
    t, g, long = {"bf16": torch.bfloat16, "fp16": torch.float16}[dtype], seeded(dtype, "wide"), 600000
    m, n = 2304, 2304
    at = torch.arange(0, m, m // 40, device="cuda")
    x, w = positive(g, m, long, t, 2.0 ** -6), positive(g, n, long, t, 2.0 ** -6)
    want = x[at].double() @ w[at].double().t()
    y, _ = ctx.rcd_linear(x, w)
    ctx.sync_status()
    assert float(((y[at][:, at].double() - want).abs() / want).max()) <= half_step(t) + 2.0 ** -11 / 20
    del w
    wt = positive(g, long, n, t, 2.0 ** -6)                # [n of the product][k]
    dx, _, _ = ctx.rcd_linear_backward(x, torch.zeros(m, n, device="cuda", dtype=t), wt, want_dw=False, want_dbias=False)
    ctx.sync_status()
    want = x[at].double() @ wt[:, at].double()
    assert float(((dx[at][:, at].double() - want).abs() / want).max()) <= half_step(t) + 2.0 ** -11 / 20
