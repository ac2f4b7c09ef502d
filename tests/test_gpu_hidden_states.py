"""Hidden states to a partition: norm, int8 projection, norm to features, partition and objective, as they are used together."""
import numpy as np
import pytest

from test_gpu_norm import ctx, rcd, rows, seeded, steps_of  # noqa: F401  (fixtures)

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def orc():
    from oracle import rcd_oracle
    return rcd_oracle


def hidden_states(seed, L, M, d, dtype):
    """L classes of M rows around a few centres each, and their labels, interleaved."""
    import torch
    g = seeded("hidden", seed, L, M, d)
    centres = torch.randn(L, 4, d, generator=g, device="cuda") * 3
    which = torch.randint(0, 4, (L, M), generator=g, device="cuda")
    x = torch.gather(centres, 1, which[:, :, None].expand(L, M, d)) + torch.randn(L, M, d, generator=g, device="cuda")
    order = torch.randperm(L * M, generator=g, device="cuda")
    labels = torch.arange(L, device="cuda", dtype=torch.int32).repeat_interleave(M)[order].contiguous()
    return x.reshape(L * M, d)[order].to(dtype).contiguous(), labels


@pytest.mark.parametrize("dtype,L,M,d,W", [("bf16", 3, 150, 256, [1, 1, 2]), ("fp32", 2, 90, 100, [1, 3]), ("fp16", 4, 40, 77, [2, 1, 1, 4])])
def test_partition_of_rows_as_they_come(rcd, ctx, orc, dtype, L, M, d, W):
    """int8 features: the integers are the stepwise arithmetic's, and the partition of them the oracle's, pick by pick."""
    import torch
    x, y = hidden_states(1, L, M, d, {"bf16": torch.bfloat16, "fp32": torch.float32, "fp16": torch.float16}[dtype])
    want = steps_of(x, None, None, 0.0, rcd.RCD_FEATURE_SCALE)
    assert torch.equal(ctx.features(x, rcd.RCD_FEAT_I8), want)
    a, order, values = ctx.rcd_partition(x, y, W, L, normalize=rcd.RCD_FEAT_I8)
    ctx.sync_status()
    ref = orc.partition(want.cpu().numpy(), y.cpu().numpy(), W, L, variant="incremental")
    assert np.array_equal(a.cpu().numpy(), ref.assignment) and np.array_equal(order.cpu().numpy(), ref.order)
    assert np.array_equal(values.cpu().numpy(), ref.part_values)
    values2, total = ctx.rcd_objective(x, y, a, len(W), L, normalize=rcd.RCD_FEAT_I8)
    assert torch.equal(values2, values) and int(total) == int(values.sum())
    # what is passed as features stays what it was
    a2, _, _ = ctx.rcd_partition(want, y, W, L)
    assert torch.equal(a, a2)


def test_unit_rows(rcd, ctx):
    """bf16 features: rows of length 1, a row of zeros left alone; entries are rounded once, half a step each."""
    import torch
    x, y = hidden_states(2, 2, 60, 130, torch.float32)
    x[5] = 0
    f = ctx.features(x, rcd.RCD_FEAT_BF16)
    want = x.double() / x.double().norm(dim=1, keepdim=True).clamp(min=1e-300)
    assert f.dtype == torch.bfloat16 and not f[5].any()
    assert bool(((f.double() - want).abs() <= want.abs() * (2.0 ** -8 + 2.0 ** -17)).all())
    a, _, _ = ctx.rcd_partition(x, y, [1, 1], 2, normalize=rcd.RCD_FEAT_BF16)
    b, _, _ = ctx.rcd_partition(f, y, [1, 1], 2)
    ctx.sync_status()
    assert torch.equal(a, b)
    with pytest.raises(ValueError):
        ctx.features(x, 7)
    with pytest.raises(TypeError):
        ctx.rcd_partition(x, y, [1, 1], 2)                # rows as they come, without being asked to


def test_from_hidden_states_to_a_partition(rcd, ctx, orc):
    """norm with residual to int8 -> int8 projection with scales, bias, activation -> norm to int8 features -> partition, and back through
    the bf16 projection's and the norm's gradients; the whole also as one captured graph up to the features."""
    import torch
    L, M, d, n = 3, 120, 512, 128
    x, y = hidden_states(3, L, M, d, torch.bfloat16)
    g = seeded("chain")
    r, w = rows(g, L * M, d, torch.bfloat16), torch.randn(n, d, generator=g, device="cuda").bfloat16() * d ** -0.5
    nw, b = 1 + 0.1 * torch.randn(d, generator=g, device="cuda"), 0.1 * torch.randn(n, generator=g, device="cuda")
    wq, ws = ctx.rcd_quantize_rows(w)

    def chain():
        q, s, h = ctx.rcd_rms_norm(x, residual=r, weight=nw, out_dtype=torch.int8, want_sum=True)
        z, _ = ctx.rcd_linear(q, wq, bias=b, activation=rcd.RCD_ACT_GELU, x_scales=s, w_scales=ws)
        return q, s, h, z, ctx.features(z, rcd.RCD_FEAT_I8)

    q, s, h, z, f = chain()
    # the 8-bit projection stands for the exact one on the values that the integers stand for: bf16's half step and the
    # epilogue's few fp32 steps around it
    exact = (q.double() * s.double()[:, None]) @ (wq.double() * ws.double()[:, None]).t() + b.double()
    exact = exact * torch.special.ndtr(exact)
    assert bool(((z.double() - exact).abs() <= exact.abs() * 2.0 ** -8 + 2.0 ** -18 * (1 + exact.abs())).all())
    assert torch.equal(f, steps_of(z, None, None, 0.0, rcd.RCD_FEATURE_SCALE))
    a, order, values = ctx.rcd_partition(f, y, [1, 2, 1], L)
    ctx.sync_status()
    ref = orc.partition(f.cpu().numpy(), y.cpu().numpy(), [1, 2, 1], L, variant="incremental")
    assert np.array_equal(a.cpu().numpy(), ref.assignment) and np.array_equal(values.cpu().numpy(), ref.part_values)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        outs = chain()
    x.copy_(hidden_states(4, L, M, d, torch.bfloat16)[0])
    graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(p, o) for p, o in zip(outs, chain()))

    # training the projection: gradients of sum(c * act(norm(h) w^T + b)) against autograd in 64 bits on the same rounded values
    hh, c = outs[2], rows(g, L * M, n, torch.bfloat16)
    t, _, _ = ctx.rcd_rms_norm(hh, weight=nw)
    _, pre = ctx.rcd_linear(t, w, bias=b, activation=rcd.RCD_ACT_SILU, want_preact=True)
    dt, dw, db = ctx.rcd_linear_backward(c, t, w, preact=pre, activation=rcd.RCD_ACT_SILU)
    dh, dnw = ctx.rcd_rms_norm_backward(dt, hh, weight=nw)
    h64, nw64, w64, b64 = (v.double().requires_grad_() for v in (hh, nw, w, b))
    t64 = h64 / (h64.square().mean(1, keepdim=True) + 1e-6).sqrt() * nw64
    loss = (torch.nn.functional.silu(t64 @ w64.t() + b64) * c.double()).sum()
    loss.backward()
    for got, want in ((dh, h64.grad), (dnw, nw64.grad), (dw, w64.grad), (db, b64.grad)):
        # t, pre, dz, dt and the result are rounded to bf16 (2^-8 each, of independent signs over hundreds of terms): 2 % of the norm is
        # five of them added up without any cancelling
        assert float((got.double() - want).norm() / want.norm()) <= 5 * 2.0 ** -8


def test_a_rank_normalises_its_own_classes(rcd, ctx):
    import torch
    from paper_2211_00839_b200 import distributed
    x, y = hidden_states(5, 3, 50, 64, torch.bfloat16)
    a = distributed.partition_sharded_gpu(ctx, x, y, [1, 2], 3, normalize=rcd.RCD_FEAT_I8)
    b, _, _ = ctx.rcd_partition(x, y, [1, 2], 3, normalize=rcd.RCD_FEAT_I8)
    ctx.sync_status()
    assert torch.equal(a, b)
