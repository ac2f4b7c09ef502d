"""What the norms and products record about a wait that ran out is reported, whatever call comes after them."""
import pytest

from test_gpu_norm import rcd  # noqa: F401  (fixture)

pytestmark = pytest.mark.gpu


@pytest.fixture()
def ctx(rcd):
    with rcd.Context(0) as c:
        yield c


def expired(rcd, ctx):
    """The waits of the norm's ring and of the product run out (a few thousand polls), as the others' do."""
    with pytest.raises(rcd.RcdError) as e:
        ctx.sync_status()
    assert e.value.status == 5                             # RCD_ERR_TIMEOUT


def calls(rcd, ctx):
    """Calls that may follow an operator, by name."""
    import torch
    x = torch.randn(60, 64, device="cuda").bfloat16()
    y = torch.arange(60, device="cuda", dtype=torch.int32) % 2
    none = torch.empty(0, 64, device="cuda", dtype=torch.bfloat16)
    return {
        "norm": lambda: ctx.rcd_rms_norm(x),
        "norm of many rows": lambda: ctx.rcd_rms_norm(torch.ones(9000, 1024, device="cuda")),
        "norm's gradients": lambda: ctx.rcd_rms_norm_backward(x, x),
        "quantized": lambda: ctx.rcd_quantize_rows(x),
        "product of few rows": lambda: ctx.rcd_linear(x[:4], x),
        "product": lambda: ctx.rcd_linear(x, x),
        "product's gradients": lambda: ctx.rcd_linear_backward(x[:, :60].contiguous(), x, x),
        "bias's gradient": lambda: ctx.rcd_linear_backward(x[:, :60].contiguous(), x, x, want_dx=False, want_dw=False),
        "partition": lambda: ctx.rcd_partition(x, y, [1, 1], 2),
        "partition of rows as they come": lambda: ctx.rcd_partition(x, y, [1, 1], 2, normalize=rcd.RCD_FEAT_I8),
        "objective": lambda: ctx.rcd_objective(x, y, y, 2, 2, normalize=rcd.RCD_FEAT_BF16),
        "similarity": lambda: ctx.rcd_similarity(x),
        "no rows": lambda: (ctx.rcd_rms_norm(none), ctx.rcd_linear(none, x)),
    }


def test_an_expired_wait_outlives_the_calls_behind_it(rcd, ctx):
    for name, call in calls(rcd, ctx).items():
        ctx.selftest_bounded_wait()
        call()
        expired(rcd, ctx)
        call()
        ctx.sync_status()                                  # reported once, and the context goes on


def test_calls_without_rows_report_no_older_error(rcd, ctx):
    import torch
    none = torch.empty(0, 64, device="cuda", dtype=torch.bfloat16)
    w = torch.ones(64, 64, device="cuda", dtype=torch.bfloat16)
    for call in (lambda: ctx.rcd_rms_norm(none), lambda: ctx.rcd_quantize_rows(none), lambda: ctx.rcd_rms_norm_backward(none, none, weight=w[0]),
                 lambda: ctx.rcd_linear(none, w), lambda: ctx.rcd_linear_backward(none, none, w)):
        ctx.selftest_bounded_wait()
        expired(rcd, ctx)
        call()
        ctx.sync_status()


def test_replayed_graphs_leave_other_calls_status_alone(rcd, ctx):
    import torch
    x = torch.randn(300, 64, device="cuda").bfloat16()
    ctx.rcd_linear(x, x)
    ctx.sync_status()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y = ctx.rcd_linear(ctx.rcd_rms_norm(x)[0], x)[0]
    ctx.selftest_bounded_wait()
    graph.replay()
    expired(rcd, ctx)
    graph.replay()
    ctx.rcd_rms_norm(x)
    ctx.sync_status()
    assert torch.equal(y, ctx.rcd_linear(ctx.rcd_rms_norm(x)[0], x)[0])
