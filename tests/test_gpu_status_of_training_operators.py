"""What an expired wait has recorded is reported, whichever call of the training operators comes after it, and none of them reports an older error."""
import pytest

from test_gpu_norm import rcd  # noqa: F401  (fixture)
from test_gpu_status_of_operators import ctx, expired  # noqa: F401  (fixture)

pytestmark = pytest.mark.gpu


def calls(ctx):
    import torch
    x = torch.randn(60, 64, device="cuda").bfloat16()
    y = torch.arange(60, device="cuda", dtype=torch.int32)
    lse = torch.full((60,), 5.0, device="cuda")
    none = torch.empty(0, 64, device="cuda", dtype=torch.bfloat16)
    wide = torch.randn(300, 430, device="cuda").bfloat16()
    large = torch.randn(1500, 1100, device="cuda").bfloat16()
    many = torch.randn(700, 64, device="cuda").bfloat16()
    return {
        "loss": lambda: ctx.rcd_linear_cross_entropy(x, x, y),
        "loss with a join": lambda: ctx.rcd_linear_cross_entropy(x, many, y),
        "its gradients": lambda: ctx.rcd_linear_cross_entropy_backward(x, x, y, lse),
        "its gradients in pieces": lambda: ctx.rcd_linear_cross_entropy_backward(x.half(), many.half(), y, lse, piece=128),
        "update by a CTA": lambda: ctx.rcd_orthogonalize(x),
        "update by a cluster": lambda: ctx.rcd_orthogonalize(torch.ones(64, 1000, device="cuda")),
        "update, all steps in one launch": lambda: ctx.rcd_orthogonalize(wide),
        "update in launches of their own": lambda: ctx.rcd_orthogonalize(large),
        "no rows": lambda: (ctx.rcd_linear_cross_entropy(none, x, y[:0]), ctx.rcd_linear_cross_entropy_backward(none, x, y[:0], lse[:0]), ctx.rcd_orthogonalize(none)),
    }


def test_an_expired_wait_outlives_the_calls_behind_it(rcd, ctx):
    for name, call in calls(ctx).items():
        call()
        ctx.sync_status()
        ctx.selftest_bounded_wait()
        call()
        expired(rcd, ctx)
        call()
        ctx.sync_status()                                  # reported once, and the context goes on


def test_replayed_graphs_leave_other_calls_status_alone(rcd, ctx):
    import torch
    for name, call in calls(ctx).items():
        call()
        ctx.sync_status()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            call()
        ctx.selftest_bounded_wait()
        if name != "no rows":
            graph.replay()
        expired(rcd, ctx)
        if name != "no rows":
            graph.replay()
        call()                                             # (the context's last call is this one, not the self-test)
        ctx.sync_status()
