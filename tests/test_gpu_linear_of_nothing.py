"""Gradients of products without rows or without columns: what is written, and what is refused."""
import ctypes as C

import pytest

from test_gpu_norm import ctx, rcd  # noqa: F401  (fixtures)

pytestmark = pytest.mark.gpu


def test_no_columns_of_any_rank(ctx):
    import torch
    x, w = torch.ones(2, 3, 64, device="cuda", dtype=torch.bfloat16), torch.empty(0, 64, device="cuda", dtype=torch.bfloat16)
    y, z = ctx.rcd_linear(x, w, want_preact=True)
    assert y.shape == (2, 3, 0) and z.shape == (2, 3, 0)
    dx, dw, db = ctx.rcd_linear_backward(y, x, w)
    ctx.sync_status()
    assert dx.shape == (2, 3, 64) and not dx.any() and dw.shape == (0, 64) and db.shape == (0,)


def args_of(rcd, rows, n, k):
    a = rcd.RcdLinearBackArgs()
    a.rows, a.n, a.k, a.type, a.dw_type = rows, n, k, rcd.RCD_ELEM_BF16, rcd.RCD_ELEM_F32
    a.ld_dy, a.ldx, a.ldw, a.ld_dx, a.ld_dw = n, k, k, k, k
    return a


def test_outputs_are_checked_where_there_is_nothing_to_sum(rcd, ctx):
    import torch
    dx = torch.ones(4, 64, device="cuda", dtype=torch.bfloat16)
    a = args_of(rcd, 4, 0, 64)
    a.dx = dx.data_ptr()
    run = lambda: rcd.lib.rcd_linear_backward(ctx._h, C.byref(a), None, 0, None)  # noqa: E731
    for ld, at in ((63, 0), (64, 1)):                       # rows shorter than themselves; not on its type
        a.ld_dx, a.dx = ld, dx.data_ptr() + at
        assert run() == 1
        torch.cuda.synchronize()
        assert bool((dx == 1).all())
    a.ld_dx, a.dx = 64, dx.data_ptr()
    assert run() == 0
    torch.cuda.synchronize()
    assert not dx.any()


def test_zeros_in_rows_far_apart(rcd, ctx):
    """Rows of the gradients 2^31 bytes and more from each other."""
    import torch
    ld = 1 << 30
    far = torch.ones(2 * ld + 64, device="cuda", dtype=torch.float32)
    a = args_of(rcd, 0, 3, 64)
    a.dw, a.ld_dw = far.data_ptr(), ld
    assert rcd.lib.rcd_linear_backward(ctx._h, C.byref(a), None, 0, None) == 0
    torch.cuda.synchronize()
    for row in range(3):
        assert not far[row * ld:row * ld + 64].any()
    assert bool((far[64:1 << 20] == 1).all()) and bool((far[ld + 64:ld + (1 << 20)] == 1).all())
