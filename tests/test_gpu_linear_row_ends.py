"""Outputs whose rows start on 16 bytes and end elsewhere: what lies between the rows, and behind the last one, stays as it was."""
import ctypes as C

import pytest

from test_gpu_linear import rounded, whole
from test_gpu_norm import ctx, kind, rcd, seeded  # noqa: F401  (fixtures)

pytestmark = pytest.mark.gpu

MARK = 77


def framed(m, n, dtype):
    """Rows of n elements on 16 bytes in a buffer of marks, which ends with the last row's last element."""
    import torch
    size = torch.empty(0, dtype=dtype).element_size()
    ld = (n * size + 15) // 16 * 16 // size
    buf = torch.full((m * ld + 64,), MARK, device="cuda", dtype=dtype)
    return buf, buf.as_strided((m, n), (ld, 1)), ld


def untouched(buf, view):
    view.fill_(MARK)
    return bool((buf == MARK).all())


@pytest.mark.parametrize("m,n,k", [(40, 1, 64), (87, 119, 476), (300, 117, 64), (300, 129, 72), (1300, 333, 512), (5000, 509, 256), (20000, 130, 128), (300, 255, 40000)])
@pytest.mark.parametrize("dtype,out", [("bf16", "bf16"), ("fp16", "fp32"), ("bf16", "fp32"), ("int8", "bf16"), ("int8", "fp32")])
@pytest.mark.parametrize("residual", [False, True])
def test_forward(rcd, ctx, m, n, k, dtype, out, residual):
    import torch
    t, o, g = kind(dtype), kind(out), seeded(m, n, k, dtype, out, "ends")
    x, w = whole(g, m, k, t, most=2), whole(g, n, k, t, most=2)
    want = x.double() @ w.double().t()
    rbuf, r, rld = framed(m, n, o)
    r.copy_(whole(g, m, n, o))
    (ybuf, y, yld), (zbuf, z, zld) = framed(m, n, o), framed(m, n, o)
    for keep in (False, True):
        a = rcd.RcdLinearArgs()
        a.rows, a.n, a.k, a.type, a.y_type = m, n, k, {"bf16": rcd.RCD_ELEM_BF16, "fp16": rcd.RCD_ELEM_F16, "int8": rcd.RCD_ELEM_I8}[dtype], rcd.RCD_ELEM_BF16 if out == "bf16" else rcd.RCD_ELEM_F32
        a.x, a.ldx, a.w, a.ldw, a.y, a.ldy = x.data_ptr(), k, w.data_ptr(), k, y.data_ptr(), yld
        if residual:
            a.residual, a.ld_residual = r.data_ptr(), rld
        if keep:
            a.preact, a.ld_preact = z.data_ptr(), zld
        need = C.c_size_t()
        assert rcd.lib.rcd_linear_workspace_bytes(ctx._h, C.byref(a), C.byref(need)) == 0
        ws = torch.empty(max(need.value, 1), device="cuda", dtype=torch.uint8)
        assert rcd.lib.rcd_linear(ctx._h, C.byref(a), C.c_void_p(ws.data_ptr()), need, None) == 0
        ctx.sync_status()
        assert torch.equal(y, rounded(want + (r.double() if residual else 0), o)) and untouched(ybuf, y)
        if keep:
            assert torch.equal(z, rounded(want, o))
        assert untouched(zbuf, z)


@pytest.mark.parametrize("m,n,k", [(300, 64, 117), (87, 119, 333), (5000, 72, 509), (1300, 333, 1001), (40000, 100, 255)])
@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("dw_fp32", [False, True])
def test_gradients(rcd, ctx, m, n, k, dtype, dw_fp32):
    import torch
    t, g = kind(dtype), seeded(m, n, k, dtype, "ends")
    dy, x, w = whole(g, m, n, t, most=2), whole(g, m, k, t, most=2), whole(g, n, k, t, most=2)
    (xbuf, dx, xld), (wbuf, dw, wld) = framed(m, k, t), framed(n, k, torch.float32 if dw_fp32 else t)
    a = rcd.RcdLinearBackArgs()
    a.rows, a.n, a.k, a.type = m, n, k, rcd.RCD_ELEM_BF16 if dtype == "bf16" else rcd.RCD_ELEM_F16
    a.dw_type = rcd.RCD_ELEM_F32 if dw_fp32 else a.type
    a.dy, a.ld_dy, a.x, a.ldx, a.w, a.ldw = dy.data_ptr(), n, x.data_ptr(), k, w.data_ptr(), k
    a.dx, a.ld_dx, a.dw, a.ld_dw = dx.data_ptr(), xld, dw.data_ptr(), wld
    need = C.c_size_t()
    assert rcd.lib.rcd_linear_backward_workspace_bytes(ctx._h, C.byref(a), C.byref(need)) == 0
    ws = torch.empty(max(need.value, 1), device="cuda", dtype=torch.uint8)
    assert rcd.lib.rcd_linear_backward(ctx._h, C.byref(a), C.c_void_p(ws.data_ptr()), need, None) == 0
    ctx.sync_status()
    assert torch.equal(dx, rounded(dy.double() @ w.double(), t)) and untouched(xbuf, dx)
    assert torch.equal(dw, rounded(dy.double().t() @ x.double(), torch.float32 if dw_fp32 else t)) and untouched(wbuf, dw)
