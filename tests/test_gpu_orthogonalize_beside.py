"""Stacked gradients and their updates as slices of one buffer: taken where no byte is shared, refused where one is."""
import pytest

from test_gpu_norm import ctx, kind, rcd, seeded  # noqa: F401  (fixtures)
from test_gpu_orthogonalize import gradient

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("batch,rows,cols", [(3, 64, 96), (2, 33, 70), (3, 300, 430), (2, 1500, 1100)])
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_slices_of_one_buffer(rcd, ctx, batch, rows, cols, dtype):
    import torch
    t = kind(dtype)
    g = gradient(seeded("beside", rows), batch, rows, cols, t)
    want = ctx.rcd_orthogonalize(g)
    wide = 1 if dtype == "bf16" else 2                     # bf16 elements in one of g's

    def check(buf, mine, out):
        mine.copy_(g)
        before = buf.clone()
        assert ctx.rcd_orthogonalize(mine, out=out) is out
        assert torch.equal(out, want) and torch.equal(mine, g)
        out.zero_()
        again = before.view(torch.bfloat16)
        again.as_strided(out.shape, out.stride(), out.storage_offset()).zero_()
        assert torch.equal(buf.view(torch.int16), before.view(torch.int16))
    # every second matrix
    buf = torch.full((batch, 2, rows, cols), 7.0, device="cuda", dtype=t)
    check(buf, buf[:, 0], buf.view(torch.bfloat16)[:, 1, :, :cols])
    # the right half of every row
    buf = torch.full((batch, rows, 2 * cols), 7.0, device="cuda", dtype=t)
    check(buf, buf[:, :, :cols], buf.view(torch.bfloat16)[:, :, wide * cols:wide * cols + cols])
    ctx.sync_status()


def test_shared_bytes_are_refused(rcd, ctx):
    import torch
    buf = torch.zeros(5, 40, 60, device="cuda", dtype=torch.bfloat16)
    for g, out in ((buf, buf), (buf[:-1], buf[1:]), (buf[::2], buf[::2]), (buf[:, :20], buf[:, 19:39]), (buf[:, :, :30], buf[:, :, 29:59]), (buf[:, :, :30], buf[:, :, :30]),
                   (buf[:2, :, :30], buf.flatten(0, 1)[39:119].view(2, 40, 60)[:, :, :30]), (buf[:2], buf.flatten()[:4800 + 59].as_strided((2, 40, 60), (2400, 60, 1), 59))):
        with pytest.raises(rcd.RcdError) as e:
            ctx.rcd_orthogonalize(g, out=out)
        assert e.value.status == 1 and "overlaps" in str(e.value)
    ctx.sync_status()
