"""Activations and their slopes far below zero, relative to the value: what is left of 1 - erf or 1 - tanh there."""
import math

import pytest

from test_gpu_linear import ACTS, U, act64, code
from test_gpu_norm import ctx, rcd  # noqa: F401  (fixtures)

pytestmark = pytest.mark.gpu

# where each activation's exponential stays in fp32's normal range
LOWEST = {"relu": -1e30, "gelu": -12.5, "gelu_tanh": -9.5, "silu": -80.0}


def steps(z, act):
    """Roundings, in units of fp32.  The exponential's argument is off by a few units of itself (three for z^2 / 2: the square, the product, the
    factor; five for the tanh form's polynomial), and so is its result by as many times the argument; beside it the instructions (4 and 2
    units) and the few products around them, and for GELU the polynomial in fp32 (ten steps, and its fit)."""
    if act == "gelu":
        return 32 + 2 * z * z
    if act == "gelu_tanh":
        return 24 + 10 * math.sqrt(2 / math.pi) * (z.abs() + 0.044715 * z.abs() ** 3)
    return 16 + 4 * z.abs()


def normal64(z):
    """The normal distribution far below zero, without a difference of near numbers."""
    import torch
    return 0.5 * torch.special.erfc(-z / math.sqrt(2))


def values(act):
    import torch
    return torch.linspace(max(LOWEST[act], -80.0), 12.5, 6001).to(torch.bfloat16).cuda()


@pytest.mark.parametrize("act", ACTS[1:])
@pytest.mark.parametrize("rows", [True, False])                       # through the product's tiles, and through the form for few rows
def test_values(rcd, ctx, act, rows):
    import torch
    z = values(act)
    one = torch.ones(1, 8, device="cuda", dtype=torch.bfloat16)
    one[:, 1:] = 0
    many = torch.zeros(z.numel(), 8, device="cuda", dtype=torch.bfloat16)
    many[:, 0] = z
    x, w = (many, one) if rows else (one, many)
    y, _ = ctx.rcd_linear(x, w, activation=code(rcd, act), out_dtype=torch.float32)
    ctx.sync_status()
    zz = z.double()
    want = {"gelu": lambda: zz * normal64(zz), "gelu_tanh": lambda: zz * torch.sigmoid(2 * math.sqrt(2 / math.pi) * (zz + 0.044715 * zz ** 3))}.get(act, lambda: act64(zz, act)[0])()
    off = (y.reshape(-1).double() - want).abs() - (want.abs() * steps(zz, act) * U + 2.0 ** -126)
    assert float(off.max()) <= 0, (float(zz[off.argmax()]), float(off.max() / want[off.argmax()]))


@pytest.mark.parametrize("act", ACTS[1:])
def test_slopes(rcd, ctx, act):
    """A slope is a sum of two terms, of unlike signs below zero: its error is theirs."""
    import torch
    z = values(act).reshape(1, -1)
    n = z.shape[1]
    x, w = torch.zeros(1, 8, device="cuda", dtype=torch.bfloat16), torch.zeros(n, 8, device="cuda", dtype=torch.bfloat16)
    _, _, db = ctx.rcd_linear_backward(torch.ones_like(z), x, w, preact=z, activation=code(rcd, act), want_dx=False, want_dw=False)
    ctx.sync_status()
    zz = z.reshape(-1).double()
    c = 2 * math.sqrt(2 / math.pi)
    if act == "relu":
        first, second = (zz > 0).double(), torch.zeros_like(zz)
    elif act == "gelu":
        first, second = normal64(zz), zz * torch.exp(-zz * zz / 2) / math.sqrt(2 * math.pi)
    else:
        u = zz if act == "silu" else c * (zz + 0.044715 * zz ** 3)
        du = torch.ones_like(zz) if act == "silu" else c * (1 + 3 * 0.044715 * zz * zz)
        first, second = torch.sigmoid(u), zz * torch.sigmoid(u) * torch.sigmoid(-u) * du
    off = (db.double() - first - second).abs() - ((first.abs() + second.abs()) * steps(zz, act) * U + 2.0 ** -126)
    assert float(off.max()) <= 0, (float(zz[off.argmax()]), float(off.max()))
