"""gelu and its slope over their whole range, relative to their own values: a layer of one weight, which is 1."""
import math

import pytest
import torch

from paper_2308_14129_amd import ops
from tests.test_gpu_ops import DEV, F64, TYPES, U, close, half, tiny

pytestmark = [pytest.mark.gpu, pytest.mark.timeout(300)]


@pytest.mark.parametrize("dtype", ["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("rows", [16, 40_001])  # the kernel of few rows, and tiles
def test_gelu_relative_to_its_value(rows, dtype):
    t = TYPES[dtype]
    h = half(t)
    z = torch.linspace(-12.5, 12.5, 40_001, device=DEV, dtype=F64).to(t)
    one = torch.ones(1, 1, dtype=t, device=DEV)
    for at in (range(0, 40_001, 2003) if rows == 16 else [0]):
        x = z[at : at + rows].view(-1, 1)
        y, kept = ops.linear(x, one, activation="gelu", keep=True)
        slope = ops.linear_backward(torch.ones_like(x), x, one, kept, "gelu", dw=False, dbias=False)[0]
        assert torch.equal(kept, x)
        Z = x.to(F64)
        phi = 0.5 * torch.special.erfc(-Z / math.sqrt(2))
        # the tail's polynomial is 1 U off, its chain of ten operations and the reciprocal add 12 U at most; the
        # exponential's argument z^2 / 2 is rounded three times (1.5 z^2 U of the value) and the exponential is 4 U off; two products
        rel = (20 + 1.5 * Z * Z) * U
        Y = Z * phi
        close(y, Y, h * Y.abs() + (1 + h) * rel * Y.abs() + tiny(t) + 2.0**-126, "y")
        more = Z * torch.exp(-Z * Z / 2) / math.sqrt(2 * math.pi)
        S = phi + more
        close(slope, S, h * S.abs() + (1 + h) * rel * (phi + more.abs()) + tiny(t) + 2.0**-126, "slope")


@pytest.mark.parametrize("dtype", ["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("act", ["none", "relu", "gelu", "silu"])
@pytest.mark.parametrize("rows", [4, 64])
def test_activations_at_infinity(rows, act, dtype):
    """Their limits, and those of their slopes; a NaN stays one (relu's slope has none)."""
    t = TYPES[dtype]
    inf = math.inf
    x = torch.tensor([inf, -inf, 3.0e38 if dtype != "fp16" else 65504.0, -3.0e38 if dtype != "fp16" else -65504.0] * (rows // 4), device=DEV).to(t).view(-1, 1)
    one = torch.ones(1, 1, dtype=t, device=DEV)
    y, z = ops.linear(x, one, activation=act, keep=True)
    slope = ops.linear_backward(torch.ones_like(x), x, one, z, act, dw=False, dbias=False)[0]
    low = act == "none"
    assert torch.equal(y, torch.where(x > 0, x, x if low else torch.zeros_like(x)))
    assert torch.equal(slope, torch.where(x > 0, torch.ones_like(x), torch.full_like(x, float(low))))
    y, z = ops.linear(torch.full_like(x, math.nan), one, activation=act, keep=True)
    slope = ops.linear_backward(torch.ones_like(x), x, one, z, act, dw=False, dbias=False)[0]
    assert torch.isnan(y).all() and (torch.isnan(slope).all() or act in ("none", "relu"))
