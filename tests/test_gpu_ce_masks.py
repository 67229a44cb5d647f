"""Softmax cross entropy whose candidates are masked by a large finite bias, the type's lowest value among them."""
import math

import pytest
import torch

from paper_2308_14129_amd import ops
from tests.test_gpu_ops import DEV, F64, TYPES, U, close, gen_of, half, rnd, tiny

pytestmark = [pytest.mark.gpu, pytest.mark.timeout(300)]

# by tiles; narrow 16-bit rows, with and without a column for the bias, of 64 and of 128 columns
SHAPES = [(90, 500, 96), (300, 2049, 40), (2100, 16_100, 48), (2100, 16_100, 64), (2100, 16_100, 100), (1100, 31_000, 128)]


def masks(t):
    return [-1e4 if t is torch.float16 else -1e9, torch.finfo(t).min] if t is torch.float16 else [-1e9, -1e30, torch.finfo(t).min]


@pytest.mark.parametrize("dtype", ["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_finite_masks_are_what_infinite_ones_are(shape, dtype):
    """Whole tiles and ranges of candidates at either end, and every third of those between: as -infinity, bit for bit (no
    logit is within 200 of another one's mask)."""
    n, V, d = shape
    t, gen = TYPES[dtype], gen_of(n + V + d)
    x, w, b = rnd(gen, n, d, dtype=t), rnd(gen, V, d, std=1.5 * d**-0.5, dtype=t), rnd(gen, V, std=0.5, dtype=t)
    off = torch.zeros(V, dtype=torch.bool, device=DEV)
    off[: V // 3] = True
    off[-(V // 3):] = True
    off[::3] = True
    labels = torch.nonzero(~off).flatten()[torch.randint(0, int((~off).sum()), (n,), device=DEV, generator=gen)].to(torch.int32)
    labels[::7] = -1
    want = ops.softmax_ce(x, w, labels, b.masked_fill(off, -math.inf))
    for name in ("loss", "lse", "mean", "dx", "dw", "dbias"):
        assert torch.isfinite(getattr(want, name)).all(), name
    for mask in masks(t):
        print(f"[mask] {shape} {dtype} {mask}", flush=True)
        got = ops.softmax_ce(x, w, labels, b.masked_fill(off, mask))
        for name in ("loss", "lse", "mean", "dx", "dw", "dbias"):
            assert torch.equal(getattr(got, name), getattr(want, name)), (mask, name)
