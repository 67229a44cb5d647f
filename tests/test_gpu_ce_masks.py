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


@pytest.mark.parametrize("dtype", ["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("shape", SHAPES, ids=str)
@pytest.mark.parametrize("weighted", [False, True])
def test_nothing_but_finite_masks_leaves_equal_probabilities(shape, dtype, weighted):
    """Every candidate of every row under the same mask, beside which the products round away: probabilities of 1 / V.  (Under a
    mask of 1e4 the products are not below half a step of the logits: they and a step are what logits may differ by.)"""
    n, V, d = shape
    t, gen = TYPES[dtype], gen_of(n + V + d + 1)
    h = half(t)
    x, w = rnd(gen, n, d, dtype=t), rnd(gen, V, d, std=1e-4, dtype=t)
    labels = torch.randint(-1, V, (n,), device=DEV, generator=gen, dtype=torch.int32)
    rs = rnd(gen, n) if weighted else None
    on = labels >= 0
    X, W = x.to(F64), w.to(F64)
    s = rs.to(F64) if weighted else torch.full((n,), 1.0 / int(on.sum()), dtype=F64, device=DEV)
    s = torch.where(on, s, torch.zeros_like(s)).unsqueeze(1)
    hot = torch.zeros(n, V, dtype=F64, device=DEV).scatter_(1, labels.long().clamp(min=0).unsqueeze(1), 1.0)
    P = (1.0 / V - hot) * s
    # the exponential of 0 and the sum: a relative error of 412 U (400 sums as elsewhere); each operand's rounding, and P's smallest step
    exact = 412 * U / V * s.abs() + 4 * U * P.abs()
    products = float((X @ W.t()).abs().max())
    step = s.abs().max() * (tiny(t) if dtype != "fp16" else 2.0**-25 * 2.0**-14)
    under = s.abs().max() * 2.0**-126
    DX, DW, DB = P @ W, P.t() @ X, P.sum(0)
    for mask in masks(t):
        print(f"[all masked] {shape} {dtype} weighted {weighted} {mask}", flush=True)
        b = torch.full((V,), mask, dtype=t, device=DEV)
        mask = float(b[0].to(F64))
        ulp = 2 * U * abs(mask)
        differ = 0.0 if products < ulp / 4 else products + ulp
        off = exact + 2.1 * differ / V * s.abs()
        off_p = (off + h * P.abs() + step) * on.unsqueeze(1)
        r = ops.softmax_ce(x, w, labels, b, rs)
        lse = mask + math.log(V)
        # (the products are below 0.01; a step of fp32 at the mask)
        assert ((r.lse.to(F64) - lse).abs() <= 2 * U * abs(lse) + 0.01 + 400 * U).all()
        # the loss is the logarithm of V, not the difference of two numbers of the mask's size
        loss = torch.where(on, math.log(V), 0.0)
        assert ((r.loss.to(F64) - loss).abs() <= 0.02 + 2.0**-7 * (abs(mask) < 1e5)).all()
        close(r.dx, DX, h * DX.abs() + 1.01 * (off_p @ W.abs() + (V + 8) * U * (P.abs() @ W.abs())) + (V + 8) * under + tiny(t), "dx")
        close(r.dw, DW, h * DW.abs() + 1.01 * (off_p.t() @ X.abs() + (n + 8) * U * (P.abs().t() @ X.abs())) + (n + 8) * under + tiny(t), "dw")
        close(r.dbias, DB, h * DB.abs() + 1.01 * ((off + step).sum(0) + 70 * U * P.abs().sum(0) + h * P.abs().sum(0)) + tiny(t), "dbias")
