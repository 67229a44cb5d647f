"""Softmax cross entropy of narrow 16-bit rows whose logits stay in registers, at sizes that take that way."""
import math

import pytest
import torch

from paper_2308_14129_amd import ops
from tests.test_gpu_ops import DEV, F64, TYPES, U, check_ce, close, gen_of, half, reference_ce, rnd, tiny
from tests.test_ops_ways import goes_narrow

pytestmark = [pytest.mark.gpu, pytest.mark.timeout(300)]


def narrow(n, V, d, dtype, grad=True):
    assert goes_narrow(ops._lib(), n, V, d, dtype, grad), "this size does not test what it is here for"


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("n,V,d", [(2100, 16_100, 100), (2100, 16_100, 48), (3000, 12_000, 64), (1000, 34_000, 96), (90, 500, 100)])
@pytest.mark.parametrize("weighted", [False, True])
def test_bias_gradient_is_summed_before_p_is_rounded(n, V, d, weighted, dtype):
    """A candidate of probability 0.3 that is the label of three rows in ten: its gradient cancels, and the rounding of 0.3 and
    -0.7, the same in every row, would not."""
    t, gen = TYPES[dtype], gen_of(n + d)
    h = half(t)
    x, w, b = rnd(gen, n, d, dtype=t), rnd(gen, V, d, std=1e-6, dtype=t), rnd(gen, V, std=0.1, dtype=t)
    b[7] = math.log(0.3 / 0.7) + float(torch.logsumexp(torch.cat([b[:7], b[8:]]).to(F64), 0))
    labels = torch.where(torch.rand(n, device=DEV, generator=gen) < 0.3, 7, 11).to(torch.int32)
    rs = torch.full((n,), 1.0 / n, device=DEV) if weighted else None
    r = ops.softmax_ce(x, w, labels, b, rs)
    logits, lse, _, _, s, p, hot = reference_ce(x, w, labels, b, rs, 1.0)
    size = x.to(F64).abs() @ w.to(F64).abs().t() + b.to(F64).abs()
    err_l = (d + 2) * U * size
    near = (logits - lse.unsqueeze(1)).abs()
    err_lse = (p * (err_l + (8 + 2 * near) * U)).sum(1) + 400 * U + 4 * U * lse.abs()
    P = (p - hot) * s.unsqueeze(1)
    off = p * s.abs().unsqueeze(1) * (err_l + err_lse.unsqueeze(1) + (12 + 2 * near) * U) + 4 * U * P.abs()
    DB = P.sum(0)
    close(r.dbias, DB, h * DB.abs() + 1.01 * (off.sum(0) + 70 * U * P.abs().sum(0)) + tiny(t), "dbias")


def check_call(x, w, labels, b, rs=None, scale=1.0):
    """Every output of a call against its formula in 64 bits, within the bounds of check_ce."""
    n, d = x.shape
    V, t = w.shape[0], x.dtype
    h = half(t)
    r = ops.softmax_ce(x, w, labels, b, rs, scale)
    logits, lse, loss, mean, s, p, hot = reference_ce(x, w, labels, b, rs, scale)
    X, W = x.to(F64), w.to(F64)
    err_l = (d + 2) * U * (X.abs() @ W.abs().t() + b.to(F64).abs())
    near = torch.where(p > 0, (logits - lse.unsqueeze(1)).abs(), torch.zeros_like(p))
    err_lse = (p * (err_l + (8 + 2 * near) * U)).sum(1) + 400 * U + 4 * U * lse.abs()
    close(r.lse, lse, err_lse, "lse")
    close(r.loss, loss, err_lse + err_l.amax(1) + 2 * U * (loss.abs() + lse.abs()), "loss")
    P = (p - hot) * s.unsqueeze(1)
    top = s.abs().max()
    off = p * s.abs().unsqueeze(1) * (err_l + err_lse.unsqueeze(1) + (12 + 2 * near) * U) + 4 * U * P.abs()
    live = (s != 0).to(F64).unsqueeze(1)
    off_p = (off + h * P.abs() + top * (tiny(t) if t is not torch.float16 else 2.0**-39)) * live
    under, A = top * 2.0**-126, P.abs()
    DX, DW, DB = P @ W, P.t() @ X, P.sum(0)
    close(r.dx, DX, h * DX.abs() + 1.01 * (off_p @ W.abs() + (V + 8) * U * (A @ W.abs())) + (V + 8) * under + tiny(t), "dx")
    close(r.dw, DW, h * DW.abs() + 1.01 * (off_p.t() @ X.abs() + (n + 8) * U * (A.t() @ X.abs())) + (n + 8) * under + tiny(t), "dw")
    close(r.dbias, DB, h * DB.abs() + 1.01 * (off.sum(0) + 70 * U * A.sum(0)) + n * under + tiny(t), "dbias")
    return r


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("n,V,d,bias", [(100, 1_000_003, 128, False), (100, 1_000_003, 128, True), (64, 1_000_001, 60, True), (3, 1_000_000, 20, False),
                                        (100, 200_003, 128, False), (6000, 140_000, 100, True)])
def test_statistics_over_long_ranges(n, V, d, bias, dtype):
    """Every streamed tile has to be there before it is read; what was not, showed now and then."""
    narrow(n, V, d, dtype, grad=False)
    r = check_ce(n, V, d, dtype, bias=bias, seed=n, grad=False)
    gen = gen_of(n)
    t = TYPES[dtype]
    x, w = rnd(gen, n, d, dtype=t), rnd(gen, V, d, std=1.5 * d**-0.5, dtype=t)
    b = rnd(gen, V, std=0.5, dtype=t) if bias else None
    labels = torch.zeros(n, dtype=torch.int32, device=DEV)
    for _ in range(8):
        assert torch.equal(ops.softmax_ce(x, w, labels, b, grad=False).lse, r.lse)


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("n,V,d", [(600, 400_000, 128), (600, 400_000, 60), (6000, 40_000, 100), (6000, 40_000, 128), (6000, 40_000, 64), (40_000, 4000, 96)])
def test_gradients_over_long_ranges(n, V, d, dtype):
    """About twenty streamed tiles a workgroup in either gradient."""
    narrow(n, V, d, dtype)
    gen, t = gen_of(n + d), TYPES[dtype]
    x, w, b = rnd(gen, n, d, dtype=t), rnd(gen, V, d, std=1.5 * d**-0.5, dtype=t), rnd(gen, V, std=0.5, dtype=t)
    labels = torch.randint(-V // 8, V, (n,), device=DEV, generator=gen, dtype=torch.int32)
    r = check_call(x, w, labels, b, scale=512.0)
    for _ in range(4):
        for name, want in r._asdict().items():
            assert torch.equal(getattr(ops.softmax_ce(x, w, labels, b, scale=512.0), name), want), name


SHAPES = [(2100, 16_100, 100), (2100, 16_100, 48), (2100, 16_100, 64), (1000, 34_000, 128), (300, 112_000, 96), (64, 530_000, 33), (34_000, 1000, 127)]


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("weighted,scale", [(False, 1.0), (True, -0.5), (False, -2.0)])
@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_every_output(shape, weighted, scale, dtype):
    n, V, d = shape
    narrow(n, V, d, dtype)
    gen, t = gen_of(n + d), TYPES[dtype]
    x, w, b = rnd(gen, n, d, dtype=t), rnd(gen, V, d, std=1.5 * d**-0.5, dtype=t), rnd(gen, V, std=0.5, dtype=t)
    labels = torch.randint(-V // 8, V, (n,), device=DEV, generator=gen, dtype=torch.int32)
    check_call(x, w, labels, b, rnd(gen, n) if weighted else None, scale * (512 if dtype == "fp16" else 1))


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("spread", [60.0, 400.0])
@pytest.mark.parametrize("shape", SHAPES[:5], ids=str)
def test_far_logits(shape, spread, dtype):
    """Logits of hundreds, and of thousands: one candidate takes all, and a row's largest logit moves far."""
    n, V, d = shape
    narrow(n, V, d, dtype)
    gen, t = gen_of(n + d), TYPES[dtype]
    x, w, b = rnd(gen, n, d, dtype=t), rnd(gen, V, d, std=spread * d**-0.5, dtype=t), rnd(gen, V, std=0.5, dtype=t)
    labels = torch.randint(-V // 8, V, (n,), device=DEV, generator=gen, dtype=torch.int32)
    check_call(x, w, labels, b, scale=512.0)


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("order", ["up", "down", "far up"])
@pytest.mark.parametrize("shape", SHAPES[:4], ids=str)
def test_logits_in_order(shape, order, dtype):
    """A bias that grows, or falls, along the vocabulary: the running maximum moves with every tile, or never again; "far up": from
    -3000 on, through the size from which a row's differences are formed first."""
    n, V, d = shape
    narrow(n, V, d, dtype)
    gen, t = gen_of(n + d), TYPES[dtype]
    x, w = rnd(gen, n, d, dtype=t), rnd(gen, V, d, std=0.5 * d**-0.5, dtype=t)
    b = torch.linspace(-3000 if order == "far up" else -120, 1, V, device=DEV, dtype=F64)
    b = (b.flip(0) if order == "down" else b).to(t)
    labels = torch.randint(-V // 8, V, (n,), device=DEV, generator=gen, dtype=torch.int32)
    check_call(x, w, labels, b, scale=512.0)
