"""Softmax cross entropy of narrow 16-bit rows whose logits stay in registers."""
import math

import pytest
import torch

from paper_2308_14129_amd import ops
from tests.test_gpu_ops import DEV, F64, TYPES, U, close, gen_of, half, reference_ce, rnd, tiny

pytestmark = [pytest.mark.gpu, pytest.mark.timeout(300)]


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
