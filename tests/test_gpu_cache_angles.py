"""Rotations by far angles (ops.cache_append): the quarter turns of an angle beyond 2^53 are still counted right."""
import math

import pytest
import torch

from paper_2308_14129_amd import ops
from tests.paged import DEV, F64, U, close, gen_of, make_cache, tiny

pytestmark = [pytest.mark.gpu, pytest.mark.timeout(120)]


def turned(k, positions, freq):
    """The host's cosine and sine take an angle as it is."""
    d = k.shape[-1] // 2
    angles = [[float(p) * f for f in freq] for p in positions]
    c, s = (torch.tensor([[f(a) for a in row] for row in angles], dtype=F64)[:, None, :] for f in (math.cos, math.sin))
    a, b = k[..., :d].to(F64), k[..., d:].to(F64)
    return torch.cat([a * c - b * s, b * c + a * s], -1), torch.cat([(a * c).abs() + (b * s).abs(), (b * c).abs() + (a * s).abs()], -1)


def append(positions, freq):
    n, d = positions.numel(), 2 * len(freq)
    k_cache, v_cache = make_cache(n, 1, 1, d, torch.float32, "rows")
    table = torch.arange(n, dtype=torch.int32, device=DEV)[:, None]
    k = torch.randn(n, 1, d, device=DEV, generator=gen_of(5))
    ops.cache_append(k_cache, v_cache, table, torch.ones(n, dtype=torch.int32, device=DEV), k, k, freq=torch.tensor(freq, dtype=F64, device=DEV),
                     positions=positions.to(DEV))
    return k.cpu(), k_cache[:, 0].cpu()


# angles up to 2^55.7 (counts of 2^53 turns), nanoseconds of decades, and up to the largest that there are cosines for
CASES = {"2 pi, 2^53": ("int64", 2.0**53, [2 * math.pi, 1.0, 6.5, 0.1]), "nanoseconds": ("fp64", 1.7e18, [1.0, 2 * math.pi, 1e-3, 1e-9]),
         "2^54": ("fp64", 2.0**54, [1.0, 1.0, 1.0, 1.0]), "2^64": ("fp64", 2.0**64, [1.0, 0.5, 0.75, 1e-8])}


@pytest.mark.parametrize("case", CASES)
def test_far_angles(case):
    kind, top, freq = CASES[case]
    r = torch.rand(1500, dtype=F64, generator=torch.Generator().manual_seed(9)) * 2 - 1
    r[:4] = torch.tensor([1.0, -1.0, 0.5, -0.25], dtype=F64)
    positions = (r * top).long() if kind == "int64" else r * top
    k, got = append(positions, freq)
    want, mag = turned(k, positions.tolist(), freq)
    close(got, want, 8 * U * mag + tiny(torch.float32), case)  # products and their sum, cosine and sine rounded


def test_angles_that_have_no_cosine():
    """Beyond 2^64 neighbouring angles are thousands of turns apart: NaN, not some number."""
    positions = torch.tensor([2.0**65, -(2.0**70), 1e300, float("inf"), float("nan"), 3.0], dtype=F64)
    _, got = append(positions, [1.0, 1.0, 1.0, 1.0])
    assert torch.isnan(got[:5]).all() and torch.isfinite(got[5]).all()
