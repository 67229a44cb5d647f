"""Queries that are turned in place while many tokens enter the cache (ops.cache_append): several tokens of a workgroup at a time, rows whose
pieces read each other's columns."""
import pytest
import torch

from paper_2308_14129_amd import ops
from tests.paged import DEV, F64, TYPES, U, close, gen_of, half, tiny

pytestmark = [pytest.mark.gpu, pytest.mark.timeout(120)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("tokens", [2_048, 9_001, 20_011])
@pytest.mark.parametrize("qh, heads, dim, rotary, interleaved", [(6, 2, 128, 128, False), (4, 1, 128, 96, False), (3, 1, 50, 50, True), (5, 3, 256, 256, False),
                                                                 (2, 1, 33, 24, False), (3, 2, 100, 100, False), (2, 2, 72, 34, True)])
def test_queries_turned_in_place(qh, heads, dim, rotary, interleaved, tokens, dtype):
    t, gen, size, seqs = TYPES[dtype], gen_of(dim + tokens), 16, 3
    counts = [tokens // 2, 7, tokens - tokens // 2 - 7]
    starts = torch.tensor([0, counts[0], counts[0] + 7, tokens], dtype=torch.int32, device=DEV)
    lengths = torch.tensor(counts, dtype=torch.int32, device=DEV)
    width = -(-max(counts) // size)
    table = torch.randperm(seqs * width, device=DEV, generator=gen).to(torch.int32).view(seqs, width)
    caches = [torch.zeros(seqs * width, size, heads, dim, dtype=t, device=DEV) for _ in range(4)]
    qkv = torch.randn(tokens, qh + 2 * heads, dim, device=DEV, generator=gen).to(t)
    mine = qkv.clone()
    freq = 1000.0 ** (-torch.arange(rotary // 2, device=DEV, dtype=F64) / (rotary // 2))
    positions = torch.rand(tokens, device=DEV, generator=gen, dtype=F64) * 1e6

    def call(k_cache, v_cache, x, out):
        return ops.cache_append(k_cache, v_cache, table, lengths, x[:, qh : qh + heads], x[:, qh + heads :], starts=starts, q=x[:, :qh], freq=freq,
                                positions=positions, interleaved=interleaved, q_out=out)

    apart = call(caches[0], caches[1], qkv, None)
    for turn in range(2):  # again, from the same numbers
        mine.copy_(qkv)
        got = call(caches[2], caches[3], mine, mine[:, :qh])
        assert torch.equal(got, apart) and torch.equal(mine[:, qh:], qkv[:, qh:])
        assert torch.equal(caches[0], caches[2]) and torch.equal(caches[1], caches[3])
    angle = torch.outer(positions, freq)[:, None, :]
    c, s = angle.cos(), angle.sin()
    first, second = (slice(0, rotary, 2), slice(1, rotary, 2)) if interleaved else (slice(0, rotary // 2), slice(rotary // 2, rotary))
    want = qkv[:, :qh].to(F64)
    tol = torch.zeros_like(want)
    a, b = want[..., first].clone(), want[..., second].clone()
    want[..., first], want[..., second] = a * c - b * s, b * c + a * s
    # products and their sum, cosine and sine: 8 units of the terms, then one rounding to the type
    tol[..., first], tol[..., second] = 8 * U * ((a * c).abs() + (b * s).abs()), 8 * U * ((b * c).abs() + (a * s).abs())
    tol[..., :rotary] += half(t) * want[..., :rotary].abs() + tiny(t)
    close(got, want, tol, "q")
