"""The attention's line of tiles where it is long (ops.cache_attend): wavefronts that go through the same rows together, several blocks of query
heads, units that many workgroups share.  Values are ones in the column of a stretch of the sequence's rows, so that a column of the output is
that stretch's weight: a tile that is lost or counted twice moves it by a per cent and more, its error is a few roundings."""
import pytest
import torch

from paper_2308_14129_amd import ops
from tests.paged import DEV, F64, TYPES, U, close, gather, gen_of, half, make_cache, make_table, tiny

pytestmark = [pytest.mark.gpu, pytest.mark.timeout(120)]

MIXED = [20_001, 3, 0, 9_999, 700, 64, 1, 12_345, 33, 5_000]
CASES = {
    # heads, group, dim, page, lengths, pages of a table (rows they hold, beside the lengths, are what the launch is planned by), window, layout
    "rows of 200 (100) bytes, two heads": (2, 1, 50, 20, MIXED, 3000, 0, "rows"),
    "three heads, one left over": (3, 2, 50, 20, MIXED, 3000, 0, "rows"),
    "five heads, three left over, whole pages": (5, 4, 36, 16, MIXED, 4000, 0, "rows"),
    "three heads of three blocks": (3, 70, 24, 16, MIXED[:6], 4000, 0, "rows"),
    "six heads, window": (6, 1, 40, 48, MIXED, 1300, 7_001, "kv"),
    "heads of whole lines, few sequences": (8, 8, 128, 16, [30_011, 17, 29_000, 30_011], 1900, 0, "rows"),
    "heads of whole lines, an odd number": (7, 1, 64, 20, [30_011, 17, 25_000], 1900, 0, "rows"),
    "two blocks of query heads, apart": (1, 40, 128, 16, MIXED, 2000, 0, "rows"),
    "two blocks of query heads, heads outside": (2, 40, 64, 20, MIXED[:4], 2000, 3_333, "heads"),
    "two blocks of query heads, together": (2, 40, 64, 16, [15_000, 70, 9_001], 3000, 0, "rows"),
    "wide heads": (3, 20, 200, 16, [9_000, 5, 4_100], 2000, 0, "rows"),
    "wide heads, rows one by one": (2, 2, 256, 12, [9_000, 5, 4_100], 7500, 0, "rows"),
    "many short ones among them": (4, 2, 36, 16, [1, 2, 40, 0] * 60 + [8_000, 16_001] + [5, 33] * 40, 1100, 0, "rows"),
}


def filled(case, t, gen):
    heads, group, dim, size, lengths, width, window, layout = case
    table, pages, _ = make_table(lengths, size, width, 1, gen)
    k_cache, v_cache = make_cache(pages, size, heads, dim, t, layout)
    for i, n in enumerate(lengths):
        p = torch.arange(n, device=DEV)
        first = max(0, n - window) if window else 0
        page = table[i].long()[p // size]
        k_cache[page, p % size] = (torch.randn(n, heads, dim, device=DEV, generator=gen) * 0.5).to(t)
        stretch = ((p - first).clamp(min=0) * dim // max(1, n - first)).clamp(max=dim - 1)
        v_cache[page, p % size] = torch.nn.functional.one_hot(stretch, dim).to(t)[:, None, :].expand(n, heads, dim)
    q = torch.randn(len(lengths), heads * group, dim, device=DEV, generator=gen).to(t)
    return q, k_cache, v_cache, table, torch.tensor(lengths, dtype=torch.int32, device=DEV)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("case", CASES)
def test_weights_of_stretches(case, dtype):
    heads, group, dim, size, lengths, width, window, _ = CASES[case]
    t, gen, scale = TYPES[dtype], gen_of(len(case)), dim**-0.5
    q, k_cache, v_cache, table, L = filled(CASES[case], t, gen)
    print(f"[attend] {case} {dtype}", flush=True)
    out, lse = ops.cache_attend(q, k_cache, v_cache, table, L, window=window, lse=True)
    torch.cuda.synchronize()
    # All terms are positive.  A score is off by d + 3 roundings of its terms, a weight by twice the largest of them, an exponential's 4 units and
    # its argument's rounding, in 16-bit types 2^-17 of itself; a sum by a rounding for every row that one wavefront goes through (a stretch of
    # the line, which is dealt to 1024 wavefronts or more) and for every factor and part: 1024 are more than there are here.
    for i, n in enumerate(lengths):
        first = max(0, n - window) if window else 0
        if n == first:
            assert not out[i].any() and (lse[i] == float("-inf")).all()
            continue
        k, ok = gather(k_cache, table, i, first, n)
        assert ok.all()
        Q, K = q[i].to(F64).view(heads, group, dim), k.permute(1, 0, 2).contiguous()
        s = scale * torch.matmul(Q, K.transpose(1, 2).contiguous())
        size_s = scale * torch.matmul(Q.abs(), K.abs().transpose(1, 2).contiguous())
        l = torch.logsumexp(s, -1)
        off = 2 * (dim + 3) * U * size_s.amax(-1) + 4 * U * (2 + s.amax(-1) - s.amin(-1)) + 1024 * U
        if t is not torch.float32:
            off = off + 2.0**-17
        stretch = (torch.arange(n - first, device=DEV) * dim // (n - first)).clamp(max=dim - 1)
        w = torch.zeros(heads, group, dim, dtype=F64, device=DEV).index_add_(2, stretch, torch.exp(s - l[..., None]))
        tol = w * (half(t) + 2.02 * off[..., None]) + tiny(t)
        close(out[i].view(heads, group, dim), w, tol, f"out of sequence {i}")
        close(lse[i].view(heads, group), l, off * 1.01 + 8 * U * (l.abs() + s.abs().amax(-1)), f"lse of sequence {i}")
    again = ops.cache_attend(q, k_cache, v_cache, table, L, window=window, lse=True)
    assert torch.equal(again[0], out) and torch.equal(again[1], lse)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("case", ["three heads, one left over", "heads of whole lines, an odd number", "two blocks of query heads, together", "wide heads, rows one by one"])
def test_windows_and_views_of_long_lines(case, dtype):
    """What a window does not see may be NaN; an output among other values leaves them as they are."""
    heads, group, dim, size, lengths, width, _, layout = CASES[case]
    t, gen, window = TYPES[dtype], gen_of(3), 4_000
    q, k_cache, v_cache, table, L = filled((heads, group, dim, size, lengths, width, window, layout), t, gen)
    want, sums = ops.cache_attend(q, k_cache, v_cache, table, L, window=window, lse=True)
    assert torch.isfinite(want).all()
    for i, n in enumerate(lengths):
        if n > window:
            p = torch.arange(n - window, device=DEV)
            page = table[i].long()[p // size]
            k_cache[page, p % size] = float("nan")
            v_cache[page, p % size] = float("inf")
    around = torch.full((len(lengths), heads * group + 2, dim + 3), 7.0, dtype=t, device=DEV)
    into = around[:, 1:-1, 1:-2]
    got, sums_got = ops.cache_attend(q, k_cache, v_cache, table, L, window=window, out=into, lse=True)
    assert got is into and torch.equal(into, want) and torch.equal(sums_got, sums)
    into.fill_(7.0)
    assert (around == 7.0).all()
    assert torch.isnan(ops.cache_attend(q, k_cache, v_cache, table, L)[L > window]).all()
