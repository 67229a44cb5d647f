"""Scores of -infinity in the attention over a paged cache: rows that carry no weight for one query, and count for the queries beside it."""
import pytest
import torch

from paper_2308_14129_amd import ops
from tests.paged import DEV, TYPES, attention, close, gen_of, make_cache, make_table

pytestmark = [pytest.mark.gpu, pytest.mark.timeout(120)]

# which rows of a sequence of n score -infinity for the first queries of a head
LOW = {
    "the first tile": lambda n: range(0, min(n - 1, 36)),
    "the last row, alone in its tile": lambda n: [n - 1],
    "whole tiles between others": lambda n: range(min(n - 1, 64), min(n - 1, 128)),
    "all but the last": lambda n: range(0, n - 1),
    "all but the first": lambda n: range(1, n),
}


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("group", [1, 2, 4, 17])
@pytest.mark.parametrize("size, width", [(16, 12), (16, 17), (12, 23), (16, 400), (12, 500)])  # one launch; the line of tiles over many workgroups
@pytest.mark.parametrize("low", LOW)
def test_rows_of_no_weight_for_one_query(low, size, width, group, dtype):
    t, gen, heads, dim = TYPES[dtype], gen_of(size + group), 2, 64
    lengths = [n for n in (257, 161, 65, 33, 17, 2) if n <= size * width]
    rows_of = [[r for r in LOW[low](n)] for n in lengths]
    table, pages, _ = make_table(lengths, size, width, 1, gen)
    k_cache, v_cache = make_cache(pages, size, heads, dim, t, "rows")
    # without the rows of no weight, and with them as the other queries see them
    left = [n - len(r) for n, r in zip(lengths, rows_of)]
    table_a, pages_a, _ = make_table(left, size, width, 1, gen)
    k_a, v_a = make_cache(pages_a, size, heads, dim, t, "rows")
    # q times k is beyond fp32's range in the first column (fp16 does not reach it: infinite keys, which nobody's zero meets)
    half_range = t is torch.float16
    for i, n in enumerate(lengths):
        p = torch.arange(n, device=DEV)
        k = torch.randn(n, heads, dim, device=DEV, generator=gen).to(t)
        v = torch.randn(n, heads, dim, device=DEV, generator=gen).to(t)
        k[..., 0] = 0.0
        stays = torch.ones(n, dtype=torch.bool, device=DEV)
        stays[rows_of[i]] = False
        at = torch.arange(left[i], device=DEV)
        page = table_a[i].long()[at // size]
        k_a[page, at % size], v_a[page, at % size] = k[stays], v[stays]
        k[~stays, :, 0] = float("-inf") if half_range else -3e38
        page = table[i].long()[p // size]
        k_cache[page, p % size], v_cache[page, p % size] = k, v
    q = torch.randn(len(lengths), heads * group, dim, device=DEV, generator=gen).to(t)
    first = torch.arange(heads * group, device=DEV) % group < (group if half_range else (group + 1) // 2)
    q[..., 0] = torch.where(first, 40.0, 0.0).to(t)
    i32 = dict(dtype=torch.int32, device=DEV)
    L = torch.tensor(lengths, **i32)
    print(f"[attend] -infinity: {low}, pages of {size}, {width} of them, group {group}, {dtype}", flush=True)
    out, lse = ops.cache_attend(q, k_cache, v_cache, table, L, lse=True)
    torch.cuda.synchronize()
    ref, rl, tol, tl = attention(q, k_a, v_a, table_a, torch.tensor(left, **i32), dim**-0.5, 0)
    close(out[:, first], ref[:, first], tol[:, first], "out")
    close(lse[:, first], rl[:, first], tl[:, first], "lse")
    if not half_range:
        k_cache[..., 0] = 0.0
        ref, rl, tol, tl = attention(q, k_cache, v_cache, table, L, dim**-0.5, 0)
        close(out[:, ~first], ref[:, ~first], tol[:, ~first], "out beside them")
        close(lse[:, ~first], rl[:, ~first], tl[:, ~first], "lse beside them")
