"""The optimiser's handle, its lists and streams on the device."""
import gc

import pytest
import torch

from paper_2308_14129_amd import ops

pytestmark = [pytest.mark.gpu, pytest.mark.timeout(120)]
DEV = "cuda:0"


def make(seed, n=5000):
    gen = torch.Generator(device=DEV).manual_seed(seed)
    lists = [[torch.randn(n, device=DEV, generator=gen) for _ in range(3)] for _ in range(3)]
    lists.append([torch.rand(n, device=DEV, generator=gen) for _ in range(3)])
    return lists, torch.zeros(1, dtype=torch.int64, device=DEV)


def test_changed_lists_do_not_change_the_steps():
    (p, g, m, v), step = make(1)
    want = ops.AdamW(p, g, m, v, step)
    want.step(1e-2, max_norm=1.0)
    want.step(1e-2, max_norm=1.0)
    torch.cuda.synchronize()
    (q, h, n, w), count = make(1)
    opt = ops.AdamW(q, h, n, w, count)
    mine = list(q)
    opt.step(1e-2, max_norm=1.0)
    for l in (q, h, n, w):
        l[0] = torch.full_like(l[0], 3.0)
        l[1].data = torch.full_like(l[1], 5.0)
        l.pop()
    gc.collect()
    junk = [torch.full((5000,), float("nan"), device=DEV) for _ in range(64)]  # (whatever was freed would be in here)
    opt.step(1e-2, max_norm=1.0)
    torch.cuda.synchronize()
    assert int(count) == 2 and len(junk) == 64
    assert torch.equal(mine[0], p[0]) and torch.equal(mine[2], p[2])


def test_memory_of_a_dropped_handle_waits_for_the_stream_that_steps():
    (p, g, m, v), step = make(2)
    opt = ops.AdamW(p, g, m, v, step)
    size, at = opt.ws.numel(), opt.ws.data_ptr()
    spare = [torch.empty(size, dtype=torch.uint8, device=DEV) for _ in range(16)]  # (so that the allocator need not ask the driver, which waits)
    opt.step(1e-2)
    del spare
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        torch.cuda._sleep(400_000_000)
        opt.step(1e-2)
    del opt
    gc.collect()
    taken = [torch.empty(size, dtype=torch.uint8, device=DEV) for _ in range(8)]
    busy = not side.query()
    assert busy and at not in [t.data_ptr() for t in taken]
    torch.cuda.synchronize()
    assert int(step) == 2
