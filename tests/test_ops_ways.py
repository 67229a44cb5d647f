"""Which calls of the loss keep their logits in registers (no GPU needed): the tests of that way are at sizes that take it."""
from ctypes import byref

import pytest

from tests.test_ops_refusals import HOST, lib, make_ce  # noqa: F401

DTYPES = {"fp32": 0, "bf16": 1, "fp16": 2}


def goes_narrow(lib, n, V, d, dtype, grad=True):  # noqa: F811
    """Of a call without a device (the addresses are never read)."""
    p = make_ce(rows=n, vocab=V, dim=d, dtype=DTYPES[dtype], ldx=d, ldw=d, lddx=d, lddw=d)
    if not grad:
        p.dx = p.dw = p.dbias = None
    way = lib.tig_debug_softmax_ce_narrow(byref(p))
    assert way >= 0
    return way == 1


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
def test_narrow_rows_with_many_logits(lib, dtype):  # noqa: F811
    for n, V in ((2048, 16_384), (2100, 16_000), (4, 1 << 23), (1 << 20, 32)):
        assert goes_narrow(lib, n, V, 128, dtype) and goes_narrow(lib, n, V, 1, dtype) and not goes_narrow(lib, n, V, 129, dtype)
        assert not goes_narrow(lib, n, V // 2, 128, dtype) and not goes_narrow(lib, n, V, 64, "fp32")
    assert goes_narrow(lib, 1, 1 << 17, 100, dtype, grad=False) and not goes_narrow(lib, 1, (1 << 17) - 1, 100, dtype, grad=False)
    assert not goes_narrow(lib, 100, 200_003, 128, dtype) and not goes_narrow(lib, 1, 1 << 17, 100, "fp32", grad=False)
