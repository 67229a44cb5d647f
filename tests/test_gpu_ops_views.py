"""Tensors of one call that are views of one buffer without sharing an element are taken."""
import pytest
import torch

from paper_2308_14129_amd import ops, tig

pytestmark = [pytest.mark.gpu, pytest.mark.timeout(120)]
DEV = "cuda:0"


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("rows", [1, 9, 200])
def test_views_of_one_buffer(rows, dtype):
    gen = torch.Generator(device=DEV).manual_seed(rows)
    w, b = torch.randn(40, 64, device=DEV, generator=gen).to(dtype), torch.randn(40, device=DEV, generator=gen).to(dtype)
    flat = torch.randn(2 * rows, 160, device=DEV, generator=gen).to(dtype)
    x, res = flat[:rows, 3:67].clone(), flat[:rows, 110:150].clone()
    want, z = ops.linear(x, w, b, res, "gelu", keep=True)
    # side by side
    for a, c in ((67, 67), (67, 109), (0, 43)):
        buf = flat.clone()
        lo = 3 if a else 43
        buf[:rows, lo : lo + 64] = x
        got = ops.linear(buf[:rows, lo : lo + 64], w, b, res, "gelu", out=buf[:rows, a if a == 0 else c : (a if a == 0 else c) + 40])
        assert torch.equal(got, want) and torch.equal(buf[:rows, lo : lo + 64], x)
    # every other row
    buf = torch.zeros(2 * rows, 64, device=DEV, dtype=dtype)
    buf[::2] = x
    got = ops.linear(buf[::2], w, b, res, "gelu", out=buf[1::2, :40])
    assert torch.equal(got, want) and torch.equal(buf[::2], x) and not buf[1::2, 40:].any()
    # one behind the other, and the residual itself
    buf = torch.zeros(rows * (64 + 40), device=DEV, dtype=dtype)
    buf[: rows * 64] = x.flatten()
    got = ops.linear(buf[: rows * 64].view(rows, 64), w, b, res, "gelu", out=buf[rows * 64 :].view(rows, 40))
    assert torch.equal(got, want)
    r = res.clone()
    assert torch.equal(ops.linear(x, w, b, r, "gelu", out=r), want)
    for bad in (x[:, :40], w[:1].expand(rows, 64)[:, :40] if rows == 1 else x[:, 24:]):
        before = bad.clone()
        with pytest.raises(tig.TigError) as e:
            ops.linear(x, w, b, res, "gelu", out=bad)
        assert e.value.status == tig.TIG_EINVAL and torch.equal(bad, before)
    # gradients: dy and x side by side
    buf = flat.clone()
    buf[:rows, :64], buf[:rows, 64:104] = x, res
    for p, q in zip(ops.linear_backward(buf[:rows, 64:104], buf[:rows, :64], w, z, "gelu"), ops.linear_backward(res, x, w, z, "gelu")):
        assert torch.equal(p, q)
