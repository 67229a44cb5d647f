"""What the operators of a trained head refuse, before anything reaches a GPU (no GPU needed)."""
import ctypes
import os
from ctypes import byref, c_size_t, c_void_p

import pytest

from paper_2308_14129_amd import ops, tig


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(tig.LIB_PATH):
        from paper_2308_14129_amd import build
        build.build()
    return ops._lib()


HOST = 0x10000  # an address that is never read: every call here is refused first


def make_linear(**kw):
    p = ops.tig_linear(ctypes.sizeof(ops.tig_linear), 1, 1, 0, 100, 64, 32)
    for n in ("x", "w", "y", "z", "dy", "dx", "dw", "dbias"):
        setattr(p, n, HOST)
    p.ldx = p.ldw = p.lddx = p.lddw = 64
    p.ldy = p.ldz = p.lddy = p.ldr = 32
    for k, v in kw.items():
        setattr(p, k, v)
    return p


@pytest.mark.parametrize("bad", [
    dict(struct_size=8), dict(dtype=3), dict(dtype=-1), dict(activation=4), dict(activation=-1), dict(reserved=1), dict(rows=-1),
    dict(rows=2**31), dict(rows=2**26 + 1), dict(in_dim=0), dict(out_dim=0), dict(in_dim=2**20 + 1, ldx=2**21, ldw=2**21), dict(ldx=63), dict(ldw=63), dict(ldy=31),
    dict(ldz=31), dict(residual=HOST, ldr=31), dict(ldx=2**22 + 1), dict(x=None), dict(w=None), dict(y=None), dict(x=HOST + 1), dict(bias=HOST + 1),
    dict(y=HOST + 1)], ids=str)
def test_linear_forward_refuses(lib, bad):
    need = c_size_t(0)
    p = make_linear(**bad)
    assert lib.tig_linear_workspace_bytes(byref(p), 0, byref(need)) == tig.TIG_EINVAL
    assert lib.tig_linear_forward(byref(p), HOST, 1 << 40, None) == tig.TIG_EINVAL
    assert b"linear" in lib.tig_last_error(None)


@pytest.mark.parametrize("bad", [
    dict(dy=None), dict(z=None), dict(x=None), dict(w=None), dict(lddy=31), dict(lddx=63), dict(lddw=63), dict(ldz=31), dict(dx=HOST + 1),
    dict(dtype=0, dy=HOST + 2)], ids=str)
def test_linear_backward_refuses(lib, bad):
    p = make_linear(**bad)
    assert lib.tig_linear_backward(byref(p), HOST, 1 << 40, None) == tig.TIG_EINVAL


def test_linear_workspace_is_checked(lib):
    need = c_size_t(0)
    p = make_linear()
    assert lib.tig_linear_workspace_bytes(byref(p), 1, byref(need)) == tig.TIG_OK and need.value > 0
    assert lib.tig_linear_workspace_bytes(byref(p), 1, None) == tig.TIG_EINVAL
    assert lib.tig_linear_workspace_bytes(None, 1, byref(need)) == tig.TIG_EINVAL
    assert lib.tig_linear_backward(byref(p), HOST, need.value - 1, None) == tig.TIG_ENOSPACE
    assert lib.tig_linear_backward(byref(p), HOST + 128, need.value, None) == tig.TIG_EINVAL
    assert lib.tig_linear_backward(byref(p), None, need.value, None) == tig.TIG_EINVAL
    p = make_linear(rows=0, x=None, dy=None)
    assert lib.tig_linear_forward(byref(p), None, 0, None) == tig.TIG_OK  # nothing to do


def make_ce(**kw):
    p = ops.tig_softmax_ce(ctypes.sizeof(ops.tig_softmax_ce), 1, 100, 1000, 64)
    for n in ("x", "w", "labels", "loss", "dx", "dw"):
        setattr(p, n, HOST)
    p.scale = 1.0
    p.ldx = p.ldw = p.lddx = p.lddw = 64
    for k, v in kw.items():
        setattr(p, k, v)
    return p


@pytest.mark.parametrize("bad", [
    dict(struct_size=8), dict(dtype=9), dict(reserved=1), dict(rows=-1), dict(rows=2**24 + 1), dict(vocab=0), dict(vocab=2**31), dict(vocab=2**28 + 1), dict(dim=0),
    dict(dim=2**16 + 1, ldx=2**17, ldw=2**17, lddx=2**17, lddw=2**17), dict(x=None), dict(w=None), dict(labels=None), dict(ldx=63), dict(ldw=63),
    dict(lddx=63), dict(lddw=63), dict(w=HOST + 1), dict(labels=HOST + 2), dict(loss=HOST + 2), dict(scale=float("nan")), dict(scale=float("inf"))], ids=str)
def test_softmax_ce_refuses(lib, bad):
    p, need = make_ce(**bad), c_size_t(0)
    assert lib.tig_softmax_ce_workspace_bytes(byref(p), byref(need)) == tig.TIG_EINVAL
    assert lib.tig_softmax_ce_run(byref(p), HOST, 1 << 40, None) == tig.TIG_EINVAL


def test_softmax_ce_workspace_is_checked(lib):
    p, need = make_ce(), c_size_t(0)
    assert lib.tig_softmax_ce_workspace_bytes(byref(p), byref(need)) == tig.TIG_OK and need.value > 0
    assert lib.tig_softmax_ce_run(byref(p), HOST, need.value - 1, None) == tig.TIG_ENOSPACE
    assert lib.tig_softmax_ce_run(byref(p), None, need.value, None) == tig.TIG_EINVAL
    assert lib.tig_softmax_ce_run(byref(p), HOST + 64, need.value, None) == tig.TIG_EINVAL
    assert lib.tig_softmax_ce_run(None, HOST, need.value, None) == tig.TIG_EINVAL


def make_adamw(cfg=(), **kw):
    c = ops.tig_adamw_config(ctypes.sizeof(ops.tig_adamw_config), 32, 0.9, 0.999, 1e-8, HOST)
    for k, v in dict(cfg).items():
        setattr(c, k, v)
    t = (ops.tig_adamw_tensor * 1)()
    t[0].param = t[0].grad = t[0].m = t[0].v = HOST
    t[0].n = 100
    for k, v in kw.items():
        setattr(t[0], k, v)
    return c, t


@pytest.mark.parametrize("bad", [
    dict(cfg=dict(struct_size=8)), dict(cfg=dict(state_bits=16)), dict(cfg=dict(beta1=1.0)), dict(cfg=dict(beta2=-0.1)), dict(cfg=dict(eps=0.0)),
    dict(cfg=dict(eps=1e-60)), dict(cfg=dict(step=None)), dict(cfg=dict(step=HOST + 4)), dict(dtype=5), dict(n=-1), dict(param=None), dict(grad=None),
    dict(m=None), dict(v=None), dict(m_scale=HOST), dict(cfg=dict(state_bits=8)), dict(weight_decay=-1.0), dict(weight_decay=float("nan")),
    dict(param=HOST + 2), dict(m=HOST + 2), dict(master=HOST + 2)], ids=str)
def test_adamw_refuses(lib, bad):
    c, t = make_adamw(**bad)
    need, h = c_size_t(0), c_void_p(None)
    assert lib.tig_adamw_workspace_bytes(byref(c), t, 1, byref(need)) == tig.TIG_EINVAL
    assert lib.tig_adamw_create(byref(c), t, 1, HOST, 1 << 40, None, byref(h)) == tig.TIG_EINVAL and not h.value
    assert b"adamw" in lib.tig_last_error(None)


def test_adamw_workspace_and_numbers_are_checked(lib):
    c, t = make_adamw()
    need, h = c_size_t(0), c_void_p(None)
    assert lib.tig_adamw_workspace_bytes(byref(c), t, 1, byref(need)) == tig.TIG_OK and need.value > 0
    assert lib.tig_adamw_create(byref(c), t, 1, HOST, need.value - 1, None, byref(h)) == tig.TIG_ENOSPACE
    assert lib.tig_adamw_create(byref(c), t, 1, None, need.value, None, byref(h)) == tig.TIG_EINVAL
    assert lib.tig_adamw_create(byref(c), t, 1, HOST, need.value, None, None) == tig.TIG_EINVAL
    assert lib.tig_adamw_create(byref(c), t, -1, HOST, need.value, None, byref(h)) == tig.TIG_EINVAL
    assert lib.tig_adamw_step(None, 1e-3, 1.0, 0.0, None, None) == tig.TIG_EINVAL


@pytest.mark.parametrize("which", ["param", "m", "v", "master", "between tensors", "v_scale"])
def test_adamw_refuses_arrays_that_overlap(lib, which):
    eight = which == "v_scale"
    c, _ = make_adamw(cfg=dict(state_bits=8 if eight else 32))
    t = (ops.tig_adamw_tensor * 2)()
    at = 1 << 20
    for q in t:
        q.n, q.grad = 1000, HOST  # (gradients may be shared)
        for name in ("param", "m", "v", "master") + (("m_scale", "v_scale") if eight else ()):
            setattr(q, name, HOST + at)
            at += 4000
    if which == "between tensors":
        t[1].param = t[0].param + 3996
    elif which == "v_scale":
        t[0].v_scale = t[0].m_scale + 12
    else:
        setattr(t[1], which, getattr(t[0], which))
    need, h = c_size_t(0), c_void_p(None)
    assert lib.tig_adamw_workspace_bytes(byref(c), t, 2, byref(need)) == tig.TIG_OK
    assert lib.tig_adamw_create(byref(c), t, 2, HOST, need.value, None, byref(h)) == tig.TIG_EINVAL and not h.value
    assert b"overlap" in lib.tig_last_error(None)


def test_python_entry_points_refuse():
    import torch
    x, w = torch.zeros(4, 8), torch.zeros(6, 8)
    labels = torch.zeros(4, dtype=torch.int32)
    for call in (
        lambda: ops.linear(x, w),                                             # not on a GPU
        lambda: ops.linear(x[0], w),
        lambda: ops.linear(x, torch.zeros(6, 9)),
        lambda: ops.linear(x, w.double()),
        lambda: ops.linear(x.double(), w.double()),
        lambda: ops.linear(x, w, activation="tanh"),
        lambda: ops.linear(x, w, bias=torch.zeros(5)),
        lambda: ops.linear(x.t().contiguous().t(), w),                        # columns not adjacent
        lambda: ops.linear(x[:1].expand(4, 8), w),                            # rows on top of each other
        lambda: ops.linear_backward(torch.zeros(4, 6), x, w, None, "relu"),
        lambda: ops.softmax_ce(x, w, labels.long()),
        lambda: ops.softmax_ce(x, w, labels[:3]),
        lambda: ops.softmax_ce(x, w, labels, bias=torch.zeros(4)),
        lambda: ops.AdamW([x], [x], [x], [x], torch.zeros(1, dtype=torch.int64)),
        lambda: ops.AdamW([x], [x], [x], [], torch.zeros(1, dtype=torch.int64)),
        lambda: ops.AdamW([x], [w], [x], [x], torch.zeros(1, dtype=torch.int64)),
        lambda: ops.AdamW([x], [x], [x], [x], torch.zeros(1)),
    ):
        with pytest.raises(tig.TigError) as e:
            call()
        assert e.value.status == tig.TIG_EINVAL


def test_struct_sizes():
    assert ctypes.sizeof(ops.tig_linear) == 16 + 3 * 8 + 10 * 8 + 8 * 8
    assert ctypes.sizeof(ops.tig_softmax_ce) == 8 + 3 * 8 + 5 * 8 + 8 + 6 * 8 + 4 * 8
    assert ctypes.sizeof(ops.tig_adamw_tensor) == 72 and ctypes.sizeof(ops.tig_adamw_config) == 40
