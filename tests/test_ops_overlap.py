"""Outputs on top of what the same call reads or writes are refused, before anything reaches a GPU (no GPU needed)."""
import ctypes
from ctypes import byref, c_size_t, c_void_p

import pytest

from paper_2308_14129_amd import ops, tig
from tests.test_ops_refusals import HOST, lib, make_ce, make_linear  # noqa: F401

MB = 1 << 20


def apart(p, names):
    for i, n in enumerate(names):
        setattr(p, n, HOST + (i + 1) * MB)
    return p


def forward(**kw):
    p = apart(make_linear(), ("x", "w", "y", "z", "bias", "residual"))
    p.ldr = 32
    for k, v in kw.items():
        setattr(p, k, v)
    return p


def backward(**kw):
    p = apart(make_linear(), ("x", "w", "y", "z", "dy", "dx", "dw", "dbias"))
    for k, v in kw.items():
        setattr(p, k, v)
    return p


X, W, Y, Z, BIAS, RES = (HOST + k * MB for k in range(1, 7))

# 100 rows of 64 -> 32 in bf16: rows of 128 and 64 bytes
FORWARD = [
    dict(y=X), dict(y=X + 100 * 128 - 2), dict(y=X - 99 * 64), dict(y=W), dict(y=W + 32 * 128 - 2), dict(y=BIAS), dict(y=BIAS + 62), dict(y=RES + 2),
    dict(y=RES, ldy=40), dict(y=RES + 64), dict(z=X), dict(z=W), dict(z=BIAS), dict(z=RES), dict(z=Y), dict(z=Y + 2), dict(y=X + 64, ldy=48), dict(y=X + 62, ldy=64),
    dict(y=X, ldy=64, ldx=64), dict(y=X + 128, ldy=128, ldx=128, in_dim=64, out_dim=65, ldw=65, ldz=65, ldr=65),
    dict(rows=3, y=X), dict(rows=1, y=X + 126), dict(rows=16, z=X + 2000),
]
# in place of y and z: DY is the fifth
DY, DX, DW, DB = (HOST + k * MB for k in range(5, 9))
BACKWARD = [
    dict(dx=DY), dict(dx=X), dict(dx=W), dict(dx=Z), dict(dw=DY), dict(dw=X), dict(dw=W + 2), dict(dw=Z), dict(dbias=DY + 64), dict(dbias=X), dict(dbias=W),
    dict(dbias=Z), dict(dx=DW), dict(dx=DB), dict(dw=DB), dict(dw=DX + 100 * 128 - 2),
]


@pytest.mark.parametrize("bad", FORWARD, ids=str)
def test_linear_forward_refuses_outputs_on_top_of_others(lib, bad):  # noqa: F811
    p, need = forward(**bad), c_size_t(0)
    assert lib.tig_linear_workspace_bytes(byref(p), 0, byref(need)) == tig.TIG_OK
    assert lib.tig_linear_forward(byref(p), HOST, need.value, None) == tig.TIG_EINVAL
    assert b"overlap" in lib.tig_last_error(None)


@pytest.mark.parametrize("bad", BACKWARD, ids=str)
def test_linear_backward_refuses_outputs_on_top_of_others(lib, bad):  # noqa: F811
    p, need = backward(**bad), c_size_t(0)
    assert lib.tig_linear_workspace_bytes(byref(p), 1, byref(need)) == tig.TIG_OK
    assert lib.tig_linear_backward(byref(p), HOST, need.value, None) == tig.TIG_EINVAL
    assert b"overlap" in lib.tig_last_error(None)


CE = ("x", "w", "bias", "labels", "row_scale", "loss", "lse", "mean", "dx", "dw", "dbias")


@pytest.mark.parametrize("out", CE[5:])
@pytest.mark.parametrize("on", CE)
def test_softmax_ce_refuses_outputs_on_top_of_others(lib, out, on):  # noqa: F811
    if out == on:
        return
    for shift in (0, 4):
        p, need = apart(make_ce(), CE), c_size_t(0)
        if shift and (out == "mean" or on == "mean"):
            continue
        setattr(p, out, getattr(p, on) + shift)
        assert lib.tig_softmax_ce_workspace_bytes(byref(p), byref(need)) == tig.TIG_OK
        assert lib.tig_softmax_ce_run(byref(p), HOST, need.value, None) == tig.TIG_EINVAL
        assert b"overlap" in lib.tig_last_error(None)


def make_two(eight=False):
    """Two tensors of 1000 fp32 elements, nothing of which overlaps; the counter and the workspace lie apart as well."""
    c = ops.tig_adamw_config(ctypes.sizeof(ops.tig_adamw_config), 8 if eight else 32, 0.9, 0.999, 1e-8, HOST)
    t = (ops.tig_adamw_tensor * 2)()
    at = MB
    for q in t:
        q.n = 1000
        for name in ("param", "grad", "m", "v", "master") + (("m_scale", "v_scale") if eight else ()):
            setattr(q, name, HOST + at)
            at += 4000
    return c, t


WORKSPACE = HOST + 64 * MB


@pytest.mark.parametrize("eight", [False, True])
@pytest.mark.parametrize("which", ["param", "m", "v", "master", "other's param", "other's m", "counter", "workspace", "param in workspace", "counter in m"])
def test_adamw_refuses_gradients_counter_or_workspace_on_what_it_writes(lib, which, eight):  # noqa: F811
    c, t = make_two(eight)
    if which == "counter":
        t[1].grad = HOST - 3996
    elif which == "workspace":
        t[0].grad = WORKSPACE - 3996
    elif which == "param in workspace":
        t[0].param = WORKSPACE
    elif which == "counter in m":
        c.step = t[1].m + 992
    else:
        on = t[1] if "other" in which else t[0]
        t[0].grad = getattr(on, which.split()[-1]) + (996 if eight and which.split()[-1] in "mv" else 3996)
    need, h = c_size_t(0), c_void_p(None)
    assert lib.tig_adamw_workspace_bytes(byref(c), t, 2, byref(need)) == tig.TIG_OK
    assert lib.tig_adamw_create(byref(c), t, 2, WORKSPACE, need.value, None, byref(h)) == tig.TIG_EINVAL and not h.value
    assert b"overlap" in lib.tig_last_error(None)
