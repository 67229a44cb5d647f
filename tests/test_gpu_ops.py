"""Operators of a trained head (ops.linear, ops.softmax_ce, ops.AdamW) against their formulas in 64 bits.

Tolerances are bounds: h = eps / 2 of a type for every rounding to it, 2^-24 for every fp32 operation of a chain, times the sum
of the terms' magnitudes.  An fp32 exponential is taken as 4 units in the last place off, with its argument's rounding on top."""
import math

import numpy as np
import pytest
import torch

from paper_2308_14129_amd import ops

pytestmark = [pytest.mark.gpu, pytest.mark.timeout(300)]

DEV = "cuda:0"
F64 = torch.float64
U = 2.0**-24
TYPES = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}


def half(t):
    return torch.finfo(t).eps / 2


def tiny(t):  # half of the smallest step
    return torch.finfo(t).tiny * torch.finfo(t).eps / 2


def rnd(gen, *shape, std=1.0, dtype=torch.float32, pad=0, shift=0):
    """Random tensor whose rows lie `pad` elements further apart than they have to, `shift` elements into their allocation."""
    n = int(np.prod(shape[:-1])) if len(shape) > 1 else 1
    ld = shape[-1] + pad
    base = torch.full((shift + n * ld,), float("nan"), dtype=dtype, device=DEV)
    t = base[shift:].view(*(shape[:-1]), ld)[..., : shape[-1]] if len(shape) > 1 else base[shift : shift + shape[-1]]
    t.copy_((torch.randn(*shape, device=DEV, generator=gen, dtype=torch.float64) * std).to(dtype))
    return t


def gen_of(seed):
    return torch.Generator(device=DEV).manual_seed(seed)


def close(got, ref, tol, name):
    # Beyond a type's range infinity is the right rounding: its largest value is (2 - eps) 2^e, and from half a step above that
    # on, (2 - eps / 2) 2^e, the nearest is 2^(e + 1), which the type does not have.  A value within tol of ref may lie there if
    # |ref| + tol does.  (fp16: 65520.)
    info = torch.finfo(got.dtype)
    edge = info.max / (2 - info.eps) * (2 - info.eps / 2)
    got = got.to(F64)
    over = torch.isinf(got) & (got * ref > 0) & (ref.abs() + tol >= edge)
    bad = ~((got - ref).abs() <= tol) & ~(torch.isnan(got) & torch.isnan(ref)) & ~(got == ref) & ~over
    if bad.any():
        i = tuple(int(v) for v in torch.nonzero(bad)[0])
        raise AssertionError(f"{name}: {int(bad.sum())} of {bad.numel()} off, first at {i}: {float(got[i])} for {float(ref[i])}, tolerance {float((tol + 0 * ref)[i])}")


def act64(z, act):
    if act == "relu":
        return z.clamp(min=0), (z > 0).to(F64)
    if act == "gelu":
        phi = 0.5 * torch.special.erfc(-z / math.sqrt(2))
        return z * phi, phi + z * torch.exp(-z * z / 2) / math.sqrt(2 * math.pi)
    if act == "silu":
        s = torch.sigmoid(z)
        return z * s, s + z * s * (1 - s)
    return z, torch.ones_like(z)


def check_linear(rows, k, n, dtype, act, bias, residual, seed, pad=0, shift=0, backward=True):
    print(f"[linear] {rows} x {k} x {n} {dtype} {act} pad {pad} shift {shift}", flush=True)
    t, gen = TYPES[dtype], gen_of(seed)
    h = half(t)
    x, w = rnd(gen, rows, k, dtype=t, pad=pad, shift=shift), rnd(gen, n, k, std=k**-0.5, dtype=t, pad=pad, shift=shift)
    b = rnd(gen, n, dtype=t, shift=shift) if bias else None
    res = rnd(gen, rows, n, dtype=t, pad=pad, shift=shift) if residual else None
    y, z = ops.linear(x, w, b, res, act, keep=True)
    torch.cuda.synchronize()
    X, W = x.to(F64), w.to(F64)
    Z = X @ W.t() + (b.to(F64) if bias else 0)
    size = X.abs() @ W.abs().t() + (b.to(F64).abs() if bias else 0)
    err = (k + 2) * U * size
    close(z, Z, h * Z.abs() + (1 + h) * err + tiny(t), "z")
    R = res.to(F64) if residual else torch.zeros((), dtype=F64, device=DEV)
    Y = act64(Z, act)[0] + R
    err_y = 1.2 * err + 16 * U * (Z.abs() + R.abs())  # slopes reach 1.13; erf, exp, quotient and sums
    close(y, Y, h * Y.abs() + (1 + h) * err_y + tiny(t), "y")
    assert torch.equal(y, ops.linear(x, w, b, res, act))  # without z: the same bits
    if not backward:
        return
    dy = rnd(gen, rows, n, dtype=t, pad=pad, shift=shift)
    dx, dw, db = ops.linear_backward(dy, x, w, z, act)
    torch.cuda.synchronize()
    DY = dy.to(F64)
    S = act64(z.to(F64), act)[1]
    DZ = DY * S
    err_dz = 16 * U * DY.abs() * (1 + z.to(F64).abs().clamp(max=4.0))  # (z exp(-z^2 / 2) and z g (1 - g) are below 1)
    off = h * DZ.abs() + (1 + h) * err_dz + tiny(t)
    DX, DW = DZ @ W, DZ.t() @ X
    close(dx, DX, h * DX.abs() + 1.01 * (off @ W.abs() + (n + 2) * U * (DZ.abs() @ W.abs())) + tiny(t), "dx")
    close(dw, DW, h * DW.abs() + 1.01 * (off.t() @ X.abs() + (rows + 2) * U * (DZ.abs().t() @ X.abs())) + tiny(t), "dw")
    DB = DZ.sum(0)
    close(db, DB, h * DB.abs() + 1.01 * (err_dz.sum(0) + 70 * U * DZ.abs().sum(0)) + tiny(t), "db")


LINEAR = [
    # few rows (the matrix straight into operands), around its limits
    (1, 64, 16), (1, 1, 1), (3, 100, 100), (16, 257, 33), (17, 1000, 77), (33, 48, 250), (64, 515, 129),
    # tiles, ragged in every direction
    (65, 64, 64), (129, 100, 100), (200, 172, 344), (300, 31, 65), (257, 1000, 515), (1000, 300, 100), (2500, 96, 2100),
]


@pytest.mark.parametrize("dtype", ["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("shape", LINEAR, ids=str)
def test_linear(shape, dtype):
    i = LINEAR.index(shape)
    act = ("none", "relu", "gelu", "silu")[i % 4]
    check_linear(*shape, dtype, act, bias=i % 3 != 0, residual=i % 2 == 1, seed=i)


@pytest.mark.parametrize("dtype", ["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("pad,shift", [(8, 0), (3, 0), (0, 1), (5, 3)])
def test_linear_strides_and_alignment(dtype, pad, shift):
    check_linear(130, 96, 72, dtype, "gelu", True, True, 7, pad, shift)
    check_linear(9, 96, 72, dtype, "silu", True, True, 8, pad, shift)


@pytest.mark.parametrize("act", ["none", "relu", "gelu", "silu"])
def test_linear_every_activation_in_every_form(act):
    check_linear(5, 40, 24, "fp32", act, True, True, 1)
    check_linear(140, 40, 24, "bf16", act, False, False, 2)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_linear_large_tiles_and_split_sums(dtype):
    check_linear(4096, 256, 4096, dtype, "gelu", True, True, 3)   # the largest tile in the forward pass
    check_linear(6000, 2048, 1100, dtype, "relu", True, False, 4)
    check_linear(80, 8192, 100, dtype, "none", True, False, 5)    # few tiles, a long sum


def test_linear_gradient_against_differences():
    gen = gen_of(11)
    x, w, b, dy = rnd(gen, 70, 20), rnd(gen, 12, 20), rnd(gen, 12), rnd(gen, 70, 12)
    for act in ("gelu", "silu"):
        y, z = ops.linear(x, w, b, None, act, keep=True)
        dx, dw, db = ops.linear_backward(dy, x, w, z, act)
        for name, t, g in (("x", x, dx), ("w", w, dw), ("b", b, db)):
            d = rnd(gen, *t.shape)
            f = lambda s: (act64((x.to(F64) + (s * d if name == "x" else 0)) @ (w.to(F64) + (s * d if name == "w" else 0)).t()  # noqa: E731
                                 + b.to(F64) + (s * d if name == "b" else 0), act)[0] * dy).sum()
            want = float(f(1e-5) - f(-1e-5)) / 2e-5
            got = float((g.to(F64) * d).sum())
            assert abs(got - want) <= 1e-4 * float((g.abs() * d.abs()).sum()), (act, name)


def test_linear_empty_parts_and_in_place_residual():
    gen = gen_of(5)
    x, w, b = rnd(gen, 0, 33), rnd(gen, 20, 33), rnd(gen, 20)
    y, z = ops.linear(x, w, b, None, "relu", keep=True)
    assert y.shape == (0, 20) and z.shape == (0, 20)
    dx, dw, db = ops.linear_backward(y, x, w, z, "relu")
    assert dx.shape == (0, 33) and not dw.any() and not db.any()
    for rows in (7, 150):
        x, res = rnd(gen, rows, 33), rnd(gen, rows, 20)
        want = ops.linear(x, w, b, res, "gelu")
        got = ops.linear(x, w, b, res, "gelu", out=res)
        assert got is res and torch.equal(got, want)
        z = ops.linear(x, w, b, None, "gelu", keep=True)[1]
        dy = rnd(gen, rows, 20)
        full = ops.linear_backward(dy, x, w, z, "gelu")
        for k in range(3):
            only = ops.linear_backward(dy, x, w, z, "gelu", dx=k == 0, dw=k == 1, dbias=k == 2)
            assert [o is not None for o in only] == [k == 0, k == 1, k == 2] and torch.equal(only[k], full[k])


def test_linear_infinities_stay_in_their_rows():
    gen = gen_of(6)
    for rows in (8, 100):
        x, w = rnd(gen, rows, 64, dtype=torch.bfloat16), rnd(gen, 48, 64, dtype=torch.bfloat16)
        clean = ops.linear(x, w, None, None, "relu")
        x[3, 5] = float("nan")
        x[6, 63] = float("inf")
        y = ops.linear(x, w, None, None, "relu")
        assert torch.isnan(y[3]).all()
        keep = [r for r in range(rows) if r not in (3, 6)]
        assert torch.equal(y[keep], clean[keep])


# --------------------------------------------------------------------------- softmax cross entropy


def reference_ce(x, w, labels, bias, row_scale, scale):
    X, W = x.to(F64), w.to(F64)
    logits = X @ W.t() + (bias.to(F64) if bias is not None else 0)
    n, V = logits.shape
    counted = (labels >= 0) & (labels < V)
    lse = torch.logsumexp(logits, 1) if n else logits.new_zeros(0)
    at = labels.long().clamp(0, V - 1).unsqueeze(1)
    l = logits.gather(1, at).squeeze(1)
    loss = torch.where(counted, lse - l, torch.zeros_like(lse))
    loss = torch.where(counted & (l == -math.inf), torch.full_like(loss, math.inf), loss)
    count = int(counted.sum())
    s = torch.where(counted, row_scale.to(F64) * scale if row_scale is not None else torch.full_like(lse, scale / max(1, count)), torch.zeros_like(lse))
    p = torch.exp(logits - torch.where(lse == -math.inf, torch.zeros_like(lse), lse).unsqueeze(1))
    hot = torch.zeros_like(p).scatter_(1, at, 1.0) * counted.unsqueeze(1)
    return logits, lse, loss, loss[counted].sum() / max(1, count), s, p, hot


def check_ce(n, V, d, dtype, bias=True, scale=1.0, ignored=0.2, weighted=False, seed=0, pad=0, shift=0, masked=0, spread=1.5, grad=True):
    print(f"[ce] {n} x {V} x {d} {dtype} ignored {ignored} weighted {weighted} pad {pad} shift {shift} masked {masked}", flush=True)
    t, gen = TYPES[dtype], gen_of(seed)
    h = half(t)
    x, w = rnd(gen, n, d, dtype=t, pad=pad, shift=shift), rnd(gen, V, d, std=spread * d**-0.5, dtype=t, pad=pad, shift=shift)
    b = rnd(gen, V, std=0.5, dtype=t, shift=shift) if bias else None
    labels = torch.randint(0, V, (n,), device=DEV, generator=gen, dtype=torch.int32)
    if masked:
        b[torch.randperm(V, device=DEV, generator=gen)[:masked]] = -math.inf
    drop = torch.rand(n, device=DEV, generator=gen) < ignored
    labels[drop] = torch.tensor([-1, V, -100, 2**31 - 1], device=DEV, dtype=torch.int32)[torch.arange(int(drop.sum()), device=DEV) % 4]
    rs = rnd(gen, n) if weighted else None
    r = ops.softmax_ce(x, w, labels, b, rs, scale, grad)
    torch.cuda.synchronize()
    logits, lse, loss, mean, s, p, hot = reference_ce(x, w, labels, b, rs, scale)
    X, W = x.to(F64), w.to(F64)
    size = X.abs() @ W.abs().t() + (b.to(F64).abs().nan_to_num(posinf=0) if bias else 0)
    err_l = (d + 2) * U * size
    near = torch.where(p > 0, (logits - lse.unsqueeze(1)).abs(), torch.zeros_like(p))
    # a logit's error, the exponential with its argument's rounding, up to 300 sums of a tile and a thousand parts
    err_lse = (p * (err_l + (8 + 2 * near) * U)).sum(1) + 400 * U + 4 * U * lse.abs().nan_to_num(neginf=0)
    close(r.lse, lse, err_lse, "lse")
    worst = err_l.amax(1) if n else err_lse
    close(r.loss, loss, torch.where(loss.isfinite(), err_lse + worst + 2 * U * (loss.abs() + lse.abs().nan_to_num(neginf=0)), torch.zeros_like(loss)), "loss")
    if n and torch.isfinite(mean):
        close(r.mean[0], mean, (err_lse + worst + 4 * U * lse.abs().nan_to_num(neginf=0)).mean() * n / max(1, int((s != 0).sum())) + 2 * U * mean.abs(), "mean")
    if not grad:
        return r
    P = (p - hot) * s.unsqueeze(1)
    top = s.abs().max() if n else torch.zeros((), dtype=F64, device=DEV)
    off = p * s.abs().unsqueeze(1) * (err_l + err_lse.unsqueeze(1) + (12 + 2 * near) * U) + (h + 4 * U) * P.abs()
    # below its smallest normal value a type's rounding is half of its smallest step, tiny(t), relative to S (fp16: 2^-14 of it,
    # as P is held times 2^14)
    off = off + top * (tiny(t) if dtype != "fp16" else 2.0**-25 * 2.0**-14)
    # a term of the matrix instructions' sums that is below the smallest normal fp32 value, 2^-126, may be taken as zero: at most
    # that much, times S, for each term (seen where it shows: 1.0e-38 = 0.85 * 2^-126 off for one such term)
    under = top * 2.0**-126
    DX, DW, DB = P @ W, P.t() @ X, P.sum(0)
    live = (s != 0).to(F64).unsqueeze(1)
    off, size_p = off * live, P.abs()
    if masked:
        off = off * torch.isfinite(b.to(F64))
        off = off + (h + 4 * U) * P.abs()
    close(r.dx, DX, h * DX.abs() + 1.01 * (off @ W.abs() + (V + 8) * U * (size_p @ W.abs())) + (V + 8) * under + tiny(t), "dx")
    close(r.dw, DW, h * DW.abs() + 1.01 * (off.t() @ X.abs() + (n + 8) * U * (size_p.t() @ X.abs())) + (n + 8) * under + tiny(t), "dw")
    if bias:
        close(r.dbias, DB, h * DB.abs() + 1.01 * (off.sum(0) + 70 * U * size_p.sum(0)) + tiny(t), "dbias")
    return r


CE = [(1, 1, 1), (1, 7, 5), (5, 100, 100), (200, 1000, 100), (65, 257, 33), (130, 64, 172), (33, 5000, 64), (300, 2049, 128), (70, 1030, 515)]


@pytest.mark.parametrize("dtype", ["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("shape", CE, ids=str)
def test_softmax_ce(shape, dtype):
    i = CE.index(shape)
    check_ce(*shape, dtype, bias=i % 2 == 0, scale=1024.0 if dtype == "fp16" else 1.0, ignored=0.0 if i < 3 else 0.2, weighted=i % 3 == 1, seed=i)


@pytest.mark.parametrize("dtype", ["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("pad,shift", [(8, 0), (3, 0), (0, 1), (5, 3)])
def test_softmax_ce_strides_and_alignment(dtype, pad, shift):
    check_ce(90, 500, 96, dtype, weighted=True, seed=21, pad=pad, shift=shift)


@pytest.mark.parametrize("dtype", ["fp32", "bf16", "fp16"])
def test_softmax_ce_masked_candidates(dtype):
    r = check_ce(40, 300, 48, dtype, seed=3, masked=250)
    assert torch.isinf(r.loss).any()  # labels among the masked ones
    r = check_ce(20, 100, 48, dtype, seed=4, masked=100, ignored=0.3)  # nothing left in any row
    assert (r.lse == -math.inf).all()


def test_softmax_ce_far_logits():
    check_ce(50, 400, 64, "fp32", seed=9, spread=60.0)  # logits of hundreds: one candidate takes all
    check_ce(50, 400, 64, "bf16", seed=9, spread=60.0)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_softmax_ce_in_several_pieces(dtype):
    # more rows than let all of P be held at once
    check_ce(20_000, 4000, 40, dtype, seed=13)


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("weighted,scale", [(False, 1.0), (True, 1.0), (False, -2.0), (True, -0.5)])
def test_softmax_ce_narrow_rows(dtype, weighted, scale):
    # 16-bit rows of at most 128 columns: around their tiles of 64 streamed and 192 or 256 own rows, and ranges of several tiles
    for i, shape in enumerate([(64, 64, 64), (65, 129, 65), (1000, 70, 128), (193, 4000, 127), (257, 900, 24), (2, 20_000, 100), (3000, 3, 8)]):
        check_ce(*shape, dtype, bias=i % 2 == 0, weighted=weighted, scale=scale * (512 if dtype == "fp16" else 1), seed=60 + i, masked=0)


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("n,V,d,bias", [(100, 200_003, 128, False), (100, 200_003, 128, True), (64, 150_001, 60, True), (700, 60_001, 100, True), (3, 300_000, 20, False)])
def test_softmax_ce_narrow_rows_over_many_tiles(n, V, d, bias, dtype):
    """Long ranges of streamed tiles: every tile has to be there before it is read."""
    check_ce(n, V, d, dtype, bias=bias, seed=n)


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("weighted,scale,pad,shift", [(False, 1.0, 0, 0), (True, -0.5, 8, 0), (False, -2.0, 0, 1), (True, 1.0, 3, 0)])
def test_softmax_ce_narrow_rows_and_many_logits(dtype, weighted, scale, pad, shift):
    # products of 2^25 logits and more: around tiles of 64 streamed and 192 or 256 own rows, one range and many
    shapes = [(2049, 16_385, 65), (4000, 8_400, 127), (64, 530_000, 64), (34_000, 1000, 128), (3, 11_200_000, 8), (1_200_000, 28, 24), (300, 112_000, 96)]
    for i, shape in enumerate(shapes):
        check_ce(*shape, dtype, bias=i % 2 == 0, weighted=weighted, scale=scale * (512 if dtype == "fp16" else 1), seed=80 + i, pad=pad, shift=shift)


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
def test_softmax_ce_narrow_rows_masked_candidates(dtype):
    r = check_ce(2100, 16_100, 48, dtype, seed=3, masked=16_000)
    assert torch.isinf(r.loss).any()  # labels among the masked ones
    r = check_ce(2100, 16_100, 100, dtype, seed=4, masked=16_100, ignored=0.3)  # nothing left in any row
    assert (r.lse == -math.inf).all()


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
def test_softmax_ce_narrow_rows_without_gradients(dtype):
    for i, shape in enumerate([(1, 131_072, 100), (7, 140_001, 33), (200, 131_100, 128)]):
        check_ce(*shape, dtype, bias=i != 2, seed=90 + i, grad=False)


def test_softmax_ce_wide_rows_in_several_pieces():
    check_ce(20_000, 4000, 136, "bf16", seed=14)
    check_ce(9000, 9000, 160, "fp16", seed=15, scale=1024.0, weighted=True)


@pytest.mark.parametrize("dtype", ["fp32", "bf16", "fp16"])
def test_softmax_ce_only_some_gradients(dtype):
    """Through the C entry: every subset of the gradients is what the whole set has."""
    import ctypes
    from ctypes import byref, c_size_t
    gen = gen_of(23)
    t = TYPES[dtype]
    lib = ops._lib()
    for n, V, d in ((90, 400, 100), (300, 130, 200), (2000, 300, 64), (2100, 16_000, 100), (300, 112_000, 64)):
        x, w, b = rnd(gen, n, d, dtype=t), rnd(gen, V, d, std=0.2, dtype=t), rnd(gen, V, dtype=t)
        labels = torch.randint(0, V, (n,), device=DEV, generator=gen, dtype=torch.int32)
        full = ops.softmax_ce(x, w, labels, b)
        for which in range(1, 8):
            out = [torch.full_like(q, 7.0) if which >> k & 1 else None for k, q in enumerate((x, w, b))]
            p = ops.tig_softmax_ce(ctypes.sizeof(ops.tig_softmax_ce), {"fp32": 0, "bf16": 1, "fp16": 2}[dtype], n, V, d)
            p.x, p.w, p.bias, p.labels, p.scale = x.data_ptr(), w.data_ptr(), b.data_ptr(), labels.data_ptr(), 1.0
            p.ldx = p.ldw = p.lddx = p.lddw = d
            p.dx, p.dw, p.dbias = [q.data_ptr() if q is not None else None for q in out]
            need = c_size_t(0)
            assert lib.tig_softmax_ce_workspace_bytes(byref(p), byref(need)) == 0
            ws = torch.empty(need.value, dtype=torch.uint8, device=DEV)
            assert lib.tig_softmax_ce_run(byref(p), ws.data_ptr(), need.value, torch.cuda.current_stream().cuda_stream) == 0
            for q, want in zip(out, (full.dx, full.dw, full.dbias)):
                assert q is None or torch.equal(q, want), (n, V, d, which)


def test_softmax_ce_rows_left_out_take_no_part():
    gen = gen_of(17)
    for t, n, V in ((torch.float32, 100, 333), (torch.bfloat16, 100, 333), (torch.bfloat16, 2100, 16_000)):
        x, w, b = rnd(gen, n, 64, dtype=t), rnd(gen, V, 64, std=0.1, dtype=t), rnd(gen, V, dtype=t)
        labels = torch.randint(0, V, (n,), device=DEV, generator=gen, dtype=torch.int32)
        labels[::3] = -1
        a = ops.softmax_ce(x, w, labels, b)
        x2 = x.clone()
        x2[::3] = float("nan")
        c = ops.softmax_ce(x2, w, labels, b)
        for name in ("loss", "mean", "dx", "dw", "dbias"):
            assert torch.equal(getattr(a, name), getattr(c, name)), name
        assert not a.dx[::3].any() and not a.loss[::3].any()
        none = ops.softmax_ce(x2, w, torch.full_like(labels, -1), b)
        for name in ("loss", "mean", "dx", "dw", "dbias"):
            assert not getattr(none, name).any(), name
        empty = ops.softmax_ce(x[:0], w, labels[:0], b)
        assert empty.loss.numel() == 0 and not empty.mean.any() and not empty.dw.any() and not empty.dbias.any()


def test_softmax_ce_gradient_against_differences():
    gen = gen_of(19)
    x, w, b = rnd(gen, 30, 24), rnd(gen, 90, 24, std=0.3), rnd(gen, 90)
    labels = torch.randint(0, 90, (30,), device=DEV, generator=gen, dtype=torch.int32)
    r = ops.softmax_ce(x, w, labels, b, scale=3.0)
    for t, g, name in ((x, r.dx, "x"), (w, r.dw, "w"), (b, r.dbias, "b")):
        d = rnd(gen, *t.shape).to(F64)

        def f(s):
            args = [q.to(F64) + (s * d if k == name else 0) for q, k in ((x, "x"), (w, "w"), (b, "b"))]
            logits = args[0] @ args[1].t() + args[2]
            return 3.0 * (torch.logsumexp(logits, 1) - logits.gather(1, labels.long().unsqueeze(1)).squeeze(1)).mean()

        want = float(f(1e-5) - f(-1e-5)) / 2e-5
        assert abs(float((g.to(F64) * d).sum()) - want) <= 1e-4 * float((g.abs() * d.abs()).sum()), name


# --------------------------------------------------------------------------- AdamW


def adam_tensors(gen, sizes, dtype, master, bits, shift=0):
    t = TYPES[dtype]
    s = dict(param=[], grad=[], m=[], v=[], master=[] if master else None, ms=[] if bits == 8 else None, vs=[] if bits == 8 else None)
    for n in sizes:
        p = rnd(gen, n, dtype=torch.float32, shift=shift)
        s["param"].append(rnd(gen, n, dtype=t, shift=shift).copy_(p))
        if master:
            s["master"].append(p)
        s["grad"].append(rnd(gen, n, dtype=t, std=0.1, shift=shift))
        m, v = rnd(gen, n, std=0.05, shift=shift), rnd(gen, n, std=0.1, shift=shift).square_()
        if bits == 8:
            nb = -(-n // 256)
            for name, x in (("m", m), ("v", v.sqrt())):
                base = torch.zeros(shift + n, dtype=torch.uint8, device=DEV).view(torch.float8_e4m3fn)
                full = torch.zeros(nb * 256, device=DEV)
                full[:n] = x
                top = full.view(nb, 256).abs().amax(1)
                scale = torch.where(top > 0, torch.exp2(torch.floor(torch.log2(top.double())) - 7).float(), torch.ones_like(top))
                base[shift:].copy_((full.view(nb, 256) / scale.unsqueeze(1)).view(-1)[:n].to(torch.float8_e4m3fn))
                s[name].append(base[shift:])
                s[name + "s"].append(scale)
        else:
            s["m"].append(m)
            s["v"].append(v)
    return s


def adam_object(s, step, **kw):
    return ops.AdamW(s["param"], s["grad"], s["m"], s["v"], step, masters=s["master"], m_scales=s["ms"], v_scales=s["vs"], **kw)


def widen(code, scale):
    n, nb = code.numel(), scale.numel()
    full = torch.zeros(nb * 256, dtype=F64, device=DEV)
    full[:n] = code.to(torch.float32).to(F64)
    return (full.view(nb, 256) * scale.to(F64).unsqueeze(1)).view(-1)[:n]


SIZES = [1, 5, 255, 256, 257, 4096, 4097, 10_000, 0, 100_003]


@pytest.mark.parametrize("dtype,master", [("fp32", False), ("bf16", True), ("bf16", False), ("fp16", True)])
@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("max_norm", [0.0, 0.5])
@pytest.mark.parametrize("shift", [0, 1])
def test_adamw(dtype, master, bits, max_norm, shift):
    gen = gen_of(bits + shift)
    s = adam_tensors(gen, SIZES, dtype, master, bits, shift)
    decay = [0.0 if i % 2 else 0.02 for i in range(len(SIZES))]
    step = torch.full((1,), 6, dtype=torch.int64, device=DEV)
    lr, b1, b2, eps, gs = 1e-2, 0.9, 0.99, 1e-8, 0.25
    before = {k: [q.clone() for q in v] if v else v for k, v in s.items()}
    opt = adam_object(s, step, betas=(b1, b2), eps=eps, weight_decay=decay)
    norm = opt.step(lr, grad_scale=gs, max_norm=max_norm)
    torch.cuda.synchronize()
    assert int(step) == 7
    h = half(TYPES[dtype])
    total = math.sqrt(sum(float((gs * g.to(F64)).square().sum()) for g in before["grad"]))
    c = gs
    if max_norm:
        assert abs(float(norm) - total) <= 2 * U * total
        c *= min(1.0, max_norm / total)
    for i, n in enumerate(SIZES):
        g = before["grad"][i].to(F64) * c
        p = (before["master"] if master else before["param"])[i].to(F64)
        if bits == 8:
            m0, v0 = widen(before["m"][i], before["ms"][i]), widen(before["v"][i], before["vs"][i]).square()
        else:
            m0, v0 = before["m"][i].to(F64), before["v"][i].to(F64)
        m, v = b1 * m0 + (1 - b1) * g, b2 * v0 + (1 - b2) * g * g
        size_m, update = (b1 * m0).abs() + ((1 - b1) * g).abs(), lr / (1 - b1**7) / ((v / (1 - b2**7)).sqrt() + eps)
        new = p * (1 - lr * decay[i]) - update * m
        err = 4 * U * p.abs() + update * (12 * U * size_m)
        if master:
            close(s["master"][i], new, err, f"master {i}")
            assert torch.equal(s["param"][i], s["master"][i].to(TYPES[dtype]))
        else:
            close(s["param"][i], new, (h if dtype != "fp32" else 0) * new.abs() + 1.01 * err, f"param {i}")
        if bits == 32:
            close(s["m"][i], m, 4 * U * size_m, f"m {i}")
            close(s["v"][i], v, 8 * U * v, f"v {i}")
            continue
        # a value of 8 bits is one of the two around it: less than a step of 2^-3 of its power of two (or of the smallest) away
        for name, want in (("m", m), ("v", v.sqrt())):
            scale = s[name + "s"][i]
            got = widen(s[name][i], scale)
            if n:
                assert (torch.log2(scale) == torch.round(torch.log2(scale))).all()
                top = torch.zeros(scale.numel() * 256, dtype=F64, device=DEV)
                top[:n] = want.abs()
                top = top.view(-1, 256).amax(1)
                low = (top / scale.to(F64)) * (1 + 8 * U)
                assert (low >= 128).all() and (top / scale.to(F64) * (1 - 8 * U) < 256).all()
                per = scale.to(F64).repeat_interleave(256)[:n]
                unit = torch.exp2(torch.floor(torch.log2((want.abs() / per).clamp(min=2.0**-6))) - 3) * per
                assert ((got - want).abs() <= unit * (1 + 1e-5)).all(), name
            if name == "v":
                assert (got[want > 1e-30] > 0).all()


def numpy_8bit(x, u, positive):
    """One block in float32, operation by operation."""
    top = np.abs(x).max()
    e0 = np.frexp(top)[1] - 8 if top > 0 else 0
    y = np.ldexp(np.abs(x), -e0).astype(np.float32)
    e = np.maximum(np.frexp(y)[1], -5) - 4
    q = np.ldexp(np.floor((np.ldexp(y, -e) + u).astype(np.float32)), e)
    q = np.where(x > 0, np.maximum(q, np.float32(2.0**-9)), q) if positive else np.copysign(q, x)
    return q.astype(np.float32), np.float32(np.ldexp(1.0, e0))


def test_adamw_8bit_codes_follow_their_rule_bit_for_bit():
    gen = gen_of(31)
    n = 3 * 256 + 77
    s = adam_tensors(gen, [n], "fp32", False, 8)
    s["grad"][0][300:512] = 0
    s["m"][0][256:512] = torch.zeros(256, device=DEV).to(torch.float8_e4m3fn)  # a block without anything
    s["v"][0][256:512] = torch.zeros(256, device=DEV).to(torch.float8_e4m3fn)
    s["grad"][0][256:300] = 0
    s["grad"][0][600] = 1e-12
    step = torch.zeros(1, dtype=torch.int64, device=DEV)
    opt = adam_object(s, step, betas=(0.9, 0.999))
    f = np.float32
    for t in range(1, 6):
        m0 = s["m"][0].float().cpu().numpy() * np.repeat(s["ms"][0].cpu().numpy(), 256)[:n]
        r0 = s["v"][0].float().cpu().numpy() * np.repeat(s["vs"][0].cpu().numpy(), 256)[:n]
        g = s["grad"][0].cpu().numpy()
        opt.step(1e-3)
        torch.cuda.synchronize()
        m = m0 * f(0.9) + g * f(1.0 - 0.9)
        r = np.sqrt((r0 * r0) * f(0.999) + (g * g) * f(1.0 - 0.999))
        place = np.arange(256, dtype=np.uint64) * 0x6A09E667 + t * 0x9E3779B9
        u = [(((place + k) & 0xFFFFFFFF) >> 8).astype(f) * f(2.0**-24) for k in (0, 0x80000000)]
        for b in range(4):
            at = slice(256 * b, min(n, 256 * b + 256))
            for x, uu, pos, code, scale in ((m, u[0], False, s["m"], s["ms"]), (r, u[1], True, s["v"], s["vs"])):
                q, sc = numpy_8bit(x[at], uu[: len(x[at])], pos)
                assert float(scale[0][b]) == sc
                np.testing.assert_array_equal(code[0][at].float().cpu().numpy(), q)


def test_adamw_8bit_averages_keep_moving():
    # 1 - beta2 = 0.001: a step changes sqrt(v) by far less than a code; over the steps it still follows
    n = 512
    z = lambda: torch.zeros(n, device=DEV)  # noqa: E731
    s = dict(param=[z()], grad=[torch.full((n,), 0.5, device=DEV)], m=[z().to(torch.float8_e4m3fn)], v=[z().to(torch.float8_e4m3fn)], master=None,
             ms=[torch.ones(2, device=DEV)], vs=[torch.ones(2, device=DEV)])
    opt = adam_object(s, torch.zeros(1, dtype=torch.int64, device=DEV))
    for _ in range(1000):
        opt.step(0.0)
    got = widen(s["v"][0], s["vs"][0]).mean()
    want = 0.5 * math.sqrt(1 - 0.999**1000)
    # every rounding is at most a code (1/8) off and they cancel over the steps: a fortieth is left room for
    assert abs(float(got) - want) <= want / 40
    assert abs(float(widen(s["m"][0], s["ms"][0]).mean()) - 0.5) <= 0.5 / 40


def test_adamw_skips_a_step_that_is_not_finite():
    gen = gen_of(37)
    s = adam_tensors(gen, [1000, 30], "fp32", False, 32)
    s["grad"][1][7] = float("inf")
    step = torch.full((1,), 3, dtype=torch.int64, device=DEV)
    before = {k: [q.clone() for q in v] for k, v in s.items() if v}
    opt = adam_object(s, step)
    norm = opt.step(1e-2, max_norm=1.0)
    assert not torch.isfinite(norm).any() and int(step) == 3
    for k, v in before.items():
        assert all(torch.equal(a, b) for a, b in zip(v, s[k])), k
    s["grad"][1][7] = 0.0
    assert torch.isfinite(opt.step(1e-2, max_norm=1.0)).all() and int(step) == 4


def test_adamw_without_tensors():
    step = torch.zeros(1, dtype=torch.int64, device=DEV)
    opt = ops.AdamW([], [], [], [], step)
    opt.step(1e-3, max_norm=1.0)
    assert int(step) == 1
    opt.close()


# --------------------------------------------------------------------------- together


def test_head_trained_in_a_captured_graph_equals_eager_steps():
    """Layer, loss, their gradients and the optimiser, as a training program runs them: replays of a captured step against
    eager steps, with other work of the program between them, and on a stream of its own."""
    def setup():
        gen = gen_of(41)
        t = torch.bfloat16
        e, W, b, C, cb = (rnd(gen, 150, 100, dtype=t), rnd(gen, 100, 100, std=0.1, dtype=t), rnd(gen, 100, dtype=t),
                          rnd(gen, 700, 100, std=0.1, dtype=t), rnd(gen, 700, dtype=t))
        labels = torch.randint(-1, 700, (150,), device=DEV, generator=gen, dtype=torch.int32)
        params = [W, b, C, cb]
        grads = [torch.zeros_like(q) for q in params]
        masters = [q.float() for q in params]
        m = [torch.zeros(q.numel(), device=DEV).to(torch.float8_e4m3fn) for q in params]
        v = [torch.zeros(q.numel(), device=DEV).to(torch.float8_e4m3fn) for q in params]
        sc = [[torch.ones(-(-q.numel() // 256), device=DEV) for q in params] for _ in range(2)]
        step = torch.zeros(1, dtype=torch.int64, device=DEV)
        opt = ops.AdamW(params, grads, m, v, step, masters=masters, m_scales=sc[0], v_scales=sc[1], weight_decay=0.01)

        def train():
            h, z = ops.linear(e, W, b, e, "gelu", keep=True)
            r = ops.softmax_ce(h, C, labels, cb)
            dx, dw, db = ops.linear_backward(r.dx, e, W, z, "gelu")
            for g, n in zip(grads, (dw, db, r.dw, r.dbias)):
                g.copy_(n)
            opt.step(1e-2, max_norm=1.0)
            return r.mean, dx

        return train, params + masters + m + v + sc[0] + sc[1] + [step]

    eager, state_a = setup()
    losses = [eager()[0].clone() for _ in range(8)]
    torch.cuda.synchronize()
    train, state_b = setup()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        for k in range(2):
            assert torch.equal(train()[0], losses[k])
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        mean, dx = train()
    torch.cuda.synchronize()
    for k in range(2, 8):
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(mean, losses[k]), k
        junk = torch.randn(300, 300, device=DEV)
        ops.linear(junk, junk, None, None, "relu")
        torch.cuda.synchronize()
    for a, b in zip(state_a, state_b):
        assert torch.equal(a.view(torch.uint8), b.view(torch.uint8))
    assert float(losses[-1]) < float(losses[0])


def test_results_do_not_change_from_call_to_call():
    gen = gen_of(43)
    for t in (torch.float32, torch.bfloat16):
        x, w, dy = rnd(gen, 3000, 200, dtype=t), rnd(gen, 150, 200, dtype=t), rnd(gen, 3000, 150, dtype=t)
        first = ops.linear_backward(dy, x, w)
        ce = ops.softmax_ce(x, w, torch.zeros(3000, dtype=torch.int32, device=DEV))
        for _ in range(3):
            assert all(torch.equal(a, b) for a, b in zip(first, ops.linear_backward(dy, x, w)))
            again = ops.softmax_ce(x, w, torch.zeros(3000, dtype=torch.int32, device=DEV))
            assert all(torch.equal(a, b) for a, b in zip(ce, again) if a is not None)


def test_large_calls_in_a_captured_graph_and_side_by_side_on_two_streams():
    gen = gen_of(61)
    t = torch.bfloat16

    def inputs():
        return (rnd(gen, 4096, 512, dtype=t), rnd(gen, 4096, 512, std=0.05, dtype=t), rnd(gen, 4096, dtype=t), rnd(gen, 4096, 4096, std=0.05, dtype=t),
                torch.randint(-1, 4096, (4096,), device=DEV, generator=gen, dtype=torch.int32), rnd(gen, 8200, 104, std=0.1, dtype=t))

    def calls(x, w, b, items, labels, narrow):
        y, z = ops.linear(x, w, b, activation="gelu", keep=True)
        r = ops.softmax_ce(y, items, labels)
        q = ops.softmax_ce(x[:, :96], narrow[:, :96], labels)  # narrow rows
        return (y, *r[:5], *q, *ops.linear_backward(r.dx, x, w, z, "gelu"))

    def same(got, want, what):
        for k, (p, q) in enumerate(zip(got, want)):
            assert (p is None) == (q is None) and (p is None or torch.equal(p, q)), (what, k)

    sets = [inputs() for _ in range(3)]
    eager = [calls(*s) for s in sets]
    held = [q.clone() for q in sets[0]]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        calls(*held)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = calls(*held)
    for turn in range(6):
        for q, new in zip(held, sets[turn % 3]):
            q.copy_(new)
        graph.replay()
        torch.cuda.synchronize()
        same(out, eager[turn % 3], f"replay {turn}")
        same(calls(*sets[(turn + 1) % 3]), eager[(turn + 1) % 3], f"eager beside replay {turn}")
    streams = [torch.cuda.Stream() for _ in range(2)]
    for st in streams:
        st.wait_stream(torch.cuda.current_stream())
    got = []
    for turn in range(4):
        with torch.cuda.stream(streams[turn % 2]):
            got.append(calls(*sets[turn % 3]))
    torch.cuda.synchronize()
    for turn in range(4):
        same(got[turn], eager[turn % 3], f"streams {turn}")
