"""Thin ctypes binding over the operators of a trained head in include/tig.h (tig_linear_*, tig_softmax_ce_*,
tig_adamw_*).  Argument marshalling only; PyTorch supplies device memory and the stream handle.  Every call enqueues on
the current stream of its tensors' device and does not synchronise.  No graph is recorded: linear() and softmax_ce() refuse
tensors that require a gradient where torch.is_grad_enabled(); linear_backward() and softmax_ce() give the gradients."""
from __future__ import annotations

import ctypes
import struct
from collections import namedtuple
from ctypes import POINTER, Structure, byref, c_double, c_float, c_int32, c_int64, c_size_t, c_uint32, c_void_p

import torch

from . import tig

ACTIVATIONS = tig.ACTIVATIONS


class tig_linear(Structure):
    _fields_ = [("struct_size", c_uint32), ("dtype", c_int32), ("activation", c_int32), ("reserved", c_int32),
                ("rows", c_int64), ("in_dim", c_int64), ("out_dim", c_int64), ("x", c_void_p), ("w", c_void_p),
                ("bias", c_void_p), ("residual", c_void_p), ("y", c_void_p), ("z", c_void_p), ("dy", c_void_p),
                ("dx", c_void_p), ("dw", c_void_p), ("dbias", c_void_p)] + [
                    (n, c_int64) for n in ("ldx", "ldw", "ldr", "ldy", "ldz", "lddy", "lddx", "lddw")]


class tig_softmax_ce(Structure):
    _fields_ = [("struct_size", c_uint32), ("dtype", c_int32), ("rows", c_int64), ("vocab", c_int64), ("dim", c_int64),
                ("x", c_void_p), ("w", c_void_p), ("bias", c_void_p), ("labels", c_void_p), ("row_scale", c_void_p),
                ("scale", c_float), ("reserved", c_int32), ("loss", c_void_p), ("lse", c_void_p), ("mean", c_void_p),
                ("dx", c_void_p), ("dw", c_void_p), ("dbias", c_void_p), ("ldx", c_int64), ("ldw", c_int64),
                ("lddx", c_int64), ("lddw", c_int64)]


class tig_adamw_tensor(Structure):
    _fields_ = [("param", c_void_p), ("grad", c_void_p), ("master", c_void_p), ("m", c_void_p), ("v", c_void_p),
                ("m_scale", c_void_p), ("v_scale", c_void_p), ("n", c_int64), ("dtype", c_int32),
                ("weight_decay", c_float)]


class tig_adamw_config(Structure):
    _fields_ = [("struct_size", c_uint32), ("state_bits", c_int32), ("beta1", c_double), ("beta2", c_double),
                ("eps", c_double), ("step", c_void_p)]


_ready = None


def _lib():
    global _ready
    if _ready is None:
        lib = tig.load_library()
        assert ctypes.sizeof(tig_linear) == 184 and ctypes.sizeof(tig_softmax_ce) == 160  # (what linear() and softmax_ce() pack)
        lib.tig_linear_workspace_bytes.argtypes = [c_void_p, c_int32, POINTER(c_size_t)]
        lib.tig_linear_forward.argtypes = [c_void_p, c_void_p, c_size_t, c_void_p]
        lib.tig_linear_backward.argtypes = [c_void_p, c_void_p, c_size_t, c_void_p]
        lib.tig_softmax_ce_workspace_bytes.argtypes = [c_void_p, POINTER(c_size_t)]
        lib.tig_softmax_ce_run.argtypes = [c_void_p, c_void_p, c_size_t, c_void_p]
        lib.tig_adamw_workspace_bytes.argtypes = [POINTER(tig_adamw_config), POINTER(tig_adamw_tensor), c_int64,
                                                  POINTER(c_size_t)]
        lib.tig_adamw_create.argtypes = [POINTER(tig_adamw_config), POINTER(tig_adamw_tensor), c_int64, c_void_p,
                                         c_size_t, c_void_p, POINTER(c_void_p)]
        lib.tig_adamw_step.argtypes = [c_void_p, c_double, c_double, c_double, c_void_p, c_void_p]
        lib.tig_adamw_destroy.argtypes = [c_void_p]
        lib.tig_adamw_destroy.restype = None
        for n in ("tig_linear_workspace_bytes", "tig_linear_forward", "tig_linear_backward", "tig_softmax_ce_workspace_bytes",
                  "tig_softmax_ce_run", "tig_adamw_workspace_bytes", "tig_adamw_create", "tig_adamw_step"):
            getattr(lib, n).restype = ctypes.c_int
        _ready = lib
    return _ready


def _check(rc):
    if rc != tig.TIG_OK:
        lib = tig.load_library()
        raise tig.TigError(rc, lib.tig_strerror(rc).decode() + " / " + lib.tig_last_error(None).decode())


def _refuse(text):
    raise tig.TigError(tig.TIG_EINVAL, text)


_codes = {torch.float32: 0, torch.bfloat16: 1, torch.float16: 2}


def _dtype_code(dtype):
    code = _codes.get(dtype)
    if code is None:
        _refuse(f"dtype {dtype} is none of float32, bfloat16, float16")
    return code


def _no_graph(name):
    if torch.is_grad_enabled():
        _refuse(f"{name} requires a gradient, but the operators record no graph: call them under torch.no_grad(), with linear_backward "
                "and softmax_ce's gradients for the way back")


def _matrix(t, rows, cols, dtype, device, name):
    """Address and row stride of a [rows x cols] tensor whose columns are adjacent."""
    if t is None:
        return 0, 0
    if t.shape != (rows, cols) or t.dtype is not dtype or t.device != device:
        _refuse(f"{name} is not a [{rows} x {cols}] tensor of {dtype} on {device}")
    ld, step = t.stride()
    if rows <= 1 and ld < cols:
        ld = cols
    if (step != 1 and cols > 1) or ld < cols:
        _refuse(f"{name}: columns have to be adjacent and rows may not overlap")
    if t.requires_grad:
        _no_graph(name)
    return t.data_ptr(), ld


def _vector(t, n, dtype, device, name):
    if t is None:
        return 0
    if t.shape != (n,) or t.dtype is not dtype or t.device != device or (n > 1 and t.stride(0) != 1):
        _refuse(f"{name} is not a contiguous [{n}] tensor of {dtype} on {device}")
    if t.requires_grad:
        _no_graph(name)
    return t.data_ptr()


class _On:
    """The device of a call's tensors made current where it is not, and its current stream."""
    __slots__ = ("guard", "index")

    def __init__(self, device):
        if device.type != "cuda":
            _refuse(f"tensors are on {device}, not on a GPU")
        self.index = device.index
        self.guard = None if device.index == torch._C._cuda_getDevice() else torch.cuda.device(device)

    def __enter__(self):
        if self.guard is not None:
            self.guard.__enter__()
        return torch._C._cuda_getCurrentRawStream(self.index)

    def __exit__(self, *a):
        if self.guard is not None:
            self.guard.__exit__(*a)


def _workspace(n, device):
    return torch.empty(n, dtype=torch.uint8, device=device) if n else None


def _activation(name):
    if name not in ACTIVATIONS:
        _refuse(f"activation {name!r} is none of {', '.join(ACTIVATIONS)}")
    return ACTIVATIONS[name]


# the structs as bytes: a small call is as long as its way to the launch
_linear_bytes = struct.Struct("=Iiii3q10Q8q").pack
_ce_bytes = struct.Struct("=Ii3q5Qfi6Q4q").pack
_FEW_ROWS = 16  # TIG_LINEAR_FEW_ROWS


def linear(x, w, bias=None, residual=None, activation="none", keep=False, out=None):
    """act(x w^T + bias) + residual for x [rows x in], w [out x in]; fp32, bf16 or fp16, sums in fp32.  With keep=True
    returns (y, z), z = x w^T + bias as linear_backward wants it.  out: where y goes; residual itself is fine, anything else that overlaps
    x, w, bias or residual is refused."""
    if x.dim() != 2 or w.dim() != 2:
        _refuse("x and w are matrices")
    rows, k = x.shape
    n = w.shape[0]
    dtype, dev = x.dtype, x.device
    code, act = _dtype_code(dtype), _activation(activation)
    px, ldx = _matrix(x, rows, k, dtype, dev, "x")
    pw, ldw = _matrix(w, n, k, dtype, dev, "w")
    pb = _vector(bias, n, dtype, dev, "bias")
    pr, ldr = _matrix(residual, rows, n, dtype, dev, "residual")
    y = out
    py, ldy = _matrix(y, rows, n, dtype, dev, "out")
    lib = _lib()
    with _On(dev) as stream:
        if y is None:
            y = torch.empty((rows, n), dtype=dtype, device=dev)
            py, ldy = y.data_ptr(), n
        z, pz = None, 0
        if keep:
            z = torch.empty((rows, n), dtype=dtype, device=dev)
            pz = z.data_ptr()
        p = _linear_bytes(184, code, act, 0, rows, k, n, px, pw, pb, pr, py, pz, 0, 0, 0, 0, ldx, ldw, ldr, ldy, n, 0, 0, 0)
        if rows <= _FEW_ROWS:
            _check(lib.tig_linear_forward(p, None, 0, stream))
        else:
            need = c_size_t(0)
            _check(lib.tig_linear_workspace_bytes(p, 0, byref(need)))
            ws = _workspace(need.value, dev)
            _check(lib.tig_linear_forward(p, ws.data_ptr() if ws is not None else None, need.value, stream))
    return (y, z) if keep else y


def linear_backward(dy, x, w, z=None, activation="none", dx=True, dw=True, dbias=True):
    """Gradients (dx, dw, dbias) of linear() for dy [rows x out]; None in the place of one that is not wanted.  z: what
    linear(keep=True) returned (not needed without an activation).  The residual's gradient is dy."""
    if dy.dim() != 2 or x.dim() != 2 or w.dim() != 2:
        _refuse("dy, x and w are matrices")
    rows, n = dy.shape
    k = w.shape[1]
    dtype, dev = dy.dtype, dy.device
    code, act = _dtype_code(dtype), _activation(activation)
    pd, lddy = _matrix(dy, rows, n, dtype, dev, "dy")
    px, ldx = _matrix(x, rows, k, dtype, dev, "x")
    pw, ldw = _matrix(w, n, k, dtype, dev, "w")
    pz, ldz = 0, 0
    if act:
        if z is None:
            _refuse("the backward pass of an activation needs z")
        pz, ldz = _matrix(z, rows, n, dtype, dev, "z")
    lib = _lib()
    with _On(dev) as stream:
        gx = torch.empty((rows, k), dtype=dtype, device=dev) if dx else None
        gw = torch.empty((n, k), dtype=dtype, device=dev) if dw else None
        gb = torch.empty(n, dtype=dtype, device=dev) if dbias else None
        p = _linear_bytes(184, code, act, 0, rows, k, n, px, pw, 0, 0, 0, pz, pd, gx.data_ptr() if dx else 0, gw.data_ptr() if dw else 0,
                          gb.data_ptr() if dbias else 0, ldx, ldw, 0, 0, ldz, lddy, k, k)
        need = c_size_t(0)
        _check(lib.tig_linear_workspace_bytes(p, 1, byref(need)))
        ws = _workspace(need.value, dev)
        _check(lib.tig_linear_backward(p, ws.data_ptr() if ws is not None else None, need.value, stream))
    return gx, gw, gb


SoftmaxCE = namedtuple("SoftmaxCE", "loss lse mean dx dw dbias")


def softmax_ce(x, w, labels, bias=None, row_scale=None, scale=1.0, grad=True):
    """Softmax cross entropy of rows x [rows x dim] over the candidates w [vocab x dim] (+ bias [vocab]) with int32
    labels [rows]; a label outside the vocabulary (-1) leaves its row out.  Returns SoftmaxCE(loss [rows], lse [rows],
    mean [1], dx, dw, dbias): loss and lse in fp32, gradients of scale * mean (or of scale * sum of row_scale * loss) in
    x's type, None without `grad`."""
    if x.dim() != 2 or w.dim() != 2:
        _refuse("x and w are matrices")
    rows, d = x.shape
    vocab = w.shape[0]
    dtype, dev = x.dtype, x.device
    code = _dtype_code(dtype)
    px, ldx = _matrix(x, rows, d, dtype, dev, "x")
    pw, ldw = _matrix(w, vocab, d, dtype, dev, "w")
    pb = _vector(bias, vocab, dtype, dev, "bias")
    pl = _vector(labels, rows, torch.int32, dev, "labels")
    ps = _vector(row_scale, rows, torch.float32, dev, "row_scale")
    lib = _lib()
    with _On(dev) as stream:
        stats = torch.empty(2 * rows + 1, dtype=torch.float32, device=dev)
        loss, lse, mean = stats[:rows], stats[rows : 2 * rows], stats[2 * rows :]
        at = stats.data_ptr()
        dx = torch.empty((rows, d), dtype=dtype, device=dev) if grad else None
        dw = torch.empty((vocab, d), dtype=dtype, device=dev) if grad else None
        db = torch.empty(vocab, dtype=dtype, device=dev) if grad and bias is not None else None
        p = _ce_bytes(160, code, rows, vocab, d, px, pw, pb, pl, ps, scale, 0, at, at + 4 * rows, at + 8 * rows, dx.data_ptr() if grad else 0,
                      dw.data_ptr() if grad else 0, db.data_ptr() if db is not None else 0, ldx, ldw, d, d)
        need = c_size_t(0)
        _check(lib.tig_softmax_ce_workspace_bytes(p, byref(need)))
        ws = _workspace(need.value, dev)
        _check(lib.tig_softmax_ce_run(p, ws.data_ptr(), need.value, stream))
    return SoftmaxCE(loss, lse, mean, dx, dw, db)


class AdamW:
    """AdamW over lists of tensors of any shape (contiguous).  States are the caller's: m and v in float32, or for 8 bits
    in torch.float8_e4m3fn with float32 scales, one for every 256 elements, m_scales and v_scales (v then holds sqrt(v)).
    step: int64 device tensor [1], the steps made so far.  masters: float32 tensors that are stepped in place of
    16-bit params, which receive their rounded copies (None, or None for a tensor, where there is none).

    The object steps the memory that it was given, and keeps it alive: a tensor put into one of the lists afterwards is not
    seen (gradients are copied into the given ones).  A captured step needs the object for as long as it is replayed."""

    def __init__(self, params, grads, m, v, step, masters=None, m_scales=None, v_scales=None, betas=(0.9, 0.999), eps=1e-8,
                 weight_decay=0.0):
        lists = dict(grads=grads, m=m, v=v)
        if masters is not None:
            lists["masters"] = masters
        if (m_scales is None) != (v_scales is None):
            _refuse("m_scales and v_scales go together")
        eight = m_scales is not None
        if eight:
            lists.update(m_scales=m_scales, v_scales=v_scales)
        for name, l in lists.items():
            if len(l) != len(params):
                _refuse(f"{len(params)} params, but {len(l)} {name}")
        decay = [float(weight_decay)] * len(params) if isinstance(weight_decay, (int, float)) else list(weight_decay)
        if len(decay) != len(params):
            _refuse(f"{len(params)} params, but {len(decay)} weight decays")
        if not isinstance(step, torch.Tensor) or step.dtype != torch.int64 or step.numel() != 1:
            _refuse("step is an int64 tensor of one element")
        self.device = step.device
        state = torch.float8_e4m3fn if eight else torch.float32
        table = (tig_adamw_tensor * max(1, len(params)))()

        def flat(t, n, dtype, name, i):
            if t.numel() != n or t.dtype != dtype or t.device != self.device or not t.is_contiguous():
                _refuse(f"{name}[{i}] is not a contiguous tensor of {n} {dtype} on {self.device}")
            return t.data_ptr()

        for i, q in enumerate(params):
            n, e = q.numel(), table[i]
            e.param, e.n, e.dtype, e.weight_decay = flat(q, n, q.dtype, "params", i), n, _dtype_code(q.dtype), decay[i]
            e.grad = flat(grads[i], n, q.dtype, "grads", i)
            if masters is not None and masters[i] is not None:
                e.master = flat(masters[i], n, torch.float32, "masters", i)
            e.m, e.v = flat(m[i], n, state, "m", i), flat(v[i], n, state, "v", i)
            if eight:
                e.m_scale = flat(m_scales[i], -(-n // 256), torch.float32, "m_scales", i)
                e.v_scale = flat(v_scales[i], -(-n // 256), torch.float32, "v_scales", i)
        # The handle has these tensors' addresses: aliases of them, whatever becomes of the caller's lists and tensors.
        self.kept = tuple(t.detach() for l in (params, *lists.values(), (step,)) for t in l if t is not None)
        self.norm = torch.zeros(1, dtype=torch.float32, device=self.device)
        cfg = tig_adamw_config(ctypes.sizeof(tig_adamw_config), 8 if eight else 32, betas[0], betas[1], eps, step.data_ptr())
        self.lib = _lib()
        h, need = c_void_p(None), c_size_t(0)
        with _On(self.device) as stream:
            self.stream = stream  # (the one that ws and norm belong to)
            _check(self.lib.tig_adamw_workspace_bytes(byref(cfg), table, len(params), byref(need)))
            self.ws = _workspace(need.value, self.device)
            _check(self.lib.tig_adamw_create(byref(cfg), table, len(params), self.ws.data_ptr(), need.value, stream, byref(h)))
        self.handle = h

    def step(self, lr, grad_scale=1.0, max_norm=0.0):
        """Enqueues one step; returns the device tensor [1] that receives the gradients' norm (with max_norm > 0)."""
        with _On(self.device) as stream:
            if stream != self.stream:  # (the allocator has to know, should the object go before the step has run)
                other = torch.cuda.current_stream(self.device)
                self.ws.record_stream(other)
                self.norm.record_stream(other)
            _check(self.lib.tig_adamw_step(self.handle, lr, grad_scale, max_norm, self.norm.data_ptr(), stream))
        return self.norm

    def close(self):
        if getattr(self, "handle", None):
            self.lib.tig_adamw_destroy(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass
