"""Thin ctypes binding over the operators of a trained head in include/tig.h (tig_linear_*, tig_softmax_ce_*,
tig_adamw_*).  Argument marshalling only; PyTorch supplies device memory and the stream handle.  Every call enqueues on
the current stream of its tensors' device and does not synchronise."""
from __future__ import annotations

import ctypes
from collections import namedtuple
from ctypes import POINTER, Structure, byref, c_double, c_float, c_int32, c_int64, c_size_t, c_uint32, c_void_p

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
        lib.tig_linear_workspace_bytes.argtypes = [POINTER(tig_linear), c_int32, POINTER(c_size_t)]
        lib.tig_linear_forward.argtypes = [POINTER(tig_linear), c_void_p, c_size_t, c_void_p]
        lib.tig_linear_backward.argtypes = [POINTER(tig_linear), c_void_p, c_size_t, c_void_p]
        lib.tig_softmax_ce_workspace_bytes.argtypes = [POINTER(tig_softmax_ce), POINTER(c_size_t)]
        lib.tig_softmax_ce_run.argtypes = [POINTER(tig_softmax_ce), c_void_p, c_size_t, c_void_p]
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


_codes = {}


def _dtype_code(dtype):
    if not _codes:
        import torch
        _codes.update({torch.float32: 0, torch.bfloat16: 1, torch.float16: 2})
    if dtype not in _codes:
        _refuse(f"dtype {dtype} is none of float32, bfloat16, float16")
    return _codes[dtype]


def _matrix(t, rows, cols, like, name):
    """Address and row stride of a [rows x cols] tensor whose columns are adjacent."""
    if t is None:
        return 0, 0
    if t.dim() != 2 or t.shape[0] != rows or t.shape[1] != cols or t.dtype != like.dtype or t.device != like.device:
        _refuse(f"{name} is not a [{rows} x {cols}] tensor of {like.dtype} on {like.device}")
    ld = t.stride(0) if rows > 1 else max(cols, t.stride(0))
    if (cols > 1 and t.stride(1) != 1) or ld < cols:
        _refuse(f"{name}: columns have to be adjacent and rows may not overlap")
    return t.data_ptr(), ld


def _vector(t, n, like, name, dtype=None):
    if t is None:
        return 0
    dtype = dtype or like.dtype
    if t.dim() != 1 or t.shape[0] != n or t.dtype != dtype or t.device != like.device or (n > 1 and t.stride(0) != 1):
        _refuse(f"{name} is not a contiguous [{n}] tensor of {dtype} on {like.device}")
    return t.data_ptr()


class _On:
    """The device of a call's tensors made current where it is not, and its current stream."""

    def __init__(self, device):
        import torch
        if device.type != "cuda":
            _refuse(f"tensors are on {device}, not on a GPU")
        self.guard = torch.cuda.device(device) if device.index != torch.cuda.current_device() else None
        self.device = device

    def __enter__(self):
        import torch
        if self.guard:
            self.guard.__enter__()
        return torch.cuda.current_stream().cuda_stream

    def __exit__(self, *a):
        if self.guard:
            self.guard.__exit__(*a)


def _workspace(n, device):
    import torch
    return torch.empty(n, dtype=torch.uint8, device=device) if n else None


def _activation(name):
    if name not in ACTIVATIONS:
        _refuse(f"activation {name!r} is none of {', '.join(ACTIVATIONS)}")
    return ACTIVATIONS[name]


def linear(x, w, bias=None, residual=None, activation="none", keep=False, out=None):
    """act(x w^T + bias) + residual for x [rows x in], w [out x in]; fp32, bf16 or fp16, sums in fp32.  With keep=True
    returns (y, z), z = x w^T + bias as linear_backward wants it.  out: where y goes (residual itself is fine)."""
    import torch
    if x.dim() != 2 or w.dim() != 2:
        _refuse("x and w are matrices")
    rows, k = x.shape
    n = w.shape[0]
    p = tig_linear(ctypes.sizeof(tig_linear), _dtype_code(x.dtype), _activation(activation), 0, rows, k, n)
    p.x, p.ldx = _matrix(x, rows, k, x, "x")
    p.w, p.ldw = _matrix(w, n, k, x, "w")
    p.bias = _vector(bias, n, x, "bias")
    p.residual, p.ldr = _matrix(residual, rows, n, x, "residual")
    lib = _lib()
    with _On(x.device) as stream:
        y = torch.empty((rows, n), dtype=x.dtype, device=x.device) if out is None else out
        z = torch.empty((rows, n), dtype=x.dtype, device=x.device) if keep else None
        p.y, p.ldy = _matrix(y, rows, n, x, "out")
        p.z, p.ldz = _matrix(z, rows, n, x, "z")
        need = c_size_t(0)
        _check(lib.tig_linear_workspace_bytes(byref(p), 0, byref(need)))
        ws = _workspace(need.value, x.device)
        _check(lib.tig_linear_forward(byref(p), ws.data_ptr() if ws is not None else None, need.value, stream))
    return (y, z) if keep else y


def linear_backward(dy, x, w, z=None, activation="none", dx=True, dw=True, dbias=True):
    """Gradients (dx, dw, dbias) of linear() for dy [rows x out]; None in the place of one that is not wanted.  z: what
    linear(keep=True) returned (not needed without an activation).  The residual's gradient is dy."""
    import torch
    if dy.dim() != 2 or x.dim() != 2 or w.dim() != 2:
        _refuse("dy, x and w are matrices")
    rows, n = dy.shape
    k = w.shape[1]
    p = tig_linear(ctypes.sizeof(tig_linear), _dtype_code(dy.dtype), _activation(activation), 0, rows, k, n)
    p.dy, p.lddy = _matrix(dy, rows, n, dy, "dy")
    p.x, p.ldx = _matrix(x, rows, k, dy, "x")
    p.w, p.ldw = _matrix(w, n, k, dy, "w")
    if p.activation:
        if z is None:
            _refuse("the backward pass of an activation needs z")
        p.z, p.ldz = _matrix(z, rows, n, dy, "z")
    lib = _lib()
    with _On(dy.device) as stream:
        gx = torch.empty((rows, k), dtype=dy.dtype, device=dy.device) if dx else None
        gw = torch.empty((n, k), dtype=dy.dtype, device=dy.device) if dw else None
        gb = torch.empty(n, dtype=dy.dtype, device=dy.device) if dbias else None
        p.dx, p.lddx = _matrix(gx, rows, k, dy, "dx")
        p.dw, p.lddw = _matrix(gw, n, k, dy, "dw")
        p.dbias = _vector(gb, n, dy, "dbias")
        need = c_size_t(0)
        _check(lib.tig_linear_workspace_bytes(byref(p), 1, byref(need)))
        ws = _workspace(need.value, dy.device)
        _check(lib.tig_linear_backward(byref(p), ws.data_ptr() if ws is not None else None, need.value, stream))
    return gx, gw, gb


SoftmaxCE = namedtuple("SoftmaxCE", "loss lse mean dx dw dbias")


def softmax_ce(x, w, labels, bias=None, row_scale=None, scale=1.0, grad=True):
    """Softmax cross entropy of rows x [rows x dim] over the candidates w [vocab x dim] (+ bias [vocab]) with int32
    labels [rows]; a label outside the vocabulary (-1) leaves its row out.  Returns SoftmaxCE(loss [rows], lse [rows],
    mean [1], dx, dw, dbias): loss and lse in fp32, gradients of scale * mean (or of scale * sum of row_scale * loss) in
    x's type, None without `grad`."""
    import torch
    if x.dim() != 2 or w.dim() != 2:
        _refuse("x and w are matrices")
    rows, d = x.shape
    vocab = w.shape[0]
    p = tig_softmax_ce(ctypes.sizeof(tig_softmax_ce), _dtype_code(x.dtype), rows, vocab, d)
    p.x, p.ldx = _matrix(x, rows, d, x, "x")
    p.w, p.ldw = _matrix(w, vocab, d, x, "w")
    p.bias = _vector(bias, vocab, x, "bias")
    p.labels = _vector(labels, rows, x, "labels", torch.int32)
    p.row_scale = _vector(row_scale, rows, x, "row_scale", torch.float32)
    p.scale = scale
    lib = _lib()
    with _On(x.device) as stream:
        dev = x.device
        stats = torch.empty(2 * rows + 1, dtype=torch.float32, device=dev)
        loss, lse, mean = stats[:rows], stats[rows : 2 * rows], stats[2 * rows :]
        p.loss, p.lse, p.mean = loss.data_ptr(), lse.data_ptr(), mean.data_ptr()
        dx = torch.empty((rows, d), dtype=x.dtype, device=dev) if grad else None
        dw = torch.empty((vocab, d), dtype=x.dtype, device=dev) if grad else None
        db = torch.empty(vocab, dtype=x.dtype, device=dev) if grad and bias is not None else None
        p.dx, p.lddx = _matrix(dx, rows, d, x, "dx")
        p.dw, p.lddw = _matrix(dw, vocab, d, x, "dw")
        p.dbias = _vector(db, vocab, x, "dbias")
        need = c_size_t(0)
        _check(lib.tig_softmax_ce_workspace_bytes(byref(p), byref(need)))
        ws = _workspace(need.value, dev)
        _check(lib.tig_softmax_ce_run(byref(p), ws.data_ptr(), need.value, stream))
    return SoftmaxCE(loss, lse, mean, dx, dw, db)


class AdamW:
    """AdamW over lists of tensors of any shape (contiguous).  States are the caller's: m and v in float32, or for 8 bits
    in torch.float8_e4m3fn with float32 scales, one for every 256 elements, m_scales and v_scales (v then holds sqrt(v)).
    step: int64 device tensor [1], the steps made so far.  masters: float32 tensors that are stepped in place of
    16-bit params, which receive their rounded copies (None, or None for a tensor, where there is none)."""

    def __init__(self, params, grads, m, v, step, masters=None, m_scales=None, v_scales=None, betas=(0.9, 0.999), eps=1e-8,
                 weight_decay=0.0):
        import torch
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
        self.kept = (params, grads, m, v, step, masters, m_scales, v_scales)  # the handle holds their addresses
        self.norm = torch.zeros(1, dtype=torch.float32, device=self.device)
        cfg = tig_adamw_config(ctypes.sizeof(tig_adamw_config), 8 if eight else 32, betas[0], betas[1], eps, step.data_ptr())
        self.lib = _lib()
        h, need = c_void_p(None), c_size_t(0)
        with _On(self.device) as stream:
            _check(self.lib.tig_adamw_workspace_bytes(byref(cfg), table, len(params), byref(need)))
            self.ws = _workspace(need.value, self.device)
            _check(self.lib.tig_adamw_create(byref(cfg), table, len(params), self.ws.data_ptr(), need.value, stream, byref(h)))
        self.handle = h

    def step(self, lr, grad_scale=1.0, max_norm=0.0):
        """Enqueues one step; returns the device tensor [1] that receives the gradients' norm (with max_norm > 0)."""
        with _On(self.device) as stream:
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
