"""A worker's operators: what comes before the aggregation rules.

The n workers' tokens lie one worker after the other in a T x D matrix, and each
worker's own weight gradient goes to its row of the n x d fp32 matrix that the
rules take:

    r = layernorm(x, weight, bias, y8=True, x8=True)       # y8: the linear layer's input,
    out = linear8(r.y8, checkpoint(w), b, fast=True)       # kept in 8 bits with x8
    ...                                                    # dout: the gradient of out
    weight_gradient(dout, r.y8, counts, out=grads[:, i:j].view(n, *w.shape), dbias=...)
    dy = linear8(checkpoint(dout), checkpoint(w, transposed=True), fast=True)
    dx, _, _ = layernorm_backward(dy, r.x8, r.mean, r.rstd, weight, counts, dweight=..., dbias=...)
    aggregate, sel = gar("multikrum", grads, f)

and for a residual block in 16 or 32 bits:

    h = linear(x, w0).out
    r = residual_norm(x, h, gain, post_weight=post, gate=gate, rms=True)
    up = linear(r.y, w1, b1, "gelu", pre=True)
    out = linear(up.out, w2, residual=r.s).out
    dp = linear_backward(dout, w2, up.pre, "gelu")
    dw1, _ = linear_weight_gradient(dp, r.y, counts)       # and of w2, w0 alike
    b = residual_norm_backward(r, h, dout, linear_backward(dp, w1), gain, post, gate=gate,
                               rms=True, counts=counts)
    norms = clip_gradients([dw1, b.dweight, ...], max_norm, out=grads)

Nothing here takes part in torch's autograd: a backward pass is called like a
forward pass.

Thin binding over the C-ABI of ``include/garfield_worker.h``, whose kernels do
all the computing; calls run on the current stream of their tensors' device and
share no scratch, so calls on several streams may overlap.
"""
from __future__ import annotations

import ctypes
from typing import NamedTuple

import torch

from . import GarfieldError, OK, load

BLOCK = 128  # GARFIELD_BLOCK: values that share one exponent
TYPES = {torch.float32: 0, torch.bfloat16: 1, torch.float16: 2}

_c = ctypes


class _Block8(_c.Structure):
    _fields_ = [("values", _c.c_void_p), ("exponents", _c.c_void_p), ("rows", _c.c_int64),
                ("cols", _c.c_int64), ("ld_values", _c.c_int64), ("ld_exponents", _c.c_int64)]


class _ResidualBlock(_c.Structure):
    _fields_ = [("type", _c.c_int), ("wtype", _c.c_int), ("rows", _c.c_int64),
                ("cols", _c.c_int64), ("rms", _c.c_int), ("eps", _c.c_float),
                ("scale", _c.c_float), ("weight", _c.c_void_p), ("bias", _c.c_void_p),
                ("post_weight", _c.c_void_p), ("post_bias", _c.c_void_p), ("gate", _c.c_void_p),
                ("ld_gate", _c.c_int64)]


class _ResidualGradients(_c.Structure):
    _fields_ = [(name, _c.c_void_p) for name in ("weight", "bias", "post_weight", "post_bias",
                                                 "gate")] + \
               [("ld_" + name, _c.c_int64) for name in ("weight", "bias", "post_weight",
                                                        "post_bias", "gate")]


class _Gradient(_c.Structure):
    _fields_ = [("values", _c.c_void_p), ("length", _c.c_int64), ("ld", _c.c_int64),
                ("type", _c.c_int)]


_vp, _i32, _i64, _sz, _f32 = _c.c_void_p, _c.c_int, _c.c_int64, _c.c_size_t, _c.c_float
_b8 = _c.POINTER(_Block8)
_counts_p = _c.POINTER(_i64)
_rb = _c.POINTER(_ResidualBlock)
_SIGNATURES = {
    "garfield_checkpoint": (_i32, [_vp, _i32, _i64, _i64, _i64, _i32, _b8, _vp]),
    "garfield_restore": (_i32, [_b8, _vp, _i32, _i64, _vp]),
    "garfield_layernorm": (_i32, [_vp, _i32, _i64, _i64, _i64, _vp, _vp, _i32, _f32, _vp, _i64,
                                  _vp, _vp, _b8, _b8, _vp]),
    "garfield_layernorm_backward_workspace": (_sz, [_i64, _i64, _i32, _counts_p]),
    "garfield_layernorm_backward": (_i32, [_vp, _i32, _i64, _i64, _i64, _vp, _i64, _b8, _vp, _vp,
                                           _vp, _i32, _vp, _i64, _i32, _counts_p, _vp, _i64, _vp,
                                           _i64, _vp, _sz, _vp]),
    "garfield_linear8_workspace": (_sz, [_i64, _i64, _i64]),
    "garfield_linear8": (_i32, [_b8, _b8, _vp, _i32, _vp, _i32, _i64, _vp, _sz, _vp]),
    "garfield_weight_gradient_workspace": (_sz, [_vp, _i32, _i64, _i64, _i64, _i64, _i32,
                                                 _counts_p]),
    "garfield_weight_gradient": (_i32, [_vp, _i32, _i64, _i64, _i64, _b8, _i32, _counts_p, _vp,
                                        _i64, _vp, _i64, _vp, _sz, _vp]),
    "garfield_linear_workspace": (_sz, [_vp, _i32, _i64, _i64, _i64, _vp, _i64, _i64]),
    "garfield_linear": (_i32, [_vp, _i32, _i64, _i64, _i64, _vp, _i64, _i64, _vp, _i32, _i32, _vp,
                               _i64, _vp, _i64, _vp, _i64, _vp, _sz, _vp]),
    "garfield_linear_backward_workspace": (_sz, [_vp, _i32, _i64, _i64, _i64, _vp, _i64, _i64]),
    "garfield_linear_backward": (_i32, [_vp, _i32, _i64, _i64, _i64, _vp, _i64, _i64, _i32, _vp,
                                        _i64, _vp, _i64, _vp, _i64, _vp, _sz, _vp]),
    "garfield_activation_backward": (_i32, [_vp, _i32, _i64, _i64, _i64, _i32, _vp, _i64, _vp,
                                            _i64, _vp]),
    "garfield_linear_weight_gradient_workspace": (_sz, [_vp, _i32, _i64, _i64, _i64, _vp, _i64,
                                                        _i64, _i32, _counts_p]),
    "garfield_linear_weight_gradient": (_i32, [_vp, _i32, _i64, _i64, _i64, _vp, _i64, _i64, _i32,
                                               _counts_p, _vp, _i64, _vp, _i64, _vp, _sz, _vp]),
    "garfield_residual_norm": (_i32, [_rb, _vp, _i64, _vp, _i64, _vp, _i64, _vp, _i64, _vp, _vp,
                                      _vp, _vp, _b8, _vp]),
    "garfield_residual_norm_backward_workspace": (_sz, [_rb, _i32, _counts_p]),
    "garfield_residual_norm_backward": (_i32, [_rb, _vp, _i64, _vp, _i64, _vp, _i64, _vp, _i64,
                                               _vp, _vp, _vp, _vp, _vp, _i64, _vp, _i64, _vp, _i64,
                                               _i32, _counts_p, _c.POINTER(_ResidualGradients),
                                               _vp, _sz, _vp]),
    "garfield_clip_workspace": (_sz, [_vp, _i32, _i32]),
    "garfield_gradient_norms": (_i32, [_vp, _i32, _i32, _vp, _vp, _sz, _vp]),
    "garfield_clip_gradients": (_i32, [_vp, _i32, _i32, _f32, _vp, _vp, _i64, _vp, _sz, _vp]),
}
_fn = {}


def _functions():
    global _fn
    if not _fn:
        lib, table = load(), {}
        for name, (restype, argtypes) in _SIGNATURES.items():
            table[name] = fn = getattr(lib, name)
            fn.restype, fn.argtypes = restype, argtypes
        _fn = table  # only when whole: another thread may be here
    return _fn


_empty = torch.empty
_this_device = getattr(torch._C, "_cuda_getDevice", None)
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)


def _run(name: str, device: torch.device, *args):
    """Call a function of the library on the device's current stream."""
    fn = _fn.get(name) or _functions()[name]
    i = device.index
    if i == _this_device():
        code = fn(*args, _raw_stream(i))
    else:
        with torch.cuda.device(i):
            code = fn(*args, _raw_stream(i))
    if code != OK:
        raise GarfieldError(code, name, load().garfield_strerror(code).decode())


def _matrix(x, name: str, dtype=None):
    """x's rows, columns, row distance and type."""
    if not isinstance(x, torch.Tensor) or x.dim() != 2:
        raise ValueError(f"{name} must be a 2-D tensor (one row a token)")
    if not x.is_cuda:
        raise ValueError(f"{name} must be on a GPU: this library has no CPU path")
    kind = TYPES.get(x.dtype)
    if kind is None or (dtype is not None and x.dtype != dtype):
        raise ValueError(f"{name} must be {dtype or 'float32, bfloat16 or float16'}")
    rows, cols = x.shape
    ld, step = x.stride()
    if step != 1 and cols > 1:
        raise ValueError(f"{name}'s columns must be next to each other")
    if rows < 2:
        ld = cols or 1
    elif ld < cols:
        raise ValueError(f"{name}'s rows must not overlap")
    return rows, cols, ld, kind


def _vector(v, name: str, length: int, dtypes, device):
    if (not isinstance(v, torch.Tensor) or v.dtype not in dtypes or v.shape != (length,)
            or v.device != device or not v.is_contiguous()):
        raise ValueError(f"{name} must be a contiguous 1-D tensor of {length} values of "
                         f"{' or '.join(str(d) for d in dtypes)} on {device}")
    return v.data_ptr()


def _padded(cols: int):
    """Columns of the codes and of the exponents that rows of cols values take."""
    blocks = -(-cols // BLOCK)
    return blocks * BLOCK, -(-blocks // 4) * 4


class Checkpoint:
    """A matrix of rows x cols values in 8-bit blocks (garfield_block8): codes
    ``values`` (float8_e4m3fn, rows x the columns padded with zeros to a multiple
    of 128) and ``exponents`` (uint8, one for each 128 values of a row, padded
    with 127 to a multiple of four): the value of a code is code * 2^(exponent -
    127). Made by ``checkpoint()`` and ``layernorm()``, or from tensors that hold
    such blocks."""

    __slots__ = ("rows", "cols", "device", "_held", "_at", "_flat", "_values", "_exponents")

    def __init__(self, values: torch.Tensor, exponents: torch.Tensor, cols: int):
        if (not isinstance(values, torch.Tensor) or values.dim() != 2
                or values.dtype != torch.float8_e4m3fn or not values.is_cuda):
            raise ValueError("values must be a 2-D float8_e4m3fn tensor on a GPU")
        if (not isinstance(exponents, torch.Tensor) or exponents.dim() != 2
                or exponents.dtype != torch.uint8 or exponents.device != values.device):
            raise ValueError("exponents must be a 2-D uint8 tensor on values' device")
        width, held = _padded(cols)
        rows, codes = values.shape
        rows_held, codes_held = exponents.shape
        if codes < width or rows_held != rows or codes_held < held:
            raise ValueError(f"{cols} columns need {width} codes and {held} exponents a row")
        (ldv, step), (lde, step_held) = values.stride(), exponents.stride()
        if rows < 2:
            ldv, lde = width, held
        pv, pe = values.data_ptr(), exponents.data_ptr()
        if cols > 0 and rows > 0 and (step != 1 or step_held != 1 or ldv < width or ldv % 16
                                      or lde < held or lde % 4 or pv % 16 or pe % 4):
            raise ValueError("rows of codes must start at multiples of 16 bytes, rows of exponents "
                             "at multiples of 4, their columns next to each other")
        self.rows, self.cols, self.device, self._flat = rows, cols, values.device, None
        self._values, self._exponents = values, exponents
        self._held = _Block8(pv, pe, rows, cols, ldv, lde)
        self._at = _c.byref(self._held)

    @classmethod
    def empty(cls, rows: int, cols: int, device) -> "Checkpoint":
        """Room for rows x cols values, to be written."""
        width, held = _padded(cols)
        # rows a multiple of 8 KiB apart share memory channels, which matters little: products
        # of 16384 x k with 8192 x k values take 894 us from such rows and 890 from these at
        # k = 8192, 1882 and 1923 at 16384
        ld = width if width % 8192 or not width else width + BLOCK
        c = cls.__new__(cls)
        c._flat = flat = _empty(rows * (ld + held), dtype=torch.uint8, device=device)
        c._values = c._exponents = None
        c.rows, c.cols, c.device = rows, cols, flat.device
        at = flat.data_ptr()
        c._held = _Block8(at, at + rows * ld, rows, cols, ld, held)
        c._at = _c.byref(c._held)
        return c

    @property
    def values(self) -> torch.Tensor:
        if self._values is None:
            self._values = self._flat.view(torch.float8_e4m3fn).as_strided(
                (self.rows, _padded(self.cols)[0]), (self._held.ld_values, 1))
        return self._values

    @property
    def exponents(self) -> torch.Tensor:
        if self._exponents is None:
            held = self._held
            self._exponents = self._flat.as_strided(
                (self.rows, held.ld_exponents), (held.ld_exponents, 1), self.rows * held.ld_values)
        return self._exponents

    def restore(self, dtype: torch.dtype = torch.bfloat16) -> torch.Tensor:
        """The values, rounded once to dtype (bfloat16 and float32 hold them exactly)."""
        if dtype not in TYPES:
            raise ValueError("dtype must be float32, bfloat16 or float16")
        out = _empty((self.rows, self.cols), dtype=dtype, device=self.device)
        _run("garfield_restore", self.device, self._at, out.data_ptr(), TYPES[dtype],
             max(self.cols, 1))
        return out


def checkpoint(x: torch.Tensor, transposed: bool = False) -> Checkpoint:
    """x (or its transpose) in 8-bit blocks of 128 values along a row of the result."""
    rows, cols, ld, kind = _matrix(x, "x")
    dev = x.device
    c = Checkpoint.empty(cols, rows, dev) if transposed else Checkpoint.empty(rows, cols, dev)
    _run("garfield_checkpoint", dev, x.data_ptr(), kind, rows, cols, ld, 1 if transposed else 0,
         c._at)
    return c


class LayerNorm(NamedTuple):
    """What layernorm() gives: y (or None), each row's mean and 1 / deviation
    (fp32), and the checkpoints of y and of x that were asked for (or None)."""
    y: torch.Tensor | None
    mean: torch.Tensor
    rstd: torch.Tensor
    y8: Checkpoint | None
    x8: Checkpoint | None


_WEIGHTS = {t: (torch.float32,) if t == torch.float32 else (torch.float32, t) for t in TYPES}


def layernorm(x: torch.Tensor, weight: torch.Tensor, bias: torch.Tensor | None = None,
              eps: float = 1e-5, y: bool = True, y8: bool = False,
              x8: bool = False) -> LayerNorm:
    """Layer norm of each row of x: (x - mean) * rstd * weight + bias in x's type
    (y) and in 8-bit blocks (y8), and x itself in 8-bit blocks (x8)."""
    rows, cols, ld, kind = _matrix(x, "x")
    dev, dtype = x.device, x.dtype
    pw = _vector(weight, "weight", cols, _WEIGHTS[dtype], dev)
    pb = None if bias is None else _vector(bias, "bias", cols, (weight.dtype,), dev)
    out = None
    if y:
        out = torch.empty_like(x) if ld == cols else _empty((rows, cols), dtype=dtype, device=dev)
    mean, rstd = _empty((2, rows), dtype=torch.float32, device=dev).unbind(0)
    cy = Checkpoint.empty(rows, cols, dev) if y8 else None
    cx = Checkpoint.empty(rows, cols, dev) if x8 else None
    _run("garfield_layernorm", dev, x.data_ptr(), kind, rows, cols, ld, pw, pb,
         TYPES[weight.dtype], eps, out.data_ptr() if y else None, cols, mean.data_ptr(),
         rstd.data_ptr(), cy._at if y8 else None, cx._at if x8 else None)
    return LayerNorm(out, mean, rstd, cy, cx)


def _counted(counts, rows: int):
    """The workers' tokens as a C array (None: one worker)."""
    counts = [rows] if counts is None else [int(c) for c in counts]
    if not counts or sum(counts) != rows or min(counts) < 0:
        raise ValueError(f"counts must be the workers' tokens, adding up to {rows}")
    return len(counts), (_i64 * len(counts))(*counts)


def _rows_of_workers(out, name: str, shape, device):
    """The caller's rows of the gradients, or new ones; and their distance."""
    if out is None:
        out = torch.empty(shape, dtype=torch.float32, device=device)
    length = shape[1] if len(shape) == 2 else shape[1] * shape[2]
    if not isinstance(out, torch.Tensor) or out.shape != shape or out.dtype != torch.float32 \
            or out.device != device:
        fine = False
    else:
        ld, *inner = out.stride()
        if shape[0] == 1:
            ld = length
        # columns next to each other, and rows of a matrix too, where there is more than one
        fine = (ld >= length and (inner[-1] == 1 or shape[-1] < 2)
                and (len(shape) == 2 or inner[0] == shape[2] or shape[1] < 2)) or length == 0
    if not fine:
        raise ValueError(f"{name} must be a float32 tensor of {tuple(shape)} on {device}, each "
                         "worker's values next to each other")
    return out, ld


def _workspace(name: str, device, *args):
    need = (_fn.get(name) or _functions()[name])(*args)
    return (_empty(need, dtype=torch.uint8, device=device) if need else None), need


def layernorm_backward(dy: torch.Tensor, x, mean: torch.Tensor, rstd: torch.Tensor,
                       weight: torch.Tensor, counts=None, dweight: torch.Tensor | None = None,
                       dbias: torch.Tensor | None = None):
    """(dx, dweight, dbias) of layernorm(): x is its input, as a tensor of dy's
    type or as a Checkpoint; counts the tokens of each of the n workers (None: one
    worker). dweight and dbias (n x cols, float32) may be given, e.g. columns of
    the matrix of gradients."""
    rows, cols, ld, kind = _matrix(dy, "dy")
    dev = dy.device
    if isinstance(x, Checkpoint):
        px, ldx, x8, shape = None, 0, x._at, (x.rows, x.cols)
    else:
        r, c, ldx, _ = _matrix(x, "x", dy.dtype)
        px, x8, shape = x.data_ptr(), None, (r, c)
    if shape != (rows, cols) or x.device != dev:
        raise ValueError("x must have dy's shape and device")
    pm = _vector(mean, "mean", rows, (torch.float32,), dev)
    pr = _vector(rstd, "rstd", rows, (torch.float32,), dev)
    pw = _vector(weight, "weight", cols, _WEIGHTS[dy.dtype], dev)
    n, counts = _counted(counts, rows)
    dweight, ldw = _rows_of_workers(dweight, "dweight", (n, cols), dev)
    dbias, ldb = _rows_of_workers(dbias, "dbias", (n, cols), dev)
    dx = torch.empty_like(dy) if ld == cols else _empty((rows, cols), dtype=dy.dtype, device=dev)
    ws, need = _workspace("garfield_layernorm_backward_workspace", dev, rows, cols, n, counts)
    _run("garfield_layernorm_backward", dev, dy.data_ptr(), kind, rows, cols, ld, px, ldx, x8, pm,
         pr, pw, TYPES[weight.dtype], dx.data_ptr(), cols, n, counts, dweight.data_ptr(), ldw,
         dbias.data_ptr(), ldb, ws.data_ptr() if need else None, need)
    return dx, dweight, dbias


def linear8(x8: Checkpoint, w8: Checkpoint, bias: torch.Tensor | None = None,
            dtype: torch.dtype = torch.bfloat16, fast: bool = False) -> torch.Tensor:
    """x w^T + bias of two checkpoints (rows of x by rows of w), in dtype; bias is
    float32. Sums are fp32; with fast they may be the 8-bit matrix instruction's,
    which runs at twice the rate and keeps 14 bits of every eight products."""
    if not isinstance(x8, Checkpoint) or not isinstance(w8, Checkpoint):
        raise ValueError("x8 and w8 must be checkpoints")
    dev, m, n, k = x8.device, x8.rows, w8.rows, x8.cols
    if k != w8.cols or dev != w8.device:
        raise ValueError("x8 and w8 must have the same columns and device")
    if dtype not in TYPES:
        raise ValueError("dtype must be float32, bfloat16 or float16")
    pb = None if bias is None else _vector(bias, "bias", n, (torch.float32,), dev)
    out = _empty((m, n), dtype=dtype, device=dev)
    ws, need = _workspace("garfield_linear8_workspace", dev, m, n, k)
    _run("garfield_linear8", dev, x8._at, w8._at, pb, 1 if fast else 0, out.data_ptr(),
         TYPES[dtype], n or 1, ws.data_ptr() if need else None, need)
    return out


def weight_gradient(dy: torch.Tensor, x8: Checkpoint, counts=None,
                    out: torch.Tensor | None = None, dbias: torch.Tensor | None = None):
    """(dw, dbias) of a linear layer for each worker: dw[w] = dy^T x over worker
    w's tokens (n x outputs x inputs, float32) and dbias[w] = their sum of dy. dy:
    the gradient of the layer's output; x8: the checkpoint of its input; out and
    dbias may be given, e.g. columns of the matrix of gradients (dbias is None
    where it is not given)."""
    tokens, outputs, ld, kind = _matrix(dy, "dy")
    dev = dy.device
    if not isinstance(x8, Checkpoint) or x8.rows != tokens or x8.device != dev:
        raise ValueError("x8 must be a checkpoint with dy's rows and device")
    n, counts = _counted(counts, tokens)
    out, ldw = _rows_of_workers(out, "out", (n, outputs, x8.cols), dev)
    pb, ldb = None, 0
    if dbias is not None:
        dbias, ldb = _rows_of_workers(dbias, "dbias", (n, outputs), dev)
        pb = dbias.data_ptr()
    py = dy.data_ptr()
    ws, need = _workspace("garfield_weight_gradient_workspace", dev, py, kind, tokens, outputs,
                          x8.cols, ld, n, counts)
    _run("garfield_weight_gradient", dev, py, kind, tokens, outputs, ld, x8._at, n, counts,
         out.data_ptr(), ldw, pb, ldb, ws.data_ptr() if need else None, need)
    return out, dbias


ACTIVATIONS = {None: 0, "relu": 1, "gelu": 2, "gelu_tanh": 3, "silu": 4}


def _activation(name) -> int:
    if name not in ACTIVATIONS:
        raise ValueError(f"activation must be one of {list(ACTIVATIONS)}, not {name!r}")
    return ACTIVATIONS[name]


def _like(v, name: str, rows: int, cols: int, x: torch.Tensor):
    """The pointer and row distance of a matrix of x's type and device (None: none)."""
    if v is None:
        return None, 0
    if (isinstance(v, torch.Tensor) and v.dtype is x.dtype and v.shape == (rows, cols)
            and v.is_contiguous() and v.device == x.device):
        return v.data_ptr(), cols  # as _matrix and what follows it find, in a third of the time
    r, c, ld, _ = _matrix(v, name, x.dtype)
    if (r, c) != (rows, cols) or v.device != x.device:
        raise ValueError(f"{name} must be {rows} x {cols} on {x.device}")
    return v.data_ptr(), ld


class Linear(NamedTuple):
    """What linear() gives: its result, and its sums with the bias (or None)."""
    out: torch.Tensor
    pre: torch.Tensor | None


def linear(x: torch.Tensor, w: torch.Tensor, bias: torch.Tensor | None = None,
           activation: str | None = None, residual: torch.Tensor | None = None,
           pre: bool = False) -> Linear:
    """act(x w^T + bias) + residual (rows of x by rows of w) in x's type, and with pre also
    x w^T + bias, for the backward pass. activation: None, "relu", "gelu", "gelu_tanh" or
    "silu"; w and residual are of x's type, bias float32 or of x's. Sums are fp32."""
    tokens, inputs, ldx, kind = _matrix(x, "x")
    outputs, k, ldw, _ = _matrix(w, "w", x.dtype)
    dev, dtype = x.device, x.dtype
    if k != inputs or w.device != dev:
        raise ValueError("x and w must have the same columns and device")
    act = _activation(activation)
    pb = None if bias is None else _vector(bias, "bias", outputs, _WEIGHTS[dtype], dev)
    pr, ldr = _like(residual, "residual", tokens, outputs, x)
    out = x.new_empty((tokens, outputs))
    kept = torch.empty_like(out) if pre else None
    px, pw, ld = x.data_ptr(), w.data_ptr(), outputs or 1
    ws, need = _workspace("garfield_linear_workspace", dev, px, kind, tokens, inputs, ldx, pw,
                          outputs, ldw)
    _run("garfield_linear", dev, px, kind, tokens, inputs, ldx, pw, outputs, ldw, pb,
         0 if bias is None else TYPES[bias.dtype], act, pr, ldr, out.data_ptr(), ld,
         kept.data_ptr() if pre else None, ld, ws.data_ptr() if need else None, need)
    return Linear(out, kept)


def linear_backward(dy: torch.Tensor, w: torch.Tensor, pre: torch.Tensor | None = None,
                    activation: str | None = None,
                    residual: torch.Tensor | None = None) -> torch.Tensor:
    """The gradient of a linear layer's input, dy w, on through what came before it: times
    the slope at pre of that layer's activation, plus a gradient that comes by another way.
    All in dy's type; pre is what linear() kept of the layer before."""
    tokens, outputs, ld, kind = _matrix(dy, "dy")
    k, inputs, ldw, _ = _matrix(w, "w", dy.dtype)
    dev = dy.device
    if k != outputs or w.device != dev:
        raise ValueError("dy's columns must be w's rows, on one device")
    act = _activation(activation)
    if (pre is None) != (activation is None):
        raise ValueError("pre and activation go together")
    pp, ldp = _like(pre, "pre", tokens, inputs, dy)
    pr, ldr = _like(residual, "residual", tokens, inputs, dy)
    dx = dy.new_empty((tokens, inputs))
    py, pw = dy.data_ptr(), w.data_ptr()
    ws, need = _workspace("garfield_linear_backward_workspace", dev, py, kind, tokens, outputs, ld,
                          pw, inputs, ldw)
    _run("garfield_linear_backward", dev, py, kind, tokens, outputs, ld, pw, inputs, ldw, act, pp,
         ldp, pr, ldr, dx.data_ptr(), inputs or 1, ws.data_ptr() if need else None, need)
    return dx


def activation_backward(dy: torch.Tensor, pre: torch.Tensor, activation: str) -> torch.Tensor:
    """dy times the activation's slope at pre: the gradient of linear()'s sums from that of
    its result, in dy's type."""
    rows, cols, ld, kind = _matrix(dy, "dy")
    if activation is None:
        raise ValueError("activation_backward needs an activation")
    act = _activation(activation)
    if pre is None:
        raise ValueError("activation_backward needs pre")
    pp, ldp = _like(pre, "pre", rows, cols, dy)
    dp = _empty((rows, cols), dtype=dy.dtype, device=dy.device)
    _run("garfield_activation_backward", dy.device, dy.data_ptr(), kind, rows, cols, ld, act, pp,
         ldp, dp.data_ptr(), cols or 1)
    return dp


def linear_weight_gradient(dy: torch.Tensor, x: torch.Tensor, counts=None,
                           out: torch.Tensor | None = None, dbias: torch.Tensor | None = None):
    """weight_gradient() with the layer's input as it is: x is a matrix of dy's type."""
    tokens, outputs, ld, kind = _matrix(dy, "dy")
    rows, inputs, ldx, _ = _matrix(x, "x", dy.dtype)
    dev = dy.device
    if rows != tokens or x.device != dev:
        raise ValueError("x must have dy's rows and device")
    n, counts = _counted(counts, tokens)
    out, ldw = _rows_of_workers(out, "out", (n, outputs, inputs), dev)
    pb, ldb = None, 0
    if dbias is not None:
        dbias, ldb = _rows_of_workers(dbias, "dbias", (n, outputs), dev)
        pb = dbias.data_ptr()
    py, px = dy.data_ptr(), x.data_ptr()
    ws, need = _workspace("garfield_linear_weight_gradient_workspace", dev, py, kind, tokens,
                          outputs, ld, px, inputs, ldx, n, counts)
    _run("garfield_linear_weight_gradient", dev, py, kind, tokens, outputs, ld, px, inputs, ldx, n,
         counts, out.data_ptr(), ldw, pb, ldb, ws.data_ptr() if need else None, need)
    return out, dbias


class ResidualNorm(NamedTuple):
    """What residual_norm() gives: the stream s, its norm y (or None) and y's checkpoint
    (or None), and the mean and 1 / deviation of each row (fp32): of s, and of the block's
    result (None for a norm that is not there; no means with rms)."""
    s: torch.Tensor
    y: torch.Tensor | None
    y8: Checkpoint | None
    mean: torch.Tensor | None
    rstd: torch.Tensor | None
    post_mean: torch.Tensor | None
    post_rstd: torch.Tensor | None


def _residual_block(like: torch.Tensor, rows, cols, kind, weight, bias, post_weight, post_bias,
                    gate, scale, eps, rms):
    dev, allowed = like.device, _WEIGHTS[like.dtype]
    if rms and (bias is not None or post_bias is not None):
        raise ValueError("with rms a norm has no bias")
    if (bias is not None and weight is None) or (post_bias is not None and post_weight is None):
        raise ValueError("a bias needs its weight")
    wtype = pw = pb = ppw = ppb = pg = None
    ld_gate = 0
    if weight is not None:
        pw, wtype = _vector(weight, "weight", cols, allowed, dev), weight.dtype
        allowed = (wtype,)  # the others' too
        if bias is not None:
            pb = _vector(bias, "bias", cols, allowed, dev)
    if post_weight is not None:
        ppw, wtype = _vector(post_weight, "post_weight", cols, allowed, dev), post_weight.dtype
        allowed = (wtype,)
        if post_bias is not None:
            ppb = _vector(post_bias, "post_bias", cols, allowed, dev)
    if gate is not None:
        if isinstance(gate, torch.Tensor) and gate.dim() == 1:
            pg, wtype = _vector(gate, "gate", cols, allowed, dev), gate.dtype
        else:
            pg, ld_gate = _like(gate, "gate", rows, cols, like)
    return _ResidualBlock(kind, 0 if wtype is None else TYPES[wtype], rows, cols, 1 if rms else 0,
                          eps, scale, pw, pb, ppw, ppb, pg, ld_gate)


def residual_norm(x: torch.Tensor, h: torch.Tensor, weight: torch.Tensor | None = None,
                  bias: torch.Tensor | None = None, post_weight: torch.Tensor | None = None,
                  post_bias: torch.Tensor | None = None, gate: torch.Tensor | None = None,
                  scale: float = 1.0, eps: float = 1e-5, rms: bool = False, y: bool = True,
                  y8: bool = False) -> ResidualNorm:
    """The residual around a block with the norms before and after it: s = scale * x +
    gate * N_post(h) and y = N(s), in x's type and in 8-bit blocks (y8). x: the residual stream;
    h: the block's result. N is a layer norm of rows, with rms one by their root mean square;
    weight None: no y, post_weight None: h as it is. gate: a value for each column, or a matrix
    like x; weights, biases and a gate of columns are all float32 or all of x's type."""
    rows, cols, ldx, kind = _matrix(x, "x")
    if h is None:
        raise ValueError("h must be a 2-D tensor (one row a token)")
    ph, ldh = _like(h, "h", rows, cols, x)
    dev, dtype = x.device, x.dtype
    if cols == 0:
        raise ValueError("x must have columns")
    b = _residual_block(x, rows, cols, kind, weight, bias, post_weight, post_bias, gate, scale,
                        eps, rms)
    normed = weight is not None
    if y8 and not normed:
        raise ValueError("y8 needs a weight")
    s = torch.empty_like(x) if ldx == cols else _empty((rows, cols), dtype=dtype, device=dev)
    out = torch.empty_like(s) if y and normed else None
    cy = Checkpoint.empty(rows, cols, dev) if y8 else None
    post = post_weight is not None
    flat = _empty(((normed + post) * (1 if rms else 2), rows), dtype=torch.float32, device=dev)
    at, apart, mean, post_mean = flat.data_ptr(), 4 * rows, None, None
    left = iter(flat.unbind(0))  # in the order of their places
    places = [None] * 4
    if normed:
        if not rms:
            mean, places[0], at = next(left), at, at + apart
        rstd, places[1], at = next(left), at, at + apart
    if post:
        if not rms:
            post_mean, places[2], at = next(left), at, at + apart
        post_rstd, places[3] = next(left), at
    _run("garfield_residual_norm", dev, _c.byref(b), x.data_ptr(), ldx, ph, ldh, s.data_ptr(),
         cols, None if out is None else out.data_ptr(), cols, *places, cy._at if y8 else None)
    return ResidualNorm(s, out, cy, mean, rstd if normed else None, post_mean,
                        post_rstd if post else None)


class ResidualNormBackward(NamedTuple):
    """What residual_norm_backward() gives: the gradients of x and h, and of each worker
    those of the parameters that there are (n x cols, float32); dgate is that of a gate of
    columns, or a matrix like dx for a gate like x."""
    dx: torch.Tensor
    dh: torch.Tensor
    dweight: torch.Tensor | None
    dbias: torch.Tensor | None
    dpost_weight: torch.Tensor | None
    dpost_bias: torch.Tensor | None
    dgate: torch.Tensor | None


def residual_norm_backward(r: ResidualNorm, h: torch.Tensor, ds: torch.Tensor | None = None,
                           dy: torch.Tensor | None = None, weight: torch.Tensor | None = None,
                           post_weight: torch.Tensor | None = None,
                           post_bias: torch.Tensor | None = None,
                           gate: torch.Tensor | None = None, scale: float = 1.0,
                           rms: bool = False, counts=None, dweight: torch.Tensor | None = None,
                           dbias: torch.Tensor | None = None,
                           dpost_weight: torch.Tensor | None = None,
                           dpost_bias: torch.Tensor | None = None,
                           dgate: torch.Tensor | None = None) -> ResidualNormBackward:
    """The gradients of residual_norm() from that of y (dy) and what reaches s by other ways
    (ds; one of the two may be None). r: what residual_norm() gave (s and the statistics are
    read); h and the parameters as they were given to it; counts the tokens of each of the n
    workers (None: one worker). dweight, dbias, dpost_weight, dpost_bias and a dgate of columns
    (n x cols, float32) may be given, e.g. columns of the matrix of gradients. Biases have
    gradients wherever they may have been (not with rms)."""
    rows, cols, ldh, kind = _matrix(h, "h")
    dev = h.device
    if ds is None and dy is None:
        raise ValueError("ds or dy must be given")
    if dy is not None and weight is None:
        raise ValueError("dy needs a weight")
    if cols == 0:
        raise ValueError("h must have columns")
    b = _residual_block(h, rows, cols, kind, weight, None, post_weight, post_bias, gate, scale,
                        0.0, rms)
    (pds, ldds), (pdy, lddy) = _like(ds, "ds", rows, cols, h), _like(dy, "dy", rows, cols, h)
    ps, lds = _like(r.s, "r.s", rows, cols, h)
    stats = [None] * 4
    for i, (name, asked) in enumerate((("mean", dy is not None and not rms),
                                       ("rstd", dy is not None),
                                       ("post_mean", post_weight is not None and not rms),
                                       ("post_rstd", post_weight is not None))):
        if asked:
            stats[i] = _vector(getattr(r, name), "r." + name, rows, (torch.float32,), dev)
    n, counts = _counted(counts, rows)
    by_columns = gate is not None and gate.dim() == 1
    if dgate is not None and not by_columns:
        raise ValueError("dgate is given for a gate of columns only")
    biased = not rms
    sums, pointers, apart = [], [], []
    for name, given, there in (
            ("dweight", dweight, weight is not None), ("dbias", dbias, biased and weight is not None),
            ("dpost_weight", dpost_weight, post_weight is not None),
            ("dpost_bias", dpost_bias, biased and post_weight is not None),
            ("dgate", dgate, by_columns)):
        ld = pointer = None
        if there:
            given, ld = _rows_of_workers(given, name, (n, cols), dev)
            pointer = given.data_ptr()
        elif given is not None:
            raise ValueError(f"{name} was given, but there is no such parameter")
        sums.append(given)
        pointers.append(pointer)
        apart.append(ld or 0)
    to = _ResidualGradients(*pointers, *apart)
    dx = torch.empty_like(h) if ldh == cols else _empty((rows, cols), dtype=h.dtype, device=dev)
    dh = torch.empty_like(dx)
    by_tokens = gate is not None and not by_columns
    dg = torch.empty_like(dx) if by_tokens else None
    at = _c.byref(b)
    ws, need = _workspace("garfield_residual_norm_backward_workspace", dev, at, n, counts)
    _run("garfield_residual_norm_backward", dev, at, pds, ldds, pdy, lddy, ps, lds, h.data_ptr(),
         ldh, *stats, dx.data_ptr(), cols, dh.data_ptr(), cols, dg.data_ptr() if by_tokens else None,
         cols, n, counts, _c.byref(to), ws.data_ptr() if need else None, need)
    if by_tokens:
        sums[4] = dg
    return ResidualNormBackward(dx, dh, *sums)


def _tensors(grads):
    """The workers' tensors as garfield_clip_gradients takes them: their count, the workers,
    a C array of garfield_gradient, the device and the values of a worker."""
    grads = [grads] if isinstance(grads, torch.Tensor) else list(grads)
    if not grads:
        raise ValueError("grads must hold a tensor")
    words, n, d = [], None, 0
    for g in grads:
        kind = TYPES.get(g.dtype) if isinstance(g, torch.Tensor) else None
        shape = () if kind is None else g.shape
        if len(shape) < 1 or not g.is_cuda:
            raise ValueError("grads must be float32, bfloat16 or float16 tensors on a GPU, "
                             "their first dimension the workers")
        if n is None:
            n, dev, index = shape[0], g.device, g.get_device()
        if shape[0] != n or n < 1 or g.get_device() != index:
            raise ValueError("grads must have the same workers (one at least) and device")
        length = ld = g.numel() // n
        if not g.is_contiguous() and length:
            ld = g.stride(0) if n > 1 else length
            if ld < length or not g[0].is_contiguous():
                raise ValueError("each worker's values of a tensor must be next to each other, "
                                 "and the workers' must not overlap")
        words += (g.data_ptr(), length, ld, kind)  # a _Gradient's
        d += length
    return len(grads), n, (_i64 * len(words))(*words), dev, d


def gradient_norms(grads) -> torch.Tensor:
    """The norm of each worker's gradient over all its tensors (float32). grads: tensors of
    any types and shapes whose first dimension is the workers, e.g. n x d or n x outputs x
    inputs (a list, or one tensor)."""
    count, n, held, dev, _ = _tensors(grads)
    norms = _empty(n, dtype=torch.float32, device=dev)
    ws, need = _workspace("garfield_clip_workspace", dev, held, count, n)
    _run("garfield_gradient_norms", dev, held, count, n, norms.data_ptr(),
         ws.data_ptr() if need else None, need)
    return norms


def clip_gradients(grads, max_norm: float, out: torch.Tensor | None = None) -> torch.Tensor:
    """Clip each worker's gradient to max_norm: all its tensors' values times max_norm / norm
    where its norm over all of them is larger. In place, or with out (n x d, float32) the
    tensors one after the other into the workers' rows of out, e.g. the matrix that the rules
    take; out shares no memory with them. Returns the norms before (float32). grads as for
    gradient_norms()."""
    count, n, held, dev, d = _tensors(grads)
    if not max_norm >= 0:
        raise ValueError("max_norm must be 0 or more")
    po, ld = None, 0
    if out is not None:
        out, ld = _rows_of_workers(out, "out", (n, d), dev)
        po = out.data_ptr()
    norms = _empty(n, dtype=torch.float32, device=dev)
    ws, need = _workspace("garfield_clip_workspace", dev, held, count, n)
    _run("garfield_clip_gradients", dev, held, count, n, max_norm, norms.data_ptr(), po, ld,
         ws.data_ptr() if need else None, need)
    return norms
