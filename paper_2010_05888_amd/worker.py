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


_vp, _i32, _i64, _sz, _f32 = _c.c_void_p, _c.c_int, _c.c_int64, _c.c_size_t, _c.c_float
_b8 = _c.POINTER(_Block8)
_counts_p = _c.POINTER(_i64)
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
