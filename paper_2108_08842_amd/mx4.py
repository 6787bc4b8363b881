"""4-bit operands and their products (include/eden_mx4.h): a linear layer's forward pass and gradients on the 4-bit matrix cores.

    w4, wt4 = quantize(w), quantize(w, transpose=True)                     # once for each step
    y, z = linear(x, w4, bias, activation="gelu", checkpoint=True)         # x is rounded to the nearest in the call; z: the activation's input in 8 bits
    xt4 = quantize(x, transpose=True)                                      # kept for the weight gradient: 17 bytes for 32 values
    noise = Stochastic(seed, id=layer)                                     # gradients are rounded stochastically: their expectation stays
    dx = linear_input_grad(quantize(dz, rounding=noise), wt4)              # or, through the activation in front of the layer, activation=, checkpoint=
    dyt4, db = quantize(dz, transpose=True, rounding=noise, sums=True)
    dw = linear_weight_grad(dyt4, xt4)                                     # fp32: what Context.encode takes

A block of 32 values has a power of two, the smallest that reaches its largest value with a 6, and codes for 0, 1/2, 1, 3/2, 2, 3, 4, 6 and a sign.  Blocks lie along the
rows of what is rounded, products sum along them: hence the transposes.  Both operands of a product are Mx4 of (rows, depth).

Tensors, streams, errors and autograd are as in layers.py: float32, float16 or bfloat16 on the GPU, dimensions in front of the last are rows at one distance, what
does not fit raises EdenError before anything is launched.  Where autograd records, quantize refuses what requires a gradient, weights among it (torch.no_grad() or detach()).
"""
from __future__ import annotations

import ctypes

import torch

from . import blocks, eden, layers
from .layers import _act, _check, _dtype, _DTYPES, _elsewhere, _gradient_lost, _new_checkpoint, _On, _output, _refuse, _rows, _same, _saved, _stream

EXPORTS = ["eden_mx4_bytes", "eden_mx4_quantize", "eden_mx4_sums_bytes", "eden_mx4_restore", "eden_mx4_workspace_bytes", "eden_mx4_linear", "eden_mx4_input_grad", "eden_mx4_weight_grad"]
CHUNK = 256                                                       # columns of a row's 128 bytes of codes and 8 exponents
MOST_ROWS, MOST_COLUMNS = 2 ** 27, 2 ** 22
OWN_ROWS, OWN_VALUES = 16, 16384                                 # up to here linear rounds x without a workspace
_lib = None


def lib():
    """The built library with this header's entry points declared."""
    global _lib
    if _lib is not None:
        return _lib
    L = eden.lib()
    vp, u64, u32, sz, ci = ctypes.c_void_p, ctypes.c_uint64, ctypes.c_uint32, ctypes.c_size_t, ctypes.c_int
    for name, args, result in (("eden_mx4_bytes", [u64, u64], sz), ("eden_mx4_sums_bytes", [u64, u64], sz), ("eden_mx4_workspace_bytes", [u64, u64, u64, ci], sz),
                               ("eden_mx4_quantize", [vp, u64, u64, u64, u32, ci, ctypes.c_char_p, vp, sz, vp, ci, vp, sz, vp], ci),
                               ("eden_mx4_restore", [vp, u64, u64, u32, vp, u64, vp], ci),
                               ("eden_mx4_linear", [vp, u64, vp, vp, vp, vp, u64, vp, u64, vp, sz, u64, u64, u64, u32, u32, vp, sz, vp], ci),
                               ("eden_mx4_input_grad", [vp, vp, vp, u32, vp, u64, vp, u64, u64, u64, u64, u32, vp, sz, vp], ci),
                               ("eden_mx4_weight_grad", [vp, vp, vp, u64, u64, u64, u64, ci, vp, sz, vp], ci)):
        f = getattr(L, name)
        f.argtypes, f.restype = args, result
    _lib = L
    return L


def _bytes(rows, cols):
    chunks = -(-cols // CHUNK)
    return chunks * (rows * (CHUNK // 2) + (rows + rows % 2) * 8)


def _sizes(rows, cols, what):
    if rows > MOST_ROWS or cols > MOST_COLUMNS:
        _refuse(f"{what}: {rows} x {cols}, at most {MOST_ROWS} rows of {MOST_COLUMNS}")


def mx4_bytes(rows: int, cols: int) -> int:
    return int(lib().eden_mx4_bytes(rows, cols))


class Stochastic:
    """Rounding that keeps the expectation, from 16 bits of the counter hash of (seed, id, row, column).  seed: a number, or an int64 tensor on the GPU that is read when
    the kernels run."""

    __slots__ = ("seed", "id")

    def __init__(self, seed, id: int = 0):
        self.seed, self.id = seed, id


class Mx4:
    """The 4 bits of a rows x cols matrix in a buffer of mx4_bytes(rows, cols) bytes."""

    __slots__ = ("buffer", "rows", "cols")

    def __init__(self, buffer, rows: int, cols: int):
        _sizes(rows, cols, "Mx4")
        need = _bytes(rows, cols)
        if buffer.dtype is not torch.uint8 or not buffer.is_cuda or not buffer.is_contiguous() or buffer.numel() < need:
            _refuse(f"Mx4: a contiguous uint8 buffer of {need} bytes on the GPU is needed")
        if buffer.numel() and buffer.data_ptr() % 16:
            _refuse("Mx4: the buffer does not begin at a multiple of 16 bytes")
        self.buffer, self.rows, self.cols = buffer, rows, cols

    def restore(self, dtype=torch.bfloat16, out=None, stream=None):
        """The values it stands for."""
        device = self.buffer.device
        if _elsewhere(device, stream):
            with _On(device, stream):
                return self.restore(dtype, out)
        if out is None:
            code = _DTYPES.get(dtype)
            if code is None:
                _refuse(f"restore: {dtype}")
            out = torch.empty((self.rows, self.cols), dtype=dtype, device=device)
        else:
            code = _dtype(out, "restore: out")
            if out.device != device:
                _refuse(f"restore: out on {out.device}, the 4 bits on {device}")
            if out.requires_grad:
                _gradient_lost("restore: out")
        p, ld, rows, cols = _rows(out, "restore: out")
        if rows != self.rows or cols != self.cols:
            _refuse(f"restore: out is {rows} x {cols}, the 4 bits {self.rows} x {self.cols}")
        _check((_lib or lib()).eden_mx4_restore(self.buffer.data_ptr(), rows, cols, code, p, ld, _stream(device)), "eden_mx4_restore")
        return out


def quantize(x, transpose: bool = False, rounding: Stochastic = None, into: Mx4 = None, sums=False, accumulate: bool = False, stream=None):
    """The 4 bits of x, or of its transpose.  `rounding`: None for the nearest; `into`: an Mx4 of the same size that is overwritten.  With `sums` (transpose only; True, or a
    float32 tensor that is written or, with `accumulate`, added to) also the sums of x's columns: (Mx4, sums).  x is refused where it requires a gradient and autograd records."""
    dtype = _dtype(x, "quantize: x")
    device = x.device
    if _elsewhere(device, stream):
        with _On(device, stream):
            return quantize(x, transpose, rounding, into, sums, accumulate)
    L = _lib or lib()
    if x.requires_grad:
        _gradient_lost("quantize: x")                              # (here, since an Mx4 no longer says where it comes from)
    p, ld, rows, cols = _rows(x, "quantize: x")
    r, c = (cols, rows) if transpose else (rows, cols)
    _sizes(r, c, "quantize")
    with_sums = sums is not False and sums is not None
    if with_sums and not transpose:
        _refuse("quantize: sums go with transpose")
    if accumulate and (not with_sums or sums is True):
        _refuse("quantize: nothing to accumulate in")
    if into is None:
        into = Mx4.__new__(Mx4)
        into.buffer, into.rows, into.cols = torch.empty(_bytes(r, c), dtype=torch.uint8, device=device), r, c
    elif (into.rows, into.cols) != (r, c) or into.buffer.device != device:
        _refuse(f"quantize: into is {into.rows} x {into.cols} on {into.buffer.device}, expected {r} x {c} on {device}")
    random = None if rounding is None else blocks._RANDOM_ARGS.pack(*blocks._random(rounding.seed, rounding.id, 0, device, "quantize"))
    total, tp, ws, wsp, size = None, None, None, None, 0
    if with_sums:
        total, tp, _ = _output(None if sums is True else sums, (cols,), x, "quantize: sums", torch.float32)
        size = L.eden_mx4_sums_bytes(rows, cols)
        if size:
            ws = torch.empty(size, dtype=torch.uint8, device=device)
            wsp = ws.data_ptr()
    buffer = into.buffer
    _check(L.eden_mx4_quantize(p, ld, rows, cols, dtype, 1 if transpose else 0, random, buffer.data_ptr(), buffer.numel(), tp, 1 if accumulate else 0, wsp, size, _stream(device)),
           "eden_mx4_quantize")
    return (into, total) if with_sums else into


def _operand(v, rows, depth, device, what):
    """Address of a packed operand of that size; rows: None for any."""
    if not isinstance(v, Mx4):
        _refuse(f"{what}: 4 bits (Mx4) are needed, got {type(v).__name__}")
    if (rows is not None and v.rows != rows) or v.cols != depth or v.buffer.device != device:
        _refuse(f"{what}: {v.rows} x {v.cols} on {v.buffer.device}, expected {'any' if rows is None else rows} x {depth} on {device}")
    return v.buffer.data_ptr()


def _workspace(L, rows, cols, depth, quantizes, device):
    size = L.eden_mx4_workspace_bytes(rows, cols, depth, quantizes)
    if not size:
        return None, None, 0
    t = torch.empty(size, dtype=torch.uint8, device=device)
    return t, t.data_ptr(), size


def _like(dtype, other, device, what):
    """A tensor that has the type and device of a call without one: that of `other`, or of `dtype`."""
    if other is not None:
        if dtype is not None and other.dtype is not dtype:
            _refuse(f"{what}: {other.dtype}, expected {dtype}")
        return other
    return torch.empty(0, dtype=dtype or torch.bfloat16, device=device)


def linear(x, w: Mx4, bias=None, activation: str = "none", residual=None, checkpoint=False, dtype=None, out=None, stream=None):
    """act(x^ w^T + bias) + residual; x: a tensor, rounded to the nearest, or its Mx4 (then `dtype` is the result's, bfloat16 if there is no residual or bias to go by).
    `checkpoint`: True or a Checkpoint to be overwritten: returns (y, 8-bit checkpoint of x^ w^T + bias)."""
    packed = isinstance(x, Mx4)
    device = x.buffer.device if packed else x.device
    if not packed:
        _dtype(x, "linear: x")
    if _elsewhere(device, stream):
        with _On(device, stream):
            return linear(x, w, bias, activation, residual, checkpoint, dtype, out)
    L = _lib or lib()
    act = _act(activation, "linear")
    if packed:
        m, k, xp, ldx, x4p = x.rows, x.cols, None, 0, x.buffer.data_ptr()
        like = _like(dtype, residual if residual is not None else bias if bias is not None else out, device, "linear")
        shape = (m, w.rows if isinstance(w, Mx4) else 0)
    else:
        if x.requires_grad:
            _gradient_lost("linear: x")
        like = _like(dtype, x, device, "linear: x")
        x4p = None
        xp, ldx, m, k = _rows(x, "linear: x")
        _sizes(m, k, "linear: x")
        shape = (m, w.rows if isinstance(w, Mx4) else 0) if x.dim() == 2 else x.shape[:-1] + (w.rows if isinstance(w, Mx4) else 0,)
    wp = _operand(w, None, k, device, "linear: w")
    n = w.rows
    code = _dtype(like, "linear")
    bp = rp = None
    ldr = n
    if bias is not None:
        _same(bias, like, "linear: bias")
        if bias.dim() != 1 or bias.shape[0] != n or (n > 1 and bias.stride(0) != 1):
            _refuse(f"linear: bias is {tuple(bias.shape)} with stride {bias.stride()}, expected {n} neighbours")
        bp = bias.data_ptr()
    if residual is not None:
        _same(residual, like, "linear: residual")
        if residual.shape != shape:
            _refuse(f"linear: residual is {tuple(residual.shape)}, expected {tuple(shape)}")
        rp, ldr, _, _ = _rows(residual, "linear: residual")
    y, yp, ldy = _output(out, shape, like, "linear: out", like.dtype)
    c, cp, capacity = None, None, 0
    if checkpoint is not False and checkpoint is not None:
        c = _new_checkpoint(None if checkpoint is True else checkpoint, m, n, device)
        cp, capacity = c.buffer.data_ptr(), c.buffer.numel()
    ws, wsp, size = None, None, 0
    if not (m <= OWN_ROWS and m * k <= OWN_VALUES) or packed:
        ws, wsp, size = _workspace(L, m, n, k, 0 if packed else 1, device)
    _check(L.eden_mx4_linear(xp, ldx, x4p, wp, bp, rp, ldr, yp, ldy, cp, capacity, m, n, k, code, act, wsp, size, _stream(device)), "eden_mx4_linear")
    return y if c is None else (y, c)


def linear_input_grad(dz: Mx4, wt: Mx4, activation: str = "none", checkpoint=None, residual=None, dtype=None, out=None, stream=None):
    """(dz w) * act'(z) + residual, wt: the 4 bits of w's transpose; z: the checkpoint of the input of the activation in front of the layer (none without one).
    `dtype`: the result's, bfloat16 if there is no residual or `out` to go by."""
    if not isinstance(dz, Mx4):
        _refuse(f"linear_input_grad: dz: 4 bits (Mx4) are needed, got {type(dz).__name__}")
    device = dz.buffer.device
    if _elsewhere(device, stream):
        with _On(device, stream):
            return linear_input_grad(dz, wt, activation, checkpoint, residual, dtype, out)
    L = _lib or lib()
    act = _act(activation, "linear_input_grad")
    m, n = dz.rows, dz.cols
    wp = _operand(wt, None, n, device, "linear_input_grad: wt")
    k = wt.rows
    if (checkpoint is None) != (act == 0):
        _refuse("linear_input_grad: an activation and the checkpoint of its input go together")
    sp = None if checkpoint is None else _saved(checkpoint, m, k, device, "linear_input_grad")
    shape = residual.shape if residual is not None else out.shape if out is not None else (m, k)
    like = _like(dtype, residual if residual is not None else out, device, "linear_input_grad")
    code = _dtype(like, "linear_input_grad")
    rp, ldr = None, k
    if residual is not None:
        _same(residual, like, "linear_input_grad: residual")
        rp, ldr, rows, cols = _rows(residual, "linear_input_grad: residual")
        if (rows, cols) != (m, k):
            _refuse(f"linear_input_grad: residual is {tuple(residual.shape)}, expected {m} x {k}")
    dx, xp, ldx = _output(out, shape, like, "linear_input_grad: out", like.dtype)
    if tuple(dx.shape) != (m, k) and _rows(dx, "linear_input_grad: out")[2:] != (m, k):
        _refuse(f"linear_input_grad: out is {tuple(dx.shape)}, expected {m} x {k}")
    ws, wsp, size = _workspace(L, m, k, n, 0, device)
    _check(L.eden_mx4_input_grad(dz.buffer.data_ptr(), wp, sp, act, rp, ldr, xp, ldx, m, n, k, code, wsp, size, _stream(device)), "eden_mx4_input_grad")
    return dx


def linear_weight_grad(dyt: Mx4, xt: Mx4, out=None, accumulate: bool = False, stream=None):
    """dy^T x (fp32) from the 4 bits of both transposes.  `out`: where to write it, for instance a part of the vector that Context.encode takes; `accumulate`: add to
    what it holds."""
    if not isinstance(dyt, Mx4):
        _refuse(f"linear_weight_grad: dyt: 4 bits (Mx4) are needed, got {type(dyt).__name__}")
    device = dyt.buffer.device
    if _elsewhere(device, stream):
        with _On(device, stream):
            return linear_weight_grad(dyt, xt, out, accumulate)
    L = _lib or lib()
    n, m = dyt.rows, dyt.cols
    xp = _operand(xt, None, m, device, "linear_weight_grad: xt")
    k = xt.rows
    if accumulate and out is None:
        _refuse("linear_weight_grad: nothing to accumulate in")
    dw, wp, ldw = _output(out, (n, k), dyt.buffer, "linear_weight_grad: out", torch.float32)
    ws, wsp, size = _workspace(L, n, k, m, 0, device)
    _check(L.eden_mx4_weight_grad(dyt.buffer.data_ptr(), xp, wp, ldw, m, n, k, 1 if accumulate else 0, wsp, size, _stream(device)), "eden_mx4_weight_grad")
    return dw
