"""Layer operators (include/eden_layers.h): a linear layer that is trained from 8-bit activation checkpoints.

    y, z = linear(x, w, bias, activation="gelu", residual=r, checkpoint=True)     # z: the activation's input in 8 bits
    kept = save_checkpoint(x)                                                     # the layer's input in 8 bits
    dz = activation_grad(dy, z, "gelu")
    dw, db = linear_weight_grad(dz, kept, bias=True)                              # fp32: what Context.encode takes
    dx = linear_input_grad(dz, w)       # or, through the activation in front of the layer, activation=, checkpoint=

Tensors are torch CUDA(HIP) tensors of float32, float16 or bfloat16 with unit distance between the last dimension's elements; dimensions
in front of it are rows.  Argument checks, allocation and marshalling only: every step runs in the HIP kernels, on the current
stream or the one given.  What does not fit raises EdenError (ERR_INVALID_ARG) before anything is launched.

An `out` must not overlap an operand, except that linear's and linear_input_grad's may be the residual itself and activation_grad's dy itself.  With `stream` the operands have
to be ready on that stream and to stay until its work is done; results and workspaces are allocated on it.

The calls record nothing for autograd: the backward pass is made of calls as above, by hand or in the two halves of a torch.autograd.Function.
Where autograd records, an operand or an `out` that requires a gradient is refused, since the gradient would be lost (`torch.no_grad()` or `detach()` says
that none is expected); save_checkpoint takes it.
"""
from __future__ import annotations

import ctypes

import torch

from . import eden
from .eden import EdenError

F32, F16, BF16 = 0, 1, 2
BLOCK = 32                                                        # columns of a checkpoint block
ACTIVATIONS = {"none": 0, "relu": 1, "gelu": 2, "gelu_tanh": 3, "silu": 4}
EXPORTS = ["eden_checkpoint_bytes", "eden_checkpoint_save", "eden_checkpoint_restore", "eden_layers_workspace_bytes", "eden_layers_copying_bytes", "eden_linear",
           "eden_linear_weight_grad", "eden_linear_input_grad", "eden_activation_grad"]

_DTYPES = {torch.float32: F32, torch.float16: F16, torch.bfloat16: BF16}
_lib = None


def lib():
    """The built library with this header's entry points declared."""
    global _lib
    if _lib is not None:
        return _lib
    L = eden.lib()
    vp, u64, u32, sz, ci = ctypes.c_void_p, ctypes.c_uint64, ctypes.c_uint32, ctypes.c_size_t, ctypes.c_int
    L.eden_checkpoint_bytes.argtypes = [u64, u64]
    L.eden_checkpoint_bytes.restype = sz
    L.eden_layers_workspace_bytes.argtypes = [u64, u64, u64, u32]
    L.eden_layers_workspace_bytes.restype = sz
    L.eden_layers_copying_bytes.argtypes = [u64, u64, u64, u32]
    L.eden_layers_copying_bytes.restype = sz
    for name, args in (("eden_checkpoint_save", [vp, u64, u64, u64, u32, vp, sz, vp]),
                       ("eden_checkpoint_restore", [vp, u64, u64, u32, vp, u64, vp]),
                       ("eden_linear", [vp, u64, vp, u64, vp, vp, u64, vp, u64, vp, sz, u64, u64, u64, u32, u32, vp, sz, vp]),
                       ("eden_linear_weight_grad", [vp, u64, vp, vp, u64, vp, u64, u64, u64, u32, ci, vp, sz, vp]),
                       ("eden_linear_input_grad", [vp, u64, vp, u64, vp, u32, vp, u64, vp, u64, u64, u64, u64, u32, vp, sz, vp]),
                       ("eden_activation_grad", [vp, u64, vp, u32, vp, u64, u64, u64, u32, vp])):
        f = getattr(L, name)
        f.argtypes, f.restype = args, ci
    _lib = L
    return L


def _refuse(what):
    raise EdenError(eden.ERR_INVALID_ARG, what)


def _check(rc, what):
    if rc != eden.OK:
        raise EdenError(rc, what)


def _dtype(t, what):
    code = _DTYPES.get(t.dtype)
    if code is None or not t.is_cuda:
        _refuse(f"{what}: a float32, float16 or bfloat16 tensor on the GPU is needed, got {t.dtype} on {t.device}")
    return code


def _rows(t, what):
    """(address, distance between rows, rows, columns) of a tensor seen as a matrix of its last dimension."""
    if t.dim() == 2:
        rows, cols = t.shape
        ld, unit = t.stride()
    else:
        if t.dim() == 0:
            _refuse(f"{what}: at least one dimension is needed")
        cols = t.shape[-1]
        if t.numel() == 0:                                        # nothing is read or written: only the sizes count
            rows = 1
            for s in t.shape[:-1]:
                rows *= s
            return t.data_ptr(), cols, rows, cols
        try:
            m = t.view(-1, cols)
        except RuntimeError:
            _refuse(f"{what}: the dimensions in front of the last are not rows at one distance")
        rows, (ld, unit) = m.shape[0], m.stride()
    if rows and cols and ((cols > 1 and unit != 1) or (rows > 1 and ld < cols)):
        _refuse(f"{what}: rows must not overlap and the last dimension's elements must be neighbours, strides {tuple(t.stride())}")
    return t.data_ptr(), ld if rows > 1 else cols, rows, cols


def _gradient_lost(what):
    """For a tensor that requires a gradient: refused where autograd records."""
    if torch.is_grad_enabled():
        _refuse(f"{what} requires a gradient, but nothing is recorded for autograd (torch.no_grad() or detach() where none is expected)")


def _same(t, like, what):
    if t.dtype is not like.dtype or t.device != like.device:
        _refuse(f"{what}: {t.dtype} on {t.device}, expected {like.dtype} on {like.device}")
    if t.requires_grad:
        _gradient_lost(what)


def _output(out, shape, like, what, dtype=None):
    """(tensor, address, distance between rows) of `out`, or of a new tensor of that shape of like's type (or `dtype`) on its device."""
    if out is None:
        out = like.new_empty(shape) if dtype is None else like.new_empty(shape, dtype=dtype)
        return out, out.data_ptr(), shape[-1]
    dtype = dtype or like.dtype
    if tuple(out.shape) != tuple(shape) or out.dtype is not dtype or out.device != like.device:
        _refuse(f"{what}: {tuple(out.shape)} of {out.dtype} on {out.device}, expected {tuple(shape)} of {dtype} on {like.device}")
    if out.requires_grad:
        _gradient_lost(what)
    address, ld, _, _ = _rows(out, what)
    return out, address, ld


def _act(name, what):
    code = ACTIVATIONS.get(name)
    if code is None:
        _refuse(f"{what}: unknown activation {name!r}")
    return code


class _On:
    """Makes the tensors' device current and, where a stream is given, has torch allocate on it, so that memory freed on
    return is reused behind the call's kernels."""

    __slots__ = ("stacked",)

    def __init__(self, device, stream):
        if stream is not None and stream.device != device:
            _refuse(f"stream on {stream.device}, tensors on {device}")
        self.stacked = torch.cuda.device(device) if stream is None else torch.cuda.stream(stream)

    def __enter__(self):
        return self.stacked.__enter__()

    def __exit__(self, *e):
        return self.stacked.__exit__(*e)


def _elsewhere(device, stream):
    """Whether a call has to change the current device or stream first."""
    return stream is not None or torch.cuda.current_device() != device.index


def _stream(device):
    """Address of the device's current stream (the device is the current one)."""
    try:
        return torch._C._cuda_getCurrentRawStream(device.index)
    except AttributeError:
        return torch.cuda.current_stream(device).cuda_stream


def _workspace(L, rows, cols, depth, dtype, device, addresses, elements):
    """A workspace; `addresses`: those of the operands or-ed together, `elements`: distances and widths: multiples of 16 bytes need no copies."""
    whole = addresses % 16 == 0 and elements % (4 if dtype == F32 else 8) == 0
    size = (L.eden_layers_workspace_bytes if whole else L.eden_layers_copying_bytes)(rows, cols, depth, dtype)
    if not size:
        return None, None, 0
    t = torch.empty(size, dtype=torch.uint8, device=device)
    return t, t.data_ptr(), size


def checkpoint_bytes(rows: int, cols: int) -> int:
    return int(lib().eden_checkpoint_bytes(rows, cols))


class Checkpoint:
    """The 8-bit checkpoint of a rows x cols matrix in a buffer of checkpoint_bytes(rows, cols) bytes (33 for 32 values)."""

    __slots__ = ("buffer", "rows", "cols")

    def __init__(self, buffer, rows: int, cols: int):
        need = rows * -(-cols // BLOCK) * (BLOCK + 1)
        if buffer.dtype is not torch.uint8 or not buffer.is_cuda or not buffer.is_contiguous() or buffer.numel() < need:
            _refuse(f"Checkpoint: a contiguous uint8 buffer of {need} bytes on the GPU is needed")
        self.buffer, self.rows, self.cols = buffer, rows, cols

    def restore(self, dtype=torch.bfloat16, out=None, stream=None):
        """The values it stands for (exact in bfloat16 and float32)."""
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
                _refuse(f"restore: out on {out.device}, the checkpoint on {device}")
        p, ld, rows, cols = _rows(out, "restore: out")
        if rows != self.rows or cols != self.cols:
            _refuse(f"restore: out is {rows} x {cols}, the checkpoint {self.rows} x {self.cols}")
        _check((_lib or lib()).eden_checkpoint_restore(self.buffer.data_ptr(), rows, cols, code, p, ld, _stream(device)), "eden_checkpoint_restore")
        return out


def _new_checkpoint(into, rows, cols, device):
    if into is None:
        c = Checkpoint.__new__(Checkpoint)
        c.buffer, c.rows, c.cols = torch.empty(rows * -(-cols // BLOCK) * (BLOCK + 1), dtype=torch.uint8, device=device), rows, cols
        return c
    if (into.rows, into.cols) != (rows, cols) or into.buffer.device != device:
        _refuse(f"checkpoint of {into.rows} x {into.cols} on {into.buffer.device}, expected {rows} x {cols} on {device}")
    return into


def _saved(c, rows, cols, device, what):
    if c.rows != rows or c.cols != cols or c.buffer.device != device:
        _refuse(f"{what}: checkpoint of {c.rows} x {c.cols} on {c.buffer.device}, expected {rows} x {cols} on {device}")
    return c.buffer.data_ptr()


def save_checkpoint(x, into=None, stream=None) -> Checkpoint:
    """The 8-bit checkpoint of x; `into`: a Checkpoint of the same size that is overwritten."""
    dtype = _dtype(x, "save_checkpoint: x")
    device = x.device
    if _elsewhere(device, stream):
        with _On(device, stream):
            return save_checkpoint(x, into)
    p, ld, rows, cols = _rows(x, "save_checkpoint: x")
    c = _new_checkpoint(into, rows, cols, device)
    buffer = c.buffer
    _check((_lib or lib()).eden_checkpoint_save(p, ld, rows, cols, dtype, buffer.data_ptr(), buffer.numel(), _stream(device)), "eden_checkpoint_save")
    return c


def linear(x, w, bias=None, activation: str = "none", residual=None, checkpoint=False, out=None, stream=None):
    """act(x w^T + bias) + residual.  `checkpoint`: True or a Checkpoint to be overwritten: returns (y, checkpoint of x w^T + bias)."""
    dtype = _dtype(x, "linear: x")
    device = x.device
    if _elsewhere(device, stream):
        with _On(device, stream):
            return linear(x, w, bias, activation, residual, checkpoint, out)
    L = _lib or lib()
    if x.requires_grad:
        _gradient_lost("linear: x")
    act = _act(activation, "linear")
    xp, ldx, m, k = _rows(x, "linear: x")
    _same(w, x, "linear: w")
    if w.dim() != 2 or w.shape[1] != k:
        _refuse(f"linear: w is {tuple(w.shape)}, x has {k} columns")
    wp, ldw, n, _ = _rows(w, "linear: w")
    bp = rp = None
    ldr = n
    if bias is not None:
        _same(bias, x, "linear: bias")
        if bias.dim() != 1 or bias.shape[0] != n or (n > 1 and bias.stride(0) != 1):
            _refuse(f"linear: bias is {tuple(bias.shape)} with stride {bias.stride()}, expected {n} neighbours")
        bp = bias.data_ptr()
    shape = (m, n) if x.dim() == 2 else x.shape[:-1] + (n,)
    if residual is not None:
        _same(residual, x, "linear: residual")
        if residual.shape != shape:
            _refuse(f"linear: residual is {tuple(residual.shape)}, expected {tuple(shape)}")
        rp, ldr, _, _ = _rows(residual, "linear: residual")
    y, yp, ldy = _output(out, shape, x, "linear: out")
    c, cp, capacity = None, None, 0
    if checkpoint is not False and checkpoint is not None:
        c = _new_checkpoint(None if checkpoint is True else checkpoint, m, n, device)
        cp, capacity = c.buffer.data_ptr(), c.buffer.numel()
    ws, wsp, size = None, None, 0
    if m > 16 or (m > 4 and dtype != F32):                         # fewer rows use none
        ws, wsp, size = _workspace(L, m, n, k, dtype, device, xp | wp, ldx | ldw | k)
    _check(L.eden_linear(xp, ldx, wp, ldw, bp, rp, ldr, yp, ldy, cp, capacity, m, n, k, dtype, act, wsp, size, _stream(device)), "eden_linear")
    return y if c is None else (y, c)


def linear_weight_grad(dy, saved: Checkpoint, bias: bool = False, out=None, bias_out=None, accumulate: bool = False, stream=None):
    """dy^T x (fp32) from the checkpoint of x; with `bias` (dw, sum of dy's rows).  `out`, `bias_out`: where to write them, for instance
    parts of the vector that Context.encode takes; `accumulate`: add to what they hold."""
    dtype = _dtype(dy, "linear_weight_grad: dy")
    device = dy.device
    if _elsewhere(device, stream):
        with _On(device, stream):
            return linear_weight_grad(dy, saved, bias, out, bias_out, accumulate)
    L = _lib or lib()
    if dy.requires_grad:
        _gradient_lost("linear_weight_grad: dy")
    dp, ldy, m, n = _rows(dy, "linear_weight_grad: dy")
    k = saved.cols
    sp = _saved(saved, m, k, device, "linear_weight_grad")
    if accumulate and (out is None or (bias and bias_out is None)):
        _refuse("linear_weight_grad: nothing to accumulate in")
    dw, wp, ldw = _output(out, (n, k), dy, "linear_weight_grad: out", torch.float32)
    db, bp = None, None
    if bias or bias_out is not None:
        db, bp, _ = _output(bias_out, (n,), dy, "linear_weight_grad: bias_out", torch.float32)
    ws, wsp, size = _workspace(L, n, k, m, dtype, device, dp, ldy | n) if dtype == BF16 else _workspace(L, n, k, m, dtype, device, 0, 0)
    _check(L.eden_linear_weight_grad(dp, ldy, sp, wp, ldw, bp, m, n, k, dtype, 1 if accumulate else 0, wsp, size, _stream(device)), "eden_linear_weight_grad")
    return dw if db is None else (dw, db)


def linear_input_grad(dz, w, activation: str = "none", checkpoint: Checkpoint = None, residual=None, out=None, stream=None):
    """(dz w) * act'(z) + residual; z: the checkpoint of the input of the activation in front of the layer (none without one)."""
    dtype = _dtype(dz, "linear_input_grad: dz")
    device = dz.device
    if _elsewhere(device, stream):
        with _On(device, stream):
            return linear_input_grad(dz, w, activation, checkpoint, residual, out)
    L = _lib or lib()
    if dz.requires_grad:
        _gradient_lost("linear_input_grad: dz")
    act = _act(activation, "linear_input_grad")
    dp, ldz, m, n = _rows(dz, "linear_input_grad: dz")
    _same(w, dz, "linear_input_grad: w")
    if w.dim() != 2 or w.shape[0] != n:
        _refuse(f"linear_input_grad: w is {tuple(w.shape)}, dz has {n} columns")
    wp, ldw, _, k = _rows(w, "linear_input_grad: w")
    if (checkpoint is None) != (act == 0):
        _refuse("linear_input_grad: an activation and the checkpoint of its input go together")
    sp = None if checkpoint is None else _saved(checkpoint, m, k, device, "linear_input_grad")
    rp, ldr = None, k
    shape = (m, k) if dz.dim() == 2 else dz.shape[:-1] + (k,)
    if residual is not None:
        _same(residual, dz, "linear_input_grad: residual")
        if residual.shape != shape:
            _refuse(f"linear_input_grad: residual is {tuple(residual.shape)}, expected {tuple(shape)}")
        rp, ldr, _, _ = _rows(residual, "linear_input_grad: residual")
    dx, xp, ldx = _output(out, shape, dz, "linear_input_grad: out")
    ws, wsp, size = _workspace(L, m, k, n, dtype, device, dp | wp, ldz | ldw | n | k)
    _check(L.eden_linear_input_grad(dp, ldz, wp, ldw, sp, act, rp, ldr, xp, ldx, m, n, k, dtype, wsp, size, _stream(device)), "eden_linear_input_grad")
    return dx


def activation_grad(dy, saved: Checkpoint, activation: str, out=None, stream=None):
    """dy * act'(z), z from its checkpoint."""
    dtype = _dtype(dy, "activation_grad: dy")
    device = dy.device
    if _elsewhere(device, stream):
        with _On(device, stream):
            return activation_grad(dy, saved, activation, out)
    if dy.requires_grad:
        _gradient_lost("activation_grad: dy")
    act = _act(activation, "activation_grad")
    dp, ldy, rows, cols = _rows(dy, "activation_grad: dy")
    sp = _saved(saved, rows, cols, device, "activation_grad")
    dz, zp, ldz = _output(out, dy.shape, dy, "activation_grad: out")
    _check((_lib or lib()).eden_activation_grad(dp, ldy, sp, act, zp, ldz, rows, cols, dtype, _stream(device)), "eden_activation_grad")
    return dz
