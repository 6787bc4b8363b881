"""Operators around a residual block (include/eden_blocks.h): dropout, norms, and the join of a block's branches with the norm of the next block.

    drop = Dropout(0.1, seed, id=layer)                       # seed: a number, or an int64 tensor on the GPU that is read when the kernels run
    pre, post = Norm("rms", w1), Norm("layer", w2, b2)
    h = norm(x, pre)                                          # in front of the first block
    r, h = join(x, f, gate=g, dropout=drop, post=post, pre=pre)      # x + g * dropout(post(f)), and pre of it for the next block
    grads = join_grad(dr, f, dh=dh, r=r, gate=g, dropout=drop, post=post, pre=pre)     # .dx .df .gate .post_weight .post_bias .pre_weight .pre_bias
    grads = norm_grad(dh, x, pre)                             # .dx .pre_weight .pre_bias
    y = dropout(x, drop); dx = dropout(dy, drop)

Tensors, streams, errors and autograd are as in layers.py: float32, float16 or bfloat16 on the GPU, dimensions in front of the last are rows at one distance, what
does not fit raises EdenError before anything is launched.  Rows have up to MOST_COLUMNS columns.  Gradients that are sums over rows are float32.

A gate has a value for each column, or rows of them: g x columns next to x of g * n rows, n consecutive rows to each (one gate for each sequence of a batch).

Masks are not kept: dropout drops a value if 16 bits of the counter hash of (seed, id, row, column) are below round(65536 p); the backward pass names the same
Dropout.  Calls that share seed and id drop the same places.
"""
from __future__ import annotations

import ctypes
import operator
import struct
from typing import NamedTuple, Optional

import torch

from . import eden, layers
from .layers import _check, _dtype, _elsewhere, _gradient_lost, _On, _output, _refuse, _rows, _same, _stream

MOST_COLUMNS = 16384
NORMS = {"rms": 1, "layer": 2}
EXPORTS = ["eden_dropout", "eden_join", "eden_join_grad", "eden_join_workspace_bytes"]
_lib = None


class RandomArgs(ctypes.Structure):
    _fields_ = [("seed", ctypes.c_uint64), ("seed_at", ctypes.c_void_p), ("id", ctypes.c_uint32), ("threshold", ctypes.c_uint32)]


class NormArgs(ctypes.Structure):
    _fields_ = [("kind", ctypes.c_uint32), ("eps", ctypes.c_float), ("weight", ctypes.c_void_p), ("bias", ctypes.c_void_p)]


def _fields(kind, names):
    return [(name, kind) for name in names.split()]


class JoinArgs(ctypes.Structure):
    _fields_ = (_fields(ctypes.c_uint64, "rows cols") + _fields(ctypes.c_void_p, "x f gate r h") + _fields(ctypes.c_uint64, "ldx ldf ld_gate ldr ldh gates")
                + _fields(NormArgs, "post pre") + _fields(RandomArgs, "random") + _fields(ctypes.c_float, "x_scale scale") + _fields(ctypes.c_uint32, "dtype"))


class JoinGradArgs(ctypes.Structure):
    _fields_ = (_fields(ctypes.c_uint64, "rows cols") + _fields(ctypes.c_void_p, "dr dh r f gate dx df") + _fields(ctypes.c_uint64, "lddr lddh ldr ldf ld_gate lddx lddf gates")
                + _fields(ctypes.c_void_p, "gate_grad post_weight_grad post_bias_grad pre_weight_grad pre_bias_grad") + _fields(ctypes.c_uint64, "ld_gate_grad")
                + _fields(NormArgs, "post pre") + _fields(RandomArgs, "random") + _fields(ctypes.c_float, "x_scale scale") + _fields(ctypes.c_uint32, "dtype branch accumulate")
                + _fields(ctypes.c_void_p, "workspace") + _fields(ctypes.c_size_t, "workspace_bytes"))


# The same structures as strings of bytes: a call packs its arguments at once (a ctypes field at a time takes the longer part of a short call)
_RANDOM, _NORM = "QPII", "IfPP"
_RANDOM_ARGS = struct.Struct(_RANDOM)
_JOIN_ARGS = struct.Struct("QQ5P6Q" + 2 * _NORM + _RANDOM + "ffI4x")
_JOIN_GRAD_ARGS = struct.Struct("QQ7P8Q5PQ" + 2 * _NORM + _RANDOM + "ffIII4xPN")


def lib():
    """The built library with this header's entry points declared."""
    global _lib
    if _lib is not None:
        return _lib
    L = eden.lib()
    vp, u64, u32 = ctypes.c_void_p, ctypes.c_uint64, ctypes.c_uint32
    L.eden_join_workspace_bytes.argtypes, L.eden_join_workspace_bytes.restype = [u64, u64, u64, u32], ctypes.c_size_t
    for name, args in (("eden_dropout", [vp, u64, vp, u64, u64, u64, u32, ctypes.c_char_p, vp]), ("eden_join", [ctypes.c_char_p, vp]),
                       ("eden_join_grad", [ctypes.c_char_p, vp])):
        f = getattr(L, name)
        f.argtypes, f.restype = args, ctypes.c_int
    _lib = L
    return L


def _random(seed, number, threshold, device, what):
    """The fields of RandomArgs for a seed that is a number, or an int64 tensor on the device."""
    try:
        number = operator.index(number)
    except TypeError:
        _refuse(f"{what}: an id is a whole number, got {number!r}")
    if not 0 <= number < 2 ** 32:
        _refuse(f"{what}: id {number} is not in 0 .. 2^32 - 1")
    if not isinstance(seed, torch.Tensor):
        try:
            return operator.index(seed) & (2 ** 64 - 1), 0, number, threshold
        except TypeError:
            _refuse(f"{what}: a seed is a whole number or a tensor, got {type(seed).__name__}")
    if seed.dtype is not torch.int64 or seed.numel() != 1 or (device is not None and seed.device != device) or not seed.is_cuda:
        _refuse(f"{what}: a seed tensor is one int64 on the operands' device, got {seed.numel()} of {seed.dtype} on {seed.device}")
    return 0, seed.data_ptr(), number, threshold


class Dropout:
    """Drops a value with probability p (rounded to 1/65536), the others are multiplied by 1 / (1 - p)."""

    __slots__ = ("p", "seed", "id", "threshold")

    def __init__(self, p: float, seed, id: int = 0):
        threshold = round(65536 * p) if 0.0 <= p < 1.0 else -1
        if not 0 <= threshold <= 65535:
            _refuse(f"Dropout: p = {p} is not in 0 .. 1 - 2^-16")
        self.p, self.seed, self.id, self.threshold = p, seed, id, threshold

    def _args(self, device, what):
        return _random(self.seed, self.id, self.threshold, device, what)


class Norm:
    """rms: v / sqrt(mean(v^2) + eps) * weight; layer: (v - mean) / sqrt(var + eps) * weight + bias.  Without weight ones, without bias zeros."""

    __slots__ = ("kind", "weight", "bias", "eps", "code")

    def __init__(self, kind: str, weight=None, bias=None, eps: float = 1e-5):
        self.kind, self.weight, self.bias, self.eps, self.code = kind, weight, bias, eps, NORMS.get(kind)
        if self.code is None:
            _refuse(f"Norm: unknown kind {kind!r}")
        if kind == "rms" and bias is not None:
            _refuse("Norm: an rms norm has no bias")
        if not 0.0 <= eps <= 3.4028234e38:
            _refuse(f"Norm: eps = {eps}")

    def _args(self, like, cols, what):
        weight, bias = self.weight, self.bias
        return (self.code, self.eps, 0 if weight is None else _vector(weight, like, cols, what, "a norm's weight"),
                0 if bias is None else _vector(bias, like, cols, what, "a norm's bias"))


_NO_NORM, _NO_RANDOM = (0, 0.0, 0, 0), (0, 0, 0, 0)


# The checks of operands: first the one that nearly all pass, then what is wrong or another layout.  `what` and `name` are put together only for a message.

def _fits(t, like, shape):
    return t.dtype is like.dtype and t.shape == shape and t.is_contiguous() and not t.requires_grad and t.get_device() == like.get_device()


def _vector(v, like, cols, what, name):
    if _fits(v, like, (cols,)):
        return v.data_ptr()
    _same(v, like, f"{what}: {name}")
    if v.dim() != 1 or v.shape[0] != cols or (cols > 1 and v.stride(0) != 1):
        _refuse(f"{what}: {name} is {tuple(v.shape)} with stride {v.stride()}, expected {cols} neighbours")
    return v.data_ptr()


def _matrix(t, like, shape, what, name):
    """(address, distance between rows) of an operand of that shape."""
    if _fits(t, like, shape):
        return t.data_ptr(), shape[-1]
    what = f"{what}: {name}"
    _same(t, like, what)
    if t.shape != shape:
        _refuse(f"{what} is {tuple(t.shape)}, expected {tuple(shape)}")
    return _rows(t, what)[:2]


def _gate(gate, like, rows, cols, what):
    """(address, distance between rows, rows) of a gate."""
    if gate.dim() == 1:
        return _vector(gate, like, cols, what, "gate"), cols, 1
    _same(gate, like, f"{what}: gate")
    address, ld, groups, width = _rows(gate, f"{what}: gate")
    if width != cols or groups < 1 or rows % groups:
        _refuse(f"{what}: gate is {tuple(gate.shape)}, expected {cols} columns and a number of rows that divides {rows}")
    return address, ld, groups


def _result(out, shape, like, what, name):
    """(tensor, address, distance between rows) of `out`, or of a new tensor."""
    if out is None:
        out = like.new_empty(shape)
        return out, out.data_ptr(), shape[-1]
    return _output(out, shape, like, f"{what}: {name}")


def _narrow(cols, what):
    if cols > MOST_COLUMNS:
        _refuse(f"{what}: rows of {cols} columns, at most {MOST_COLUMNS}")


def _finite(what, *numbers):
    for n in numbers:
        if not -3.4028234e38 <= n <= 3.4028234e38:
            _refuse(f"{what}: a scale of {n}")


def dropout(x, drop: Optional[Dropout], out=None, stream=None):
    """x / (1 - p) where kept, 0 elsewhere.  The gradient is the same call on that of the result.  `out` may be x."""
    dtype = _dtype(x, "dropout: x")
    device = x.device
    if _elsewhere(device, stream):
        with _On(device, stream):
            return dropout(x, drop, out)
    if x.requires_grad:
        _gradient_lost("dropout: x")
    xp, ldx, rows, cols = _rows(x, "dropout: x")
    _narrow(cols, "dropout")
    random = drop._args(device, "dropout") if drop is not None else _NO_RANDOM
    y, yp, ldy = _output(out, x.shape, x, "dropout: out")
    _check((_lib or lib()).eden_dropout(xp, ldx, yp, ldy, rows, cols, dtype, _RANDOM_ARGS.pack(*random), _stream(device)), "eden_dropout")
    return y


def norm(x, pre: Norm, out=None, stream=None):
    """The norm of x's rows.  `out` may be x."""
    return _join("norm", x, None, None, 1.0, 1.0, None, None, pre, None, out, stream)[1]


def join(x, f, gate=None, scale: float = 1.0, x_scale: float = 1.0, dropout: Optional[Dropout] = None, post: Optional[Norm] = None, pre: Optional[Norm] = None, out=None,
         norm_out=None, stream=None):
    """r = x_scale x + scale gate * dropout(post(f)); with `pre` (r, pre(r)).  `out` may be x or f, `norm_out` may be x or f.  Both scales, and scale / (1 - p), are finite in
    float32."""
    if f is None:
        _refuse("join: f is missing")
    r, h = _join("join", x, f, gate, scale, x_scale, dropout, post, pre, out, norm_out, stream)
    return r if pre is None else (r, h)


def _join(what, x, f, gate, scale, x_scale, drop, post, pre, out, norm_out, stream):
    dtype = _dtype(x, f"{what}: x")
    device = x.device
    if _elsewhere(device, stream):
        with _On(device, stream):
            return _join(what, x, f, gate, scale, x_scale, drop, post, pre, out, norm_out, None)
    L = _lib or lib()
    if x.requires_grad:
        _gradient_lost(f"{what}: x")
    _finite(what, scale, x_scale)
    xp, ldx, rows, cols = _rows(x, f"{what}: x")
    _narrow(cols, what)
    shape = x.shape
    r = h = None
    fp = gp = rp = hp = 0
    ldf = ldg = ldr = ldh = cols
    gates, random, post_args = 1, _NO_RANDOM, _NO_NORM
    if f is not None:
        fp, ldf = _matrix(f, x, shape, what, "f")
        if gate is not None:
            gp, ldg, gates = _gate(gate, x, rows, cols, what)
        if drop is not None:
            random = drop._args(device, what)
        if post is not None:
            post_args = post._args(x, cols, what)
        r, rp, ldr = _result(out, shape, x, what, "out")
    if pre is not None:
        pre_args = pre._args(x, cols, what)
        h, hp, ldh = _result(norm_out, shape, x, what, "out" if f is None else "norm_out")
    elif f is None:
        _refuse("norm: without a norm")
    elif norm_out is not None:
        _refuse("join: norm_out without pre")
    else:
        pre_args = _NO_NORM
    args = _JOIN_ARGS.pack(rows, cols, xp, fp, gp, rp, hp, ldx, ldf, ldg, ldr, ldh, gates, *post_args, *pre_args, *random, x_scale, scale, dtype)
    _check(L.eden_join(args, _stream(device)), "eden_join")
    return r, h


class JoinGrads(NamedTuple):
    """Gradients of a join; None where there is nothing.  Those of the gate and of the norms' weights and biases are float32."""
    dx: Optional[torch.Tensor] = None
    df: Optional[torch.Tensor] = None
    gate: Optional[torch.Tensor] = None
    post_weight: Optional[torch.Tensor] = None
    post_bias: Optional[torch.Tensor] = None
    pre_weight: Optional[torch.Tensor] = None
    pre_bias: Optional[torch.Tensor] = None


def norm_grad(dh, x, pre: Norm, residual=None, into: JoinGrads = JoinGrads(), accumulate: bool = False, stream=None) -> JoinGrads:
    """The gradients of norm(x, pre) from that of its result; dx is added to `residual`, the gradient that reaches x past the norm."""
    if dh is None or pre is None:
        _refuse("norm_grad: dh and pre are needed")
    return _join_grad("norm_grad", residual, None, dh, x, None, 1.0, 1.0, None, None, pre, into, accumulate, False, stream)


def join_grad(dr, f=None, dh=None, r=None, gate=None, scale: float = 1.0, x_scale: float = 1.0, dropout: Optional[Dropout] = None, post: Optional[Norm] = None,
              pre: Optional[Norm] = None, into: JoinGrads = JoinGrads(), accumulate: bool = False, stream=None) -> JoinGrads:
    """The gradients of a join from those of its results: dr of r and dh of pre(r), either may be None for zeros.  f and r: as join took and returned them (f is
    needed with a gate or `post`, r with dh).  `into`: tensors that are written, for instance parts of the vector that Context.encode takes; `accumulate`: the
    float32 ones among them are added to.  into.dx may be dr, dh or r; into.df may be f."""
    return _join_grad("join_grad", dr, f, dh, r, gate, scale, x_scale, dropout, post, pre, into, accumulate, True, stream)


def _join_grad(what, dr, f, dh, r, gate, scale, x_scale, drop, post, pre, into, accumulate, branch, stream):
    like = dr if dr is not None else dh
    if like is None:
        _refuse(f"{what}: neither dr nor dh")
    dtype = _dtype(like, f"{what}: the gradient")
    device = like.device
    if _elsewhere(device, stream):
        with _On(device, stream):
            return _join_grad(what, dr, f, dh, r, gate, scale, x_scale, drop, post, pre, into, accumulate, branch, None)
    L = _lib or lib()
    _finite(what, scale, x_scale)
    shape = like.shape
    _, _, rows, cols = _rows(like, f"{what}: the gradient")
    _narrow(cols, what)
    df = None
    drp = dhp = rp = fp = gp = dfp = 0
    lddr = lddh = ldr = ldf = ldg = lddf = cols
    gates, random, post_args, pre_args = 1, _NO_RANDOM, _NO_NORM, _NO_NORM
    if dr is not None:
        drp, lddr = _matrix(dr, like, shape, what, "dr")
    if pre is not None:
        pre_args = pre._args(like, cols, what)
        if dh is not None:
            if r is None:
                _refuse(f"{what}: dh without r")
            dhp, lddh = _matrix(dh, like, shape, what, "dh")
            rp, ldr = _matrix(r, like, shape, what, "r")
    elif dh is not None:
        _refuse(f"{what}: dh without pre")
    if gate is not None:
        gp, ldg, gates = _gate(gate, like, rows, cols, what)
    if drop is not None:
        random = drop._args(device, what)
    if post is not None:
        post_args = post._args(like, cols, what)
    if gate is not None or post is not None:
        if f is None:
            _refuse(f"{what}: f is needed with a gate or post")
        fp, ldf = _matrix(f, like, shape, what, "f")
    dx, dxp, lddx = _result(into.dx, shape, like, what, "into.dx")
    if branch:
        df, dfp, lddf = _result(into.df, shape, like, what, "into.df")
    elif into.df is not None:
        _refuse(f"{what}: into.df without a branch")
    sums, addresses, ld_gate_grad, fresh, sizes = [None] * 5, [0] * 5, cols, [], []
    there = (gate is not None, post is not None and post.weight is not None, post is not None and post.bias is not None, pre is not None and pre.weight is not None,
             pre is not None and pre.bias is not None)
    for i in range(5):
        given = into[2 + i]
        if not there[i]:
            if given is not None:
                _refuse(f"{what}: into.{into._fields[2 + i]} without one")
        elif given is not None:
            sums[i], addresses[i], ld = _output(given, gate.shape if i == 0 else (cols,), like, f"{what}: into.{into._fields[2 + i]}", torch.float32)
            if i == 0:
                ld_gate_grad = ld
        elif accumulate:
            _refuse(f"{what}: nothing to accumulate in for {into._fields[2 + i]}")
        else:
            fresh.append(i)
            sizes.append(gates * cols if i == 0 else cols)
    if fresh:
        # new ones are parts of one allocation
        flat = like.new_empty(sum(sizes), dtype=torch.float32)
        for i, part in zip(fresh, flat.split_with_sizes(sizes) if len(fresh) > 1 else (flat,)):
            addresses[i] = part.data_ptr()
            sums[i] = part if i or gate.dim() == 1 else part.view(gate.shape)
    ws, size = None, 0
    if any(addresses):
        size = L.eden_join_workspace_bytes(rows, cols, gates, dtype)
        if size:
            ws = torch.empty(size, dtype=torch.uint8, device=device)
    args = _JOIN_GRAD_ARGS.pack(rows, cols, drp, dhp, rp, fp, gp, dxp, dfp, lddr, lddh, ldr, ldf, ldg, lddx, lddf, gates, *addresses, ld_gate_grad, *post_args, *pre_args, *random, x_scale, scale,
                                dtype, 1 if branch else 0, 1 if accumulate else 0, 0 if ws is None else ws.data_ptr(), size)
    _check(L.eden_join_grad(args, _stream(device)), "eden_join_grad")
    return JoinGrads(dx, df, *sums)
