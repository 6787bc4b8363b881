"""The layer operators in 64 bits, for their tests: numpy / torch on the CPU, no code of the library."""
import math

import numpy as np
import torch

EPS = 2.0 ** -24                                                   # half the distance of fp32 numbers next to 1
ROUND = {torch.float32: 2.0 ** -24, torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}      # twice a rounding to nearest (relative)
TINY = {torch.float32: 2.0 ** -126, torch.float16: 2.0 ** -24, torch.bfloat16: 2.0 ** -126}


def encode(x):
    """(codes int8 rows x 32 blocks, exponents uint8 rows x blocks) of an fp32 numpy matrix."""
    rows, cols = x.shape
    blocks = (cols + 31) // 32
    codes, exps = np.zeros((rows, blocks * 32), np.int8), np.zeros((rows, blocks), np.uint8)
    for r in range(rows):
        for b in range(blocks):
            part = x[r, 32 * b:32 * b + 32].astype(np.float64)
            if not np.all(np.isfinite(part)):
                exps[r, b] = 255
                continue
            a = np.abs(part).max()
            field = 0 if a < 2.0 ** -126 else int(math.frexp(a)[1]) + 126
            t = max(1, field - 6)
            q = np.clip(np.rint(part * 2.0 ** (127 - t)), -127, 127)
            codes[r, 32 * b:32 * b + len(part)] = q.astype(np.int8)
            exps[r, b] = t
    return codes, exps


def decode(codes, exps, cols):
    unit = np.where(exps == 255, np.nan, np.exp2(exps.astype(np.float64) - 127))
    return (codes.astype(np.float64) * np.repeat(unit, 32, axis=1))[:, :cols]


def pack(codes, exps):
    return torch.from_numpy(np.concatenate([codes.view(np.uint8).reshape(-1), exps.reshape(-1)]))


def unpack(buffer, rows, cols):
    blocks = (cols + 31) // 32
    b = buffer.cpu().numpy()
    return b[:rows * blocks * 32].view(np.int8).reshape(rows, blocks * 32), b[rows * blocks * 32:rows * blocks * 33].reshape(rows, blocks)


def values(checkpoint):
    return torch.from_numpy(decode(*unpack(checkpoint.buffer, checkpoint.rows, checkpoint.cols), checkpoint.cols))


def act(z, name):
    if name == "relu":
        return torch.clamp(z, min=0.0)
    if name == "gelu":
        return z * 0.5 * torch.erfc(-z / math.sqrt(2.0))
    if name == "gelu_tanh":
        return z * torch.sigmoid(2.0 * math.sqrt(2.0 / math.pi) * (z + 0.044715 * z ** 3))
    if name == "silu":
        return z * torch.sigmoid(z)
    return z


def slope(z, name):
    if name == "none":
        return torch.ones_like(z)
    if name == "relu":
        return (z > 0).double()
    z = z.clone().requires_grad_(True)
    return torch.autograd.grad(act(z, name).sum(), z)[0]


def product_bound(a, b, depth):
    """Elementwise bound of an fp32 sum of `depth` products a b^T: each of at most depth + 4 roundings is off by 2^-23 of the sum of the
    sizes at most (products of bf16 terms are exact; the left out ones are below 2^-22 of it together)."""
    return (depth + 8) * 2.0 ** -23 * (a.abs() @ b.abs().t())


def norm_bound(depth, dtype):
    """Bound of the relative 2-norm of the error of a sum of products of independent values: a rounding of 2^-23 at most of each
    partial sum, the partial sums growing like the square root of their length, rounding errors independent; and the result's own."""
    return 2.0 ** -23 * (math.sqrt(depth) + 4) + ROUND[dtype]


def rel(a, b):
    d = float(torch.linalg.vector_norm(a.double() - b.double()))
    n = float(torch.linalg.vector_norm(b.double()))
    return d / n if n else (math.inf if d else 0.0)
