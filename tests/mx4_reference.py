"""4-bit operands in 64 bits, for their tests: numpy and the oracle's hash, no code of the library."""
import math

import numpy as np
import torch

from tests import blocks_reference as blocks_ref

GRID = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])


def draws(seed, number, rows, cols):
    return blocks_ref.bits16(seed, blocks_ref.STREAM_ROUNDING, number, rows, cols).numpy()


def encode(x, bits=None):
    """(codes rows x 32 blocks with bit 3 for the sign, exponents rows x blocks) of an fp32 numpy matrix; bits: its 16 random bits, or None for the nearest."""
    x = np.asarray(x, dtype=np.float32)
    rows, cols = x.shape
    blocks = (cols + 31) // 32
    full = np.zeros((rows, blocks * 32), np.float32)
    full[:, :cols] = x
    parts = full.reshape(rows, blocks, 32).astype(np.float64)
    with np.errstate(all="ignore"):
        largest = np.abs(parts).max(axis=2)
        finite = np.isfinite(largest)
        t = np.zeros((rows, blocks), np.int64)
        # the smallest t with largest <= 6 2^(t - 127)
        safe = np.where(finite & (largest > 0), largest, 1.0)
        _, e = np.frexp(safe / 6.0)
        e = e - (safe <= 6.0 * np.ldexp(1.0, e - 1))
        t = np.where(finite & (largest > 0), np.maximum(e + 127, 0), 0)
        v = np.abs(np.where(finite[..., None], parts, 0.0)) * np.ldexp(1.0, 127 - t)[..., None]
    low = np.searchsorted(GRID, v, side="right") - 1
    high = np.minimum(low + 1, 7)
    share = np.where(high > low, (v - GRID[low]) / np.maximum(GRID[high] - GRID[low], 0.5), 0.0)
    if bits is None:
        up = (share > 0.5) | ((share == 0.5) & (low % 2 == 1))
    else:
        d = np.zeros((rows, blocks * 32), np.int64)
        d[:, :cols] = bits
        up = d.reshape(v.shape) + 0.5 < 65536.0 * share
    code = np.where(up, high, low) + 8 * np.signbit(parts)
    code = np.where(finite[..., None], code, 0)
    return code.reshape(rows, blocks * 32).astype(np.uint8), np.where(finite, t, 255).astype(np.uint8)


def decode(codes, exps, cols):
    unit = np.where(exps == 255, np.nan, np.ldexp(1.0, exps.astype(np.int64) - 127))
    return (GRID[codes & 7] * np.where(codes & 8, -1.0, 1.0) * np.repeat(unit, 32, axis=1))[:, :cols]


def size(rows, cols):
    chunks = (cols + 255) // 256
    return chunks * (128 * rows + 8 * (rows + rows % 2))


def pack(codes, exps):
    rows, width = codes.shape
    chunks = (width + 255) // 256
    full, e = np.zeros((rows, chunks * 256), np.uint8), np.zeros((rows + rows % 2, chunks * 8), np.uint8)
    full[:, :width], e[:rows, :width // 32] = codes, exps
    e = e.reshape(-1, chunks, 8).transpose(1, 0, 2)
    return torch.from_numpy(np.concatenate([(full[:, 0::2] | (full[:, 1::2] << 4)).reshape(-1), e.reshape(-1)]))


def unpack(buffer, rows, cols):
    """(codes rows x 256 chunks, exponents rows x 8 chunks), the fill among them."""
    b, chunks = buffer.cpu().numpy(), (cols + 255) // 256
    codes = b[:rows * chunks * 128].reshape(rows, chunks * 128)
    both = np.empty((rows, chunks * 256), np.uint8)
    both[:, 0::2], both[:, 1::2] = codes & 15, codes >> 4
    exps = b[rows * chunks * 128:size(rows, cols)].reshape(chunks, rows + rows % 2, 8)[:, :rows].transpose(1, 0, 2).reshape(rows, chunks * 8)
    return both, exps


def values(x, bits=None):
    """What the 4 bits of a torch matrix stand for, in 64 bits."""
    x = x.float().cpu().numpy()
    return torch.from_numpy(decode(*encode(x, bits), x.shape[1]))


def norm_bound(depth, dtype):
    """Bound of the relative 2-norm of the error of a sum of exact products of independent values: a rounding of each of the partial sums, which grow like the square root of
    their length, and the result's own."""
    return 2.0 ** -23 * (math.sqrt(depth) + 4) + blocks_ref.ROUND[dtype]
