"""The operators around a residual block in 64 bits, for their tests: torch on the CPU and the oracle's hash, no code of the library.

Results come with elementwise bounds of what fp32 arithmetic may be off by: e = 2^-24 is a rounding, a sum of positive numbers along a row (at most 32 in a lane one
after the other, 10 steps between lanes) is off by 44 e of itself, a mean of v by 44 e mean|v|."""
import numpy as np
import torch

from oracle import eden_oracle as oracle

E = 2.0 ** -24
ROUND = {torch.float32: 2.0 ** -24, torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}
TINY = {torch.float32: 2.0 ** -149, torch.float16: 2.0 ** -25, torch.bfloat16: 2.0 ** -134}         # half a step of the subnormal numbers
STREAM_DROPOUT, STREAM_ROUNDING = 5, 6


def bits16(seed, stream, number, rows, cols):
    """The 16 random bits of each element."""
    per_row = (cols + 3) // 4
    words = oracle.hash_words(oracle.stream_key(seed % 2 ** 64, stream, number), 0, rows * per_row).astype("<u8")
    return torch.from_numpy(words.view("<u2").reshape(rows, 4 * per_row)[:, :cols].astype(np.int64))


def kept(seed, number, threshold, rows, cols):
    return bits16(seed, STREAM_DROPOUT, number, rows, cols) >= threshold


class Normed:
    """A norm of the rows of v (bound: of v's own error), its gradient, and bounds of both."""

    def __init__(self, v, kind, weight, bias, eps):
        self.layer, k = kind == "layer", v.shape[1]
        self.weight = torch.ones(k, dtype=torch.float64) if weight is None else weight
        self.bias = torch.zeros(k, dtype=torch.float64) if bias is None else bias
        mean = v.mean(dim=1, keepdim=True) if self.layer else torch.zeros(v.shape[0], 1, dtype=torch.float64)
        self.rho = ((v - mean).square().mean(dim=1, keepdim=True) + eps) ** -0.5
        self.n = (v - mean) * self.rho
        # the sum 44, its mean, eps and the square root 4 more, of which the root takes half; the product 1; v - mean: the mean's error and a rounding
        off = 46 * E * v.abs().mean(dim=1, keepdim=True) + E * v.abs() if self.layer else torch.zeros_like(v)
        self.n_off = 28 * E * self.n.abs() + self.rho * off
        self.value = self.n * self.weight + self.bias
        self.off = self.n_off * self.weight.abs() + 2 * E * ((self.n * self.weight).abs() + self.bias.abs())

    def value_off(self, off):
        """Bound of the value where v itself is off by `off`."""
        spread = off + self.n.abs() * (off * self.n.abs()).mean(dim=1, keepdim=True)
        return self.off + 1.01 * self.rho * (spread + (off.mean(dim=1, keepdim=True) if self.layer else 0.0)) * self.weight.abs()

    def grad(self, d, off):
        """(gradient of v, its bound, gradients of weight and bias, their bounds) from the value's gradient d, itself off by `off`."""
        def mean(x):
            return x.mean(dim=1, keepdim=True)
        g, g_off = d * self.weight, off * self.weight.abs() + 2 * E * (d * self.weight).abs()
        inner, inner_off = mean(g * self.n), mean(g_off * self.n.abs() + g.abs() * self.n_off) + 46 * E * mean((g * self.n).abs())
        total, total_off = g - self.n * inner, g_off + self.n_off * inner.abs() + self.n.abs() * inner_off
        size = g.abs() + (self.n * inner).abs()
        if self.layer:
            total, total_off, size = total - mean(g), total_off + mean(g_off) + 46 * E * mean(g.abs()), size + mean(g).abs()
        # rho is off by 26 e of itself, and three roundings
        return (self.rho * total, self.rho * (total_off + 32 * E * size), (d * self.n).sum(0), summed(d * self.n, off * self.n.abs() + d.abs() * self.n_off), d.sum(0),
                summed(d, off))


def summed(terms, off):
    """Bound of a sum over rows in any order."""
    return off.sum(0) + (terms.shape[0] + 24) * E * terms.abs().sum(0)


def by_row(gate, rows):
    return gate if gate is None or gate.dim() == 1 else gate.repeat_interleave(rows // gate.shape[0], dim=0)


def join(x, f, gate, scale, x_scale, mask, p, post, pre):
    """{"r": (value, bound), "h": ...}; mask: kept places or None, p: the exact probability; post, pre: (kind, weight, bias, eps) or None."""
    r, r_off, out = x, torch.zeros_like(x), {}
    if f is not None:
        u, off = f, torch.zeros_like(f)
        if post is not None:
            n = Normed(f, *post)
            u, off = n.value, n.off
        if mask is not None:
            u, off = torch.where(mask, u / (1.0 - p), 0.0), torch.where(mask, off / (1.0 - p), 0.0)
        factor = scale * (1.0 if gate is None else by_row(gate, x.shape[0]))
        r = x_scale * x + factor * u
        r_off = abs_(factor) * off + 6 * E * (abs_(factor) * u.abs() + abs(x_scale) * x.abs())
        out["r"] = (r, r_off)
    if pre is not None:
        n = Normed(r, *pre)
        out["h"] = (n.value, n.value_off(r_off))
    return out


def abs_(v):
    return v.abs() if isinstance(v, torch.Tensor) else abs(v)


def join_grad(dr, f, dh, r, gate, scale, x_scale, mask, p, post, pre):
    out, like = {}, dr if dr is not None else dh
    d = torch.zeros_like(like) if dr is None else dr
    off = torch.zeros_like(like)
    if pre is not None:
        more, more_off, w, w_off, b, b_off = Normed(r, *pre).grad(torch.zeros_like(like) if dh is None else dh, torch.zeros_like(like))
        d, off = d + more, more_off + 2 * E * (d.abs() + more.abs())
        out["pre_weight"], out["pre_bias"] = (w, w_off), (b, b_off)
    out["dx"] = (x_scale * d, abs(x_scale) * (off + E * d.abs()))
    back = scale / (1.0 - p)
    keep = torch.ones_like(d, dtype=torch.bool) if mask is None else mask
    d, off = torch.where(keep, back * d, 0.0), torch.where(keep, abs(back) * (off + 4 * E * d.abs()), 0.0)
    n = None if post is None else Normed(f, *post)
    if gate is not None:
        u, u_off = (f, torch.zeros_like(f)) if n is None else (n.value, n.off)
        terms, terms_off = torch.where(keep, d * u, 0.0), torch.where(keep, off * u.abs() + d.abs() * u_off + 2 * E * (d * u).abs(), 0.0)
        groups = 1 if gate.dim() == 1 else gate.shape[0]
        parts = [(a.sum(0), summed(a, b)) for a, b in zip(terms.chunk(groups), terms_off.chunk(groups))]
        out["gate"] = tuple(torch.stack(t).reshape(gate.shape) for t in zip(*parts))
        factor = by_row(gate, d.shape[0])
        off = off * factor.abs() + E * (d * factor).abs()
        d = d * factor
    out["df"] = (d, off)
    if n is not None:
        v, v_off, w, w_off, b, b_off = n.grad(d, off)
        out["df"], out["post_weight"], out["post_bias"] = (v, v_off), (w, w_off), (b, b_off)
    return out
