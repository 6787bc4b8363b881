"""Distributed training of a small residual block on one GPU: every sender computes its gradient with the layer operators, from 8-bit
activation checkpoints, and sends it through EDEN; the receiver's mean updates the weights.

    python -m paper_2108_08842_amd.train --senders 4 --budget 1 --steps 60
    python -m paper_2108_08842_amd.train --budget 0        # the exact mean of the gradients, for comparison
    python -m paper_2108_08842_amd.train --norm rms --dropout 0.1 --four-bit

The block is y = x + W2 act(W1 x + b1) + b2.  Its backward pass reads what it kept of the forward pass in 8 bits (33 bytes for 32
values): the block's input, the activation's input and its output.  The weight and bias gradients are written straight into the flat fp32 vector that
eden_encode takes.  Data are synthetic: a block of the same shape with other weights is to be imitated.

With a norm it is y = x + gate * dropout(W2 act(W1 norm(x) + b1) + b2), with a gate for each column; the norm's weight (and bias) and the gate are trained too.  With
--four-bit the products are taken of 4-bit operands: activations and weights rounded to the nearest, gradients stochastically; the inputs of both layers are then kept in 4 bits.
"""
from __future__ import annotations

import argparse

import torch

from . import blocks, eden, layers, mx4


class Block:
    """Weights of y = x + W2 act(W1 x + b1) + b2 as parts of one flat fp32 vector, and a sender's forward and backward pass.  `norm`: "rms" or "layer", with a gate behind the
    branch; `dropout`: its probability in the branch; `four_bit`: products of 4-bit operands."""

    def __init__(self, width: int, hidden: int, dtype, activation: str, generator, norm: str = "none", dropout: float = 0.0, four_bit: bool = False):
        self.width, self.hidden, self.dtype, self.activation = width, hidden, dtype, activation
        self.norm, self.dropout, self.four_bit = norm, dropout, four_bit
        self.shapes = [(hidden, width), (hidden,), (width, hidden), (width,)]
        if norm != "none":
            self.shapes += [(width,)] * (3 if norm == "layer" else 2)           # gate, norm's weight, bias
        self.flat = torch.zeros(sum(torch.Size(s).numel() for s in self.shapes), device="cuda")
        w1, _, w2, _, *others = self.parts(self.flat)
        w1.normal_(0.0, width ** -0.5, generator=generator)
        w2.normal_(0.0, hidden ** -0.5, generator=generator)
        for one in others[:2]:
            one.fill_(1.0)

    def parts(self, flat):
        out, at = [], 0
        for s in self.shapes:
            n = torch.Size(s).numel()
            out.append(flat[at:at + n].view(s))
            at += n
        return out

    def weights(self):
        """The weights in the compute type: made once for each step.  With 4 bits those of both layers' weights and of their transposes behind them."""
        out = [p.to(self.dtype) for p in self.parts(self.flat)]
        if self.four_bit:
            out += [mx4.quantize(out[i], transpose=t) for i in (0, 2) for t in (False, True)]
        return out

    def _around(self, weights, seed):
        """Norm in front of the branch, gate and dropout behind it, or None."""
        drop = blocks.Dropout(self.dropout, seed) if self.dropout else None
        if self.norm == "none":
            return None, None, drop
        gate, w = weights[4:6]
        return blocks.Norm(self.norm, w, weights[6] if self.norm == "layer" else None), gate, drop

    def forward(self, weights, x, seed: int = 0):
        """y and what the backward pass needs, in 8 or 4 bits."""
        w1, b1, w2, b2 = weights[:4]
        norm, gate, drop = self._around(weights, seed)
        n = x if norm is None else blocks.norm(x, norm)
        if self.four_bit:
            w1_four, _, w2_four, _ = weights[-4:]
            kept_n = mx4.quantize(n, transpose=True)
            h, kept_z = mx4.linear(n, w1_four, b1, activation=self.activation, checkpoint=True)
            kept_h = mx4.quantize(h, transpose=True)
        else:
            kept_n = layers.save_checkpoint(n)
            h, kept_z = layers.linear(n, w1, b1, activation=self.activation, checkpoint=True)
            kept_h = layers.save_checkpoint(h)
        plain = gate is None and drop is None
        f = mx4.linear(h, w2_four, b2, residual=x if plain else None) if self.four_bit else layers.linear(h, w2, b2, residual=x if plain else None)
        if plain:
            return f, (kept_n, kept_z, kept_h, x if norm is not None else None, None, seed)
        return blocks.join(x, f, gate=gate, dropout=drop), (kept_n, kept_z, kept_h, x if norm is not None else None, f if gate is not None else None, seed)

    def backward(self, weights, dy, kept, gradient):
        """Writes the gradient of all weights into the flat vector `gradient` and returns that of x."""
        w1, _, w2, _ = weights[:4]
        kept_n, kept_z, kept_h, x, f, seed = kept
        norm, gate, drop = self._around(weights, seed)
        dw1, db1, dw2, db2, *others = self.parts(gradient)
        df = dy
        if gate is not None or drop is not None:
            df = blocks.join_grad(dy, f, gate=gate, dropout=drop, into=blocks.JoinGrads(gate=others[0] if others else None)).df
        if self.four_bit:
            _, w1_turned, _, w2_turned = weights[-4:]
            rounding = [mx4.Stochastic(seed, i) for i in range(4)]
            df_turned, _ = mx4.quantize(df, transpose=True, rounding=rounding[0], sums=db2)
            mx4.linear_weight_grad(df_turned, kept_h, out=dw2)
            dz = mx4.linear_input_grad(mx4.quantize(df, rounding=rounding[1]), w2_turned, activation=self.activation, checkpoint=kept_z, dtype=self.dtype)
            dz_turned, _ = mx4.quantize(dz, transpose=True, rounding=rounding[2], sums=db1)
            mx4.linear_weight_grad(dz_turned, kept_n, out=dw1)
            dz_four = mx4.quantize(dz, rounding=rounding[3])
            if norm is None:
                return mx4.linear_input_grad(dz_four, w1_turned, residual=dy)
            dn = mx4.linear_input_grad(dz_four, w1_turned, dtype=self.dtype)
        else:
            layers.linear_weight_grad(df, kept_h, out=dw2, bias_out=db2)
            dz = layers.linear_input_grad(df, w2, activation=self.activation, checkpoint=kept_z)
            layers.linear_weight_grad(dz, kept_n, out=dw1, bias_out=db1)
            if norm is None:
                return layers.linear_input_grad(dz, w1, residual=dy)
            dn = layers.linear_input_grad(dz, w1)
        into = blocks.JoinGrads(pre_weight=others[1], pre_bias=others[2] if self.norm == "layer" else None)
        return blocks.norm_grad(dn, x, norm, residual=dy, into=into).dx


def train(senders=4, rows=512, width=256, hidden=1024, budget=1.0, steps=60, rate=0.05, dtype=torch.bfloat16, activation="gelu", seed=0, norm="none",
          dropout=0.0, four_bit=False):
    """Losses (mean squared error of each step, before its update).  budget: bits per coordinate (0: the exact mean)."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    teacher = Block(width, hidden, dtype, activation, g, norm)
    student = Block(width, hidden, dtype, activation, g, norm, dropout, four_bit)
    d = student.flat.numel()
    ctx = eden.Context(d_max=d, n_max=senders, device=torch.cuda.current_device()) if budget else None
    gradients = [torch.zeros(d, device="cuda") for _ in range(senders)]
    mean = torch.empty(d, device="cuda")
    ids, bits = list(range(senders)), [int(round(256 * budget))] * senders
    losses = []
    for step in range(steps):
        weights, target = student.weights(), teacher.weights()
        loss = torch.zeros((), device="cuda")
        for c in range(senders):
            x = torch.randn(rows, width, generator=g, device="cuda").to(dtype)
            y, kept = student.forward(weights, x, seed=step * senders + c)
            error = y.float() - teacher.forward(target, x)[0].float()
            loss += error.square().mean() / senders
            student.backward(weights, (error / rows).to(dtype), kept, gradients[c])
        if budget:
            ctx.decode_mean(ctx.encode(gradients, ids, bits, seed=step), ids, bits, d, step, mean)
        else:
            torch.mean(torch.stack(gradients), dim=0, out=mean)
        student.flat.sub_(mean, alpha=rate)
        losses.append(loss)
    return torch.stack(losses).tolist()


def main():
    p = argparse.ArgumentParser(description=__doc__.split("\n\n")[0])
    p.add_argument("--senders", type=int, default=4)
    p.add_argument("--rows", type=int, default=512, help="rows of a sender's batch")
    p.add_argument("--width", type=int, default=256)
    p.add_argument("--hidden", type=int, default=1024)
    p.add_argument("--budget", type=float, default=1.0, help="bits per coordinate (1/2, 1, 2, .., 8); 0: the exact mean")
    p.add_argument("--steps", type=int, default=60)
    p.add_argument("--rate", type=float, default=0.05)
    p.add_argument("--activation", choices=[a for a in layers.ACTIVATIONS if a != "none"], default="gelu")
    p.add_argument("--norm", choices=["none", "rms", "layer"], default="none")
    p.add_argument("--dropout", type=float, default=0.0)
    p.add_argument("--four-bit", action="store_true", help="products of 4-bit operands")
    a = p.parse_args()
    inputs = sum(mx4.mx4_bytes(c, a.rows) if a.four_bit else layers.checkpoint_bytes(a.rows, c) for c in (a.width, a.hidden)) + layers.checkpoint_bytes(a.rows, a.hidden)
    more = 0 if a.norm == "none" else 2 * 2 * a.rows * a.width                   # the norm's input and the gate's
    print(f"kept for the backward pass: {inputs + more} bytes a sender in 8{' and 4' if a.four_bit else ''} bits, {2 * a.rows * (a.width + 2 * a.hidden) + more} in bf16", flush=True)
    losses = train(a.senders, a.rows, a.width, a.hidden, a.budget, a.steps, a.rate, activation=a.activation, norm=a.norm, dropout=a.dropout, four_bit=a.four_bit)
    for i in range(0, len(losses), max(1, len(losses) // 10)):
        print(f"step {i}: loss {losses[i]:.5f}", flush=True)
    print(f"step {len(losses) - 1}: loss {losses[-1]:.5f}")


if __name__ == "__main__":
    main()
