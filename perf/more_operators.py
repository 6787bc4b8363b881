"""Cases of the operators around and inside a residual block that is trained with 4-bit products.

A case is a plain dict:
  op     "dropout"    y = x / (1 - p) where kept, 0 elsewhere
         "join"       r = a x + s gate * dropout(post(f)), h = pre(r); without a branch f: h = pre(x)
         "join_grad"  from the gradients of r and h: those of x, f, the gate, the norms' weights and biases
         "quantize"   a matrix, or its transpose, to 4 bits and back; with the sums of the columns where asked
         "linear"     y = act(x^ w^T + bias) + residual, x^ the 4-bit values of x, w from its 4 bits; where asked with the 8-bit checkpoint of what is inside act
         "igrad"      dx = (dz^ w) * act'(z) + residual, dz^ rounded stochastically to 4 bits, w from the 4 bits of its transpose, z from its checkpoint
         "wgrad"      dw = dy^T x from the 4 bits of both transposes, those of dy made in the call, and db = sums of dy over the rows
  m, n, k   rows; features out and in ("wgrad", "igrad" as in "linear"); the others have k columns
  dtype     "f32", "f16", "bf16"
  p         probability of dropout
  branch, gates, post, pre   whether there is f; 0: no gate, 1: one for each column, more: as many groups of rows with gates of their own; "none", "rms", "layer"
  transpose, stochastic, bias, residual, checkpoint, act   whether or which
  pad       elements between the rows of the first operand

Random numbers: word j of a key is the j-th output of splitmix64 started at the key, the key follows from seed, stream (5: dropout, 6: rounding) and id.  A row of c
columns has ceil(c / 4) words, a column 16 bits of one.  Dropout keeps a value whose bits are at least round(65536 p).

4 bits: blocks of 32 columns, a power of two 2^(t - 127) for each and codes for 0, 1/2, 1, 3/2, 2, 3, 4, 6 and a sign.  2^(t - 127) is the smallest that reaches the block's largest
|x| with a 6 (t at least 0).  Rounding is to the nearest (ties to the even code), or up where the 16 bits and a half are below 65536 times what a value is above the code below.
Of a transpose, rows and columns are the transpose's.  A row's codes are filled up with zeros to 256 columns and packed two to a byte, the first in the low half.  Behind all rows' codes,
for every 256 columns, eight bytes t of each row; the rows are filled up to an even number there.
"""
import math

import torch

own = False

_TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
_ACTS = ["none", "relu", "gelu", "gelu_tanh", "silu"]
_EPS = {"rms": 1e-6, "layer": 1e-5}
_SEED, _ID = 20241, 3


def _case(name, op, m, n, k, dtype, **more):
    c = {"name": name, "op": op, "m": m, "n": n, "k": k, "dtype": dtype, "p": 0.0, "branch": True, "gates": 0, "post": "none", "pre": "none", "transpose": False,
         "stochastic": False, "bias": False, "residual": False, "checkpoint": False, "act": "none", "pad": 0}
    c.update(more)
    return c


def listed():
    return [
        # a short sequence in full precision, odd sizes: a call that is all latency
        _case("dropout_33x1001_f32", "dropout", 33, 0, 1001, "f32", p=0.1),
        # the activations of a long batch, rows inside a wider matrix
        _case("dropout_8192x8192_bf16", "dropout", 8192, 0, 8192, "bf16", p=0.1, pad=8),
        # one token between two blocks: the sum and the next block's norm
        _case("join_1x4096_bf16", "join", 1, 0, 4096, "bf16", pre="rms"),
        # the end of a block and the norm of the next in a training step on a long batch, gates of their own for each of sixteen sequences
        _case("join_8192x4096_bf16", "join", 8192, 0, 4096, "bf16", p=0.1, gates=16, post="layer", pre="rms"),
        # all gradients of a ragged batch in full precision
        _case("join_grad_77x1000_f32", "join_grad", 77, 0, 1000, "f32", p=0.2, gates=1, post="layer", pre="layer"),
        # the gradients of a long batch
        _case("join_grad_8192x4096_bf16", "join_grad", 8192, 0, 4096, "bf16", p=0.1, gates=1, post="rms", pre="rms"),
        # the activations of a short batch of odd length
        _case("quantize_301x1000_f16", "quantize", 301, 0, 1000, "f16"),
        # the gradient of a wide layer for its weight gradient: transposed, unbiased, with the bias gradient
        _case("quantize_8192x16384_bf16", "quantize", 8192, 0, 16384, "bf16", transpose=True, stochastic=True, bias=True),
        # a single token through a wide layer: the weights are read once for it
        _case("linear_1x4096x16384_bf16", "linear", 1, 16384, 4096, "bf16", act="gelu", bias=True),
        # an ordinary batch of odd length
        _case("linear_1021x2048x5000_f16", "linear", 1021, 5000, 2048, "f16", act="relu", bias=True, residual=True),
        # the widening layer of a training step on a long batch, which keeps what the backward pass needs
        _case("linear_8192x4096x16384_bf16", "linear", 8192, 16384, 4096, "bf16", act="gelu", bias=True, checkpoint=True),
        # the weight gradient of a long batch
        _case("wgrad_8192x4096x8192_bf16", "wgrad", 8192, 4096, 8192, "bf16", bias=True),
    ]


_MOST_FLOPS = 2.0 * 8192 * 4096 * 16384


def draw(rng):
    def size(low, high):
        v = int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))
        kind = rng.random()                     # whole tiles, whole vectors of eight, or anything odd
        v = -(-v // 64) * 64 if kind < 0.45 and v >= 48 else -(-v // 8) * 8 if kind < 0.75 else v | 1
        return max(low, min(high, v))

    op = rng.choice(["dropout", "join", "join", "join_grad", "join_grad", "quantize", "quantize", "linear", "linear", "igrad", "wgrad"])
    dtype = rng.choice(["bf16", "bf16", "f16", "f32"])
    m = max(1, int(round(math.exp(rng.uniform(0.0, math.log(8192))))))
    pad = rng.choice([0, 0, 0, 8, 3])
    if op in ("dropout", "join", "join_grad", "quantize"):
        k = size(32, 16384)
        m = max(1, min(m, (1 << (25 if op[:4] == "join" else 26)) // k))
        if op == "dropout":
            return _case("drawn", op, m, 0, k, dtype, p=rng.choice([0.05, 0.1, 0.3, 0.5]), pad=pad)
        if op == "quantize":
            transpose = rng.random() < 0.5
            return _case("drawn", op, m, 0, k, dtype, transpose=transpose, stochastic=rng.random() < 0.5, bias=transpose and rng.random() < 0.5, pad=pad)
        branch = rng.random() < 0.75
        gates = rng.choice([0, 1, 1, 4]) if branch else 0
        if gates > 1:
            m = -(-m // gates) * gates
        return _case("drawn", op, m, 0, k, dtype, branch=branch, gates=gates, p=rng.choice([0.0, 0.1, 0.25]) if branch else 0.0,
                     post=rng.choice(["none", "rms", "layer"]) if branch else "none", pre=rng.choice(["none", "rms", "layer"][0 if branch else 1:]), pad=pad)
    n, k = size(32, 16384), size(32, 8192)
    if op == "linear" and rng.random() < 0.3:
        m = rng.choice([1, 2, 4, 8, 16])
    m = max(1, min(m, int(_MOST_FLOPS / (2.0 * n * k))))
    act = "none" if op == "wgrad" else rng.choice(_ACTS)
    checkpoint = act != "none" if op == "igrad" else op == "linear" and m > 16 and rng.random() < 0.5
    return _case("drawn", op, m, n, k, dtype, act=act, bias=op != "igrad" and rng.random() < 0.6, residual=op != "wgrad" and rng.random() < 0.4,
                 checkpoint=checkpoint, pad=pad)


# ---- inputs

def _matrix(g, rows, cols, dtype, pad=0, scale=1.0, outliers=False, padding=False):
    """Rows of normal values; `outliers`: a few columns twenty times as large, as activations have; `padding`: some rows all zero."""
    x = torch.randn(rows, cols + pad, generator=g, device="cuda", dtype=torch.float32).mul_(scale)
    if outliers:
        x[:, torch.randint(0, cols, (max(1, cols // 256),), generator=g, device="cuda")] *= 20.0
    if padding and rows > 16:
        x[torch.randint(0, rows, (rows // 64 + 1,), generator=g, device="cuda")] = 0.0
    return x.to(dtype)[:, :cols]


def _packed(x):
    """The buffer of the 4 bits of an fp32 matrix, rounded to the nearest."""
    rows, cols = x.shape
    chunks = -(-cols // 256)
    code, t = _four_bits(x, None)
    code = torch.nn.functional.pad(code.reshape(rows, -1), (0, 256 * chunks - code.shape[1] * 32)).to(torch.uint8)
    t = torch.nn.functional.pad(t, (0, 8 * chunks - t.shape[1], 0, rows % 2)).to(torch.uint8)
    codes = code[:, 0::2] | (code[:, 1::2] << 4)
    return torch.cat([codes.reshape(-1), t.view(rows + rows % 2, chunks, 8).transpose(0, 1).reshape(-1)])


def _checkpoint(z):
    """The buffer of an fp32 matrix's 8-bit checkpoint."""
    q, t = _block_codes(z)
    return torch.cat([q.to(torch.int8).view(torch.uint8).reshape(-1), t.to(torch.uint8).reshape(-1)])


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    dtype, m, n, k, op, pad = _TYPES[case["dtype"]], case["m"], case["n"], case["k"], case["op"], case["pad"]
    s = {"case": case, "dtype": dtype, "seed": _SEED + seed}
    if op in ("dropout", "quantize"):
        s["x"] = _matrix(g, m, k, dtype, pad, outliers=True, padding=True)
    elif op in ("join", "join_grad"):
        s["x"] = _matrix(g, m, k, dtype, pad, outliers=True, padding=True)
        s["f"] = _matrix(g, m, k, dtype, scale=0.5, padding=True) if case["branch"] else None
        s["gate"] = _matrix(g, case["gates"], k, dtype, scale=0.3) if case["gates"] else None
        if case["gates"] == 1:
            s["gate"] = s["gate"][0]
        for name in ("post", "pre"):
            if case[name] != "none":
                s[name + "_weight"] = (1.0 + _matrix(g, 1, k, torch.float32, scale=0.1)[0]).to(dtype)
                s[name + "_bias"] = _matrix(g, 1, k, dtype, scale=0.1)[0] if case[name] == "layer" else None
        if op == "join_grad":
            s["dr"] = _matrix(g, m, k, dtype, scale=1e-2, padding=True) if case["branch"] else None
            s["dh"] = _matrix(g, m, k, dtype, scale=1e-2, padding=True) if case["pre"] != "none" else None
    elif op == "linear":
        s["x"] = _matrix(g, m, k, dtype, pad, outliers=True, padding=True)
        s["w"] = _packed(_matrix(g, n, k, torch.float32, scale=k ** -0.5))
        s["bias"] = _matrix(g, 1, n, dtype, scale=0.1)[0] if case["bias"] else None
        s["residual"] = _matrix(g, m, n, dtype) if case["residual"] else None
    elif op == "igrad":
        s["dz"] = _matrix(g, m, n, dtype, pad, scale=1e-2, padding=True)
        s["wt"] = _packed(_matrix(g, k, n, torch.float32, scale=k ** -0.5))
        s["z"] = _checkpoint(_matrix(g, m, k, torch.float32)) if case["checkpoint"] else None
        s["residual"] = _matrix(g, m, k, dtype, scale=1e-2) if case["residual"] else None
    else:
        s["dy"] = _matrix(g, m, n, dtype, pad, scale=1e-2, padding=True)
        s["xt"] = _packed(_matrix(g, k, m, torch.float32))
    return s


# ---- the plain form, in 32 bits

_PHI = 0x9E3779B97F4A7C15
_MASK = (1 << 64) - 1


def _signed(v):
    v &= _MASK
    return v - (1 << 64) if v >> 63 else v


def _mix(z):
    """splitmix64's output function on int64 tensors, whose products wrap around."""
    def down(v, by):
        return (v >> by) & ((1 << (64 - by)) - 1)
    z = (z ^ down(z, 30)) * _signed(0xBF58476D1CE4E5B9)
    z = (z ^ down(z, 27)) * _signed(0x94D049BB133111EB)
    return z ^ down(z, 31)


def _draws(seed, stream, rows, cols):
    """The 16 bits of each element, as whole numbers."""
    first = _mix(torch.tensor(_signed(seed + _PHI), device="cuda"))
    key = _mix(first + _signed(_PHI * ((stream << 32) | _ID) + _PHI))
    words = -(-cols // 4)
    w = _mix(key + (torch.arange(rows * words, device="cuda") + 1) * _signed(_PHI)).view(rows, words, 1)
    return ((w >> torch.tensor([0, 16, 32, 48], device="cuda")) & 0xFFFF).reshape(rows, 4 * words)[:, :cols]


def _dropped(v, p, seed):
    """v / (1 - p) where kept, else 0"""
    threshold = round(65536 * p)
    if threshold == 0:
        return v
    kept = _draws(seed, 5, *v.shape) >= threshold
    return torch.where(kept, v * (65536.0 / (65536 - threshold)), torch.zeros((), device=v.device))


def _four_bits(x, seed):
    """Codes (rows, blocks, 32) with their signs and exponents (rows, blocks) of an fp32 matrix; seed: of the stochastic rounding."""
    rows, cols = x.shape
    blocks = -(-cols // 32)
    x = torch.nn.functional.pad(x, (0, 32 * blocks - cols)).view(rows, blocks, 32)
    bits = x.abs().amax(dim=2).view(torch.int32)
    t = ((bits >> 23) - 2 + ((bits & 0x7FFFFF) > 0x400000).int()).clamp(min=0)
    v = x.abs() * ((254 - t) << 23).view(torch.float32)[..., None]             # 0 .. 6
    e = (v >= 2.0).int() + (v >= 4.0).int()                                    # steps of 2^(e - 1) from code 2 e + ..
    v = v * torch.where(e == 0, 2.0, torch.where(e == 1, 1.0, 0.5))            # 0 .. 4
    if seed is None:
        q = torch.round(v)
    else:
        draws = torch.nn.functional.pad(_draws(seed, 6, rows, cols), (0, 32 * blocks - cols)).view(rows, blocks, 32)
        q = torch.floor(v)
        q = q + (draws.float() + 0.5 < (v - q) * 65536.0).float()
    return q.int() + 2 * e + 8 * (x.view(torch.int32) < 0).int(), t


def _of_four_bits(code, t, cols):
    values = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], device=code.device)
    v = values[(code & 7).long()] * (1.0 - 2.0 * (code >> 3).float())
    return (v * torch.pow(2.0, (t - 127).float())[..., None]).reshape(code.shape[0], -1)[:, :cols]


def _unpacked(buffer, rows, cols):
    chunks = -(-cols // 256)
    codes = buffer[:rows * chunks * 128].view(rows, chunks * 128)
    code = torch.stack([codes & 15, codes >> 4], dim=2).view(rows, chunks * 8, 32).int()
    t = buffer[rows * chunks * 128:].view(chunks, rows + rows % 2, 8).transpose(0, 1)[:rows].reshape(rows, chunks * 8).int()
    return _of_four_bits(code, t, cols)


def _block_codes(x):
    """Codes (rows, blocks, 32) and exponents (rows, blocks) of an fp32 matrix's 8-bit checkpoint."""
    rows, cols = x.shape
    blocks = -(-cols // 32)
    x = torch.nn.functional.pad(x, (0, 32 * blocks - cols)).view(rows, blocks, 32)
    t = ((x.abs().amax(dim=2).view(torch.int32) >> 23) - 6).clamp(min=1)
    return torch.round(x * ((254 - t) << 23).view(torch.float32)[..., None]).clamp(-127, 127), t


def _block_values(q, t, cols):
    return (q * (t << 23).view(torch.float32)[..., None]).reshape(q.shape[0], -1)[:, :cols]


def _saved_values(buffer, rows, cols):
    blocks = -(-cols // 32)
    q = buffer[:rows * blocks * 32].view(torch.int8).view(rows, blocks, 32).float()
    return _block_values(q, buffer[rows * blocks * 32:].view(rows, blocks).to(torch.int32), cols)


def _activation(z, act):
    if act == "relu":
        return torch.maximum(z, torch.zeros((), device=z.device))
    if act == "gelu":
        return 0.5 * z * (1.0 + torch.erf(z * math.sqrt(0.5)))
    if act == "gelu_tanh":
        return 0.5 * z * (1.0 + torch.tanh(math.sqrt(2.0 / math.pi) * (z + 0.044715 * z * z * z)))
    if act == "silu":
        return z / (1.0 + torch.exp(-z))
    return z


def _slope(z, act):
    if act == "relu":
        return (z > 0).to(z.dtype)
    if act == "gelu":
        return 0.5 * (1.0 + torch.erf(z * math.sqrt(0.5))) + z * torch.exp(-0.5 * z * z) * (1.0 / math.sqrt(2.0 * math.pi))
    if act == "gelu_tanh":
        c = math.sqrt(2.0 / math.pi)
        t = torch.tanh(c * (z + 0.044715 * z * z * z))
        return 0.5 * (1.0 + t) + 0.5 * z * (1.0 - t * t) * c * (1.0 + 3 * 0.044715 * z * z)
    if act == "silu":
        p = 1.0 / (1.0 + torch.exp(-z))
        return p * (1.0 + z * (1.0 - p))
    return torch.ones_like(z)


def _normed(v, kind):
    """Rows without and with their mean and size taken out, and 1 / size."""
    if kind == "layer":
        v = v - v.mean(dim=1, keepdim=True)
    rho = torch.rsqrt((v * v).mean(dim=1, keepdim=True) + _EPS[kind])
    return v * rho, rho


def _norm(v, s, name):
    kind = s["case"][name]
    if kind == "none":
        return v
    v = _normed(v, kind)[0] * s[name + "_weight"].float()
    return v if kind == "rms" else v + s[name + "_bias"].float()


def _norm_grad(d, v, s, name, out):
    kind = s["case"][name]
    if kind == "none":
        return d
    unit, rho = _normed(v, kind)
    out[name + "_weight"] = (d * unit).sum(dim=0)
    if kind == "layer":
        out[name + "_bias"] = d.sum(dim=0)
    d = d * s[name + "_weight"].float()
    inner = unit * (d * unit).mean(dim=1, keepdim=True)
    return rho * (d - inner if kind == "rms" else d - d.mean(dim=1, keepdim=True) - inner)


_X_SCALE, _F_SCALE = 1.0, 0.75


def _gate_rows(s):
    gate = s["gate"].float()
    return gate if gate.dim() == 1 else gate.repeat_interleave(s["case"]["m"] // gate.shape[0], dim=0)


def _plain(s):
    case, dtype = s["case"], s["dtype"]
    m, n, k, act, op = case["m"], case["n"], case["k"], case["act"], case["op"]
    if op == "dropout":
        return {"y": _dropped(s["x"].float(), case["p"], s["seed"]).to(dtype)}
    if op == "join":
        r, out = s["x"].float(), {}
        if case["branch"]:
            b = _dropped(_norm(s["f"].float(), s, "post"), case["p"], s["seed"])
            r = _X_SCALE * r + _F_SCALE * (b * _gate_rows(s) if case["gates"] else b)
            out["r"] = r.to(dtype)
        if case["pre"] != "none":
            out["h"] = _norm(r, s, "pre").to(dtype)
        return out
    if op == "join_grad":
        r, out = s["x"].float(), {}
        d = s["dr"].float() if s["dr"] is not None else 0.0
        if case["pre"] != "none":
            d = d + _norm_grad(s["dh"].float(), r, s, "pre", out)
        if not case["branch"]:
            return out | {"dx": d.to(dtype)}
        out["dx"] = (_X_SCALE * d).to(dtype)
        if case["gates"]:
            b = _F_SCALE * _dropped(_norm(s["f"].float(), s, "post"), case["p"], s["seed"])
            out["gate"] = (d * b).view(case["gates"], -1, k).sum(dim=1).reshape(s["gate"].shape)
            d = d * _gate_rows(s)
        out["df"] = _norm_grad(_dropped(_F_SCALE * d, case["p"], s["seed"]), s["f"].float(), s, "post", out).to(dtype)
        return out
    if op == "quantize":
        x = s["x"].float()
        out = {"sums": x.sum(dim=0)} if case["bias"] else {}
        x = x.t().contiguous() if case["transpose"] else x
        return out | {"values": _of_four_bits(*_four_bits(x, s["seed"] if case["stochastic"] else None), x.shape[1]).to(dtype)}
    if op == "linear":
        z = torch.matmul(_of_four_bits(*_four_bits(s["x"].float(), None), k), _unpacked(s["w"], n, k).t())
        if case["bias"]:
            z = z + s["bias"].float()
        y = _activation(z, act)
        out = {"y": (y + s["residual"].float() if case["residual"] else y).to(dtype)}
        if case["checkpoint"]:
            out["z"] = _block_values(*_block_codes(z), n).to(torch.bfloat16)
        return out
    if op == "igrad":
        dx = torch.matmul(_of_four_bits(*_four_bits(s["dz"].float(), s["seed"]), n), _unpacked(s["wt"], k, n).t())
        if case["checkpoint"]:
            dx = dx * _slope(_saved_values(s["z"], m, k), act)
        return {"dx": (dx + s["residual"].float() if case["residual"] else dx).to(dtype)}
    dy = s["dy"].float()
    dyt = _of_four_bits(*_four_bits(dy.t().contiguous(), s["seed"]), m)
    out = {"dw": torch.matmul(dyt, _unpacked(s["xt"], k, m).t())}
    if case["bias"]:
        out["db"] = dy.sum(dim=0)
    return out


# ---- the framework's operators

def _own(s):
    from paper_2108_08842_amd import blocks, layers, mx4
    case, dtype = s["case"], s["dtype"]
    m, n, k, act, op = case["m"], case["n"], case["k"], case["act"], case["op"]
    if op in ("dropout", "join", "join_grad"):
        drop = blocks.Dropout(case["p"], s["seed"], _ID) if case["p"] else None
    if op == "dropout":
        return {"y": blocks.dropout(s["x"], drop)}
    if op in ("join", "join_grad"):
        post, pre = (None if case[name] == "none" else blocks.Norm(case[name], s[name + "_weight"], s[name + "_bias"], _EPS[case[name]]) for name in ("post", "pre"))
    if op == "join":
        if not case["branch"]:
            return {"h": blocks.norm(s["x"], pre)}
        got = blocks.join(s["x"], s["f"], gate=s["gate"], scale=_F_SCALE, x_scale=_X_SCALE, dropout=drop, post=post, pre=pre)
        return {"r": got} if pre is None else {"r": got[0], "h": got[1]}
    if op == "join_grad":
        if case["branch"]:
            got = blocks.join_grad(s["dr"], s["f"], dh=s["dh"], r=s["x"], gate=s["gate"], scale=_F_SCALE, x_scale=_X_SCALE, dropout=drop, post=post, pre=pre)
        else:
            got = blocks.norm_grad(s["dh"], s["x"], pre)
        return {name: value for name, value in got._asdict().items() if value is not None}
    rounding = mx4.Stochastic(s["seed"], _ID)
    if op == "quantize":
        got = mx4.quantize(s["x"], transpose=case["transpose"], rounding=rounding if case["stochastic"] else None, sums=case["bias"])
        return {"sums": got[1], "values": got[0].restore(dtype)} if case["bias"] else {"values": got.restore(dtype)}
    if op == "linear":
        got = mx4.linear(s["x"], mx4.Mx4(s["w"], n, k), s["bias"], activation=act, residual=s["residual"], checkpoint=case["checkpoint"])
        return {"y": got[0], "z": got[1].restore(torch.bfloat16)} if case["checkpoint"] else {"y": got}
    if op == "igrad":
        z = layers.Checkpoint(s["z"], m, k) if case["checkpoint"] else None
        return {"dx": mx4.linear_input_grad(mx4.quantize(s["dz"], rounding=rounding), mx4.Mx4(s["wt"], k, n), activation=act, checkpoint=z, residual=s["residual"], dtype=dtype)}
    dyt = mx4.quantize(s["dy"], transpose=True, rounding=rounding, sums=case["bias"])
    if case["bias"]:
        return {"dw": mx4.linear_weight_grad(dyt[0], mx4.Mx4(s["xt"], k, m)), "db": dyt[1]}
    return {"dw": mx4.linear_weight_grad(dyt, mx4.Mx4(s["xt"], k, m))}


def run(state):
    return _own(state) if own else _plain(state)


def work(case):
    m, n, k, op = case["m"], case["n"], case["k"], case["op"]
    size = {"f32": 4, "f16": 2, "bf16": 2}[case["dtype"]]
    hashes = 4 * m * k if case["p"] or case["stochastic"] else 0

    def four(rows, cols):                       # a byte for two values and one for 32
        return rows * (-(-cols // 32)) * 17

    if op == "dropout":
        return {"bytes": 2 * m * k * size, "flops": m * k + hashes}
    norms = [kind for kind in (case["post"], case["pre"]) if kind != "none"]
    rows_of_weights = case["gates"] + sum(2 if kind == "layer" else 1 for kind in norms)
    if op == "join":                            # x, f read; r, h written
        passes = (3 if case["branch"] else 1) + (case["pre"] != "none")
        return {"bytes": (m * passes + rows_of_weights) * k * size, "flops": 8 * m * k * (1 + len(norms)) + hashes}
    if op == "join_grad":                       # x where it is normed, f where its values count, dr, dh read; dx, df written; weights read, their gradients written
        needs_f = case["branch"] and (case["gates"] > 0 or case["post"] != "none")
        passes = 2 * (case["pre"] != "none") + needs_f + 1 + 2 * case["branch"]
        return {"bytes": m * passes * k * size + rows_of_weights * k * (size + 4), "flops": 16 * m * k * (1 + len(norms)) + hashes}
    if op == "quantize":                        # values, 4 bits written; 4 bits, values written
        bits = four(k, m) if case["transpose"] else four(m, k)
        return {"bytes": 2 * m * k * size + 2 * bits + (4 * k if case["bias"] else 0), "flops": 6 * m * k + hashes}
    flops = 2 * m * n * k
    if op == "linear":
        kept = m * (-(-n // 32)) * 33
        return {"bytes": size * (m * k + m * n * (2 if case["residual"] else 1) + (n if case["bias"] else 0)) + four(n, k)
                + (2 * kept + 2 * m * n if case["checkpoint"] else 0), "flops": flops}
    if op == "igrad":
        return {"bytes": size * (m * n + m * k * (2 if case["residual"] else 1)) + four(k, n) + (m * (-(-k // 32)) * 33 if case["checkpoint"] else 0), "flops": flops}
    return {"bytes": size * m * n + four(k, m) + 4 * n * k + (4 * n if case["bias"] else 0), "flops": flops}


# ---- the definition, in 64 bits

def exact(case, seed):
    import numpy as np
    s = prepare(case, seed)
    rows, n, k, op = case["m"], case["n"], case["k"], case["op"]

    def bits16(stream, count, width):
        def mix64(z):
            z = (z ^ (z >> np.uint64(30))) * np.uint64(0xBF58476D1CE4E5B9)
            z = (z ^ (z >> np.uint64(27))) * np.uint64(0x94D049BB133111EB)
            return z ^ (z >> np.uint64(31))
        with np.errstate(over="ignore"):
            phi = np.uint64(0x9E3779B97F4A7C15)
            tag = np.array([(stream << 32) + _ID], dtype=np.uint64)
            key = mix64(mix64(np.array([s["seed"]], dtype=np.uint64) + phi) + phi * tag + phi)
            per_row = (width + 3) // 4
            out = np.arange(1, count * per_row + 1, dtype=np.uint64)
            out *= phi
            out += key
            out = mix64(out)
        return torch.from_numpy(out.view(np.uint16).reshape(count, 4 * per_row)[:, :width].astype(np.int32)).cuda()      # (least significant bits first)

    def drop(v):
        if not case["p"]:
            return v
        least = round(65536 * case["p"])
        return torch.where(bits16(5, *v.shape) < least, 0.0, v / (1.0 - least / 65536.0))

    def power_of_two(e):
        return ((e.long() + 1023) << 52).view(torch.float64)

    grid = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], dtype=torch.float64, device="cuda")

    def to_four_bits(v, stochastic):
        v = v.double()
        draws = bits16(6, *v.shape) if stochastic else None
        out = torch.empty_like(v)
        for first in range(0, v.shape[1], 32):
            part = v[:, first:first + 32]
            largest = part.abs().max(dim=1, keepdim=True).values
            _, e = torch.frexp(largest / 6.0)                                  # 2^(e - 1) <= largest / 6 < 2^e
            e = torch.where(largest <= 6.0 * power_of_two(e - 1), e - 1, e).clamp(min=-127)
            unit = power_of_two(torch.where(largest > 0, e, torch.zeros_like(e)))
            a = part.abs() / unit
            low = torch.bucketize(a, grid, right=True) - 1
            high = (low + 1).clamp(max=7)
            share = torch.where(high > low, (a - grid[low]) / (grid[high] - grid[low]).clamp(min=0.5), 0.0)
            if stochastic:
                up = (draws[:, first:first + 32].double() + 0.5) / 65536.0 < share
            else:
                up = (share > 0.5) | ((share == 0.5) & (low % 2 == 1))
            out[:, first:first + 32] = grid[torch.where(up, high, low)] * unit * torch.where(part < 0, -1.0, 1.0)
        return out

    def from_four_bits(buffer, count, width):
        per_row = (width + 255) // 256
        codes = buffer[:count * per_row * 128].reshape(count, per_row * 128).to(torch.int16)
        nibbles = torch.empty(count, per_row * 256, dtype=torch.int64, device="cuda")
        nibbles[:, 0::2], nibbles[:, 1::2] = codes % 16, codes // 16
        exps = torch.empty(count, per_row * 8, dtype=torch.int64, device="cuda")
        even = (count + 1) // 2 * 2
        for c in range(per_row):
            at = count * per_row * 128 + c * even * 8
            exps[:, 8 * c:8 * c + 8] = buffer[at:at + count * 8].reshape(count, 8)
        return (torch.where(nibbles > 7, -grid[nibbles % 8], grid[nibbles % 8]) * power_of_two(exps - 127).repeat_interleave(32, dim=1))[:, :width]

    def from_checkpoint(buffer, width):
        blocks = (width + 31) // 32
        codes = buffer[:rows * blocks * 32].to(torch.int16)
        signed = torch.where(codes > 127, codes - 256, codes).reshape(rows, 32 * blocks).double()
        return (signed * power_of_two(buffer[rows * blocks * 32:].long() - 127).reshape(rows, blocks).repeat_interleave(32, dim=1))[:, :width]

    def to_checkpoint(v):
        out = torch.empty_like(v)
        for first in range(0, v.shape[1], 32):
            part = v[:, first:first + 32]
            largest = part.abs().max(dim=1, keepdim=True).values
            e = torch.frexp(largest).exponent                                  # the fp32 number's exponent field is e + 126
            unit = power_of_two(torch.where(largest > 0, e - 7, torch.full_like(e, -126)).clamp(min=-126))
            out[:, first:first + 32] = (part / unit).round().clamp(-127, 127) * unit
        return out

    def normal_cdf(v):
        return 0.5 * torch.erfc(-v / math.sqrt(2.0))

    def act(v, name):
        if name == "gelu":
            return v * normal_cdf(v)
        if name == "gelu_tanh":
            return v * torch.sigmoid(2.0 * math.sqrt(2.0 / math.pi) * (v + 0.044715 * v ** 3))
        return {"none": lambda: v, "relu": lambda: v.clamp(min=0.0), "silu": lambda: v * torch.sigmoid(v)}[name]()

    def act_slope(v, name):
        if name == "gelu":
            return normal_cdf(v) + v * torch.exp(-v * v / 2.0) / math.sqrt(2.0 * math.pi)
        if name == "gelu_tanh":
            b = 2.0 * math.sqrt(2.0 / math.pi)
            p = torch.sigmoid(b * (v + 0.044715 * v ** 3))
            return p + v * p * (1.0 - p) * b * (1.0 + 0.134145 * v ** 2)
        if name == "silu":
            p = torch.sigmoid(v)
            return p + v * p * (1.0 - p)
        return (v > 0).double() if name == "relu" else torch.ones_like(v)

    def statistics(v, kind):
        mean = v.sum(dim=1, keepdim=True) / k if kind == "layer" else torch.zeros(rows, 1, dtype=torch.float64, device="cuda")
        return mean, ((v - mean).square().sum(dim=1, keepdim=True) / k + _EPS[kind]) ** -0.5

    def norm(v, name):
        if case[name] == "none":
            return v
        mean, scale = statistics(v, case[name])
        out = (v - mean) * scale * s[name + "_weight"].double()
        return out + s[name + "_bias"].double() if case[name] == "layer" else out

    def norm_back(g, v, name, out):
        if case[name] == "none":
            return g
        mean, scale = statistics(v, case[name])
        hat = (v - mean) * scale
        out[name + "_weight"] = (g * hat).sum(dim=0)
        w = s[name + "_weight"].double()
        total = scale * (g * w) - scale * hat * ((g * w * hat).sum(dim=1, keepdim=True) / k)
        if case[name] == "layer":
            out[name + "_bias"] = g.sum(dim=0)
            total = total - scale * (g * w).sum(dim=1, keepdim=True) / k
        return total

    def gate_of_rows():
        gate = s["gate"].double().reshape(-1, k)
        return gate[torch.arange(rows, device="cuda") // (rows // gate.shape[0])]

    if op == "dropout":
        return {"y": drop(s["x"].double())}
    if op == "join":
        r, out = s["x"].double(), {}
        if case["branch"]:
            b = drop(norm(s["f"].double(), "post"))
            r = _X_SCALE * r + _F_SCALE * (gate_of_rows() * b if case["gates"] else b)
            out["r"] = r
        return out | {"h": norm(r, "pre")} if case["pre"] != "none" else out
    if op == "join_grad":
        out = {}
        d = torch.zeros(rows, k, dtype=torch.float64, device="cuda") if s["dr"] is None else s["dr"].double()
        if case["pre"] != "none":
            d = d + norm_back(s["dh"].double(), s["x"].double(), "pre", out)
        if not case["branch"]:
            return out | {"dx": d}
        out["dx"] = _X_SCALE * d
        if case["gates"]:
            b = _F_SCALE * drop(norm(s["f"].double(), "post"))
            out["gate"] = torch.stack([part.sum(dim=0) for part in (d * b).chunk(case["gates"], dim=0)]).reshape(s["gate"].shape)
            d = d * gate_of_rows()
        out["df"] = norm_back(drop(_F_SCALE * d), s["f"].double(), "post", out)
        return out
    if op == "quantize":
        x = s["x"].t().contiguous() if case["transpose"] else s["x"]
        out = {"values": to_four_bits(x, case["stochastic"])}
        return out | {"sums": s["x"].sum(dim=0, dtype=torch.float64)} if case["bias"] else out
    if op == "linear":
        z = to_four_bits(s["x"], False) @ from_four_bits(s["w"], n, k).t().contiguous()
        z = z + s["bias"].double() if case["bias"] else z
        y = act(z, case["act"])
        out = {"y": y + s["residual"].double() if case["residual"] else y}
        return out | {"z": to_checkpoint(z)} if case["checkpoint"] else out
    if op == "igrad":
        dx = to_four_bits(s["dz"], True) @ from_four_bits(s["wt"], k, n).t().contiguous()
        if case["checkpoint"]:
            dx = dx * act_slope(from_checkpoint(s["z"], k), case["act"])
        return {"dx": dx + s["residual"].double() if case["residual"] else dx}
    out = {"dw": to_four_bits(s["dy"].t().contiguous(), True) @ from_four_bits(s["xt"], k, rows).t().contiguous()}
    return out | {"db": s["dy"].sum(dim=0, dtype=torch.float64)} if case["bias"] else out
