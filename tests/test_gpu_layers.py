"""The layer operators on the GPU against 64 bits, at the sizes, types, distances and values where they can go wrong."""
import math
import zlib

import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from tests import layers_reference as ref                          # noqa: E402

TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
ACTS = ["none", "relu", "gelu", "gelu_tanh", "silu"]
# rows, features out, features in: single ones, a block more or less, a tile more or less, sums that are split over workgroups
SIZES = [(1, 1, 1), (1, 40, 7), (2, 31, 64), (3, 1000, 96), (5, 130, 2056), (16, 33, 333), (17, 128, 128), (127, 129, 31), (128, 128, 64),
         (129, 257, 191), (130, 64, 1024), (300, 72, 1500), (700, 40, 33), (1025, 24, 65)]


@pytest.fixture(scope="module")
def layers():
    from paper_2108_08842_amd import layers as m
    assert torch.cuda.is_available()
    m.lib()
    return m


def matrix(gen, rows, cols, dtype, pad=0, scale=1.0):
    """A matrix on the GPU whose rows are `pad` elements further apart than they are long, surrounded by NaN."""
    x = torch.full((rows, cols + pad), float("nan"), dtype=dtype)
    x[:, :cols] = (torch.randn(rows, cols, generator=gen, dtype=torch.float64) * scale).to(dtype)
    return x.cuda()[:, :cols]


def saved(layers, x):
    """A checkpoint made by the reference from a CPU fp32 matrix, and its values in 64 bits."""
    codes, exps = ref.encode(x.numpy())
    return layers.Checkpoint(ref.pack(codes, exps).cuda(), *x.shape), torch.from_numpy(ref.decode(codes, exps, x.shape[1]))


def gen(*key):
    return torch.Generator().manual_seed(zlib.crc32(repr(key).encode()))


# ---- checkpoints

def special_rows():
    rows = [np.zeros(70), np.full(70, -0.0), np.arange(70) - 35.0, np.linspace(-1, 1, 70), np.full(70, 1e-45), np.full(70, 2.0 ** -126), np.full(70, 2.0 ** -130),
            np.full(70, 3.4028234e38), np.geomspace(1e-38, 1e38, 70), np.full(70, 127.5), np.full(70, 127.75), np.full(70, 0.5) + np.arange(70)]
    for bad in (np.inf, -np.inf, np.nan):
        for at in (0, 31, 32, 69):
            r = np.linspace(-2, 2, 70)
            r[at] = bad
            rows.append(r)
    tiny = np.full(70, 2.0 ** -120)
    tiny[::3] = 2.0 ** -127
    rows.append(tiny)
    return torch.from_numpy(np.stack(rows).astype(np.float32))


@pytest.mark.parametrize("dtype", TYPES)
def test_checkpoint_of_special_values_is_bit_exact(layers, dtype):
    x = special_rows().to(TYPES[dtype])
    c = layers.save_checkpoint(x.cuda())
    codes, exps = ref.encode(x.float().numpy())
    got_codes, got_exps = ref.unpack(c.buffer, *x.shape)
    assert np.array_equal(got_exps, exps) and np.array_equal(got_codes, codes)
    want = torch.from_numpy(ref.decode(codes, exps, x.shape[1]))
    for out in TYPES.values():
        got = c.restore(out).cpu()
        assert torch.equal(got.isnan(), want.isnan())
        assert torch.equal(torch.nan_to_num(got, nan=0.0, posinf=math.inf, neginf=-math.inf),
                           torch.nan_to_num(want, nan=0.0).float().to(out))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,cols,pad", [(1, 1, 0), (1, 31, 0), (3, 32, 1), (2, 33, 3), (65, 1000, 0), (7, 4097, 5), (1000, 40, 8), (513, 96, 0)])
def test_checkpoint_is_bit_exact(layers, dtype, rows, cols, pad):
    x = matrix(gen(dtype, rows, cols), rows, cols, TYPES[dtype], pad, 3.0)
    codes, exps = ref.encode(x.cpu().float().numpy())
    into = layers.Checkpoint(torch.full((layers.checkpoint_bytes(rows, cols) + 64,), 0xA5, dtype=torch.uint8, device="cuda"), rows, cols)
    assert layers.save_checkpoint(x, into=into) is into
    got_codes, got_exps = ref.unpack(into.buffer, rows, cols)
    assert np.array_equal(got_exps, exps) and np.array_equal(got_codes, codes)
    assert bool((into.buffer[layers.checkpoint_bytes(rows, cols):] == 0xA5).all())
    want = ref.decode(codes, exps, cols)
    out = torch.full((rows, cols + pad), 7.0, dtype=torch.float32, device="cuda")
    into.restore(out=out[:, :cols])
    assert np.array_equal(out[:, :cols].cpu().double().numpy(), want) and bool((out[:, cols:] == 7.0).all())
    # the error is at most half a unit, a whole one where the code is clipped
    unit = np.repeat(np.exp2(exps.astype(np.float64) - 127), 32, axis=1)[:, :cols]
    d = np.abs(want - x.cpu().double().numpy())
    assert np.all(d <= unit * np.where(np.abs(want) == 127 * unit, 1.0, 0.5))


# ---- forward

@pytest.mark.parametrize("m,n,k", SIZES)
@pytest.mark.parametrize("dtype", TYPES)
def test_linear(layers, dtype, m, n, k):
    t = TYPES[dtype]
    g = gen("linear", dtype, m, n, k)
    for number, (act, with_bias, with_residual, keep, pad) in enumerate([("none", False, False, False, 0), ("gelu", True, False, True, 0), ("silu", True, True, True, 3),
                                                                         ("relu", False, True, False, 8), ("gelu_tanh", True, True, True, 1)]):
        x, w = matrix(g, m, k, t, pad), matrix(g, n, k, t, pad if number != 2 else 0, k ** -0.5)
        bias = matrix(g, 1, n, t)[0] if with_bias else None
        residual = matrix(g, m, n, t, pad) if with_residual else None
        out = torch.full((m, n + pad), 5.0, dtype=t, device="cuda")
        got = layers.linear(x, w, bias, activation=act, residual=residual, checkpoint=keep, out=out[:, :n])
        y, z8 = got if keep else (got, None)
        X, W = x.cpu().double(), w.cpu().double()
        z = X @ W.t() + (bias.cpu().double() if with_bias else 0.0)
        want = ref.act(z, act) + (residual.cpu().double() if with_residual else 0.0)
        dz = ref.product_bound(X, W, k) + 4 * ref.EPS * z.abs()
        # slopes are below 1.13; an activation is off by 16 fp32 roundings (2-byte results: exp and the quotient of z in one instruction each)
        near = 1.13 * dz + (2.0 ** -20 + 2.0 ** -23 * z.abs()) * ref.act(z, act).abs() + 2.0 ** -22 * (z.abs() + want.abs()) + ref.ROUND[t] * want.abs() + ref.TINY[t]
        assert bool(((y.cpu().double() - want).abs() <= near).all()), (act, (y.cpu().double() - want).abs().max())
        if m * n >= 64:
            # the whole result against the rounding of independent sums; a residual or bias only makes it larger
            assert ref.rel(y.cpu(), want) <= 1.5 * ref.norm_bound(k, t) + 2.0 ** -20, act
        assert bool((out[:, n:] == 5.0).all())
        if keep:
            codes, exps = ref.unpack(z8.buffer, m, n)
            unit = torch.from_numpy(np.repeat(np.exp2(exps.astype(np.float64) - 127), 32, axis=1)[:, :n])
            got = torch.from_numpy(ref.decode(codes, exps, n))
            assert bool(((got - z).abs() <= unit * torch.where(got.abs() == 127 * unit, 1.0, 0.5) + dz).all())
            assert not codes[:, n:].any()


def test_linear_checkpoint_is_that_of_z(layers):
    # fp32 and no activation: y is z, so its own checkpoint has the same bytes, whatever the path (whole, split, few rows)
    for m, n, k in [(200, 200, 100), (40, 70, 3000), (3, 100, 500), (1, 33, 4000)]:
        g = gen("z", m)
        y, c = layers.linear(matrix(g, m, k, torch.float32), matrix(g, n, k, torch.float32), checkpoint=True)
        assert torch.equal(layers.save_checkpoint(y).buffer, c.buffer)


@pytest.mark.parametrize("dtype", TYPES)
def test_linear_without_terms_rows_or_columns(layers, dtype):
    t = TYPES[dtype]
    bias = torch.tensor([1.0, -2.0, 3.0], dtype=t, device="cuda")
    y, c = layers.linear(torch.empty(2, 0, dtype=t, device="cuda"), torch.empty(3, 0, dtype=t, device="cuda"), bias, activation="relu", checkpoint=True)
    assert y.cpu().tolist() == [[1.0, 0.0, 3.0]] * 2 and c.restore(torch.float32).cpu().tolist() == [[1.0, -2.0, 3.0]] * 2
    assert layers.linear(torch.empty(0, 5, dtype=t, device="cuda"), torch.ones(3, 5, dtype=t, device="cuda")).shape == (0, 3)
    assert layers.linear(torch.ones(4, 5, dtype=t, device="cuda"), torch.empty(0, 5, dtype=t, device="cuda")).shape == (4, 0)
    dw, db = layers.linear_weight_grad(torch.empty(0, 3, dtype=t, device="cuda"), layers.save_checkpoint(torch.empty(0, 40, dtype=t, device="cuda")), bias=True)
    assert torch.equal(dw.cpu(), torch.zeros(3, 40)) and torch.equal(db.cpu(), torch.zeros(3))
    dw, db = layers.linear_weight_grad(torch.ones(5, 3, dtype=t, device="cuda"), layers.save_checkpoint(torch.empty(5, 0, dtype=t, device="cuda")), bias=True)
    assert dw.shape == (3, 0) and torch.equal(db.cpu(), torch.full((3,), 5.0))
    dx = layers.linear_input_grad(torch.empty(2, 0, dtype=t, device="cuda"), torch.empty(0, 6, dtype=t, device="cuda"), residual=torch.ones(2, 6, dtype=t, device="cuda"))
    assert torch.equal(dx.cpu(), torch.ones(2, 6, dtype=t))
    assert layers.activation_grad(torch.empty(0, 6, dtype=t, device="cuda"), layers.save_checkpoint(torch.empty(0, 6, dtype=t, device="cuda")), "gelu").shape == (0, 6)


def test_leading_dimensions_and_residual_in_place(layers):
    g = gen("dims")
    x, w, r = torch.randn(2, 3, 5, 64, generator=g).cuda(), torch.randn(48, 64, generator=g).cuda(), torch.randn(2, 3, 5, 48, generator=g).cuda()
    y, c = layers.linear(x, w, residual=r, checkpoint=True)
    flat = layers.linear(x.view(30, 64), w, residual=r.view(30, 48))
    assert y.shape == r.shape and (c.rows, c.cols) == (30, 48) and torch.equal(y.view(30, 48), flat)
    assert layers.linear(x, w, residual=r, out=r) is r and torch.equal(r, y)
    dy = torch.randn(2, 3, 5, 48, generator=g).cuda()
    want = layers.activation_grad(dy, c, "silu")
    assert want.shape == dy.shape and torch.equal(layers.activation_grad(dy, c, "silu", out=dy), want)


# ---- backward

@pytest.mark.parametrize("m,n,k", SIZES)
@pytest.mark.parametrize("dtype", TYPES)
def test_weight_grad(layers, dtype, m, n, k):
    t = TYPES[dtype]
    g = gen("wgrad", dtype, m, n, k)
    for pad in (0, 3):
        dy = matrix(g, m, n, t, pad)
        c, X = saved(layers, torch.randn(m, k, generator=g) * 10.0)
        Y = dy.cpu().double()
        want, want_b = Y.t() @ X, Y.sum(0)
        flat = torch.full((5 + n * k + 3 + n,), 4.0, device="cuda")          # a part of a longer vector, not at a multiple of 16 bytes
        out, bias_out = flat[5:5 + n * k].view(n, k), flat[5 + n * k + 3:]
        dw, db = layers.linear_weight_grad(dy, c, out=out, bias_out=bias_out)
        near = ref.product_bound(Y.t(), X.t(), m) + 2.0 ** -24 * want.abs()
        near_b = (m + 8) * 2.0 ** -23 * Y.abs().sum(0)
        assert bool(((dw.cpu().double() - want).abs() <= near).all()) and bool(((db.cpu().double() - want_b).abs() <= near_b).all())
        if n * k >= 64:
            assert ref.rel(dw.cpu(), want) <= ref.norm_bound(m, torch.float32)
        first, first_b = dw.clone(), db.clone()
        layers.linear_weight_grad(dy, c, out=out, bias_out=bias_out, accumulate=True)
        assert torch.equal(dw, first + first) and torch.equal(db, first_b + first_b)
        assert torch.equal(layers.linear_weight_grad(dy, c), first)
        assert bool((flat[:5] == 4.0).all()) and bool((flat[5 + n * k:8 + n * k] == 4.0).all())


@pytest.mark.parametrize("m,n,k", SIZES)
@pytest.mark.parametrize("dtype", TYPES)
def test_input_grad(layers, dtype, m, n, k):
    t = TYPES[dtype]
    g = gen("igrad", dtype, m, n, k)
    for act, with_residual, pad in [("none", False, 0), ("gelu", False, 3), ("silu", True, 0), ("relu", True, 8), ("gelu_tanh", True, 1)]:
        dz, w = matrix(g, m, n, t, pad), matrix(g, n, k, t, pad, n ** -0.5)
        residual = matrix(g, m, k, t, pad) if with_residual else None
        c, z = saved(layers, torch.randn(m, k, generator=g) * 2.0) if act != "none" else (None, torch.zeros(m, k, dtype=torch.float64))
        Z, W = dz.cpu().double(), w.cpu().double()
        s = ref.slope(z, act)
        product = Z @ W
        want = product * s + (residual.cpu().double() if with_residual else 0.0)
        dx = layers.linear_input_grad(dz, w, activation=act, checkpoint=c, residual=residual)
        # a slope is off by 2^-19 at most: exp is by |z| 2^-23 of itself, and the terms are below 1.2
        near = 1.13 * ref.product_bound(Z, W.t(), n) + 2.0 ** -19 * product.abs() + 4 * ref.EPS * want.abs() + ref.ROUND[t] * want.abs() + ref.TINY[t]
        assert bool(((dx.cpu().double() - want).abs() <= near).all()), act
        if m * k >= 64:
            assert ref.rel(dx.cpu(), want) <= 1.5 * ref.norm_bound(n, t) + 2.0 ** -19, act


@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("dtype", TYPES)
def test_activation_grad(layers, dtype, act):
    t = TYPES[dtype]
    for rows, cols, pad in [(1, 1, 0), (3, 33, 1), (64, 1000, 0), (257, 40, 8)]:
        g = gen("agrad", rows, cols)
        dy = matrix(g, rows, cols, t, pad)
        c, z = saved(layers, torch.randn(rows, cols, generator=g) * 3.0)
        want = dy.cpu().double() * ref.slope(z, act)
        got = layers.activation_grad(dy, c, act).cpu().double()
        near = 2.0 ** -19 * dy.cpu().double().abs() + ref.ROUND[t] * want.abs() + ref.TINY[t]
        assert bool(((got - want).abs() <= near).all())


@pytest.mark.parametrize("act", ACTS)
def test_slopes_at_the_ends_of_the_range(layers, act):
    # 127 codes times the largest and the smallest units; the slope is finite everywhere, and NaN for a block that is not finite
    far = torch.tensor([[2.0 ** 127, -2.0 ** 127] * 16 + [2.0 ** 64, -2.0 ** 64] * 16 + [100.0, -100.0] * 16 + [2.0 ** -126, -2.0 ** -126] * 16 + [0.0, -0.0] * 16
                        + [float("nan"), 1.0] * 16])
    c = layers.save_checkpoint(far.cuda())
    got = layers.activation_grad(torch.ones_like(far).cuda(), c, act).cpu()
    assert bool(got[:, :160].isfinite().all()) and bool(got[:, 160:].isnan().all() if act != "none" else (got[:, 160:] == 1.0).all())
    ends = {"none": (1.0, 1.0), "relu": (1.0, 0.0), "gelu": (1.0, 0.0), "gelu_tanh": (1.0, 0.0), "silu": (1.0, 0.0)}[act]
    assert bool((got[:, :96:2] == ends[0]).all()) and bool((got[:, 1:96:2].abs() == ends[1]).all())
    middle = {"none": 1.0, "relu": 0.0}.get(act, 0.5)
    assert bool((got[:, 128:160] == middle).all())


@pytest.mark.parametrize("act", ["none", "gelu", "gelu_tanh", "silu"])
def test_gradients_against_differences(layers, act):
    """One layer and the loss sum(c y): the gradients from the kernels against central differences of the 64-bit forward pass.
    x and z are of a kind that their checkpoints hold exactly."""
    g = gen("differences", act)
    m, n, k = 6, 5, 9
    x = torch.randint(-64, 65, (m, k), generator=g).double() / 16
    x[:, 0] = 4.0                                                  # every block's largest value: units of 1/16
    w = torch.randint(-3, 4, (n, k), generator=g).double() / 8
    b = torch.randint(-8, 9, (n,), generator=g).double() / 8
    c = torch.randn(m, n, generator=g, dtype=torch.float64)
    z = x @ w.t() + b
    codes, exps = ref.encode(z.float().numpy())
    z8 = layers.Checkpoint(ref.pack(codes, exps).cuda(), m, n)
    held = torch.from_numpy(ref.decode(codes, exps, n))            # the slope is taken here

    def loss(x, w, b):
        y = x @ w.t() + b + (held - z)                             # shifted so that it is held at the point itself
        return float((c * ref.act(y, act)).sum())

    def differences(t, f):
        d, h = torch.zeros_like(t), 1e-5
        for i in range(t.numel()):
            up, down = t.clone(), t.clone()
            up.view(-1)[i] += h
            down.view(-1)[i] -= h
            d.view(-1)[i] = (f(up) - f(down)) / (2 * h)
        return d

    dz = layers.activation_grad(c.float().cuda(), z8, act)
    kept = layers.save_checkpoint(x.float().cuda())
    assert torch.equal(ref.values(kept), x)
    dw, db = layers.linear_weight_grad(dz, kept, bias=True)
    dx = layers.linear_input_grad(dz, w.float().cuda())
    for got, want in ((dw, differences(w, lambda v: loss(x, v, b))), (db, differences(b, lambda v: loss(x, w, v))), (dx, differences(x, lambda v: loss(v, w, b)))):
        # differences: h^2 f''' / 6 ~ 1e-10 and 64-bit cancellation 1e-16 / 1e-5; fp32 gradients 1e-5
        assert bool(((got.cpu().double() - want).abs() <= 1e-5 * (1.0 + want.abs()) * 4).all())


# ---- results that fill the device: another kernel (rows of whole 16-byte pieces, two-byte types), ragged tiles, depths around its steps of 64

def wide(seed, rows, cols, dtype, pad=0, scale=1.0):
    """A matrix whose rows are `pad` elements further apart than they are long, NaN between them and behind the last."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    x = torch.full((rows * (cols + pad) + 64,), float("nan"), dtype=dtype, device="cuda")
    m = x[:rows * (cols + pad)].view(rows, cols + pad)[:, :cols]
    m.copy_(torch.randn(rows, cols, generator=g, device="cuda") * scale)
    return m


@pytest.mark.parametrize("depth,pad", [(8, 0), (56, 8), (64, 0), (72, 0), (200, 24), (1000, 0)])
@pytest.mark.parametrize("dtype", ["f16", "bf16"])
def test_large_linear(layers, dtype, depth, pad):
    t, m, n = TYPES[dtype], 3337, 3592
    x, w, bias, r = wide(1, m, depth, t, pad), wide(2, n, depth, t, pad, depth ** -0.5), wide(3, 1, n, t)[0], wide(4, m, n, t, pad)
    out = torch.full((m, n + pad), 5.0, dtype=t, device="cuda")
    y, c = layers.linear(x, w, bias, activation="gelu", residual=r, checkpoint=True, out=out[:, :n])
    z = x.double() @ w.double().t().contiguous() + bias.double()
    want = ref.act(z, "gelu") + r.double()
    dz = ref.product_bound(x.double(), w.double(), depth) + 4 * ref.EPS * z.abs()
    near = 1.13 * dz + 2.0 ** -20 * (1.0 + z.abs() + want.abs()) + ref.ROUND[t] * want.abs()
    assert bool(((y.double() - want).abs() <= near).all()) and bool((out[:, n:] == 5.0).all())
    assert ref.rel(y, want) <= 1.5 * ref.norm_bound(depth, t) + 2.0 ** -20
    codes, exps = ref.unpack(c.buffer, m, n)
    unit = torch.from_numpy(np.repeat(np.exp2(exps.astype(np.float64) - 127), 32, axis=1)[:, :n])
    got = torch.from_numpy(ref.decode(codes, exps, n))
    assert bool(((got - z.cpu()).abs() <= unit * torch.where(got.abs() == 127 * unit, 1.0, 0.5) + dz.cpu()).all()) and not codes[:, n:].any()


@pytest.mark.parametrize("depth,pad", [(8, 8), (64, 0), (72, 24), (328, 0)])
@pytest.mark.parametrize("dtype", ["f16", "bf16"])
def test_large_input_grad(layers, dtype, depth, pad):
    t, m, k = TYPES[dtype], 3337, 3592
    dz, w, r = wide(1, m, depth, t, pad), wide(2, depth, k, t, pad, depth ** -0.5), wide(4, m, k, t, pad)
    saved_z = layers.save_checkpoint(wide(5, m, k, t, 0, 2.0))
    s = ref.slope(saved_z.restore(torch.float32).double(), "silu")
    product = dz.double() @ w.double()
    want = product * s + r.double()
    dx = layers.linear_input_grad(dz, w, activation="silu", checkpoint=saved_z, residual=r)
    near = 1.13 * ref.product_bound(dz.double(), w.double().t().contiguous(), depth) + 2.0 ** -19 * product.abs() + (4 * ref.EPS + ref.ROUND[t]) * want.abs() + ref.TINY[t]
    assert bool(((dx.double() - want).abs() <= near).all())
    assert ref.rel(dx, want) <= 1.5 * ref.norm_bound(depth, t) + 2.0 ** -19


@pytest.mark.parametrize("depth,pad", [(1, 0), (63, 8), (64, 0), (65, 0), (333, 24), (1000, 0)])
def test_large_weight_grad(layers, depth, pad):
    n, k = 3592, 3589
    dy = wide(1, depth, n, torch.bfloat16, pad)
    c = layers.save_checkpoint(wide(2, depth, k, torch.bfloat16, 0, 10.0))
    X, Y = c.restore(torch.float32).double(), dy.double()
    flat = torch.full((3 + n * k + n + 2,), 4.0, device="cuda")
    out, bias_out = flat[3:3 + n * k].view(n, k), flat[3 + n * k:-2]
    layers.linear_weight_grad(dy, c, out=out, bias_out=bias_out)
    want, want_b = Y.t().contiguous() @ X, Y.sum(0)
    near = ref.product_bound(Y.t().contiguous(), X.t().contiguous(), depth) + 2.0 ** -24 * want.abs()
    assert bool(((out.double() - want).abs() <= near).all()) and ref.rel(out, want) <= ref.norm_bound(depth, torch.float32)
    assert bool(((bias_out.double() - want_b).abs() <= (depth + 8) * 2.0 ** -23 * Y.abs().sum(0)).all())
    first, first_b = out.clone(), bias_out.clone()
    layers.linear_weight_grad(dy, c, out=out, bias_out=bias_out, accumulate=True)
    assert torch.equal(out, first + first) and torch.equal(bias_out, first_b + first_b)
    assert bool((flat[:3] == 4.0).all()) and bool((flat[-2:] == 4.0).all())


@pytest.mark.parametrize("m,n,k,pad", [(1500, 1501, 1499, 0), (1501, 1504, 1496, 3), (1499, 1500, 1501, 8)])
@pytest.mark.parametrize("dtype", TYPES)
def test_large_products_of_rows_that_begin_anywhere(layers, dtype, m, n, k, pad):
    # operands are copied first where a workspace is given; the same call without one gives the same up to the order of additions
    t = TYPES[dtype]
    x, w, dy = wide(1, m, k, t, pad), wide(2, n, k, t, pad, k ** -0.5), wide(3, m, n, t, pad)
    assert layers.lib().eden_layers_copying_bytes(m, n, k, 1) > layers.lib().eden_layers_workspace_bytes(m, n, k, 1)
    X, W, Y = x.double(), w.double(), dy.double()
    y, z = layers.linear(x, w, checkpoint=True)
    want = X @ W.t().contiguous()
    assert bool(((y.double() - want).abs() <= ref.product_bound(X, W, k) + ref.ROUND[t] * want.abs() + ref.TINY[t]).all()) and ref.rel(y, want) <= ref.norm_bound(k, t)
    dx = layers.linear_input_grad(dy, w, activation="gelu_tanh", checkpoint=layers.save_checkpoint(x), residual=x)
    product = Y @ W
    want = product * ref.slope(layers.save_checkpoint(x).restore(torch.float32).double(), "gelu_tanh") + X
    near = 1.13 * ref.product_bound(Y, W.t().contiguous(), n) + 2.0 ** -19 * product.abs() + (4 * ref.EPS + ref.ROUND[t]) * want.abs() + ref.TINY[t]
    assert bool(((dx.double() - want).abs() <= near).all())
    c = layers.save_checkpoint(x)
    dw, db = layers.linear_weight_grad(dy, c, bias=True)
    want = Y.t().contiguous() @ c.restore(torch.float32).double()
    assert ref.rel(dw, want) <= ref.norm_bound(m, torch.float32) and ref.rel(db, Y.sum(0)) <= ref.norm_bound(m, torch.float32)


@pytest.mark.parametrize("m,n,k,pad", [(300, 264, 136, 0), (1100, 1000, 72, 8), (1033, 1016, 8, 0), (200, 520, 1000, 16), (32, 1000, 1928, 0), (5, 16400, 264, 0), (16, 16385, 1032, 8), (8, 20000, 136, 0)])
@pytest.mark.parametrize("dtype", ["f16", "bf16"])
def test_middle_sizes_of_whole_pieces(layers, dtype, m, n, k, pad):
    # with and without splits of the depth, and few rows next to many columns
    t = TYPES[dtype]
    x, w, bias, r = wide(1, m, k, t, pad), wide(2, n, k, t, pad, k ** -0.5), wide(3, 1, n, t)[0], wide(4, m, n, t, pad)
    y, c = layers.linear(x, w, bias, activation="relu", residual=r, checkpoint=True)
    z = x.double() @ w.double().t().contiguous() + bias.double()
    want = ref.act(z, "relu") + r.double()
    dz = ref.product_bound(x.double(), w.double(), k) + 4 * ref.EPS * z.abs()
    assert bool(((y.double() - want).abs() <= 1.01 * dz + (4 * ref.EPS + ref.ROUND[t]) * want.abs() + ref.TINY[t]).all())
    assert ref.rel(y, want) <= 1.5 * ref.norm_bound(k, t)
    codes, exps = ref.unpack(c.buffer, m, n)
    unit = torch.from_numpy(np.repeat(np.exp2(exps.astype(np.float64) - 127), 32, axis=1)[:, :n])
    got = torch.from_numpy(ref.decode(codes, exps, n))
    assert bool(((got - z.cpu()).abs() <= unit * torch.where(got.abs() == 127 * unit, 1.0, 0.5) + dz.cpu()).all()) and not codes[:, n:].any()
    if n % 8 == 0:
        g, v = wide(5, m, k, t, pad), wide(6, k, n, t, pad, k ** -0.5)
        want = g.double() @ v.double() + r.double()
        dx = layers.linear_input_grad(g, v, residual=r)
        near = 1.01 * ref.product_bound(g.double(), v.double().t().contiguous(), k) + (4 * ref.EPS + ref.ROUND[t]) * want.abs() + ref.TINY[t]
        assert bool(((dx.double() - want).abs() <= near).all())


@pytest.mark.parametrize("m", [1, 2, 3, 4, 7, 11])
@pytest.mark.parametrize("n,k,pad", [(8195, 1101, 3), (8192, 1160, 0), (16390, 1100, 0), (516, 3000, 5)])
@pytest.mark.parametrize("dtype", TYPES)
def test_few_rows_next_to_many_columns(layers, dtype, n, k, pad, m):
    t = TYPES[dtype]
    x, w, bias, r = wide(1, m, k, t, pad), wide(2, n, k, t, pad, k ** -0.5), wide(3, 1, n, t)[0], wide(4, m, n, t, pad)
    y = layers.linear(x, w, bias, activation="relu", residual=r)
    z = x.double() @ w.double().t().contiguous() + bias.double()
    want = ref.act(z, "relu") + r.double()
    near = 1.01 * ref.product_bound(x.double(), w.double(), k) + 4 * ref.EPS * z.abs() + (4 * ref.EPS + ref.ROUND[t]) * want.abs() + ref.TINY[t]
    assert bool(((y.double() - want).abs() <= near).all())


@pytest.mark.parametrize("rows,n,k,pad", [(4100, 264, 260, 0), (40, 2600, 2600, 8), (1032, 520, 513, 0)])
def test_middle_sizes_of_weight_grad(layers, rows, n, k, pad):
    dy = wide(1, rows, n, torch.bfloat16, pad)
    c = layers.save_checkpoint(wide(2, rows, k, torch.bfloat16, 0, 10.0))
    X, Y = c.restore(torch.float32).double(), dy.double()
    dw, db = layers.linear_weight_grad(dy, c, bias=True)
    want, want_b = Y.t().contiguous() @ X, Y.sum(0)
    near = ref.product_bound(Y.t().contiguous(), X.t().contiguous(), rows) + 2.0 ** -24 * want.abs()
    assert bool(((dw.double() - want).abs() <= near).all()) and ref.rel(dw, want) <= ref.norm_bound(rows, torch.float32)
    assert bool(((db.double() - want_b).abs() <= (rows + 8) * 2.0 ** -23 * Y.abs().sum(0)).all())


@pytest.mark.parametrize("m,depth,n,pad", [(129, 4, 260, 0), (300, 36, 516, 4), (1000, 1000, 1284, 0), (2100, 100, 2052, 12), (129, 3200, 1000, 0), (9000, 12, 4004, 4)])
def test_large_fp32_products(layers, m, depth, n, pad):
    # rows of whole 16-byte pieces: depths around the kernel's steps of 32, tiles that end inside the result, one and several splits
    x, w, bias, r = wide(1, m, depth, torch.float32, pad), wide(2, n, depth, torch.float32, pad, depth ** -0.5), wide(3, 1, n, torch.float32)[0], wide(4, m, n, torch.float32, pad)
    y, c = layers.linear(x, w, bias, residual=r, checkpoint=True)
    z = x.double() @ w.double().t().contiguous() + bias.double()
    want = z + r.double()
    assert bool(((y.double() - want).abs() <= ref.product_bound(x.double(), w.double(), depth) + 6 * ref.EPS * (z.abs() + want.abs())).all())
    assert ref.rel(y, want) <= ref.norm_bound(depth, torch.float32)
    assert torch.equal(layers.save_checkpoint(layers.linear(x, w, bias)).buffer, c.buffer)
    dz, v = wide(5, m, depth, torch.float32, pad), wide(6, depth, n, torch.float32, pad)
    want = dz.double() @ v.double()
    dx = layers.linear_input_grad(dz, v)
    assert bool(((dx.double() - want).abs() <= ref.product_bound(dz.double(), v.double().t().contiguous(), depth)).all())
    assert ref.rel(dx, want) <= ref.norm_bound(depth, torch.float32)


def test_large_products_give_the_same_bits_every_time(layers):
    # loads into the LDS, barriers and stages: a missing wait would show as results that come and go
    x, w, dy = wide(1, 4096, 2048, torch.bfloat16), wide(2, 4096, 2048, torch.bfloat16), wide(3, 4096, 4096, torch.bfloat16)
    c = layers.save_checkpoint(x)
    calls = [lambda: layers.linear(x, w), lambda: layers.linear_input_grad(dy, w), lambda: layers.linear_weight_grad(dy, c)]
    first = [f() for f in calls]
    for _ in range(20):
        for f, want in zip(calls, first):
            assert torch.equal(f(), want)
    assert ref.rel(first[0], x.double() @ w.double().t().contiguous()) <= ref.norm_bound(2048, torch.bfloat16)
    assert ref.rel(first[1], dy.double() @ w.double()) <= ref.norm_bound(4096, torch.bfloat16)


# ---- values that are not finite

@pytest.mark.parametrize("dtype", TYPES)
def test_values_that_are_not_finite_reach_what_they_should(layers, dtype):
    t = TYPES[dtype]
    for m in (3, 40):                                              # few rows, tiles
        x, w = torch.ones(m, 200, dtype=t), torch.ones(100, 200, dtype=t)
        x[1, 7] = float("nan")
        w[50, 199] = float("nan")
        y, c = layers.linear(x.cuda(), w.cuda(), checkpoint=True)
        bad = torch.zeros(m, 100, dtype=torch.bool)
        bad[1] = bad[:, 50] = True
        assert torch.equal(y.cpu().isnan(), bad) and bool((y.cpu()[~bad] == 200.0).all())
        blocks = bad.clone()
        blocks[:, 32:64] = True                                    # the block of a NaN
        assert torch.equal(c.restore(torch.float32).cpu().isnan(), blocks)
        x = torch.ones(m, 200, dtype=t)
        x[2, 5] = float("inf")
        y = layers.linear(x.cuda(), torch.ones(100, 200, dtype=t, device="cuda")).cpu()
        assert not bool(y[2].isfinite().any()) and bool((y[torch.arange(m) != 2] == 200.0).all())
        dy = torch.ones(m, 40, dtype=t)
        dy[0, 3] = float("inf")
        dy[1, 4] = float("nan")
        kept, _ = saved(layers, torch.ones(m, 70))
        dw, db = layers.linear_weight_grad(dy.cuda(), kept, bias=True)
        dw, db = dw.cpu(), db.cpu()
        assert bool((dw[3] == float("inf")).all()) and float(db[3]) == float("inf") and bool(dw[4].isnan().all()) and math.isnan(float(db[4]))
        rest = [i for i in range(40) if i not in (3, 4)]
        assert bool((dw[rest] == m).all()) and bool((db[rest] == m).all())


# ---- distances, streams, graphs

def test_rows_further_apart_than_32_bits_reach(layers):
    # 9 rows at a distance of 2^29 + 5 elements: byte offsets up to 2^33
    far = torch.empty(8 * (2 ** 29 + 5) + 96, dtype=torch.bfloat16, device="cuda")
    x = far.as_strided((9, 96), (2 ** 29 + 5, 1))
    g = gen("far")
    x.copy_(torch.randn(9, 96, generator=g).bfloat16())
    w, near = torch.randn(200, 96, generator=g).bfloat16().cuda(), x.contiguous()
    assert torch.equal(layers.linear(x, w), layers.linear(near, w))
    wide = far[:8 * (2 ** 29 + 5) + 96].as_strided((9, 96), (2 ** 29 + 5, 1))
    c = layers.save_checkpoint(wide)
    assert torch.equal(c.buffer, layers.save_checkpoint(near).buffer)
    dy = torch.randn(9, 96, generator=g).bfloat16().cuda()
    want = layers.linear_weight_grad(dy, c)
    x.copy_(dy)
    assert torch.equal(layers.linear_weight_grad(x, c), want)
    assert torch.equal(layers.activation_grad(x, c, "gelu"), layers.activation_grad(dy, c, "gelu"))
    v = torch.randn(96, 300, generator=g).bfloat16().cuda()
    assert torch.equal(layers.linear_input_grad(x, v), layers.linear_input_grad(dy, v))
    out = far.as_strided((9, 96), (2 ** 29 + 5, 1))
    c.restore(out=out)
    assert torch.equal(out, c.restore(torch.bfloat16))


def test_other_streams_and_repeated_calls_give_the_same_bits(layers):
    g = gen("streams")
    x, w = torch.randn(60, 2000, generator=g).cuda(), torch.randn(70, 2000, generator=g).cuda()      # a split sum
    assert layers.lib().eden_layers_workspace_bytes(60, 70, 2000, layers.F32) > 0
    want = layers.linear(x, w, activation="gelu")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = layers.linear(x, w, activation="gelu", stream=side)
    with torch.cuda.stream(side):
        again = layers.linear(x, w, activation="gelu")
    side.synchronize()
    assert torch.equal(got, want) and torch.equal(again, want)
    for _ in range(5):
        assert torch.equal(layers.linear(x, w, activation="gelu"), want)


def test_without_a_workspace(layers):
    # the same call without room to split: the same result up to the order of additions, and no write anywhere else
    from paper_2108_08842_amd import eden
    g = gen("workspace")
    m, n, k = 40, 70, 5000
    x, w = torch.randn(m, k, generator=g).cuda(), torch.randn(n, k, generator=g).cuda()
    want = layers.linear(x, w)
    L = layers.lib()
    full = L.eden_layers_workspace_bytes(m, n, k, layers.F32)
    for size in (0, 16, full // 2, full):
        y = torch.empty(m, n, device="cuda")
        ws = torch.full((full + 64,), 0x5A, dtype=torch.uint8, device="cuda")
        assert L.eden_linear(x.data_ptr(), k, w.data_ptr(), k, None, None, 0, y.data_ptr(), n, None, 0, m, n, k, layers.F32, 0, ws.data_ptr() if size else None,
                             size, eden._stream_ptr()) == 0
        assert ref.rel(y.cpu(), want.cpu()) <= 2 * ref.norm_bound(k, torch.float32)
        assert bool((ws[size:] == 0x5A).all())
        if size == full:
            assert torch.equal(y, want)


def test_graph_replays_give_the_eager_result(layers):
    g = gen("graph")
    x, w = torch.randn(300, 256, generator=g).bfloat16().cuda(), torch.randn(512, 256, generator=g).bfloat16().cuda()
    dy = torch.randn(300, 512, generator=g).bfloat16().cuda()
    kept, y, dx = layers.save_checkpoint(x), torch.empty(300, 512, dtype=torch.bfloat16, device="cuda"), torch.empty_like(x)
    z, dw, db = layers.save_checkpoint(dy), torch.empty(512, 256, device="cuda"), torch.empty(512, device="cuda")

    def step():
        layers.save_checkpoint(x, into=kept)
        layers.linear(x, w, activation="gelu", checkpoint=z, out=y)
        dz = layers.activation_grad(dy, z, "gelu")
        layers.linear_weight_grad(dz, kept, out=dw, bias_out=db)
        layers.linear_input_grad(dz, w, residual=x, out=dx)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for round in range(4):
        x.copy_(torch.randn(300, 256, generator=g).bfloat16())
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in (y, dx, dw, db, z.buffer, kept.buffer)]
        for t in (y, dx, dw, db):
            t.zero_()
        step()
        torch.cuda.synchronize()
        for a, b in zip(got, (y, dx, dw, db, z.buffer, kept.buffer)):
            assert torch.equal(a, b), round
