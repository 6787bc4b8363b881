"""The layer operators at the ends of their range, in part through the C entry points themselves."""
import zlib

import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from tests import layers_reference as ref                          # noqa: E402

TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}


@pytest.fixture(scope="module")
def layers():
    from paper_2108_08842_amd import layers as m
    assert torch.cuda.is_available()
    m.lib()
    return m


def gen(*key):
    return torch.Generator(device="cuda").manual_seed(zlib.crc32(repr(key).encode()))


def randn(g, *shape, dtype=torch.float32, scale=1.0):
    return (torch.randn(*shape, generator=g, device="cuda") * scale).to(dtype)


def stream():
    from paper_2108_08842_amd import eden
    return eden._stream_ptr()


# ---- sizes of nothing, one row

@pytest.mark.parametrize("accumulate", [0, 1])
@pytest.mark.parametrize("m,n", [(1000, 40), (8192, 64), (512, 1000), (191, 3)])
@pytest.mark.parametrize("dtype", TYPES)
def test_bias_gradient_of_an_input_without_columns_next_to_a_workspace(layers, dtype, m, n, accumulate):
    # a caller with one workspace for all calls: the sum of dy is not split where there is no column to join
    dy = randn(gen(m, n), m, n, dtype=TYPES[dtype])
    db, ws = torch.full((n,), 3.0, device="cuda"), torch.full((1 << 22,), 0x5A, dtype=torch.uint8, device="cuda")
    assert layers.lib().eden_linear_weight_grad(dy.data_ptr(), n, None, None, 0, db.data_ptr(), m, n, 0, layers._DTYPES[TYPES[dtype]], accumulate,
                                                ws.data_ptr(), ws.numel(), stream()) == 0
    want = dy.double().sum(0) + 3.0 * accumulate
    assert bool(((db.double() - want).abs() <= (m + 8) * 2.0 ** -23 * (dy.double().abs().sum(0) + 3.0)).all())


@pytest.mark.parametrize("ld", [0, 8, 16384, 2 ** 40])
def test_gradients_of_one_row_at_any_distance(layers, ld):
    # up to one row the distance says nothing: dy is read once, whatever it is
    n = k = 16384
    g = gen("row")
    dy = randn(g, 1, n, dtype=torch.bfloat16)
    dy[0, 5], dy[0, 9000] = float("inf"), float("nan")
    x = randn(g, 1, k).abs() + 1.0                                 # (no code is 0)
    c = layers.save_checkpoint(x)
    dw, db = torch.empty(n, k, device="cuda"), torch.empty(n, device="cuda")
    assert layers.lib().eden_linear_weight_grad(dy.data_ptr(), ld, c.buffer.data_ptr(), dw.data_ptr(), k, db.data_ptr(), 1, n, k, layers.BF16, 0, None, 0, stream()) == 0
    # a product of 8 and 7 bits is exact in fp32
    assert torch.equal(db.nan_to_num(nan=77.0), dy[0].float().nan_to_num(nan=77.0))
    assert torch.equal(dw.nan_to_num(nan=77.0), (dy.float().t() * c.restore(torch.float32)).nan_to_num(nan=77.0))


def test_input_gradient_of_one_feature_at_any_distance(layers):
    # w of one row at distance 0 next to dz whose rows are copied: nothing but its one row counts
    m = k = 32768
    g = gen("feature")
    dz, w = randn(g, m, 1, dtype=torch.bfloat16).abs() + 1.0, randn(g, 1, k, dtype=torch.bfloat16)
    w[0, 3] = float("inf")
    size = layers.lib().eden_layers_copying_bytes(m, k, 1, layers.BF16)
    dx, ws = torch.empty(m, k, dtype=torch.bfloat16, device="cuda"), torch.empty(size, dtype=torch.uint8, device="cuda")
    assert size and layers.lib().eden_linear_input_grad(dz.data_ptr(), 1, w.data_ptr(), 0, None, 0, None, 0, dx.data_ptr(), k, m, 1, k, layers.BF16, ws.data_ptr(), size,
                                                        stream()) == 0
    assert torch.equal(dx, dz * w)                                 # 16 bits, rounded once


# ---- precision

# a launch of k_tiles (few products) and one of the kernel with loads straight into the LDS
PAIRS = [(40, 72, 3), (2048, 2048, 128)]


@pytest.mark.parametrize("m,n,k", PAIRS)
def test_what_is_left_out_of_fp32_products(layers, m, n, k):
    """One product in each sum, the other operands zero: what is left out is below 2^-22 of it, and the additions of its parts (the largest last: the others
    are below 2^-6 of it) are off by 2^-23 of it at most."""
    g = gen("pairs", m)
    x, w = torch.zeros(m, k, device="cuda"), torch.zeros(n, k, device="cuda")
    worst = torch.tensor([1 + 2.0 ** -7 - 2.0 ** -23, 1 + 2.0 ** -8 - 2.0 ** -17, 1 + 2.0 ** -8, 1 + 2.0 ** -7 - 2.0 ** -16, 2 - 2.0 ** -23, 1.0, 1 + 2.0 ** -23], device="cuda")
    for t, at in ((x, 1), (w, 1)):
        t[:, at] = torch.rand(t.shape[0], generator=g, device="cuda") + 1.0
        t[:7, at] = worst
    want = x[:, 1].double()[:, None] * w[:, 1].double()
    v = w.t().contiguous()
    for y in (layers.linear(x, w), layers.linear_input_grad(x, v)):
        off = (y.double() - want) / want
        assert float(off.abs().max()) <= 1.5 * 2.0 ** -22


@pytest.mark.parametrize("m,n,k", PAIRS)
def test_largest_fp32_operands(layers, m, n, k):
    # numbers that round to an infinity in bf16
    big = torch.finfo(torch.float32).max
    x, w = torch.zeros(m, k, device="cuda"), torch.zeros(n, k, device="cuda")
    x[:, 0], w[:, 0] = big, 2.0 ** -20
    x[1::2, 0] = -big
    want = x[:, 0].double()[:, None] * w[:, 0].double()
    for y in (layers.linear(x, w), layers.linear_input_grad(x, w.t().contiguous()), layers.linear(w, x).t()):
        assert y.shape == want.shape and bool(((y.double() - want).abs() <= 2.0 ** -22 * want.abs()).all())
    x[0, 0] = float("inf")                                         # gives NaN, and in its own row only
    y = layers.linear(x, w)
    assert bool(y[0].isnan().all()) and bool(y[1:].isfinite().all())


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
def test_slope_of_gelu_is_rounded_once_next_to_its_zero_too(layers, dtype):
    """Every code in four units, -0.75 among them, next to which (-0.7518) the two terms of the slope cancel.  In 32 bits the slope is off by less than 2^-17 of
    itself (its polynomial 2^-18.3, exp and a quotient 2^-23 each of the terms); then half a unit of the result's type."""
    bits, least = {"f16": (11, -24), "bf16": (8, -133)}[dtype]
    for unit in (2.0 ** -8, 2.0 ** -7, 2.0 ** -6, 2.0 ** -5):
        z = torch.zeros(8, 256, device="cuda")
        codes = (torch.arange(8 * 31, device="cuda").float() - 127).view(8, 31)
        z[:, 1:32], z[:, 32:39] = codes, torch.arange(121, 128, device="cuda").float()
        z[:, ::32] = 127.0                                         # every block's largest value
        z *= unit
        c = layers.save_checkpoint(z)
        assert torch.equal(c.restore(torch.float32), z)
        got = layers.activation_grad(torch.ones(8, 256, dtype=TYPES[dtype], device="cuda"), c, "gelu").double().cpu()
        want = ref.slope(z.double().cpu(), "gelu")
        half = torch.exp2((torch.frexp(want)[1] - bits).clamp(min=least).double() - 1)
        assert bool(((got - want).abs() <= half * 1.001 + 2.0 ** -17 * want.abs()).all()), float(((got - want).abs() - half).max())


@pytest.mark.parametrize("m", [3, 40])
@pytest.mark.parametrize("dtype", ["f16", "bf16"])
def test_gelu_under_a_residual_that_nearly_cancels_it(layers, dtype, m):
    """In 32 bits gelu is off by 2^-20 + 2^-23 |z| of itself (exp of z^2 / 2, its argument rounded twice; polynomial, quotient and products 2^-21); then one
    rounding of the sum.  z is an operand itself: one product by 1."""
    t, bits, least = TYPES[dtype], {"f16": 11, "bf16": 8}[dtype], {"f16": -24, "bf16": -133}[dtype]
    z = (torch.arange(m * 40, device="cuda").double() / (m * 40) * 8 - 4).to(t).view(m, 40)
    act = ref.act(z.double(), "gelu")
    residual = (-act).to(t)
    got = layers.linear(z, torch.eye(40, dtype=t, device="cuda"), activation="gelu", residual=residual).double()
    want = act + residual.double()
    half = torch.exp2((torch.frexp(want)[1] - bits).clamp(min=least).double() - 1)
    assert bool(((got - want).abs() <= (2.0 ** -20 + 2.0 ** -23 * z.double().abs()) * act.abs() + 1.001 * half).all())


# ---- more threads than a launch can have (2^32)

def test_few_rows_next_to_more_columns_than_a_launch_has_threads_for(layers):
    # whole numbers: exact.  fp32, one row: 64 threads a column; bf16, eight rows of odd length: 32
    for m, n, k, t in ((1, 2 ** 26 + 44, 8, torch.float32), (8, 2 ** 27 + 20, 7, torch.bfloat16)):
        g = gen("wide", m)
        x, w = torch.randint(-3, 4, (m, k), generator=g, device="cuda").to(t), torch.randint(-3, 4, (4099, k), generator=g, device="cuda").to(t)
        want, w = (x.float() @ w.float().t()).to(t), w.repeat(n // 4099 + 1, 1)[:n]
        y = layers.linear(x, w)
        whole = n // 4099 * 4099
        assert torch.equal(y[:, :whole].reshape(m, -1, 4099), want[:, None].expand(m, whole // 4099, 4099)) and torch.equal(y[:, whole:], want[:, :n - whole])
        del w, y


def test_more_rows_than_a_launch_has_threads_for(layers):
    # 2^30 rows of one column take four threads each; every value fills its block's seven bits or less
    rows = 2 ** 30
    x = (torch.arange(2 ** 20 + 3, device="cuda") % 251 - 125).half().repeat(1024)[:rows].view(rows, 1)
    c = layers.save_checkpoint(x)
    assert torch.equal(c.restore(torch.float16), x)
    codes, exps = ref.encode(x[-100:].float().cpu().numpy())
    assert np.array_equal(c.buffer[(rows - 100) * 32:rows * 32].cpu().numpy().view(np.int8).reshape(100, 32), codes)
    assert np.array_equal(c.buffer[rows * 33 - 100:].cpu().numpy().reshape(100, 1), exps)
    assert torch.equal(layers.activation_grad(x, c, "relu"), x.clamp(min=0.0))


# ---- operands that require a gradient

def test_operands_that_require_a_gradient_are_refused_where_it_would_be_lost(layers):
    from paper_2108_08842_amd.eden import EdenError
    g = gen("autograd")
    x, w, b, r, dy, dw = randn(g, 6, 40), randn(g, 24, 40), randn(g, 24), randn(g, 6, 24), randn(g, 6, 24), torch.zeros(24, 40, device="cuda")
    kept, z = layers.save_checkpoint(x), layers.save_checkpoint(dy)

    def calls(x, w, b, r, dy, dw):
        return [lambda: layers.linear(x, w, b, residual=r), lambda: layers.save_checkpoint(x).restore(torch.float32), lambda: layers.linear_weight_grad(dy, kept),
                lambda: layers.linear_input_grad(dy, w), lambda: layers.linear_input_grad(r, w, residual=x), lambda: layers.activation_grad(dy, z, "gelu"),
                lambda: layers.linear_weight_grad(r, kept, out=dw), lambda: layers.linear(x, w, stream=torch.cuda.current_stream())]

    plain = {"x": x, "w": w, "b": b, "r": r, "dy": dy, "dw": dw}
    want = [f().clone() for f in calls(**plain)]
    for which, refused in (("x", {0, 4, 7}), ("w", {0, 3, 4, 7}), ("b", {0}), ("r", {0, 4, 6}), ("dy", {2, 3, 5}), ("dw", {6})):
        for number, f in enumerate(calls(**{**plain, which: plain[which].clone().requires_grad_(True)})):
            if number in refused:
                with pytest.raises(EdenError):
                    f()
            else:
                assert torch.equal(f(), want[number])
            with torch.no_grad():                                  # nobody expects one
                assert torch.equal(f(), want[number])


# ---- subnormal and non-finite operands, in every kernel that has a product

# rows, features out, features in: few rows (dots; matrix cores), tiles, a split sum, tiles with loads straight into the LDS, the same with copies
# (from 2^30 products on)
PLACES = [(1, 40, 24), (3, 70, 520), (9, 40, 264), (14, 40, 24), (40, 72, 33), (40, 72, 3000), (40, 72, 3008), (2048, 2048, 136), (1500, 1501, 499)]


@pytest.mark.parametrize("m,n,k", PLACES)
@pytest.mark.parametrize("dtype", TYPES)
def test_subnormal_operands(layers, dtype, m, n, k):
    """Whole numbers of the smallest unit next to powers of two that bring the products back into the range: every sum is exact."""
    t = TYPES[dtype]
    unit, up = {"f32": (2.0 ** -133, 2.0 ** 110), "f16": (2.0 ** -24, 2.0 ** 10), "bf16": (2.0 ** -133, 2.0 ** 110)}[dtype]
    small = torch.zeros(m, k, dtype=torch.float64, device="cuda")
    small[:, ::7] = ((torch.arange(m, device="cuda")[:, None] + torch.arange(0, k, 7, device="cuda")) % 3).double() - 1.0      # -1, 0, 1
    small[:, k - 1] = torch.arange(m, device="cuda") % 100 + 5
    small, big = (small * unit).to(t), torch.full((n, k), up, dtype=torch.float64, device="cuda").to(t)
    want = (small.double() @ big.double().t().contiguous()).to(t)
    assert bool((want != 0).any())
    assert torch.equal(layers.linear(small, big), want)
    assert torch.equal(layers.linear_input_grad(small, big.t().contiguous()), want)
    flipped = layers.linear(big, small)                            # the weights are the small ones
    assert torch.equal(flipped, want.t())
    # the weight gradient's dy, and its sums
    c = layers.save_checkpoint(torch.full((k, m), up, dtype=torch.float32, device="cuda"))
    dy = torch.zeros(k, n, dtype=torch.float64, device="cuda")
    dy[:] = (torch.arange(k, device="cuda")[:, None] + torch.arange(n, device="cuda")) % 3 * unit
    dy = dy.to(t)
    dw, db = layers.linear_weight_grad(dy, c, bias=True)
    sums = dy.double().sum(0)
    assert torch.equal(dw.double(), (sums[:, None] * up).expand(n, m)) and torch.equal(db.double(), sums)


@pytest.mark.parametrize("m,n,k", PLACES)
def test_fp32_operands_whose_terms_are_subnormal(layers, m, n, k):
    # what an operand holds below 2^-133 may be left out: at 2^-120 some 2^-13 of it
    g = gen("tiny", m, k)
    x, w = randn(g, m, k, scale=2.0 ** -120), randn(g, n, k, scale=2.0 ** 100)
    X, W = x.double(), w.double()
    for y in (layers.linear(x, w), layers.linear_input_grad(x, w.t().contiguous()), layers.linear(w, x).t()):
        near = ref.product_bound(X, W, k) + 2.0 ** -133 * W.abs().sum(1)
        assert bool(((y.double() - X @ W.t().contiguous()).abs() <= near).all())
    c = layers.save_checkpoint(randn(g, m, k, scale=2.0 ** 100))
    dy, held = randn(g, m, n, scale=2.0 ** -120), c.restore(torch.float32).double()
    dw, db = layers.linear_weight_grad(dy, c, bias=True)
    Y = dy.double()
    near = ref.product_bound(Y.t().contiguous(), held.t().contiguous(), m) + 2.0 ** -133 * held.abs().sum(0)
    assert bool(((dw.double() - Y.t().contiguous() @ held).abs() <= near).all())
    assert bool(((db.double() - Y.sum(0)).abs() <= (m + 8) * 2.0 ** -23 * Y.abs().sum(0) + m * 2.0 ** -133).all())


@pytest.mark.parametrize("m,n,k", PLACES)
@pytest.mark.parametrize("dtype", TYPES)
def test_infinities_and_nan_reach_their_own_rows_and_columns(layers, dtype, m, n, k):
    t = TYPES[dtype]
    x, w = torch.ones(m, k, dtype=t, device="cuda"), torch.ones(n, k, dtype=t, device="cuda")
    r, c = m // 2, n - 1
    x[r, k - 1], w[c, k // 2], w[3, 0] = float("inf"), float("nan"), -float("inf")
    want = x.double() @ w.double().t().contiguous()
    finite = torch.ones(m, n, dtype=torch.bool, device="cuda")
    finite[r], finite[:, c], finite[:, 3] = False, False, False
    y, z = layers.linear(x, w, checkpoint=True)
    values = z.restore(torch.float32)
    dx = layers.linear_input_grad(x, w.t().contiguous())
    for got in (y, dx):
        assert torch.equal(got.isfinite(), finite) and torch.equal(got[finite], want[finite].to(t))
        if t != torch.float32 or (m <= 16 and got is y):           # (products of fp32 terms: an infinity gives NaN)
            assert torch.equal(got.nan_to_num(nan=7.0), want.to(t).nan_to_num(nan=7.0))
    blocks = torch.nn.functional.pad(~finite, (0, -n % 32)).view(m, -1, 32).any(2).repeat_interleave(32, 1)[:, :n]
    assert torch.equal(values.isnan(), blocks)
    dy = torch.ones(m, n, dtype=t, device="cuda")
    dy[r, 0], dy[0, n - 1] = float("inf"), float("nan")
    dw, db = layers.linear_weight_grad(dy, layers.save_checkpoint(torch.ones(m, k, device="cuda")), bias=True)
    assert bool((dw[0] == float("inf")).all()) and bool(dw[n - 1].isnan().all()) and bool((dw[1:n - 1] == m).all())
    assert float(db[0]) == float("inf") and bool(db[n - 1].isnan()) and bool((db[1:n - 1] == m).all())
    kept = torch.ones(m, k, device="cuda")
    kept[r, k - 1] = float("nan")
    dw = layers.linear_weight_grad(torch.ones(m, n, dtype=t, device="cuda"), layers.save_checkpoint(kept))
    bad = torch.zeros(k, dtype=torch.bool, device="cuda")
    bad[(k - 1) // 32 * 32:] = True
    assert bool(dw[:, bad].isnan().all()) and bool((dw[:, ~bad] == m).all())


# ---- the general kernel's tiles of 128 x 128: from 256 of them on

@pytest.mark.parametrize("n,k,m,pad", [(2056, 2051, 333, 0), (2050, 2056, 64, 3), (2177, 1930, 33, 1)])
@pytest.mark.parametrize("dtype", ["f32", "f16"])
def test_weight_grad_in_large_tiles(layers, dtype, n, k, m, pad):
    g = gen("tiles", n, m)
    dy = torch.full((m, n + pad), float("nan"), dtype=TYPES[dtype], device="cuda")[:, :n]
    dy.copy_(randn(g, m, n))
    c = layers.save_checkpoint(randn(g, m, k, scale=10.0))
    X, Y = c.restore(torch.float32).double(), dy.double()
    flat = torch.full((1 + n * k + 2 + n,), 4.0, device="cuda")
    out, bias_out = flat[1:1 + n * k].view(n, k), flat[1 + n * k + 2:]
    layers.linear_weight_grad(dy, c, out=out, bias_out=bias_out)
    want, want_b = Y.t().contiguous() @ X, Y.sum(0)
    assert bool(((out.double() - want).abs() <= ref.product_bound(Y.t().contiguous(), X.t().contiguous(), m) + 2.0 ** -24 * want.abs()).all())
    assert ref.rel(out, want) <= ref.norm_bound(m, torch.float32)
    assert bool(((bias_out.double() - want_b).abs() <= (m + 8) * 2.0 ** -23 * Y.abs().sum(0)).all())
    first, first_b = out.clone(), bias_out.clone()
    layers.linear_weight_grad(dy, c, out=out, bias_out=bias_out, accumulate=True)
    assert torch.equal(out, first + first) and torch.equal(bias_out, first_b + first_b)
    assert bool((flat[:1] == 4.0).all()) and bool((flat[1 + n * k:3 + n * k] == 4.0).all())


@pytest.mark.parametrize("m,n,k,pad", [(2100, 2051, 100, 0), (2051, 2100, 333, 3), (2305, 1801, 31, 1)])
@pytest.mark.parametrize("dtype", TYPES)
def test_products_in_large_tiles_without_a_workspace(layers, dtype, m, n, k, pad):
    # rows that begin anywhere and no room for copies of them
    t, g = TYPES[dtype], gen("anywhere", m)

    def apart(rows, cols, scale=1.0):
        return torch.full((rows, cols + pad), float("nan"), dtype=t, device="cuda")[:, :cols].copy_(randn(g, rows, cols, scale=scale))

    x, w, r, L, code = apart(m, k), apart(n, k, k ** -0.5), apart(m, n), layers.lib(), layers._DTYPES[t]
    y, z = torch.full((m, n + pad), 5.0, dtype=t, device="cuda"), layers.Checkpoint(torch.empty(layers.checkpoint_bytes(m, n), dtype=torch.uint8, device="cuda"), m, n)
    assert L.eden_linear(x.data_ptr(), k + pad, w.data_ptr(), k + pad, None, r.data_ptr(), n + pad, y.data_ptr(), n + pad, z.buffer.data_ptr(), z.buffer.numel(), m, n, k, code, 0,
                         None, 0, stream()) == 0
    product = x.double() @ w.double().t().contiguous()
    want, dz = product + r.double(), ref.product_bound(x.double(), w.double(), k)
    assert bool(((y[:, :n].double() - want).abs() <= dz + (4 * ref.EPS + ref.ROUND[t]) * want.abs() + ref.TINY[t]).all()) and bool((y[:, n:] == 5.0).all())
    codes, exps = ref.unpack(z.buffer, m, n)
    unit = torch.from_numpy(np.repeat(np.exp2(exps.astype(np.float64) - 127), 32, axis=1)[:, :n])
    held = torch.from_numpy(ref.decode(codes, exps, n))
    assert bool(((held - product.cpu()).abs() <= unit * torch.where(held.abs() == 127 * unit, 1.0, 0.5) + dz.cpu()).all()) and not codes[:, n:].any()
    # dx of that size: dz is m x k, w k x n
    v, dx = apart(k, n, k ** -0.5), torch.full((m, n + pad), 5.0, dtype=t, device="cuda")
    assert L.eden_linear_input_grad(x.data_ptr(), k + pad, v.data_ptr(), n + pad, z.buffer.data_ptr(), 4, None, 0, dx.data_ptr(), n + pad, m, k, n, code, None, 0, stream()) == 0
    product = x.double() @ v.double()
    want = product * ref.slope(held, "silu").cuda()
    near = 1.13 * ref.product_bound(x.double(), v.double().t().contiguous(), k) + 2.0 ** -19 * product.abs() + (4 * ref.EPS + ref.ROUND[t]) * want.abs() + ref.TINY[t]
    assert bool(((dx[:, :n].double() - want).abs() <= near).all()) and bool((dx[:, n:] == 5.0).all())


# ---- the same bits every time

def test_checkpoints_ends_and_joined_sums_give_the_same_bits_every_time(layers):
    g = gen("again")
    bf = torch.bfloat16
    x, w, b, r = randn(g, 2304, 1024, dtype=bf), randn(g, 4096, 1024, dtype=bf, scale=2.0 ** -5), randn(g, 4096, dtype=bf), randn(g, 2304, 4096, dtype=bf)
    x32, w32 = randn(g, 40, 3000), randn(g, 72, 3000)

    def calls():
        y, z = layers.linear(x, w, b, activation="gelu", residual=r, checkpoint=True)
        s, q = layers.linear(x32, w32, activation="silu", checkpoint=True)
        dx = layers.linear_input_grad(y, w, activation="gelu", checkpoint=layers.save_checkpoint(x))
        return y, z.buffer, s, q.buffer, dx, *layers.linear_weight_grad(r, z, bias=True)

    first = calls()
    for _ in range(10):
        for got, want in zip(calls(), first):
            assert torch.equal(got, want)
