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
