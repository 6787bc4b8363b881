"""4-bit operands and their products on the GPU against 64 bits, at the sizes, types, distances and values where they can go wrong."""
import math
import zlib

import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from tests import layers_reference as lref, mx4_reference as ref   # noqa: E402

TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
ACTS = ["none", "relu", "gelu", "gelu_tanh", "silu"]
# rows, features out, features in: single ones, a block, chunk or tile more or less, sums that are split over workgroups, tiles of 256
SIZES = [(1, 1, 1), (1, 40, 7), (2, 31, 64), (2, 300, 17000), (3, 1000, 96), (5, 130, 2056), (16, 33, 333), (17, 128, 128), (127, 129, 31), (128, 128, 256), (129, 257, 191), (130, 64, 1024),
         (300, 72, 1500), (700, 40, 33), (1025, 24, 65), (64, 64, 9000)]


@pytest.fixture(scope="module")
def mx4():
    from paper_2108_08842_amd import mx4 as m
    assert torch.cuda.is_available()
    m.lib()
    return m


def gen(*key):
    return torch.Generator().manual_seed(zlib.crc32(repr(key).encode()))


def matrix(g, rows, cols, dtype, pad=0, scale=1.0):
    """A matrix on the GPU whose rows are `pad` elements further apart than they are long, surrounded by NaN."""
    x = torch.full((rows, cols + pad), float("nan"), dtype=dtype)
    x[:, :cols] = (torch.randn(rows, cols, generator=g, dtype=torch.float64) * scale).to(dtype)
    return x.cuda()[:, :cols]


def packed(mx4, x):
    """Mx4 made by the reference from a CPU matrix, and its values in 64 bits."""
    codes, exps = ref.encode(x.float().numpy())
    return mx4.Mx4(ref.pack(codes, exps).cuda(), *x.shape), torch.from_numpy(ref.decode(codes, exps, x.shape[1]))


def randn(g, *shape, scale=1.0):
    return torch.randn(*shape, generator=g, dtype=torch.float64).mul_(scale).float()


def same(got, x, bits=None):
    """Buffer against the reference's codes and exponents of x, the fill included."""
    codes, exps = ref.encode(x.float().cpu().numpy(), bits)
    got_codes, got_exps = ref.unpack(got.buffer, *x.shape)
    width = codes.shape[1]
    # (where x is an odd zero or rounds to zero, the sign is x's)
    assert np.array_equal(got_exps[:, :width // 32], exps) and not got_exps[:, width // 32:].any()
    assert np.array_equal(got_codes[:, :width], codes) and not got_codes[:, width:].any()


# ---- rounding

def special_rows():
    rows = [np.zeros(70), np.full(70, -0.0), np.arange(70) - 35.0, np.linspace(-1, 1, 70), np.full(70, 1e-45), np.full(70, 2.0 ** -126), np.full(70, 2.0 ** -127), np.full(70, 3.4028234e38),
            np.geomspace(1e-38, 1e38, 70), np.geomspace(1e-45, 1e-36, 70), np.linspace(0, 6, 70), -np.linspace(0, 6, 70), np.linspace(0, 12, 70) * 2.0 ** -127, np.linspace(0, 6, 70) * 2.0 ** 120]
    for top in (6.0, np.nextafter(np.float32(6), np.float32(7)), np.nextafter(np.float32(6), np.float32(5)), 4.0, 8.0):
        r = np.tile([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 0.2499999, 0.2500001, 4.9999995, 5.0000005, 2.0, 1e-30, 0.0], 5)      # the middle between codes, and next to it
        r[[0, 40, 69]] = top
        rows += [r, -r, r * 2.0 ** -100]
    for bad in (np.inf, -np.inf, np.nan):
        for at in (0, 31, 32, 69):
            r = np.linspace(-2, 2, 70)
            r[at] = bad
            rows.append(r)
    return torch.from_numpy(np.stack(rows).astype(np.float32))


@pytest.mark.parametrize("transpose", [False, True])
@pytest.mark.parametrize("dtype", TYPES)
def test_special_values_are_bit_exact(mx4, dtype, transpose):
    x = special_rows().to(TYPES[dtype])
    given = x.t().contiguous().cuda() if transpose else x.cuda()
    got = mx4.quantize(given, transpose=transpose)
    same(got, x)
    same(mx4.quantize(given, transpose=transpose, rounding=mx4.Stochastic(5, 6)), x, ref.draws(5, 6, *x.shape))
    want = ref.values(x)
    for out in TYPES.values():
        back = got.restore(out).cpu()
        assert torch.equal(back.isnan(), want.isnan())
        rounded = torch.nan_to_num(want, nan=0.0, posinf=math.inf, neginf=-math.inf)
        assert torch.equal(torch.nan_to_num(back, nan=0.0, posinf=math.inf, neginf=-math.inf), rounded.float().to(out))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,cols,pad", [(1, 1, 0), (1, 31, 0), (3, 32, 1), (2, 33, 3), (65, 1000, 0), (7, 4097, 5), (1000, 40, 8), (513, 256, 0), (257, 129, 1), (300, 300, 0)])
def test_rounding_is_bit_exact(mx4, dtype, rows, cols, pad):
    x = matrix(gen(dtype, rows, cols), rows, cols, TYPES[dtype], pad, 3.0)
    for transpose in (False, True):
        like = x.t().contiguous() if transpose else x
        r, c = like.shape
        for rounding, bits in ((None, None), (mx4.Stochastic(77, 5), ref.draws(77, 5, r, c))):
            into = mx4.Mx4(torch.full((mx4.mx4_bytes(r, c) + 64,), 0xA5, dtype=torch.uint8, device="cuda"), r, c)
            assert mx4.quantize(x, transpose=transpose, rounding=rounding, into=into) is into
            same(into, like, bits)
            assert bool((into.buffer[mx4.mx4_bytes(r, c):] == 0xA5).all())
            out = torch.full((r, c + pad), 7.0, dtype=torch.float32, device="cuda")
            into.restore(out=out[:, :c])
            assert np.array_equal(out[:, :c].cpu().double().numpy(), ref.values(like, bits).numpy()) and bool((out[:, c:] == 7.0).all())


@pytest.mark.parametrize("rows,cols", [(65539, 40), (32779, 300), (16391, 777)])
def test_rounding_of_many_rows_is_bit_exact(mx4, rows, cols):                    # threads that have several rows, the last ones behind the matrix
    x = matrix(gen("many", rows, cols), rows, cols, torch.bfloat16, 8)
    same(mx4.quantize(x), x)
    into = mx4.Mx4(torch.full((mx4.mx4_bytes(rows, cols) + 64,), 0xA5, dtype=torch.uint8, device="cuda"), rows, cols)
    same(mx4.quantize(x, rounding=mx4.Stochastic(8, 1), into=into), x, ref.draws(8, 1, rows, cols))
    assert bool((into.buffer[mx4.mx4_bytes(rows, cols):] == 0xA5).all())


@pytest.mark.parametrize("transpose", [False, True])
def test_stochastic_rounding_keeps_the_expectation(mx4, transpose):
    x = torch.linspace(-6.0, 6.0, 256, device="cuda").repeat(4096, 1)            # 4096 draws of each value, in blocks whose unit is at most 1
    if transpose:
        x = x[:, :4].t().repeat(64, 1).t().contiguous()
        values = mx4.quantize(x, transpose=True, rounding=mx4.Stochastic(3)).restore(torch.float32).t()
    else:
        values = mx4.quantize(x, rounding=mx4.Stochastic(3)).restore(torch.float32)
    off = (values.double().mean(0) - x.double().mean(0)).abs()
    # a step is at most 2, a draw's deviation at most 1; six deviations of the mean of 4096, and 2^-17 of a step
    assert float(off.max()) <= 6 / math.sqrt(4096) + 2.0 ** -16
    held = torch.tensor([0.0, 0.5, -1.0, 1.5, 2.0, -3.0, 4.0, 6.0], device="cuda").repeat(100, 4)
    assert torch.equal(mx4.quantize(held, rounding=mx4.Stochastic(4)).restore(torch.float32), held)
    seed = torch.tensor(41, device="cuda")
    y = torch.randn(100, 100, device="cuda")
    assert torch.equal(mx4.quantize(y, rounding=mx4.Stochastic(seed, 2)).buffer, mx4.quantize(y, rounding=mx4.Stochastic(41, 2)).buffer)
    assert not torch.equal(mx4.quantize(y, rounding=mx4.Stochastic(41, 3)).buffer, mx4.quantize(y, rounding=mx4.Stochastic(41, 2)).buffer)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,cols", [(1, 5), (31, 127), (256, 128), (257, 130), (3000, 40), (5000, 300)])
def test_sums_of_columns(mx4, dtype, rows, cols):
    x = matrix(gen("sums", dtype, rows, cols), rows, cols, TYPES[dtype], 3)
    want, size = x.double().sum(0), x.double().abs().sum(0)
    bound = (rows + 8) * 2.0 ** -24 * size
    got, sums = mx4.quantize(x, transpose=True, sums=True)
    assert bool(((sums.double() - want).abs() <= bound).all())
    flat = torch.full((cols + 8,), 3.0, device="cuda")
    again, into = mx4.quantize(x, transpose=True, sums=flat[4:4 + cols], accumulate=True)
    assert bool(((into.double() - 3.0 - want).abs() <= bound + 2.0 ** -24 * (3.0 + size)).all()) and bool((flat[:4] == 3.0).all()) and bool((flat[4 + cols:] == 3.0).all())
    assert torch.equal(again.restore(), got.restore())
    # the C entry without a workspace: the same sums in another order
    alone = torch.full((cols,), 9.0, device="cuda")
    from paper_2108_08842_amd import layers
    assert mx4.lib().eden_mx4_quantize(x.data_ptr(), cols + 3, rows, cols, layers._DTYPES[x.dtype], 1, None, got.buffer.data_ptr(), got.buffer.numel(), alone.data_ptr(), 0, None, 0,
                                       layers._stream(x.device)) == 0
    assert bool(((alone.double() - want).abs() <= bound).all())


# ---- products

def near(got, want, dz, act, t):
    """Elementwise: dz bounds what z is off by; slopes are below 1.13; an activation is off by 16 fp32 roundings (two-byte results: exp and the quotient of z in one
    instruction each)."""
    y, z = want
    got = got.cpu().double()
    limit = 1.13 * dz + (2.0 ** -20 + 2.0 ** -23 * z.abs()) * lref.act(z, act).abs() + 2.0 ** -22 * (z.abs() + y.abs()) + lref.ROUND[t] * y.abs() + lref.TINY[t]
    assert bool(((got - y).abs() <= limit).all()), (act, ((got - y).abs() / limit).max())


# (17 to 64 rows: by few rows where the result is narrow and the sum short, by tiles next to that)
@pytest.mark.parametrize("m,n,k", SIZES + [(300, 6000, 200), (2300, 3200, 300), (4, 4097, 520), (18, 4096, 40), (31, 5000, 257), (32, 33, 8192), (32, 65, 8193), (33, 131, 2056), (47, 8192, 65), (48, 8193, 65), (64, 70, 4096), (65, 70, 300)])
@pytest.mark.parametrize("dtype", TYPES)
def test_linear(mx4, dtype, m, n, k):
    t, g = TYPES[dtype], gen("linear", dtype, m, n, k)
    w, W = packed(mx4, randn(g, n, k, scale=k ** -0.5))
    for number, (act, with_bias, with_residual, keep, pad) in enumerate([("none", False, False, False, 0), ("gelu", True, False, True, 0), ("silu", True, True, True, 3),
                                                                         ("relu", False, True, False, 8), ("gelu_tanh", True, True, True, 1)]):
        if m * n > 10 ** 6 and number not in (0, 2):
            continue
        x = matrix(g, m, k, t, pad)
        bias = matrix(g, 1, n, t)[0] if with_bias else None
        residual = matrix(g, m, n, t, pad) if with_residual else None
        out = torch.full((m, n + pad), 5.0, dtype=t, device="cuda")
        got = mx4.linear(x, w, bias, activation=act, residual=residual, checkpoint=keep, out=out[:, :n])
        y, z8 = got if keep else (got, None)
        X = ref.values(x)
        z = X @ W.t() + (bias.cpu().double() if with_bias else 0.0)
        want = lref.act(z, act) + (residual.cpu().double() if with_residual else 0.0)
        dz = lref.product_bound(X, W, k) + 4 * lref.EPS * z.abs()
        near(y, (want, z), dz, act, t)
        assert bool((out[:, n:] == 5.0).all())
        if m * n >= 64:
            assert lref.rel(y.cpu(), want) <= 1.5 * ref.norm_bound(k, t) + 2.0 ** -20, act
        if keep:
            codes, exps = lref.unpack(z8.buffer, m, n)
            unit = torch.from_numpy(np.repeat(np.exp2(exps.astype(np.float64) - 127), 32, axis=1)[:, :n])
            kept = torch.from_numpy(lref.decode(codes, exps, n))
            assert bool(((kept - z).abs() <= unit * torch.where(kept.abs() == 127 * unit, 1.0, 0.5) + dz).all())
            assert not codes[:, n:].any()
        # the operand rounded before gives the same bits
        early = mx4.linear(mx4.quantize(x), w, bias, activation=act, residual=residual, checkpoint=keep, dtype=t)
        assert torch.equal(early[0] if keep else early, y) and (not keep or torch.equal(early[1].buffer, z8.buffer))


@pytest.mark.parametrize("m,n,k", SIZES + [(2300, 300, 3200)])
@pytest.mark.parametrize("dtype", TYPES)
def test_linear_input_grad(mx4, dtype, m, n, k):
    t, g = TYPES[dtype], gen("igrad", dtype, m, n, k)
    wt, WT = packed(mx4, randn(g, k, n, scale=k ** -0.5))
    dz4, DZ = packed(mx4, randn(g, m, n, scale=0.1))
    for number, act in enumerate(ACTS):
        if m * k > 10 ** 6 and number not in (0, 2):
            continue
        codes, exps = lref.encode(randn(g, m, k).numpy())
        from paper_2108_08842_amd import layers
        kept = layers.Checkpoint(lref.pack(codes, exps).cuda(), m, k) if act != "none" else None
        z = torch.from_numpy(lref.decode(codes, exps, k))
        residual = matrix(g, m, k, t, 3) if number % 2 else None
        out = torch.full((m, k + 2), 5.0, dtype=t, device="cuda")
        got = mx4.linear_input_grad(dz4, wt, activation=act, checkpoint=kept, residual=residual, out=out[:, :k])
        s = lref.slope(z, act)
        want = (DZ @ WT.t()) * s + (residual.cpu().double() if residual is not None else 0.0)
        # a slope is off by 2^-20 and a few roundings that grow with |z| (two-byte results)
        limit = lref.product_bound(DZ, WT, n) * (s.abs() + 2.0 ** -19) + (DZ @ WT.t()).abs() * (2.0 ** -19 + 2.0 ** -22 * z.abs()) + 2.0 ** -22 * want.abs() + lref.ROUND[t] * want.abs() + lref.TINY[t]
        assert bool(((got.cpu().double() - want).abs() <= limit).all()), act
        assert bool((out[:, k:] == 5.0).all())
        if residual is not None:
            assert torch.equal(mx4.linear_input_grad(dz4, wt, activation=act, checkpoint=kept, residual=residual), got)


@pytest.mark.parametrize("m,n,k", SIZES + [(200, 3000, 2400)])
def test_linear_weight_grad(mx4, m, n, k):
    g = gen("wgrad", m, n, k)
    dyt, DYT = packed(mx4, randn(g, n, m, scale=0.1))
    xt, XT = packed(mx4, randn(g, k, m))
    want, bound = DYT @ XT.t(), lref.product_bound(DYT, XT, m) + 2.0 ** -40
    out = torch.full((n, k + 3), 5.0, device="cuda")
    dw = mx4.linear_weight_grad(dyt, xt, out=out[:, :k])
    assert bool(((dw.cpu().double() - want).abs() <= bound).all()) and bool((out[:, k:] == 5.0).all())
    dw = mx4.linear_weight_grad(dyt, xt, out=out[:, :k], accumulate=True)
    assert bool(((dw.cpu().double() - 2 * want).abs() <= 2 * bound + 2.0 ** -22 * want.abs()).all()) and bool((out[:, k:] == 5.0).all())
    assert torch.equal(mx4.linear_weight_grad(dyt, xt), mx4.linear_weight_grad(dyt, xt))
    # without a workspace nothing is split
    alone = torch.empty(n, k, device="cuda")
    from paper_2108_08842_amd import layers
    assert mx4.lib().eden_mx4_weight_grad(dyt.buffer.data_ptr(), xt.buffer.data_ptr(), alone.data_ptr(), k, m, n, k, 0, None, 0, layers._stream(alone.device)) == 0
    assert bool(((alone.cpu().double() - want).abs() <= bound).all())


def test_blocks_that_are_not_finite_reach_only_their_results(mx4):
    for m in (1, 8, 40, 300):
        g = gen("nan", m)
        x, w = randn(g, m, 700), randn(g, 500, 700)
        x[0, 3], w[7, 600] = math.inf, math.nan
        y = mx4.linear(x.cuda(), mx4.quantize(w.cuda())).cpu()
        bad = y.isnan()
        assert bool(bad[0].all()) and bool(bad[:, 7].all()) and int(bad.sum()) == 500 + m - 1
        x[0, 3], w[7, 600] = 0.5, 0.5
        clean = mx4.linear(x.cuda(), mx4.quantize(w.cuda())).cpu()
        assert torch.equal(clean[1:, :7], y[1:, :7]) and torch.equal(clean[1:, 8:], y[1:, 8:])


def test_the_ends_of_the_exponents(mx4):
    """Operands of very large and very small blocks: products whose powers of two nearly cancel."""
    for m in (2, 40):
        g = gen("ends", m)
        x, w = randn(g, m, 300, scale=2.0 ** -118), randn(g, 70, 300, scale=2.0 ** 118)
        x[1], w[3] = 0.0, 0.0
        x[0] *= 2.0 ** -12                                         # subnormal numbers among them
        X, W = ref.values(x), ref.values(w)
        got = mx4.linear(x.cuda(), mx4.quantize(w.cuda())).cpu().double()
        assert bool(((got - X @ W.t()).abs() <= lref.product_bound(X, W, 300)).all())


@pytest.mark.parametrize("dtype", TYPES)
def test_nothing_to_do_and_sums_of_nothing(mx4, dtype):
    t = TYPES[dtype]
    for m in (3, 40):
        x, w = torch.empty(m, 0, dtype=t, device="cuda"), mx4.quantize(torch.empty(50, 0, dtype=t, device="cuda"))
        bias, residual = torch.randn(50, device="cuda").to(t), torch.randn(m, 50, device="cuda").to(t)
        got = mx4.linear(x, w, bias, activation="relu", residual=residual)
        assert torch.equal(got, (torch.relu(bias.float()) + residual.float()).to(t))
    assert mx4.linear(torch.empty(0, 64, dtype=t, device="cuda"), mx4.quantize(torch.ones(8, 64, dtype=t, device="cuda"))).shape == (0, 8)
    assert mx4.linear(torch.ones(2, 3, 64, dtype=t, device="cuda"), mx4.quantize(torch.ones(8, 64, dtype=t, device="cuda"))).shape == (2, 3, 8)
    empty, sums = mx4.quantize(torch.empty(0, 7, dtype=t, device="cuda"), transpose=True, sums=True)
    assert bool((sums == 0).all()) and (empty.rows, empty.cols) == (7, 0)
    held = torch.full((7,), 2.0, device="cuda")
    mx4.quantize(torch.empty(0, 7, dtype=t, device="cuda"), transpose=True, sums=held, accumulate=True)
    assert bool((held == 2.0).all())
    assert bool((mx4.linear_weight_grad(empty, mx4.quantize(torch.empty(0, 5, device="cuda"), transpose=True)) == 0).all())
    assert empty.restore().shape == (7, 0)


def test_operands_beyond_four_gigabytes(mx4):
    """Codes and results behind 2^32 bytes: the last rows against the reference."""
    n, k = 2 ** 19 + 2 ** 14 + 5, 16384                            # 4.4 GB of codes
    g = torch.Generator(device="cuda").manual_seed(1)
    buffer = torch.zeros(mx4.mx4_bytes(n, k), dtype=torch.uint8, device="cuda")
    last, chunks = 40, k // 256
    rows = torch.randn(last, k, generator=g, device="cuda")
    small = mx4.quantize(rows)
    codes = n * chunks * 128
    buffer[codes - last * chunks * 128:codes] = small.buffer[:last * chunks * 128]
    exps = buffer[codes:].view(chunks, n + n % 2, 8)
    exps[:, n - last:n] = small.buffer[last * chunks * 128:].view(chunks, last, 8)
    w = mx4.Mx4(buffer, n, k)
    for m in (1, 20):
        x = torch.randn(m, k, generator=g, device="cuda")
        y = mx4.linear(x, w)
        assert torch.equal(y[:, n - last:], mx4.linear(x, small)) or float((y[:, n - last:] - mx4.linear(x, small)).abs().max()) <= 2e-3
        assert not bool(y[:, :n - last].any())
    back = w.restore(torch.bfloat16)
    assert torch.equal(back[n - last:], small.restore(torch.bfloat16)) and not bool(back[:4].any())
    # every value is a code's and stays (where a block's largest one was rounded to 3 units, as 6 of the next smaller unit)
    assert torch.equal(mx4.quantize(back).restore(torch.bfloat16)[n - last:], back[n - last:])
    noise = mx4.quantize(back, rounding=mx4.Stochastic(1))
    assert torch.equal(noise.restore(torch.bfloat16)[n - last:], back[n - last:])


# ---- streams, graphs

def step(mx4, x, dy, w, noise, bias):
    from paper_2108_08842_amd import layers
    w4, wt4 = mx4.quantize(w), mx4.quantize(w, transpose=True)
    y, z = mx4.linear(x, w4, bias, activation="silu", checkpoint=True)
    dz = layers.activation_grad(dy, z, "silu")
    dx = mx4.linear_input_grad(mx4.quantize(dz, rounding=noise), wt4, residual=dy[:, :x.shape[1]].contiguous())
    dyt, db = mx4.quantize(dz, transpose=True, rounding=noise, sums=True)
    return [y, z.buffer, dx, db, mx4.linear_weight_grad(dyt, mx4.quantize(x, transpose=True))]


def test_captured_steps_share_nothing(mx4):
    """Two captured training steps of one layer, replayed in turn with eager work between them; each draws new numbers from its seed on the device."""
    g = gen("graph")
    n, k, m = 300, 200, 600
    w, bias = matrix(g, n, k, torch.bfloat16, 0, 0.1), matrix(g, 1, n, torch.bfloat16)[0]
    graphs = []
    for number in range(2):
        seed = torch.zeros((), dtype=torch.int64, device="cuda")
        x, dy = matrix(g, m, k, torch.bfloat16), matrix(g, m, n, torch.bfloat16, 0, 0.1)
        stream = torch.cuda.Stream()
        stream.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(stream):
            step(mx4, x, dy, w, mx4.Stochastic(seed, number), bias)
        torch.cuda.current_stream().wait_stream(stream)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            out = step(mx4, x, dy, w, mx4.Stochastic(seed, number), bias)
        graphs.append((graph, seed, x, dy, out, number))
    for replay in range(3):
        for graph, seed, x, dy, out, number in graphs:
            seed.fill_(100 * replay + number)
            x.copy_(matrix(gen("x", replay, number), m, k, torch.bfloat16))
            graph.replay()
        for graph, seed, x, dy, out, number in graphs:
            want = step(mx4, x, dy, w, mx4.Stochastic(100 * replay + number, number), bias)
            torch.cuda.synchronize()
            for a, b in zip(out, want):
                assert torch.equal(a, b)


def test_on_other_streams_at_once(mx4):
    g = gen("streams")
    n, k, m = 260, 3000, 500
    w, bias = matrix(g, n, k, torch.float16, 0, 0.1), matrix(g, 1, n, torch.float16)[0]
    x = matrix(g, m, k, torch.float16)
    want = mx4.linear(x, mx4.quantize(w), bias, activation="gelu")
    streams = [torch.cuda.Stream() for _ in range(3)]
    for s in streams:
        s.wait_stream(torch.cuda.current_stream())
    got = [mx4.linear(x, mx4.quantize(w, stream=s), bias, activation="gelu", stream=s) for s in streams]
    torch.cuda.synchronize()
    for y in got:
        assert torch.equal(y, want)


@pytest.mark.parametrize("dtype", TYPES)
def test_operands_that_begin_anywhere(mx4, dtype):
    t = TYPES[dtype]
    for rows, cols in ((40, 300), (257, 1000), (1, 4096), (3, 128)):
        g = gen("anywhere", dtype, rows)
        x, w = matrix(g, rows, cols, t), mx4.quantize(matrix(g, 90, cols, t))
        flat = torch.full((rows * cols + 8,), float("nan"), dtype=t, device="cuda")
        moved = flat[1:1 + rows * cols].view(rows, cols).copy_(x)
        for transpose in (False, True):
            for rounding in (None, mx4.Stochastic(3)):
                a, b = (mx4.quantize(v, transpose=transpose, rounding=rounding) for v in (x, moved))
                assert torch.equal(a.restore(torch.float32), b.restore(torch.float32))
        out = torch.full((rows * 90 + 8,), float("nan"), dtype=t, device="cuda")[1:1 + rows * 90].view(rows, 90)
        residual = torch.full((rows * 90 + 8,), 0.5, dtype=t, device="cuda")[3:3 + rows * 90].view(rows, 90)
        want = mx4.linear(x, w, residual=residual)
        assert torch.equal(mx4.linear(moved, w, residual=residual, out=out), want)
        assert torch.equal(mx4.linear(x, w, residual=residual, out=residual), want)


def test_transposes_beyond_two_to_the_32_elements(mx4):
    rows, cols, last = 2 ** 18 + 2 ** 15, 16384, 32
    g = torch.Generator(device="cuda").manual_seed(2)
    tail = torch.randn(last, cols, generator=g, device="cuda").bfloat16()
    x = torch.zeros(rows, cols, dtype=torch.bfloat16, device="cuda")
    x[-last:] = tail
    got, sums = mx4.quantize(x, transpose=True, rounding=mx4.Stochastic(9, 1), sums=True)
    # the last block of every packed row: its words are the last eight of a row's
    words = rows // 4
    pick = [0, 1, 777, cols - 1]
    back = got.restore(torch.float32, out=torch.empty(cols, rows, device="cuda"))
    for c in pick:
        bits = np.asarray(lref_hash(c * words + words - last // 4, last // 4)).astype("<u8").view("<u2")
        want = ref.values(tail[:, c:c + 1].t().cpu(), torch.from_numpy(bits.astype(np.int64)).view(1, last).numpy())
        assert torch.equal(back[c, -last:].cpu().double(), want[0])
        assert not bool(back[c, :-last].any())
    assert bool(((sums.double() - tail.double().sum(0)).abs() <= (last + 8) * 2.0 ** -24 * tail.double().abs().sum(0)).all())


def lref_hash(first, count):
    from oracle import eden_oracle as oracle
    from tests import blocks_reference
    return oracle.hash_words(oracle.stream_key(9, blocks_reference.STREAM_ROUNDING, 1), first, count)
