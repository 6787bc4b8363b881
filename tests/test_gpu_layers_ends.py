"""The layer operators at the ends of their range, in part through the C entry points themselves."""
import zlib

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

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
