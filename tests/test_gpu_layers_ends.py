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
