"""Results of 4-bit products in the place of the residual, in every kernel that has one: few rows, tiles of both sizes, sums that are split over workgroups."""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from tests.test_gpu_mx4 import TYPES, gen, matrix, packed, randn   # noqa: E402


@pytest.mark.parametrize("m,n,k", [(1, 300, 333), (3, 1000, 96), (16, 4099, 520), (18, 4096, 40), (48, 8192, 65), (129, 257, 191), (64, 64, 9000), (300, 72, 1500), (2300, 3200, 300)])
@pytest.mark.parametrize("dtype", TYPES)
def test_a_result_over_its_residual(dtype, m, n, k):
    from paper_2108_08842_amd import layers, mx4
    t, g = TYPES[dtype], gen("in place", dtype, m, n, k)
    w, _ = packed(mx4, randn(g, n, k, scale=k ** -0.5))
    for pad in (0, 3):
        x, bias, residual = matrix(g, m, k, t, pad), matrix(g, 1, n, t)[0], matrix(g, m, n, t, pad)
        for given in (x, mx4.quantize(x)):
            want, kept = mx4.linear(given, w, bias, activation="gelu", residual=residual, checkpoint=True, dtype=t)
            held = torch.full((m, n + pad), 5.0, dtype=t, device="cuda")
            place = held[:, :n]
            place.copy_(residual)
            got, again = mx4.linear(given, w, bias, activation="gelu", residual=place, checkpoint=True, dtype=t, out=place)
            assert got is place and torch.equal(got, want) and torch.equal(again.buffer, kept.buffer) and bool((held[:, n:] == 5.0).all())
            place.copy_(residual)
            want = mx4.linear_input_grad(mx4.quantize(x), w, activation="gelu", checkpoint=kept, residual=residual)
            assert torch.equal(mx4.linear_input_grad(mx4.quantize(x), w, activation="gelu", checkpoint=kept, residual=place, out=place), want)
            assert bool((held[:, n:] == 5.0).all())
    assert isinstance(kept, layers.Checkpoint)
