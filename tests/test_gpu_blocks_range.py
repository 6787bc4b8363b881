"""Operators around a residual block on rows near the end of the range of fp32."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from tests import blocks_reference as ref                          # noqa: E402
from tests.test_gpu_blocks import double, gen, matrix, near, vector          # noqa: E402
from tests.test_gpu_blocks_pairs import norms                      # noqa: E402

WIDE = {"f32": torch.float32, "bf16": torch.bfloat16}              # (fp16 ends at 2^16)


@pytest.fixture(scope="module")
def blocks():
    from paper_2108_08842_amd import blocks as m
    assert torch.cuda.is_available()
    m.lib()
    return m


def large(g, rows, cols, t):
    """Rows whose mean square is in fp32's range, the sum of their squares in most of them is not: sizes of 2^57 to 2^62 and, from row 4 on, an ordinary row after each such one."""
    x = torch.randn(rows, cols, generator=g, dtype=torch.float64)
    size = torch.tensor([2.0 ** 62, 2.0 ** 60, 2.0 ** 57, 2.0 ** 58.5], dtype=torch.float64).repeat(rows // 4 + 1)[:rows]
    size[5::2] = 1.0
    return (x * size[:, None]).to(t).cuda()


@pytest.mark.parametrize("cols", [5, 40, 250, 1000, 1031, 2048, 4096, 8192, 16383, 16384])
@pytest.mark.parametrize("dtype", WIDE)
def test_norms_of_large_values(blocks, dtype, cols):
    t, rows = WIDE[dtype], 23
    for kind in ("rms", "layer"):
        g = gen("large", dtype, cols, kind)
        x, f = large(g, rows, cols, t), large(g, rows, cols, t)
        pre, pre_ref = norms(blocks, g, cols, t, kind)
        post, post_ref = norms(blocks, g, cols, t, kind)
        want = ref.join(double(x), None, None, 1.0, 1.0, None, 0.0, None, pre_ref)
        near(blocks.norm(x, pre), want["h"], (kind, cols))
        # the sum of a branch with a norm behind it, and the norm of the sum: both of a call pass the range
        small = matrix(g, rows, cols, t, 0, 2.0 ** -3)
        want = ref.join(double(x), double(f), None, 0.5, 1.0, None, 0.0, post_ref, pre_ref)
        got = blocks.join(x, f, scale=0.5, post=post, pre=pre)
        near(got[0], want["r"], (kind, cols))
        near(got[1], want["h"], (kind, cols))
        want = ref.join(double(small), double(f), None, 1.0, 1.0, None, 0.0, post_ref, pre_ref)
        got = blocks.join(small, f, post=post, pre=pre)
        near(got[0], want["r"], (kind, cols))
        near(got[1], want["h"], (kind, cols))


@pytest.mark.parametrize("cols", [5, 40, 250, 1000, 1031, 2048, 4096, 8192, 16383, 16384])
@pytest.mark.parametrize("dtype", WIDE)
def test_gradients_of_norms_of_large_values(blocks, dtype, cols):
    t, rows = WIDE[dtype], 23
    for kind, size in (("rms", 1.0), ("layer", 1.0), ("rms", 2.0 ** -22), ("layer", 2.0 ** -22)):          # (1 / mean square times a small gradient is below fp32's range, dx is not)
        g = gen("large grad", dtype, cols, kind, size)
        r, f, dh, dr = large(g, rows, cols, t), large(g, rows, cols, t), matrix(g, rows, cols, t, 0, size), matrix(g, rows, cols, t, 0, size)
        pre, pre_ref = norms(blocks, g, cols, t, kind)
        post, post_ref = norms(blocks, g, cols, t, kind)
        want = ref.join_grad(None, None, double(dh), double(r), None, 1.0, 1.0, None, 0.0, None, pre_ref)
        got = blocks.norm_grad(dh, r, pre)
        for name in ("dx", "pre_weight") + (("pre_bias",) if kind == "layer" else ()):
            near(getattr(got, name), want[name], (name, kind, cols, size))
        want = ref.join_grad(double(dr), double(f), double(dh), double(r), None, 1.0, 1.0, None, 0.0, post_ref, pre_ref)
        got = blocks.join_grad(dr, f, dh=dh, r=r, post=post, pre=pre)
        for name in ("dx", "df", "pre_weight", "post_weight") + (("pre_bias", "post_bias") if kind == "layer" else ()):
            near(getattr(got, name), want[name], (name, kind, cols, size))
