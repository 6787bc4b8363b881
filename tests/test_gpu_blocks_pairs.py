"""Gradients of the join for every pair of norms, in front and behind the branch, each of which is a kernel of its own: next to a gate and dropout in all types and over all widths."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from tests import blocks_reference as ref                          # noqa: E402
from tests.test_gpu_blocks import COLUMNS, TYPES, double, gen, matrix, near, vector              # noqa: E402

KINDS = [None, "rms", "layer"]
PAIRS = [(post, pre) for post in KINDS for pre in KINDS]


@pytest.fixture(scope="module")
def blocks():
    from paper_2108_08842_amd import blocks as m
    assert torch.cuda.is_available()
    m.lib()
    return m


def norms(blocks, g, cols, t, kind):
    """A norm with weight (and bias), and the reference's."""
    if kind is None:
        return None, None
    weight, bias = vector(g, cols, t, 1.0), vector(g, cols, t) if kind == "layer" else None
    return blocks.Norm(kind, weight, bias), (kind, double(weight), double(bias), float(np.float32(1e-5)))


def check(blocks, dtype, rows, cols, post, pre, gates, p=0.25, with_dr=True):
    t, g = TYPES[dtype], gen("pairs", dtype, rows, cols, post, pre, gates)
    f, r, dr = matrix(g, rows, cols, t, 3, 0.7, -1.0), matrix(g, rows, cols, t, 0, 2.0, 0.5), matrix(g, rows, cols, t, 8, 1e-2)
    dh = matrix(g, rows, cols, t, 1, 1e-2) if pre else None
    if not with_dr and pre:
        dr = None
    gate = vector(g, cols, t, 0.5) if gates == 1 else matrix(g, gates, cols, t, 3, 0.5, 0.3)
    post, post_ref = norms(blocks, g, cols, t, post)
    pre, pre_ref = norms(blocks, g, cols, t, pre)
    drop = blocks.Dropout(p, 77, 3) if p else None
    mask, exact = (ref.kept(77, 3, drop.threshold, rows, cols), drop.threshold / 65536) if p else (None, 0.0)
    got = blocks.join_grad(dr, f, dh=dh, r=r if pre else None, gate=gate, scale=0.5, x_scale=1.5, dropout=drop, post=post, pre=pre)
    want = ref.join_grad(double(dr), double(f), double(dh), double(r), double(gate), 0.5, 1.5, mask, exact, post_ref, pre_ref)
    for name, value in got._asdict().items():
        norm = {"pre": pre, "post": post}.get(name.split("_")[0])
        there = (norm is not None and getattr(norm, name.split("_")[1]) is not None) if "_" in name else True
        assert (value is not None) == there, name
        if there:
            near(value, want[name], (name, dtype, rows, cols))


@pytest.mark.parametrize("cols", COLUMNS)
@pytest.mark.parametrize("post,pre", PAIRS)
def test_every_pair_of_norms(blocks, post, pre, cols):
    for dtype in TYPES:
        check(blocks, dtype, 1, cols, post, pre, 1)
        check(blocks, dtype, 30, cols, post, pre, 3, with_dr=False)


@pytest.mark.parametrize("rows,cols", [(5000, 40), (2100, 1000), (600, 4096), (600, 8192), (300, 12001)])
@pytest.mark.parametrize("post,pre", PAIRS)
def test_every_pair_of_norms_in_many_rows(blocks, post, pre, rows, cols):          # workgroups that go through several rows, sums of several workgroups
    check(blocks, "bf16", rows, cols, post, pre, 1)
    check(blocks, "f32", rows, cols, post, pre, 2 if rows % 2 == 0 else 1, p=0.0)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("kind", ["rms", "layer"])
def test_a_norm_in_front_without_a_gradient_of_its_result(blocks, kind, dtype):
    """dh None stands for zeros: the norm adds nothing to dx, and the gradients of its weights are sums over nothing."""
    t = TYPES[dtype]
    for rows, cols in ((1, 5), (30, 1000), (600, 96), (40, 9000)):
        g = gen("without", dtype, kind, cols)
        f, dr, gate = matrix(g, rows, cols, t), matrix(g, rows, cols, t), vector(g, cols, t, 0.5)
        pre, _ = norms(blocks, g, cols, t, kind)
        post, _ = norms(blocks, g, cols, t, "layer")
        drop = blocks.Dropout(0.25, 7)
        plain = blocks.join_grad(dr, f, gate=gate, dropout=drop, post=post)
        got = blocks.join_grad(dr, f, gate=gate, dropout=drop, post=post, pre=pre)
        for name in ("dx", "df", "gate", "post_weight", "post_bias"):
            assert torch.equal(getattr(got, name), getattr(plain, name)), name
        assert (got.pre_bias is None) == (kind == "rms")
        given = [v for v in (got.pre_weight, got.pre_bias) if v is not None]
        assert all(v.shape == (cols,) and not bool(v.any()) for v in given)
        into = blocks.JoinGrads(gate=plain.gate.clone(), post_weight=plain.post_weight.clone(), post_bias=plain.post_bias.clone(), pre_weight=torch.full((cols,), 3.0, device="cuda"),
                                pre_bias=torch.full((cols,), 4.0, device="cuda") if kind == "layer" else None)
        got = blocks.join_grad(dr, f, gate=gate, dropout=drop, post=post, pre=pre, into=into, accumulate=True)
        assert bool((got.pre_weight == 3.0).all()) and (kind == "rms" or bool((got.pre_bias == 4.0).all()))
        for name in ("gate", "post_weight", "post_bias"):
            assert torch.equal(getattr(got, name), 2.0 * getattr(plain, name)), name
