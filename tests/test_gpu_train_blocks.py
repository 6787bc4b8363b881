"""The training example with norms, dropout, a gate and 4-bit products: all operators of a block one after the other."""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from tests import blocks_reference as bref, layers_reference as lref, mx4_reference as mref          # noqa: E402

ROWS, WIDTH, HIDDEN, SEED = 150, 96, 200, 17


def made(norm, dropout, four_bit, dtype=torch.float32):
    from paper_2108_08842_amd import train
    g = torch.Generator(device="cuda").manual_seed(3)
    block = train.Block(WIDTH, HIDDEN, dtype, "gelu", g, norm, dropout, four_bit)
    block.flat.add_(0.1 * torch.randn(block.flat.shape, generator=g, device="cuda"))
    x, dy = (torch.randn(ROWS, WIDTH, generator=g, device="cuda").to(dtype) for _ in range(2))
    weights = block.weights()
    y, kept = block.forward(weights, x, seed=SEED)
    gradient = torch.full_like(block.flat, float("nan"))
    dx = block.backward(weights, dy, kept, gradient)
    return block, weights, x, dy, y, kept, gradient, dx


@pytest.mark.parametrize("norm,dropout", [("none", 0.0), ("none", 0.2), ("rms", 0.0), ("layer", 0.1), ("rms", 0.3)])
def test_gradient_of_the_block_matches_autograd(norm, dropout):
    # in fp32 the only difference from exact autograd is the 8-bit checkpoints: a relative error of about 2^-8 / sqrt(3) of a block's size in each kept value
    # (half a unit in 64 .. 127 of a block's largest value, uniform); the bar is eight times that in the 2-norm
    block, weights, x, dy, y, kept, gradient, dx = made(norm, dropout, False)
    wanted = [p.double().cpu().requires_grad_(True) for p in weights]
    x64 = x.double().cpu().requires_grad_(True)
    w1, b1, w2, b2, *others = wanted
    n = x64 if norm == "none" else bref.Normed(x64, norm, others[1], others[2] if norm == "layer" else None, 1e-5).value
    f = torch.nn.functional.gelu(n @ w1.t() + b1) @ w2.t() + b2
    if dropout:
        threshold = round(65536 * dropout)
        f = torch.where(bref.kept(SEED, 0, threshold, ROWS, WIDTH), f / (1.0 - threshold / 65536), 0.0)
    y64 = x64 + (f if norm == "none" else others[0] * f)
    grads = torch.autograd.grad((y64 * dy.double().cpu()).sum(), wanted + [x64])
    assert float((y.cpu() - y64.detach()).norm() / y64.detach().norm()) < 1e-5
    bar = 8 * 2.0 ** -8 / 3 ** 0.5
    assert len(block.parts(gradient)) == len(wanted)
    for got, want in zip(block.parts(gradient) + [dx], grads):
        assert float((got.cpu() - want).norm() / want.norm()) < bar
    # no checkpoint lies between the result and the last bias, nor the gate
    for i in (3,) + ((4,) if norm != "none" else ()):
        assert float((block.parts(gradient)[i].cpu() - grads[i]).norm() / grads[i].norm()) < 1e-5


@pytest.mark.parametrize("norm,dropout", [("none", 0.0), ("layer", 0.1)])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_four_bit_block(norm, dropout, dtype):
    """Every product of the block from the 4 bits that its operands round to: forward, both weight gradients and the input gradient, with the library's own intermediate results as inputs."""
    from paper_2108_08842_amd import blocks, layers, mx4
    block, weights, x, dy, y, kept, gradient, dx = made(norm, dropout, True, dtype)
    w1, b1, w2, b2 = (w.cpu().double() for w in weights[:4])
    pre, gate, drop = block._around(weights, SEED)
    n = x if pre is None else blocks.norm(x, pre)
    z = mref.values(n) @ mref.values(weights[0]).t() + b1
    off = 1.5 * mref.norm_bound(WIDTH, dtype) + 2.0 ** -20
    h, _ = mx4.linear(n, weights[-4], weights[1], activation="gelu", checkpoint=True)
    assert lref.rel(h.cpu(), lref.act(z, "gelu")) <= off
    f = mref.values(h) @ mref.values(weights[2]).t() + b2
    got_f = y if gate is None else kept[4]
    assert lref.rel(got_f.cpu(), f + (x.cpu().double() if gate is None else 0.0)) <= off
    df = dy if gate is None else blocks.join_grad(dy, kept[4], gate=gate, dropout=drop).df

    def rounded(v, number, turned):
        v = v.t().contiguous() if turned else v
        return mref.values(v, mref.draws(SEED, number, *v.shape))
    dw1, db1, dw2, db2 = block.parts(gradient)[:4]
    assert lref.rel(dw2.cpu(), rounded(df, 0, True) @ mref.values(h.t().contiguous()).t()) <= mref.norm_bound(ROWS, torch.float32)
    assert lref.rel(db2.cpu(), df.cpu().double().sum(0)) <= mref.norm_bound(ROWS, torch.float32)
    dz = mx4.linear_input_grad(mx4.quantize(df, rounding=mx4.Stochastic(SEED, 1)), weights[-1], activation="gelu", checkpoint=kept[1], dtype=dtype)
    slope = lref.slope(lref.values(kept[1]), "gelu")
    assert lref.rel(dz.cpu(), (rounded(df, 1, False) @ mref.values(weights[2].t().contiguous()).t()) * slope) <= off
    assert lref.rel(dw1.cpu(), rounded(dz, 2, True) @ mref.values(n.t().contiguous()).t()) <= mref.norm_bound(ROWS, torch.float32)
    assert lref.rel(db1.cpu(), dz.cpu().double().sum(0)) <= mref.norm_bound(ROWS, torch.float32)
    dn = rounded(dz, 3, False) @ mref.values(weights[0].t().contiguous()).t()
    if norm == "none":
        assert lref.rel(dx.cpu(), dn + dy.cpu().double()) <= off
    assert bool(dx.isfinite().all()) and bool(gradient.isfinite().all())


@pytest.mark.parametrize("options", [dict(norm="rms", dropout=0.1, four_bit=True), dict(norm="layer"), dict(four_bit=True), dict(dropout=0.2)])
def test_training_runs(options):
    from paper_2108_08842_amd import train
    losses = train.train(senders=2, rows=128, width=64, hidden=128, budget=1, steps=4, **options)
    again = train.train(senders=2, rows=128, width=64, hidden=128, budget=1, steps=4, **options)
    assert len(losses) == 4 and all(0.0 < v < float("inf") for v in losses) and losses == again


@pytest.mark.parametrize("norm,dropout", [("rms", 0.0), ("layer", 0.1), ("rms", 0.3)])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_four_bit_block_with_a_norm(norm, dropout, dtype):
    """What the norm, the gate and the residual do with the 4-bit products' results, against 64 bits: the gradient of x, and those of the gate and of the norm's weight and bias."""
    import numpy as np
    from paper_2108_08842_amd import blocks, mx4
    from tests.test_gpu_blocks import near
    block, weights, x, dy, y, kept, gradient, dx = made(norm, dropout, True, dtype)
    pre, gate, drop = block._around(weights, SEED)
    f, threshold = kept[4], drop.threshold if drop else 0
    mask, p = (bref.kept(SEED, 0, threshold, ROWS, WIDTH), threshold / 65536) if drop else (None, 0.0)

    def double(t):
        return None if t is None else t.cpu().double()
    joined = bref.join(double(x), double(f), double(gate), 1.0, 1.0, mask, p, None, None)
    near(y, joined["r"], "y")
    split = bref.join_grad(double(dy), double(f), None, None, double(gate), 1.0, 1.0, mask, p, None, None)
    parts = block.parts(gradient)
    near(parts[4], split["gate"], "gate")
    # the gradient that reaches the norm: both layers' products of what was rounded, each held against 64 bits by itself
    df = blocks.join_grad(dy, f, gate=gate, dropout=drop).df
    near(df, split["df"], "df")
    off = 1.5 * mref.norm_bound(WIDTH, dtype) + 2.0 ** -20

    def rounded(v, number):
        return mref.values(v, mref.draws(SEED, number, *v.shape))
    dz = mx4.linear_input_grad(mx4.quantize(df, rounding=mx4.Stochastic(SEED, 1)), weights[-1], activation="gelu", checkpoint=kept[1], dtype=dtype)
    dn = mx4.linear_input_grad(mx4.quantize(dz, rounding=mx4.Stochastic(SEED, 3)), weights[-3], dtype=dtype)
    assert lref.rel(dn.cpu(), rounded(dz, 3) @ mref.values(weights[0].t().contiguous()).t()) <= off
    want = bref.join_grad(double(dy), None, double(dn), double(x), None, 1.0, 1.0, None, 0.0, None, (norm, double(pre.weight), double(pre.bias), float(np.float32(1e-5))))
    near(dx, want["dx"], "dx")
    near(parts[5], want["pre_weight"], "norm's weight")
    if norm == "layer":
        near(parts[6], want["pre_bias"], "norm's bias")
    assert len(parts) == (7 if norm == "layer" else 6)
