"""The training example: layer operators, EDEN and the update together."""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


def test_gradient_of_the_block_matches_autograd():
    # in fp32 the only difference from exact autograd is the 8-bit checkpoints: a uniform error of at most half a unit in 64 .. 127 of a block's largest
    # value, so a relative error of about 2^-8 / sqrt(3) of a block's size in each kept value; the bar is eight times that in the 2-norm
    from paper_2108_08842_amd import layers, train
    g = torch.Generator(device="cuda").manual_seed(3)
    block = train.Block(96, 200, torch.float32, "gelu", g)
    weights = block.weights()
    x, dy = torch.randn(150, 96, generator=g, device="cuda"), torch.randn(150, 96, generator=g, device="cuda")
    y, kept = block.forward(weights, x)
    gradient = torch.zeros_like(block.flat)
    dx = block.backward(weights, dy, kept, gradient)

    wanted = [p.double().cpu().requires_grad_(True) for p in weights]
    x64 = x.double().cpu().requires_grad_(True)
    w1, b1, w2, b2 = wanted
    y64 = x64 + torch.nn.functional.gelu(x64 @ w1.t() + b1) @ w2.t() + b2
    grads = torch.autograd.grad((y64 * dy.double().cpu()).sum(), wanted + [x64])
    assert float((y.cpu() - y64).norm() / y64.norm()) < 1e-5
    bar = 8 * 2.0 ** -8 / 3 ** 0.5
    for got, want in zip(block.parts(gradient) + [dx], grads):
        assert float((got.cpu() - want).norm() / want.norm()) < bar
    # the last bias sees no checkpoint
    assert float((block.parts(gradient)[3].cpu() - grads[3]).norm() / grads[3].norm()) < 1e-5
    assert layers.checkpoint_bytes(150, 96) == kept[0].buffer.numel()


@pytest.mark.parametrize("budget", [0, 1, 4])
def test_training_lowers_the_loss(budget):
    from paper_2108_08842_amd import train
    losses = train.train(senders=4, rows=256, width=128, hidden=256, budget=budget, steps=40, rate=0.1)
    assert losses[-1] < 0.5 * losses[0]
