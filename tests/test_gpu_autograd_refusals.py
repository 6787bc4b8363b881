"""Operators around a residual block and 4-bit operands record nothing for autograd: what requires a gradient is refused where it would be lost."""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from paper_2108_08842_amd import blocks, mx4                       # noqa: E402
from paper_2108_08842_amd.eden import EdenError                    # noqa: E402
from tests.test_gpu_blocks import gen                              # noqa: E402


def flat(result):
    """The tensors of a result: what an Mx4 holds as values."""
    if isinstance(result, torch.Tensor):
        return [result.clone()]
    if isinstance(result, mx4.Mx4):
        return [result.restore(torch.float32)]
    return [t for v in result if v is not None for t in flat(v)]


def check(calls, plain, refusals):
    want = [flat(f()) for f in calls(**plain)]
    for which, refused in refusals.items():
        for number, f in enumerate(calls(**{**plain, which: plain[which].clone().requires_grad_(True)})):
            if number in refused:
                with pytest.raises(EdenError):
                    f()
            else:
                assert all(torch.equal(a, b) for a, b in zip(flat(f()), want[number])), (which, number)
            with torch.no_grad():                                  # nobody expects one
                assert all(torch.equal(a, b) for a, b in zip(flat(f()), want[number])), (which, number)


def test_operators_around_a_block():
    g = gen("refused")
    tensors = {name: torch.randn(6, 40, generator=g).cuda() for name in ("x", "f", "dr", "dh", "out")}
    tensors |= {name: torch.randn(40, generator=g).cuda() for name in ("gate", "w", "b", "v", "total")}

    def calls(x, f, dr, dh, out, gate, w, b, v, total):
        pre, post, drop = blocks.Norm("layer", w, b), blocks.Norm("rms", v), blocks.Dropout(0.25, 3)
        return [lambda: blocks.dropout(x, drop), lambda: blocks.norm(x, pre), lambda: blocks.join(x, f, gate=gate, dropout=drop, post=post, pre=pre),
                lambda: blocks.join_grad(dr, f, dh=dh, r=x, gate=gate, dropout=drop, post=post, pre=pre), lambda: blocks.norm_grad(dh, x, pre, residual=dr),
                lambda: blocks.join(x, f, out=out), lambda: blocks.dropout(f, drop, out=out), lambda: blocks.join_grad(dr, f, gate=gate, into=blocks.JoinGrads(gate=total)),
                lambda: blocks.join(x, f, stream=torch.cuda.current_stream())]
    check(calls, tensors, {"x": {0, 1, 2, 3, 4, 5, 8}, "f": {2, 3, 5, 6, 7, 8}, "dr": {3, 4, 7}, "dh": {3, 4}, "out": {5, 6}, "gate": {2, 3, 7}, "w": {1, 2, 3, 4}, "b": {1, 2, 3, 4}, "v": {2, 3},
                           "total": {7}})


def test_four_bit_operands():
    g = gen("refused", 4)
    tensors = {"x": torch.randn(6, 40, generator=g).cuda(), "w": torch.randn(24, 40, generator=g).cuda(), "b": torch.randn(24, generator=g).cuda(), "r": torch.randn(6, 24, generator=g).cuda(),
               "q": torch.randn(6, 40, generator=g).cuda(), "total": torch.zeros(40, device="cuda"), "dw": torch.zeros(24, 40, device="cuda")}
    w4, x4 = mx4.quantize(tensors["w"]), mx4.quantize(tensors["x"])
    wt4, r4, rt4, xt4 = mx4.quantize(tensors["w"], transpose=True), mx4.quantize(tensors["r"]), mx4.quantize(tensors["r"], transpose=True), mx4.quantize(tensors["x"], transpose=True)

    def calls(x, w, b, r, q, total, dw):
        return [lambda: mx4.quantize(x), lambda: mx4.quantize(x, transpose=True, rounding=mx4.Stochastic(1)), lambda: mx4.quantize(q, transpose=True, sums=total), lambda: mx4.linear(x, w4),
                lambda: mx4.linear(x4, mx4.quantize(w), b, residual=r), lambda: mx4.linear_input_grad(r4, wt4, residual=q), lambda: mx4.linear_weight_grad(rt4, xt4, out=dw),
                lambda: x4.restore(out=q.clone() if not q.requires_grad else q), lambda: mx4.quantize(x, stream=torch.cuda.current_stream())]
    check(calls, tensors, {"x": {0, 1, 3, 8}, "w": {4}, "b": {4}, "r": {4}, "q": {2, 5, 7}, "total": {2}, "dw": {6}})
