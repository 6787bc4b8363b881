"""CPU-side checks of the 4-bit operands: exports, sizes and refusals, and the reference of their tests.  Nothing is launched: every call is refused or has nothing to do."""
import os
import re
import shutil
import subprocess

import numpy as np
import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
torch = pytest.importorskip("torch")

from tests import mx4_reference as ref                             # noqa: E402


@pytest.fixture(scope="module")
def mx4():
    from paper_2108_08842_amd import eden, mx4 as m
    if not os.path.exists(eden._LIB_PATH):
        from paper_2108_08842_amd import build
        build.build(verbose=False)
    m.lib()
    return m


def test_every_declared_symbol_is_exported(mx4):
    text = open(os.path.join(ROOT, "include", "eden_mx4.h")).read()
    header = re.sub(r"/\*.*?\*/", "", text, flags=re.S)
    assert set(re.findall(r"\b(eden_[a-z_0-9]+)\s*\(", header)) == set(mx4.EXPORTS)
    for name in mx4.EXPORTS:
        assert getattr(mx4.lib(), name) is not None
    assert f"#define EDEN_MX4_ROWS {mx4.OWN_ROWS}\n" in text and f"#define EDEN_MX4_VALUES {mx4.OWN_VALUES}\n" in text


def test_header_is_plain_c(tmp_path):
    if shutil.which("gcc") is None:
        pytest.skip("no gcc")
    source = tmp_path / "c.c"
    source.write_text('#include "eden_mx4.h"\nint main(void) { return eden_mx4_bytes(1, 1) == 144 ? EDEN_OK : 1; }\n')
    subprocess.run(["gcc", "-std=c99", "-Wall", "-Wextra", "-pedantic", "-Werror", "-I", os.path.join(ROOT, "include"), "-c", str(source), "-o", str(tmp_path / "c.o")],
                   check=True, capture_output=True, text=True)


def test_sizes(mx4):
    for rows, cols in ((0, 5), (5, 0), (1, 1), (1, 256), (2, 257), (3, 33), (7, 1000), (2 ** 27, 2 ** 22)):
        assert mx4.mx4_bytes(rows, cols) == ref.size(rows, cols) == mx4._bytes(rows, cols)
    assert mx4.mx4_bytes(2 ** 27 + 1, 1) == 0 and mx4.mx4_bytes(1, 2 ** 22 + 1) == 0
    sums, space = mx4.lib().eden_mx4_sums_bytes, mx4.lib().eden_mx4_workspace_bytes
    assert sums(256, 100) == 0 and 0 < sums(8192, 100) <= 32 * 400 and sums(0, 5) == sums(5, 0) == 0
    assert space(8192, 8192, 8192, 0) == 0 and space(0, 5, 10000, 0) == 0
    assert 0 < space(100, 100, 8192, 0) <= 64 * 100 * 400
    assert space(8192, 8192, 1000, 1) == mx4.mx4_bytes(8192, 1000) and space(1, 1, 2 ** 22 + 1, 0) == 0


def test_the_reference_rounds_to_the_nearest_code():
    g = np.random.default_rng(5)
    x = (g.standard_normal((50, 70)) * np.exp2(g.integers(-20, 20, (50, 70)))).astype(np.float32)
    codes, exps = ref.encode(x)
    unit = np.repeat(np.exp2(exps.astype(np.float64) - 127), 32, axis=1)[:, :70]
    every = unit[..., None] * np.concatenate([-ref.GRID, ref.GRID])
    best = np.abs(every - x[..., None]).min(axis=2)
    assert np.array_equal(np.abs(ref.decode(codes, exps, 70) - x), best)
    # the unit is the smallest that clips nothing
    blocks = np.zeros((50, 96))
    blocks[:, :70] = np.abs(x)
    largest = blocks.reshape(50, 3, 32).max(axis=2)
    unit = np.exp2(exps.astype(np.float64) - 127)
    assert np.all(largest <= 6 * unit) and np.all(largest > 3 * unit)
    # a code's value stays where the rounding is stochastic, whatever the bits
    held = ref.decode(codes, exps, 70).astype(np.float32)
    assert np.array_equal(ref.encode(held, np.full((50, 70), 0))[0] & 7, ref.encode(held)[0] & 7)
    assert np.array_equal(ref.unpack(ref.pack(codes, exps), 50, 70)[0][:, :96], codes) and np.array_equal(ref.unpack(ref.pack(codes, exps), 50, 70)[1][:, :3], exps)


P = 4096                                                           # an address that is never used


def test_refusals(mx4):
    from paper_2108_08842_amd.blocks import RandomArgs
    L, bad, room = mx4.lib(), -1, -2

    def quantize(x=P, ldx=8, rows=4, cols=8, dtype=0, transpose=0, rounding=None, packed=P, capacity=1 << 20, sums=None, ws=None, size=0):
        return L.eden_mx4_quantize(x, ldx, rows, cols, dtype, transpose, rounding, packed, capacity, sums, 0, ws, size, None)

    assert quantize(rows=0) == quantize(cols=0) == quantize(rows=0, transpose=1) == 0
    for case in (dict(x=None), dict(packed=None), dict(packed=P + 8), dict(ldx=7), dict(x=P + 2), dict(dtype=3), dict(sums=P), dict(transpose=1, sums=P + 2), dict(ws=P + 4, size=8),
                 dict(cols=2 ** 22 + 1, ldx=2 ** 23), dict(rows=2 ** 27 + 1), dict(rows=2 ** 22 + 1, transpose=1), dict(cols=2 ** 27 + 1, ldx=2 ** 29, transpose=1),
                 dict(rows=2 ** 27, cols=2 ** 22, ldx=2 ** 22, capacity=2 ** 62), dict(rounding=bytes(RandomArgs(1, P + 4, 0, 0)))):
        assert quantize(**case) == bad, case
    assert quantize(capacity=mx4.mx4_bytes(4, 8) - 1) == room and quantize(transpose=1, capacity=mx4.mx4_bytes(8, 4) - 1) == room

    def restore(packed=P, rows=4, cols=8, dtype=0, x=P, ldx=8):
        return L.eden_mx4_restore(packed, rows, cols, dtype, x, ldx, None)

    assert restore(rows=0) == restore(cols=0) == 0
    for case in (dict(packed=None), dict(packed=P + 4), dict(x=None), dict(ldx=7), dict(dtype=3), dict(x=P + 1), dict(rows=2 ** 29)):
        assert restore(**case) == bad, case

    def linear(x=P, ldx=8, x4=None, w=P, bias=None, res=None, ldr=4, y=P, ldy=4, z=None, cap=0, m=3, n=4, k=8, dtype=0, act=0, ws=P, size=1 << 20):
        return L.eden_mx4_linear(x, ldx, x4, w, bias, res, ldr, y, ldy, z, cap, m, n, k, dtype, act, ws, size, None)

    assert linear(m=0) == linear(n=0) == 0
    for case in (dict(x=None), dict(x4=P), dict(x=None, x4=P + 8), dict(w=None), dict(w=P + 8), dict(y=None), dict(dtype=3), dict(act=5), dict(ldx=7), dict(ldy=3), dict(res=P, ldr=3), dict(x=P + 2),
                 dict(bias=P + 2), dict(res=P + 1), dict(z=P + 8, cap=1 << 20), dict(m=2 ** 27 + 1), dict(n=2 ** 27 + 1), dict(k=2 ** 22 + 1), dict(ws=P + 4)):
        assert linear(**case) == bad, case
    assert linear(x=None, x4=P, m=2 ** 27, n=2 ** 27, ldy=2 ** 27) == bad
    assert linear(z=P, cap=3 * 33 - 1) == room and linear(m=17, ws=None) == room and linear(m=17, size=mx4.mx4_bytes(17, 8) - 1) == room and linear(m=1, k=2 ** 14 + 1, ldx=2 ** 16, size=64) == room

    def inputs(dz=P, wt=P, c=None, act=0, res=None, ldr=8, dx=P, ldx=8, m=2, n=4, k=8, dtype=1, ws=None):
        return L.eden_mx4_input_grad(dz, wt, c, act, res, ldr, dx, ldx, m, n, k, dtype, ws, 0, None)

    assert inputs(m=0) == inputs(k=0) == 0
    for case in (dict(dz=None), dict(wt=None), dict(dx=None), dict(dz=P + 8), dict(wt=P + 4), dict(ldx=7), dict(res=P, ldr=7), dict(c=P), dict(act=2), dict(act=2, c=P + 1), dict(act=7, c=P),
                 dict(dtype=4), dict(ws=P + 8), dict(n=2 ** 22 + 1)):
        assert inputs(**case) == bad, case

    def weight(dyt=P, xt=P, dw=P, ldw=8, m=2, n=4, k=8, ws=None):
        return L.eden_mx4_weight_grad(dyt, xt, dw, ldw, m, n, k, 0, ws, 0, None)

    assert weight(n=0) == weight(k=0) == 0
    for case in (dict(dyt=None), dict(xt=None), dict(dw=None), dict(ldw=7), dict(dyt=P + 8), dict(xt=P + 2), dict(dw=P + 2), dict(ws=P + 8), dict(m=2 ** 22 + 1), dict(n=2 ** 27 + 1)):
        assert weight(**case) == bad, case


def test_calls_that_do_not_fit_are_refused(mx4):
    from paper_2108_08842_amd.eden import EdenError
    x = torch.ones(4, 8)
    for call in (lambda: mx4.quantize(x), lambda: mx4.linear(x, None), lambda: mx4.linear_input_grad(x, x), lambda: mx4.linear_weight_grad(x, x),
                 lambda: mx4.Mx4(torch.zeros(10 ** 4, dtype=torch.uint8), 4, 8), lambda: mx4.Mx4(torch.zeros(1, dtype=torch.uint8), 2 ** 27 + 1, 8)):
        with pytest.raises(EdenError):
            call()
