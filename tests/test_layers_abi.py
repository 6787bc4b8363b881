"""CPU-side checks of the layer operators: exports, sizes and refusals.  Nothing is launched: every call is refused or has nothing to do."""
import os
import re
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
torch = pytest.importorskip("torch")


@pytest.fixture(scope="module")
def layers():
    from paper_2108_08842_amd import eden, layers as m
    if not os.path.exists(eden._LIB_PATH):
        from paper_2108_08842_amd import build
        build.build(verbose=False)
    m.lib()
    return m


def test_every_declared_symbol_is_exported(layers):
    header = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", "eden_layers.h")).read(), flags=re.S)
    assert set(re.findall(r"\b(eden_[a-z_]+)\s*\(", header)) == set(layers.EXPORTS)
    for name in layers.EXPORTS:
        assert getattr(layers.lib(), name) is not None


def test_header_is_plain_c(tmp_path):
    if shutil.which("gcc") is None:
        pytest.skip("no gcc")
    source = tmp_path / "c.c"
    source.write_text('#include "eden_layers.h"\nint main(void) { return eden_checkpoint_bytes(1, 1) == 33 ? EDEN_OK : 1; }\n')
    subprocess.run(["gcc", "-std=c99", "-Wall", "-Wextra", "-pedantic", "-Werror", "-I", os.path.join(ROOT, "include"), "-c", str(source), "-o", str(tmp_path / "c.o")],
                   check=True, capture_output=True, text=True)


def test_checkpoint_bytes(layers):
    for rows, cols in ((0, 5), (1, 1), (1, 32), (3, 33), (7, 1000), (2 ** 30, 2 ** 30)):
        assert layers.checkpoint_bytes(rows, cols) == rows * ((cols + 31) // 32) * 33
    assert layers.checkpoint_bytes(2 ** 30 + 1, 1) == 0 and layers.checkpoint_bytes(1, 2 ** 30 + 1) == 0


def test_workspace_is_for_long_sums_of_small_results_only(layers):
    size = layers.lib().eden_layers_workspace_bytes
    assert size(8192, 8192, 8192, layers.BF16) == 0 and size(128, 128, 100, layers.BF16) == 0 and size(0, 5, 10000, layers.F32) == 0
    assert 0 < size(100, 100, 8192, layers.F16) <= 64 * (100 * 101 * 4)
    assert size(1, 1, 1, 3) == 0 and size(2 ** 30 + 1, 1, 1, 0) == 0


def test_room_for_copies_is_for_large_products(layers):
    plain, copying = layers.lib().eden_layers_workspace_bytes, layers.lib().eden_layers_copying_bytes
    assert copying(4001, 4001, 4001, layers.BF16) >= plain(4001, 4001, 4001, layers.BF16) + 2 * 2 * 4001 * 4001
    assert copying(4001, 4001, 4001, layers.F32) >= plain(4001, 4001, 4001, layers.F32) + 2 * 4 * 4001 * 4001
    assert copying(100, 100, 8192, layers.F16) == plain(100, 100, 8192, layers.F16) and copying(5, 5, 0, layers.F16) == 0
    assert copying(2 ** 30 + 1, 1, 1, 0) == 0 and copying(1, 1, 1, 9) == 0


P = 4096                                                           # an address that is never used


def test_refusals(layers):
    L = layers.lib()
    bad, room = -1, -2

    def linear(x=P, ldx=8, w=P, ldw=8, bias=None, res=None, ldr=4, y=P, ldy=4, z=None, cap=0, m=2, n=4, k=8, dtype=0, act=0, ws=None, size=0):
        return L.eden_linear(x, ldx, w, ldw, bias, res, ldr, y, ldy, z, cap, m, n, k, dtype, act, ws, size, None)

    assert linear(m=0) == linear(n=0) == 0                         # nothing to do
    for case in (dict(x=None), dict(w=None), dict(y=None), dict(dtype=3), dict(act=5), dict(ldx=7), dict(ldw=7), dict(ldy=3), dict(res=P, ldr=3), dict(x=P + 2), dict(w=P + 1),
                 dict(bias=P + 2), dict(res=P + 1), dict(z=P + 8, cap=1 << 20), dict(m=2 ** 30 + 1), dict(n=2 ** 30 + 1), dict(k=2 ** 30 + 1), dict(ws=P + 4, size=1 << 20),
                 dict(m=2 ** 30, n=2 ** 30, ldy=2 ** 30)):
        assert linear(**case) == bad, case
    assert linear(z=P, cap=2 * 33 - 1) == room

    def weight(dy=P, ldy=4, c=P, dw=P, ldw=8, db=None, m=2, n=4, k=8, dtype=0, ws=None):
        return L.eden_linear_weight_grad(dy, ldy, c, dw, ldw, db, m, n, k, dtype, 0, ws, 0, None)

    assert weight(n=0) == weight(k=0) == 0
    for case in (dict(dy=None), dict(c=None), dict(dw=None), dict(ldy=3), dict(ldw=7), dict(c=P + 8), dict(dw=P + 2), dict(db=P + 2), dict(dtype=9), dict(m=2 ** 30 + 1), dict(ws=P + 8)):
        assert weight(**case) == bad, case

    def inputs(dz=P, ldz=4, w=P, ldw=8, c=None, act=0, res=None, ldr=8, dx=P, ldx=8, m=2, n=4, k=8, dtype=1, ws=None):
        return L.eden_linear_input_grad(dz, ldz, w, ldw, c, act, res, ldr, dx, ldx, m, n, k, dtype, ws, 0, None)

    assert inputs(m=0) == inputs(k=0) == 0
    for case in (dict(dz=None), dict(w=None), dict(dx=None), dict(ldz=3), dict(ldw=7), dict(ldx=7), dict(res=P, ldr=7), dict(c=P), dict(act=2), dict(act=2, c=P + 1), dict(act=7, c=P),
                 dict(dtype=4), dict(dz=P + 1), dict(ws=P + 8)):
        assert inputs(**case) == bad, case

    def gradient(dy=P, ldy=8, c=P, act=2, dz=P, ldz=8, rows=2, cols=8, dtype=2):
        return L.eden_activation_grad(dy, ldy, c, act, dz, ldz, rows, cols, dtype, None)

    assert gradient(rows=0) == gradient(cols=0) == 0
    for case in (dict(dy=None), dict(c=None), dict(dz=None), dict(ldy=7), dict(ldz=7), dict(act=5), dict(dtype=3), dict(dz=P + 1), dict(rows=2 ** 30, cols=2 ** 30, ldy=2 ** 30, ldz=2 ** 30)):
        assert gradient(**case) == bad, case

    def save(x=P, ldx=8, rows=2, cols=8, dtype=0, c=P, cap=66):
        return L.eden_checkpoint_save(x, ldx, rows, cols, dtype, c, cap, None)

    assert save(rows=0) == save(cols=0, cap=0) == 0 and save(cap=65) == room
    for case in (dict(x=None), dict(c=None), dict(c=P + 4), dict(ldx=7), dict(x=P + 1), dict(dtype=3), dict(cols=2 ** 30 + 1)):
        assert save(**case) == bad, case

    def restore(c=P, rows=2, cols=8, dtype=0, x=P, ldx=8):
        return L.eden_checkpoint_restore(c, rows, cols, dtype, x, ldx, None)

    assert restore(rows=0) == restore(cols=0) == 0
    for case in (dict(x=None), dict(c=None), dict(c=P + 4), dict(ldx=7), dict(x=P + 1), dict(dtype=3), dict(rows=2 ** 30 + 1)):
        assert restore(**case) == bad, case


def test_tensors_that_are_not_on_the_gpu_are_refused(layers):
    from paper_2108_08842_amd.eden import EdenError
    x, w = torch.ones(2, 8), torch.ones(4, 8)
    for call in (lambda: layers.linear(x, w), lambda: layers.save_checkpoint(x), lambda: layers.linear_input_grad(x, w.t()),
                 lambda: layers.Checkpoint(torch.zeros(66, dtype=torch.uint8), 2, 8)):
        with pytest.raises(EdenError):
            call()


@pytest.mark.parametrize("dtype", [0, 1, 2])
def test_no_room_for_copies_below_two_to_the_30_products(layers, dtype):
    plain, copying = layers.lib().eden_layers_workspace_bytes, layers.lib().eden_layers_copying_bytes
    for size in ((831, 831, 831), (301, 2001, 1001), (1023, 1024, 1024), (255, 8192, 8192), (8192, 255, 8192)):
        assert copying(*size, dtype) == plain(*size, dtype)
    for size in ((1025, 1024, 1024), (1235, 1235, 1235), (256, 8192, 8192)):
        assert copying(*size, dtype) > plain(*size, dtype)
