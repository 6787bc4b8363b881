"""CPU-side checks of the operators around a residual block: exports, sizes and refusals, and the reference of their tests.  Nothing is launched: every call is
refused or has nothing to do."""
import ctypes
import os
import re
import shutil
import struct
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
torch = pytest.importorskip("torch")

from tests import blocks_reference as ref                          # noqa: E402


@pytest.fixture(scope="module")
def blocks():
    from paper_2108_08842_amd import blocks as m, eden
    if not os.path.exists(eden._LIB_PATH):
        from paper_2108_08842_amd import build
        build.build(verbose=False)
    m.lib()
    return m


def test_every_declared_symbol_is_exported(blocks):
    header = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", "eden_blocks.h")).read(), flags=re.S)
    assert set(re.findall(r"\b(eden_[a-z_]+)\s*\(", header)) == set(blocks.EXPORTS)
    for name in blocks.EXPORTS:
        assert getattr(blocks.lib(), name) is not None


def test_header_is_plain_c_and_the_binding_has_its_layout(blocks, tmp_path):
    if shutil.which("gcc") is None:
        pytest.skip("no gcc")
    source = tmp_path / "c.c"
    fields = {"eden_join_args": blocks.JoinArgs, "eden_join_grad_args": blocks.JoinGradArgs, "eden_norm": blocks.NormArgs, "eden_random": blocks.RandomArgs}
    lines = [f'printf("%zu\\n", sizeof({c}));' for c in fields]
    lines += [f'printf("%zu\\n", offsetof({c}, {f[0]}));' for c, s in fields.items() for f in s._fields_]
    source.write_text('#include <stdio.h>\n#include "eden_blocks.h"\nint main(void) {\n' + "\n".join(lines) + "\nreturn 0; }\n")
    subprocess.run(["gcc", "-std=c99", "-Wall", "-Wextra", "-pedantic", "-Werror", "-I", os.path.join(ROOT, "include"), str(source), "-o", str(tmp_path / "c")], check=True,
                   capture_output=True, text=True)
    got = [int(v) for v in subprocess.run([str(tmp_path / "c")], check=True, capture_output=True, text=True).stdout.split()]
    want = [ctypes.sizeof(s) for s in fields.values()] + [getattr(s, f[0]).offset for s in fields.values() for f in s._fields_]
    assert got == want
    assert [blocks._JOIN_ARGS.size, blocks._JOIN_GRAD_ARGS.size, struct.calcsize(blocks._NORM), blocks._RANDOM_ARGS.size] == want[:4]


def test_arguments_are_packed_as_the_structures_are(blocks):
    """Every field a number of its own: the packed bytes are those of the structure."""
    for kind, packed in ((blocks.JoinArgs, blocks._JOIN_ARGS), (blocks.JoinGradArgs, blocks._JOIN_GRAD_ARGS)):
        a, flat = kind(), []
        for name, field in kind._fields_:
            for part, of in [(name, None)] if not issubclass(field, ctypes.Structure) else [(f[0], name) for f in field._fields_]:
                flat.append(len(flat) + 1)
                setattr(a if of is None else getattr(a, of), part, flat[-1])
        assert packed.pack(*flat) == bytes(a)


def test_workspace(blocks):
    size = blocks.lib().eden_join_workspace_bytes
    assert size(0, 64, 1, 0) == size(64, 0, 1, 0) == size(1, 64, 1, 0) == 0
    assert size(64, 64, 1, 3) == size(64, 16385, 1, 0) == size(2 ** 30 + 1, 64, 1, 0) == size(64, 64, 65, 0) == size(64, 64, 7, 0) == 0
    assert 0 < size(8192, 4096, 1, 2) <= 64 << 20
    assert 0 < size(8192, 4096, 8192, 2) <= 64 << 20


P = 4096                                                           # an address that is never used


def test_refusals(blocks):
    L, bad = blocks.lib(), -1

    def dropout(x=P, ldx=8, y=P, ldy=8, rows=2, cols=8, dtype=0, threshold=5, seed_at=None):
        return L.eden_dropout(x, ldx, y, ldy, rows, cols, dtype, bytes(blocks.RandomArgs(1, seed_at, 0, threshold)), None)

    assert dropout(rows=0) == dropout(cols=0) == 0
    for case in (dict(x=None), dict(y=None), dict(ldx=7), dict(ldy=7), dict(x=P + 2), dict(dtype=3), dict(threshold=65536), dict(seed_at=P + 4), dict(rows=2 ** 30 + 1), dict(cols=16385, ldx=16385, ldy=16385)):
        assert dropout(**case) == bad, case
    assert L.eden_dropout(P, 8, P, 8, 2, 8, 0, None, None) == bad

    def fill(a, given):
        for name, value in given.items():
            if "__" in name:
                part, field = name.split("__")
                setattr(getattr(a, part), field, value)
            else:
                setattr(a, name, value)
        return a

    def join(**given):
        a = blocks.JoinArgs(rows=4, cols=8, x=P, f=P, r=P, h=P, ldx=8, ldf=8, ldr=8, ldh=8, gates=1, x_scale=1.0, scale=1.0)
        a.pre.kind = 1
        return L.eden_join(bytes(fill(a, given)), None)

    assert join(rows=0) == join(cols=0) == 0 and L.eden_join(None, None) == bad
    inf = float("inf")
    for case in (dict(x=None), dict(h=None), dict(pre__kind=0), dict(pre__kind=3), dict(post__kind=3), dict(dtype=3), dict(ldx=7), dict(ldf=7), dict(ldr=7), dict(ldh=7), dict(x=P + 2), dict(f=P + 1),
                 dict(r=P + 1), dict(h=P + 3), dict(gate=P, gates=3, ld_gate=8), dict(gate=P, gates=0, ld_gate=8), dict(gate=P + 1, ld_gate=8), dict(gate=P, gates=2, ld_gate=7), dict(pre__eps=-1.0),
                 dict(pre__eps=inf), dict(post__kind=2, post__eps=float("nan")), dict(pre__bias=P), dict(pre__weight=P + 1), dict(post__weight=P), dict(scale=inf), dict(x_scale=float("nan")), dict(f=None),
                 dict(f=None, r=None, gate=P, ld_gate=8), dict(f=None, r=None, post__kind=1), dict(f=None, r=None, random__threshold=3), dict(random__threshold=65536), dict(random__seed_at=P + 4),
                 dict(cols=16385), dict(rows=2 ** 30 + 1), dict(r=None, h=None, pre__kind=0)):
        assert join(**case) == bad, case

    def grad(**given):
        a = blocks.JoinGradArgs(rows=4, cols=8, dr=P, dh=P, r=P, f=P, dx=P, df=P, lddr=8, lddh=8, ldr=8, ldf=8, lddx=8, lddf=8, gates=1, x_scale=1.0, scale=1.0, branch=1)
        a.pre.kind = a.post.kind = 2
        return L.eden_join_grad(bytes(fill(a, given)), None)

    assert grad(cols=0) == grad(dx=None, df=None) == 0 and L.eden_join_grad(None, None) == bad
    for case in (dict(r=None), dict(f=None), dict(pre__kind=0), dict(lddr=7), dict(lddh=7), dict(ldr=7), dict(ldf=7), dict(lddx=7), dict(lddf=7), dict(dr=P + 1), dict(dx=P + 2), dict(workspace=P + 8),
                 dict(gate=P, gates=3, ld_gate=8), dict(gate_grad=P, gates=2, ld_gate_grad=7), dict(gate_grad=P + 2, gates=1), dict(pre__kind=1, pre_bias_grad=P), dict(post__kind=1, post_bias_grad=P),
                 dict(post__kind=0, post_weight_grad=P), dict(pre__kind=0, dh=None, pre_weight_grad=P), dict(pre_weight_grad=P + 2), dict(branch=0), dict(branch=0, df=None), dict(branch=0, df=None, post__kind=0, dh=None), dict(dtype=7),
                 dict(random__threshold=70000), dict(cols=20000), dict(rows=2 ** 31), dict(scale=inf)):
        assert grad(**case) == bad, case


def test_calls_that_do_not_fit_are_refused(blocks):
    from paper_2108_08842_amd.eden import EdenError
    x = torch.ones(4, 8)
    for call in (lambda: blocks.dropout(x, blocks.Dropout(0.1, 1)), lambda: blocks.norm(x, blocks.Norm("rms")), lambda: blocks.join(x, x), lambda: blocks.join_grad(x, x), lambda: blocks.join(x, None),
                 lambda: blocks.join_grad(None), lambda: blocks.Dropout(1.0, 1), lambda: blocks.Dropout(-0.1, 1), lambda: blocks.Dropout(float("nan"), 1), lambda: blocks.Norm("batch"),
                 lambda: blocks.Norm("rms", None, x[0]), lambda: blocks.Norm("layer", eps=-1.0), lambda: blocks.Norm("layer", eps=float("inf")), lambda: blocks.Norm("layer", eps=1e39), lambda: blocks.norm_grad(None, x, blocks.Norm("rms"), residual=x),
                 lambda: blocks.norm_grad(x, x, None), lambda: blocks.Dropout(0.1, 1, 2 ** 32)._args(None, "x"), lambda: blocks.Dropout(0.1, torch.tensor(3))._args(None, "x"),
                 lambda: blocks.Dropout(0.1, 1.5)._args(None, "x")):
        with pytest.raises(EdenError):
            call()


def test_seeds_are_whole_numbers_of_any_kind(blocks):
    import numpy as np
    for seed, want in ((0, 0), (-1, 2 ** 64 - 1), (2 ** 64 + 5, 5), (np.int64(-3), 2 ** 64 - 3), (np.uint64(2 ** 64 - 1), 2 ** 64 - 1)):
        assert blocks.Dropout(0.5, seed, 7)._args(None, "x") == (want, 0, 7, 32768)


def test_ids_are_whole_numbers_of_any_kind(blocks):
    import numpy as np
    from paper_2108_08842_amd import mx4
    from paper_2108_08842_amd.eden import EdenError

    def args(number):
        rounding = mx4.Stochastic(5, number)                       # as mx4.quantize reads it
        assert blocks._random(rounding.seed, rounding.id, 0, None, "x")[2] == number
        return blocks.Dropout(0.5, 5, number)._args(None, "x")
    for number in (0, 2 ** 32 - 1, np.int32(7), np.uint64(9), torch.tensor(3)):
        assert args(number) == (5, 0, int(number), 32768) and len(blocks._RANDOM_ARGS.pack(*args(number))) == 24
    for bad in (1.5, 2.0, "3", None, torch.tensor(1.5), -1, 2 ** 32, np.int64(-1), float("nan")):
        for call in (lambda: blocks.Dropout(0.5, 5, bad)._args(None, "x"), lambda: blocks._random(5, bad, 0, None, "quantize")):
            with pytest.raises(EdenError):
                call()


def test_scales_that_leave_the_range_with_dropout_are_refused(blocks):
    """scale 65536 / (65536 - threshold) multiplies what is kept: infinite, it would make NaN of the zeros of what is dropped."""
    L, most, half = blocks.lib(), 3.4028234e38, 32768
    for rows, scale, threshold, want in ((0, most, 0, 0), (0, most / 2.01, half, 0), (4, most / 1.9, half, -1), (4, -most, 1, -1), (0, 1e33, 65535, 0), (4, 1e34, 65535, -1)):
        a = blocks.JoinArgs(rows=rows, cols=8, x=P, f=P, r=P, ldx=8, ldf=8, ldr=8, gates=1, x_scale=1.0, scale=scale)
        a.random.threshold = threshold
        assert L.eden_join(bytes(a), None) == want, (scale, threshold)
        a = blocks.JoinGradArgs(rows=rows, cols=8, dr=P, f=P, dx=None if rows == 0 else P, lddr=8, ldf=8, lddx=8, lddf=8, gates=1, x_scale=1.0, scale=scale, branch=1)
        a.random.threshold = threshold
        assert L.eden_join_grad(bytes(a), None) == want, (scale, threshold)


def test_the_reference_gradients_against_autograd():
    """The formulas of the tests' reference, in 64 bits, against torch's own differentiation of the forward formulas."""
    g = torch.Generator().manual_seed(4)
    rows, cols = 6, 20

    def rand(*s):
        return torch.randn(*s, generator=g, dtype=torch.float64)
    for gate_rows in (None, 1, 3):
        for post in (None, "rms", "layer"):
            for pre in (None, "rms", "layer"):
                leaves = {"x": rand(rows, cols), "f": rand(rows, cols)}
                if gate_rows:
                    leaves["gate"] = rand(gate_rows, cols)
                norms = {}
                for name, kind in (("post", post), ("pre", pre)):
                    if kind:
                        leaves[name + "_weight"] = rand(cols)
                        if kind == "layer":
                            leaves[name + "_bias"] = rand(cols)
                for v in leaves.values():
                    v.requires_grad_(True)
                for name, kind in (("post", post), ("pre", pre)):
                    norms[name] = (kind, leaves[name + "_weight"], leaves.get(name + "_bias"), 1e-5) if kind else None
                mask, p = ref.kept(3, 1, 16384, rows, cols), 0.25
                out = ref.join(leaves["x"], leaves["f"], leaves.get("gate"), 0.7, 1.3, mask, p, norms["post"], norms["pre"])
                dr, dh = rand(rows, cols), rand(rows, cols)
                total = (out["r"][0] * dr).sum() + ((out["h"][0] * dh).sum() if pre else 0.0)
                want = dict(zip(leaves, torch.autograd.grad(total, list(leaves.values()))))
                with torch.no_grad():
                    got = ref.join_grad(dr, leaves["f"], dh if pre else None, out["r"][0], leaves.get("gate"), 0.7, 1.3, mask, p, norms["post"], norms["pre"])
                for name, value in want.items():
                    mine = got[{"x": "dx", "f": "df"}.get(name, name)][0]
                    assert torch.allclose(mine, value, rtol=1e-10, atol=1e-12), (gate_rows, post, pre, name)
