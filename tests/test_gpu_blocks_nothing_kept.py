"""Gradients of rows that dropout takes out as a whole."""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from tests import blocks_reference as ref                          # noqa: E402
from tests.test_gpu_blocks import gen, matrix, vector              # noqa: E402
from tests.test_gpu_blocks_pairs import norms                      # noqa: E402


@pytest.fixture(scope="module")
def blocks():
    from paper_2108_08842_amd import blocks as m
    assert torch.cuda.is_available()
    m.lib()
    return m


@pytest.mark.parametrize("cols", [1, 5, 8, 12, 40])
def test_rows_of_which_nothing_is_kept(blocks, cols):
    """Whatever reaches a dropped place: df is 0 where a whole row is dropped, behind every kind of norm, also where the row's r and its gradient are not finite."""
    rows, seed = 400, 9
    drop = blocks.Dropout(60000 / 65536, seed, 2)
    mask = ref.kept(seed, 2, drop.threshold, rows, cols)
    nothing = ~mask.any(1)
    assert int(nothing.sum()) > 8
    for t in (torch.float32, torch.bfloat16):
        for post in (None, "rms", "layer"):
            for pre in (None, "rms", "layer"):
                g = gen("nothing", cols, post, pre)
                f, r, dr, dh = (matrix(g, rows, cols, t) for _ in range(4))
                bad = torch.arange(rows) % 2 == 0
                r[bad.cuda(), 0], dr[bad.cuda(), 0] = float("inf"), float("nan")
                got = blocks.join_grad(dr, f, dh=dh if pre else None, r=r if pre else None, gate=vector(g, cols, t, 0.5), dropout=drop, post=norms(blocks, g, cols, t, post)[0],
                                       pre=norms(blocks, g, cols, t, pre)[0])
                df = got.df.cpu()
                assert bool((df[nothing] == 0).all()), (t, post, pre)
                assert bool(df[~bad].isfinite().all()), (t, post, pre)
