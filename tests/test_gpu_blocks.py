"""The operators around a residual block on the GPU against 64 bits, at the sizes, types, distances and values where they can go wrong."""
import math
import zlib

import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from tests import blocks_reference as ref                          # noqa: E402

TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
# rows that are shorter than a vector, end inside one, fill 8 .. 64 lanes, several waves, one column more than that, the longest
COLUMNS = [1, 3, 8, 64, 65, 128, 250, 513, 1000, 1024, 1031, 2048, 4097, 8192, 8200, 16384]


@pytest.fixture(scope="module")
def blocks():
    from paper_2108_08842_amd import blocks as m
    assert torch.cuda.is_available()
    m.lib()
    return m


def gen(*key):
    return torch.Generator().manual_seed(zlib.crc32(repr(key).encode()))


def matrix(g, rows, cols, dtype, pad=0, scale=1.0, shift=0.0):
    """A matrix on the GPU whose rows are `pad` elements further apart than they are long, surrounded by NaN."""
    x = torch.full((rows, cols + pad), float("nan"), dtype=dtype)
    x[:, :cols] = (torch.randn(rows, cols, generator=g, dtype=torch.float64) * scale + shift).to(dtype)
    return x.cuda()[:, :cols]


def vector(g, cols, dtype, shift=0.0, scale=0.3):
    return (torch.randn(cols, generator=g, dtype=torch.float64) * scale + shift).to(dtype).cuda()


def double(t):
    return None if t is None else t.cpu().double()


def near(got, want, what):
    value, off = want
    got = got.cpu()
    limit = off + (ref.ROUND[got.dtype] * (1.0 + 2.0 ** -20) * (value.abs() + off)) + ref.TINY[got.dtype]
    worst = ((got.double() - value).abs() / limit).max() if got.numel() else 0.0
    assert float(worst) <= 1.0, (what, float(worst))


# ---- dropout

@pytest.mark.parametrize("rows,cols,pad", [(1, 1, 0), (1, 4096, 0), (3, 7, 1), (33, 1001, 0), (130, 64, 8), (5, 16384, 0), (700, 33, 3)])
@pytest.mark.parametrize("dtype", TYPES)
def test_dropout_is_bit_exact(blocks, dtype, rows, cols, pad):
    t = TYPES[dtype]
    x = matrix(gen(dtype, rows, cols), rows, cols, t, pad, 3.0)
    for p, seed, number in ((0.1, 7, 0), (0.5, 2 ** 64 - 3, 2 ** 32 - 1), (65535 / 65536, -5, 1), (1e-9, 3, 4), (0.0, 1, 1)):
        out = torch.full((rows, cols + pad), 5.0, dtype=t, device="cuda")
        got = blocks.dropout(x, blocks.Dropout(p, seed, number), out=out[:, :cols]).cpu()
        threshold = round(65536 * p)
        mask = ref.kept(seed, number, threshold, rows, cols)
        want = torch.where(mask, x.cpu().float() * torch.tensor(65536.0 / (65536 - threshold), dtype=torch.float32), torch.zeros(())).to(t)
        assert torch.equal(got, want) and bool((out[:, cols:] == 5.0).all())
    again = x.clone()
    drop = blocks.Dropout(0.3, 9, 2)
    want = blocks.dropout(x, drop)
    assert blocks.dropout(again, drop, out=again) is again and torch.equal(again, want)
    assert torch.equal(blocks.dropout(x, None), x)


def test_what_is_dropped_may_be_anything(blocks):
    for t in TYPES.values():
        x = torch.full((64, 100), float("nan"), dtype=t, device="cuda")
        x[::2] = float("inf")
        mask = ref.kept(3, 1, 32768, 64, 100)
        y = blocks.dropout(x, blocks.Dropout(0.5, 3, 1)).cpu()
        assert bool((y[~mask] == 0).all()) and bool((y[mask] == x.cpu()[mask])[::1].logical_or(y[mask].isnan()).all())
        f = torch.where(mask.cuda(), torch.ones((), dtype=t, device="cuda"), x)
        got = blocks.join(torch.zeros_like(f), f, dropout=blocks.Dropout(0.5, 3, 1))
        assert torch.equal(got.cpu(), torch.where(mask, 2.0, 0.0).to(t))
        d = torch.where(mask.cuda(), torch.ones((), dtype=t, device="cuda"), x)
        grads = blocks.join_grad(d, f, gate=torch.ones(100, dtype=t, device="cuda"), dropout=blocks.Dropout(0.5, 3, 1))
        assert torch.equal(grads.df.cpu(), torch.where(mask, 2.0, 0.0).to(t)) and torch.equal(grads.gate.cpu(), 2.0 * mask.sum(0).float())


def test_seed_on_the_device(blocks):
    x = matrix(gen("seed"), 40, 300, torch.bfloat16)
    for seed in (5, -17, 2 ** 63 - 1):
        at = torch.tensor(seed, dtype=torch.int64, device="cuda")
        assert torch.equal(blocks.dropout(x, blocks.Dropout(0.4, at, 3)), blocks.dropout(x, blocks.Dropout(0.4, seed, 3)))
    assert not torch.equal(blocks.dropout(x, blocks.Dropout(0.4, 5, 3)), blocks.dropout(x, blocks.Dropout(0.4, 5, 4)))
    kept = (blocks.dropout(torch.ones(1000, 1000, device="cuda"), blocks.Dropout(0.3, 1)) != 0).double().mean()
    assert abs(float(kept) - 0.7) < 5 * math.sqrt(0.21) / 1000


# ---- join

def setting(blocks, g, rows, cols, t, number, pad=0):
    """Keyword arguments of one of several kinds of join: for the library, and for the reference."""
    gate, p, post, pre, scale, x_scale = [(None, 0.0, None, "rms", 1.0, 1.0), ("columns", 0.25, None, None, 0.5, 1.0), ("groups", 0.1, "layer", "rms", 1.0, 1.0),
                                          (None, 0.0, "rms", "layer", -0.75, 0.5), ("columns", 0.5, "rms", "rms", 1.0, 1.0), ("groups", 0.0, "layer", "layer", 2.0, 3.0),
                                          ("rows", 0.1, "bare", "bare", 1.0, 1.0)][number]
    groups = {"groups": max(q for q in (1, 2, 3, 5) if rows % q == 0), "rows": rows}.get(gate, 1)
    gates = None if gate is None else vector(g, cols, t, 0.5) if gate == "columns" else matrix(g, groups, cols, t, pad, 0.5, 0.3)
    drop = blocks.Dropout(p, 1000 + number, number) if p else None

    def norm(kind):
        if kind is None:
            return None, None
        weight = None if kind == "bare" else vector(g, cols, t, 1.0)
        bias = vector(g, cols, t) if kind == "layer" else None
        kind = "layer" if kind == "bare" else kind
        eps = 1e-5 if kind == "layer" else 1e-6
        return blocks.Norm(kind, weight, bias, eps), (kind, double(weight), double(bias), float(np.float32(eps)))
    post, post_ref = norm(post)
    pre, pre_ref = norm(pre)
    mask = ref.kept(1000 + number, number, drop.threshold, rows, cols) if drop else None
    exact_p = drop.threshold / 65536 if drop else 0.0
    return (dict(gate=gates, scale=scale, x_scale=x_scale, dropout=drop, post=post, pre=pre),
            dict(gate=double(gates), scale=scale, x_scale=x_scale, mask=mask, p=exact_p, post=post_ref, pre=pre_ref))


def check_join(blocks, dtype, rows, cols, number, pad):
    t, g = TYPES[dtype], gen("join", dtype, rows, cols, number)
    kw, kw_ref = setting(blocks, g, rows, cols, t, number, pad)
    x, f = matrix(g, rows, cols, t, pad, 2.0, 0.5), matrix(g, rows, cols, t, 0, 0.7, -1.0)
    r = torch.full((rows, cols + pad), 7.0, dtype=t, device="cuda")
    got = blocks.join(x, f, out=r[:, :cols], **kw)
    got = {"r": got} if kw["pre"] is None else {"r": got[0], "h": got[1]}
    want = ref.join(double(x), double(f), **kw_ref)
    assert set(got) == set(want) and bool((r[:, cols:] == 7.0).all())
    for name in want:
        near(got[name], want[name], (name, number))


@pytest.mark.parametrize("cols", COLUMNS)
@pytest.mark.parametrize("dtype", TYPES)
def test_join(blocks, dtype, cols):
    for number in range(7):
        for rows in (1, 30):
            check_join(blocks, dtype, rows, cols, number, (0, 3, 8)[number % 3])


def test_join_of_many_rows(blocks):
    for rows, cols in ((70000, 8), (1200, 1000)):
        check_join(blocks, "bf16", rows, cols, 2, 0)


@pytest.mark.parametrize("kind", ["rms", "layer"])
@pytest.mark.parametrize("dtype", TYPES)
def test_norm(blocks, dtype, kind):
    t = TYPES[dtype]
    for rows, cols in ((1, 1), (1, 4096), (5, 100), (301, 128), (17, 9000)):
        g = gen("norm", dtype, kind, cols)
        x, w, b = matrix(g, rows, cols, t, 3, 1.0, 3.0), vector(g, cols, t, 1.0), vector(g, cols, t) if kind == "layer" else None
        want = ref.join(double(x), None, None, 1.0, 1.0, None, 0.0, None, (kind, double(w), double(b), float(np.float32(1e-5))))
        near(blocks.norm(x, blocks.Norm(kind, w, b)), want["h"], (rows, cols))
        y = x.clone()
        assert blocks.norm(y, blocks.Norm(kind, w, b), out=y) is y and torch.equal(y, blocks.norm(x, blocks.Norm(kind, w, b)))


def test_special_rows(blocks):
    """Rows of zeros, of one value, with an infinity or a NaN: only those rows show it."""
    for kind in ("rms", "layer"):
        x = matrix(gen("special"), 8, 500, torch.float32)
        x[1], x[2], x[3, 7], x[4, 9] = 0.0, 1000.25, float("inf"), float("nan")
        h = blocks.norm(x, blocks.Norm(kind, eps=1e-5))
        assert bool(h[3].isnan().any()) and bool(h[4].isnan().all()) and bool(h[[0, 1, 2, 5, 6, 7]].isfinite().all())
        assert bool((h[1] == 0).all())
        want = ref.Normed(double(x[[0, 2, 5]]), kind, None, None, float(np.float32(1e-5)))
        near(h[[0, 2, 5]], (want.value, want.off), kind)
        dx = blocks.norm_grad(torch.ones_like(x), x, blocks.Norm(kind, torch.ones(500, device="cuda"), eps=1e-5))
        assert bool(dx.dx[[0, 1, 2, 5, 6, 7]].isfinite().all()) and bool(dx.dx[4].isnan().all())
        # without eps a row of zeros has no size; the others do not notice
        bare = blocks.norm(x, blocks.Norm(kind, eps=0.0))
        assert bool(bare[1].isnan().all()) and bool(bare[[0, 5, 6, 7]].isfinite().all())


# ---- gradients

def check_grad(blocks, dtype, rows, cols, number, pad, run=None):
    t, g = TYPES[dtype], gen("grad", dtype, rows, cols, number)
    kw, kw_ref = setting(blocks, g, rows, cols, t, number, pad)
    f, r = matrix(g, rows, cols, t, pad, 0.7, -1.0), matrix(g, rows, cols, t, 0, 2.0, 0.5)
    dr = matrix(g, rows, cols, t, pad, 1e-2) if number != 3 else None
    dh = matrix(g, rows, cols, t, 0, 1e-2) if kw["pre"] is not None else None
    got = (run or blocks.join_grad)(dr, f, dh=dh, r=r if dh is not None else None, **kw)
    want = ref.join_grad(double(dr), double(f), double(dh), double(r), **kw_ref)
    for name, value in got._asdict().items():
        norm = {"pre": kw["pre"], "post": kw["post"]}.get(name.split("_")[0])
        there = getattr(norm, name.split("_")[1]) is not None if "_" in name and norm is not None else name in want
        assert (value is not None) == there, name
        if there:
            near(value, want[name], (name, number, rows))
    return got


@pytest.mark.parametrize("cols", COLUMNS)
@pytest.mark.parametrize("dtype", TYPES)
def test_join_grad(blocks, dtype, cols):
    for number in range(7):
        for rows in (1, 30):
            check_grad(blocks, dtype, rows, cols, number, (0, 3, 8)[number % 3])


@pytest.mark.parametrize("rows,cols", [(5000, 40), (3001, 129), (2100, 1000), (600, 8192), (600, 8200), (300, 12001)])
@pytest.mark.parametrize("number", [2, 4, 5, 6])
def test_join_grad_of_many_rows(blocks, rows, cols, number):
    check_grad(blocks, "bf16", rows, cols, number, 0)


@pytest.mark.parametrize("rows,gates,cols", [(600, 300, 8200), (1200, 600, 40), (1030, 515, 1001), (9, 9, 16384)])
@pytest.mark.parametrize("kind", [None, "rms", "layer"])
def test_more_gates_than_workgroups(blocks, rows, gates, cols, kind):          # workgroups that have several gates one after the other
    g = gen("gates", rows, cols, kind)
    f, dr = (matrix(g, rows, cols, torch.float32) for _ in range(2))
    gate = matrix(g, gates, cols, torch.float32, 0, 0.5)
    w = vector(g, cols, torch.float32, 1.0)
    post = blocks.Norm(kind, w) if kind else None
    got = blocks.join_grad(dr, f, gate=gate, post=post)
    want = ref.join_grad(double(dr), double(f), None, None, double(gate), 1.0, 1.0, None, 0.0, (kind, double(w), None, float(np.float32(1e-5))) if kind else None, None)
    near(got.gate, want["gate"], (kind, cols))
    near(got.df, want["df"], (kind, cols))
    if kind:
        near(got.post_weight, want["post_weight"], (kind, cols))
    held = torch.full_like(got.gate, 3.0)
    added = blocks.join_grad(dr, f, gate=gate, into=blocks.JoinGrads(gate=held), accumulate=True) if not kind else None
    assert added is None or bool(((held - 3.0 - got.gate).abs() <= 2.0 ** -23 * (3.0 + got.gate.abs())).all())


@pytest.mark.parametrize("kind", ["rms", "layer"])
def test_norm_grad(blocks, kind):
    for dtype, t in TYPES.items():
        for rows, cols in ((1, 7), (100, 64), (257, 1000), (33, 4096)):
            g = gen("norm_grad", dtype, kind, cols)
            x, dh, past = matrix(g, rows, cols, t, 3, 1.0, 3.0), matrix(g, rows, cols, t, 0, 0.1), matrix(g, rows, cols, t, 1, 0.1)
            w, b = vector(g, cols, t, 1.0), vector(g, cols, t) if kind == "layer" else None
            for residual in (None, past):
                got = blocks.norm_grad(dh, x, blocks.Norm(kind, w, b), residual=residual)
                want = ref.join_grad(double(residual), None, double(dh), double(x), None, 1.0, 1.0, None, 0.0, None, (kind, double(w), double(b), float(np.float32(1e-5))))
                near(got.dx, want["dx"], (kind, cols))
                near(got.pre_weight, want["pre_weight"], (kind, cols))
                assert (got.pre_bias is None) == (b is None) and got.df is None and got.gate is None
                if b is not None:
                    near(got.pre_bias, want["pre_bias"], (kind, cols))


def test_gradients_are_written_into_a_vector_and_added_to(blocks):
    for rows, cols, number in ((1, 100, 5), (30, 1000, 5), (900, 1000, 2), (900, 64, 5)):
        g = gen("into", rows, cols)
        kw, _ = setting(blocks, g, rows, cols, torch.float32, number)
        f, r, dr, dh = (matrix(g, rows, cols, torch.float32) for _ in range(4))
        plain = blocks.join_grad(dr, f, dh=dh, r=r, **kw)
        names = [n for n, v in plain._asdict().items() if v is not None and n not in ("dx", "df")]
        flat = torch.full((sum(getattr(plain, n).numel() + 3 for n in names),), 2.0, device="cuda")
        parts, at = {}, 0
        for n in names:
            like = getattr(plain, n)
            parts[n] = flat[at:at + like.numel()].view(like.shape)
            at += like.numel() + 3
        keep = {"dx": dr.clone(), "df": f.clone()}
        got = blocks.join_grad(keep["dx"], keep["df"], dh=dh, r=r, into=blocks.JoinGrads(dx=keep["dx"], df=keep["df"], **parts), **kw)
        assert got.dx is keep["dx"] and torch.equal(got.dx, plain.dx) and torch.equal(got.df, plain.df)
        for n in names:
            assert torch.equal(parts[n], getattr(plain, n)), n
        got = blocks.join_grad(dr, f, dh=dh, r=r, into=blocks.JoinGrads(**parts), accumulate=True, **kw)
        for n in names:
            assert torch.equal(parts[n], getattr(plain, n) * 2), n
        gaps = torch.ones_like(flat, dtype=torch.bool)
        at = 0
        for n in names:
            gaps[at:at + parts[n].numel()] = False
            at += parts[n].numel() + 3
        assert bool((flat[gaps] == 2.0).all())


def test_any_workspace_gives_the_gradients(blocks):
    from paper_2108_08842_amd import layers
    for rows, cols, number in ((500, 300, 5), (600, 1000, 2), (64, 64, 6), (301, 64, 4)):
        def run(dr, f, dh=None, r=None, size=0, **kw):
            # the binding with a workspace of another size
            full, fake = blocks.lib(), type("L", (), {})()
            fake.eden_join_workspace_bytes = lambda *a: size
            fake.eden_join_grad = full.eden_join_grad
            blocks._lib = fake
            try:
                return blocks.join_grad(dr, f, dh=dh, r=r, **kw)
            finally:
                blocks._lib = full
        need = int(blocks.lib().eden_join_workspace_bytes(rows, cols, 1, layers.F32))
        assert need > 0
        for size in (0, 16, 5000 * 4, 100000, need):
            check_grad(blocks, "f32", rows, cols, number, 0, run=lambda *a, size=size, **k: run(*a, size=size, **k))


def test_nothing_to_do(blocks):
    for rows, cols in ((0, 64), (5, 0), (0, 0)):
        x = torch.empty(rows, cols, device="cuda")
        w = torch.ones(cols, device="cuda")
        assert blocks.dropout(x, blocks.Dropout(0.1, 1)).shape == x.shape
        assert blocks.join(x, x, pre=blocks.Norm("rms", w))[1].shape == x.shape
        into = blocks.JoinGrads(gate=torch.full((cols,), 3.0, device="cuda"), pre_weight=torch.full((cols,), 3.0, device="cuda"))
        got = blocks.join_grad(x, x, dh=x, r=x, gate=w, pre=blocks.Norm("rms", w), into=into, accumulate=True)
        assert bool((got.gate == 3.0).all()) and bool((got.pre_weight == 3.0).all())
        got = blocks.join_grad(x, x, dh=x, r=x, gate=w, pre=blocks.Norm("rms", w))
        assert bool((got.gate == 0.0).all()) and bool((got.pre_weight == 0.0).all())      # a sum over nothing


def test_batches_and_gates_of_sequences(blocks):
    g = gen("batch")
    x, f = (torch.randn(3, 5, 40, generator=g).cuda() for _ in range(2))
    gate = torch.randn(3, 40, generator=g).cuda()
    r = blocks.join(x, f, gate=gate)
    assert r.shape == x.shape and torch.allclose(r, x + gate[:, None] * f, rtol=1e-6, atol=1e-6)
    grads = blocks.join_grad(x, f, gate=gate)
    assert grads.gate.shape == gate.shape and torch.allclose(grads.gate, (x * f).sum(1), rtol=1e-5, atol=1e-5)
    assert torch.allclose(grads.df, x * gate[:, None]) and torch.equal(grads.dx, x)


# ---- streams, graphs, both directions together

def test_on_another_stream(blocks):
    g = gen("stream")
    kw, _ = setting(blocks, g, 300, 500, torch.bfloat16, 4)
    x, f, dr, dh = (matrix(g, 300, 500, torch.bfloat16) for _ in range(4))
    want, want_grads = blocks.join(x, f, **kw), blocks.join_grad(dr, f, dh=dh, r=x, **kw)
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    got, got_grads = blocks.join(x, f, stream=stream, **kw), blocks.join_grad(dr, f, dh=dh, r=x, stream=stream, **kw)
    stream.synchronize()
    for a, b in zip(list(want) + list(want_grads), list(got) + list(got_grads)):
        assert (a is None and b is None) or torch.equal(a, b)


def test_captured_calls_draw_new_numbers_from_a_seed_on_the_device(blocks):
    g = gen("graph")
    seed = torch.zeros((), dtype=torch.int64, device="cuda")
    kw, _ = setting(blocks, g, 200, 600, torch.bfloat16, 4)
    kw["dropout"] = blocks.Dropout(0.3, seed, 2)
    x, f, dr, dh = (matrix(g, 200, 600, torch.bfloat16) for _ in range(4))

    def step():
        r, h = blocks.join(x, f, **kw)
        return [blocks.dropout(h, kw["dropout"]), r, h] + [v for v in blocks.join_grad(dr, f, dh=dh, r=r, **kw) if v is not None]
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        step()
    torch.cuda.current_stream().wait_stream(stream)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        captured = step()
    before = None
    for replay in range(4):
        seed.fill_(11 * replay)
        f.copy_(matrix(gen("graph", replay), 200, 600, torch.bfloat16))
        graph.replay()
        torch.cuda.synchronize()
        kw["dropout"] = blocks.Dropout(0.3, 11 * replay, 2)
        for a, b in zip(captured, step()):
            assert torch.equal(a, b)
        zeros = captured[0] == 0
        assert before is None or not torch.equal(zeros, before)
        before = zeros.clone()


def test_two_calls_at_once_and_the_same_bits_every_time(blocks):
    g = gen("twice")
    kw, _ = setting(blocks, g, 2000, 700, torch.float32, 5)
    f, r, dr, dh = (matrix(g, 2000, 700, torch.float32) for _ in range(4))
    want = blocks.join_grad(dr, f, dh=dh, r=r, **kw)
    streams = [torch.cuda.Stream() for _ in range(2)]
    for s in streams:
        s.wait_stream(torch.cuda.current_stream())
    got = [blocks.join_grad(dr, f, dh=dh, r=r, stream=s, **kw) for s in streams for _ in range(2)]
    torch.cuda.synchronize()
    for other in got:
        for a, b in zip(want, other):
            assert torch.equal(a, b)


def test_gradients_against_differences(blocks):
    """A small join in fp32, moved along random directions: (L(+t) - L(-t)) / 2t in 64 bits of the reference, gradients of the library."""
    rows, cols = 6, 40
    g = gen("differences")
    kw, kw_ref = setting(blocks, g, rows, cols, torch.float32, 5)
    x, f, wr, wh = (matrix(g, rows, cols, torch.float32) for _ in range(4))

    def loss(x64, f64, gate):
        out = ref.join(x64, f64, **dict(kw_ref, gate=gate))
        return float((out["r"][0] * double(wr)).sum() + (out["h"][0] * double(wh)).sum())
    r, _ = blocks.join(x, f, **kw)
    got = blocks.join_grad(wr, f, dh=wh, r=r, **kw)
    base = [double(x), double(f), kw_ref["gate"]]
    for i, grad in enumerate((got.dx, got.df, got.gate)):
        for _ in range(5):
            way = torch.randn(base[i].shape, generator=g, dtype=torch.float64)
            t = 1e-4
            ends = [loss(*[b + s * t * way if j == i else b for j, b in enumerate(base)]) for s in (1.0, -1.0)]
            slope = (ends[0] - ends[1]) / (2 * t)
            # r, rounded to fp32, and the gradients' own roundings: 1e-5 of the sum of sizes is a hundred of them; the third derivative's t^2 is below that
            assert abs(slope - float((double(grad) * way).sum())) <= 1e-5 * float((double(grad) * way).abs().sum()) + 1e-5


# ---- ends of the range

@pytest.mark.parametrize("cols", [5, 250, 1000, 1031, 4097, 8190, 16383])
@pytest.mark.parametrize("dtype", TYPES)
def test_results_in_the_place_of_operands(blocks, dtype, cols):
    """A result over the operand it replaces, with and without the sums over a row that keep a row's waves together."""
    t = TYPES[dtype]
    for number in (1, 4, 5):
        g = gen("place", dtype, cols, number)
        kw, _ = setting(blocks, g, 40, cols, t, number)
        x, f, dr, dh = (matrix(g, 40, cols, t, 3) for _ in range(4))
        want = blocks.join(x, f, **kw)
        want = (want, None) if kw["pre"] is None else want
        for place in (x, f):
            x2, f2 = x.clone(), f.clone()
            out = x2 if place is x else f2
            got = blocks.join(x2, f2, out=out, norm_out=None if kw["pre"] is None else (f2 if place is x else x2), **kw)
            got = (got, None) if kw["pre"] is None else got
            assert got[0] is out and torch.equal(got[0], want[0]) and (want[1] is None or torch.equal(got[1], want[1]))
        dh = dh if kw["pre"] is not None else None
        want = blocks.join_grad(dr, f, dh=dh, r=x, **kw)
        for place in range(3):
            if place and dh is None:
                continue
            operands = [dr.clone(), dh.clone() if dh is not None else None, x.clone()]
            f2 = f.clone()
            got = blocks.join_grad(operands[0], f2, dh=operands[1], r=operands[2], into=blocks.JoinGrads(dx=operands[place], df=f2), **kw)
            for a, b in zip(want, got):
                assert (a is None and b is None) or torch.equal(a, b)
        y = x.clone()
        assert torch.equal(blocks.dropout(y, blocks.Dropout(0.4, 3), out=y), blocks.dropout(x, blocks.Dropout(0.4, 3)))


@pytest.mark.parametrize("dtype", TYPES)
def test_operands_that_begin_anywhere(blocks, dtype):
    t = TYPES[dtype]
    for cols in (64, 1000, 1031, 4096):
        g = gen("anywhere", dtype, cols)
        kw, _ = setting(blocks, g, 20, cols, t, 5)

        def moved(v):
            if v is None:
                return None
            flat = torch.full((v.numel() + 8,), float("nan"), dtype=v.dtype, device="cuda")
            return flat[1:1 + v.numel()].view(v.shape).copy_(v)
        x, f, dr, dh = (matrix(g, 20, cols, t) for _ in range(4))
        kw2 = dict(kw, gate=moved(kw["gate"]), post=blocks.Norm("layer", moved(kw["post"].weight), moved(kw["post"].bias)), pre=blocks.Norm("layer", moved(kw["pre"].weight), moved(kw["pre"].bias)))
        for a, b in zip(blocks.join(x, f, **kw), blocks.join(moved(x), moved(f), out=moved(x), norm_out=moved(x), **kw2)):
            assert torch.equal(a, b)
        into = blocks.JoinGrads(dx=moved(x), df=moved(x))
        for a, b in zip(blocks.join_grad(dr, f, dh=dh, r=x, **kw), blocks.join_grad(moved(dr), moved(f), dh=moved(dh), r=moved(x), into=into, **kw2)):
            assert torch.equal(a, b)
        assert torch.equal(blocks.dropout(moved(x), blocks.Dropout(0.2, 1), out=moved(x)), blocks.dropout(x, blocks.Dropout(0.2, 1)))


def test_more_rows_than_workgroups_and_elements_than_32_bits_count(blocks):
    """The last rows of 2^32 elements and more, in more rows than the join has workgroups."""
    rows, cols, last, t = 2 ** 18 + 2 ** 15, 16384, 8, torch.bfloat16
    g = gen("large")
    words = (cols + 3) // 4
    bits = np.asarray(ref.oracle.hash_words(ref.oracle.stream_key(5, ref.STREAM_DROPOUT, 2), (rows - last) * words, last * words)).astype("<u8").view("<u2")
    mask = torch.from_numpy(bits.reshape(last, 4 * words)[:, :cols].astype(np.int64)) >= 16384

    def ending(tail):
        x = torch.zeros(rows, cols, dtype=t, device="cuda")
        x[-last:] = tail
        return x
    tails = [matrix(g, last, cols, t) for _ in range(4)]
    x, f = ending(tails[0]), ending(tails[1])
    drop, w = blocks.Dropout(0.25, 5, 2), vector(g, cols, t, 1.0)
    want = ref.join(double(tails[0]), double(tails[1]), None, 1.0, 1.0, mask, 0.25, None, ("rms", double(w), None, float(np.float32(1e-5))))
    r, h = blocks.join(x, f, dropout=drop, pre=blocks.Norm("rms", w), norm_out=f)
    near(r[-last:], want["r"], "r")
    near(h[-last:], want["h"], "h")
    assert not bool(h[:-last].any())
    y = blocks.dropout(x, drop, out=x)
    assert torch.equal(y[-last:].cpu(), torch.where(mask, tails[0].cpu().float() * torch.tensor(65536.0 / 49152, dtype=torch.float32), torch.zeros(())).to(t))
    dr, dh = ending(tails[2]), ending(tails[3])
    got = blocks.join_grad(dr, dh=dh, r=r, dropout=drop, pre=blocks.Norm("rms", w), into=blocks.JoinGrads(dx=dr, df=h))
    want = ref.join_grad(double(tails[2]), None, double(tails[3]), double(r[-last:]), None, 1.0, 1.0, mask, 0.25, None, ("rms", double(w), None, float(np.float32(1e-5))))
    near(got.dx[-last:], want["dx"], "dx")
    near(got.df[-last:], want["df"], "df")
    # (the zeros in front add nothing)
    near(got.pre_weight, (want["pre_weight"][0], want["pre_weight"][1] + 64 * ref.E * want["pre_weight"][0].abs()), "pre_weight")
