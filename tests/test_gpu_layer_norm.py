"""GPU layer norm and its gradients against the fp64 reference.

Tolerances.  fp32 arithmetic on n terms: a sum held in fp32 over lanes is off
by at most about log2(n) + 64 half steps (64 terms a thread, then a tree) of
2^-24 of the sum of magnitudes, below 1e-5 for every size here; relative to
values that the sums are added to, 2e-5 covers each fp32 output.  bf16 outputs
add one rounding, half a step: 2^-8 of the value with eps / 2 = 2^-8 for bf16.
"""
import numpy as np
import pytest
import torch

import paper_2609_23153_amd as sa
from gpu_helpers import say
from oracle import layer_norm as R

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
F32 = 2e-5


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.fail("GPU tests need a GPU")
    sa.library()
    yield
    torch.cuda.synchronize()


def make(rows, cols, dtype, groups, pad=0, seed=0, shift=0.3):
    g = torch.Generator().manual_seed(1000 * rows + cols + seed)
    rnd = lambda *s: torch.randn(*s, generator=g)
    x = (rnd(rows, cols) * torch.exp(0.5 * rnd(rows, 1)) + shift * rnd(rows, 1)).to(dtype)
    dy = rnd(rows, cols).to(dtype)
    w = None if groups == 0 else (1 + 0.3 * rnd(groups, cols))
    b = None if groups == 0 else 0.3 * rnd(groups, cols)
    on = lambda t: None if t is None else t.to(DEV)

    def padded(t):  # rows with `pad` more elements between them
        buf = torch.full((rows, cols + pad), 7.0, dtype=dtype, device=DEV)
        buf[:, :cols] = t.to(DEV)
        return buf[:, :cols]

    return padded(x), padded(dy), on(w), on(b), padded


def near(got, want, scale, what):
    """|got - want| <= tol * scale, scale the magnitudes that the sums hold."""
    got = got.double().cpu().numpy()
    err = np.abs(got - want)
    say(f"  {what}: worst {float((err / scale).max()) if err.size else 0.0:.2e} of the bound")
    assert np.all(err <= scale), what


SHAPES = [(1, 1), (1, 8), (3, 7), (5, 64), (7, 511), (4, 512), (9, 513), (64, 1536), (33, 1531),
          (6, 2048), (10, 2049), (12, 5120), (5, 6144), (6, 6145), (3, 8960), (2, 16384), (3, 16383),
          (3000, 96), (50, 9), (700, 15), (21, 127), (40, 128), (17, 129), (9, 1023), (9, 1025),
          (10, 4095), (5, 4097), (4, 12287), (4, 12288), (3, 12289), (5000, 100)]


def check(rows, cols, dtype, groups, pad=0, eps=1e-6, shift=0.3):
    x, dy, w, b, padded = make(rows, cols, dtype, groups, pad, shift=shift)
    y = padded(torch.zeros(rows, cols, dtype=dtype))
    out, mean, rstd = sa.sparse_attn_layer_norm(x, w, b, eps=eps, y=y)
    assert out.data_ptr() == y.data_ptr()
    xs = x.double().cpu().numpy()
    wn = None if w is None else w.double().cpu().numpy()
    ry, rm, rr = R.layer_norm(xs, wn, None if b is None else b.double().cpu().numpy(), eps)
    half = torch.finfo(dtype).eps / 2 if dtype == torch.bfloat16 else 0.0
    size = np.abs(xs).max(1)
    near(mean, rm, F32 * size + 1e-30, "mean")
    near(rstd, rr, F32 * rr * np.maximum(1, (size * rr) ** 2 * 2.0 ** -20), "rstd")
    # y: the row's largest normalised value times the weights carries the fp32 error
    amp = (size * rr)[:, None] * (1.0 if wn is None else np.abs(wn).max()) + 1.0
    near(out, ry, half * np.abs(ry) + F32 * amp, "y")
    if pad:
        tail = y.as_strided((rows, pad), (cols + pad, 1), cols) if rows > 1 else None
        assert tail is None or bool((tail == 7.0).all()), "rows' padding was written"
    dx, dw, db = sa.sparse_attn_layer_norm_bwd(dy, x, mean, rstd, w)
    ds = dy.double().cpu().numpy()
    rdx, rdw, rdb = R.layer_norm_bwd(ds, xs, mean.double().cpu().numpy(),
                                     rstd.double().cpu().numpy(), wn, max(groups, 1))
    xh = np.abs((xs - mean.double().cpu().numpy()[:, None]) * rstd.double().cpu().numpy()[:, None])
    g = np.abs(ds) * (1.0 if wn is None else np.abs(np.repeat(wn, rows // groups, 0)))
    amp = rstd.double().cpu().numpy()[:, None] * (
        g + g.mean(1, keepdims=True) + xh * (g * xh).mean(1, keepdims=True))
    near(dx, rdx, half * np.abs(rdx) + F32 * amp + 1e-30, "dx")
    split = lambda t: t.reshape(max(groups, 1), -1, cols).sum(1)
    # (x - mean) rstd carries three fp32 roundings of values up to |x| rstd
    reach = np.abs(ds) * (xh + size[:, None] * rstd.double().cpu().numpy()[:, None])
    near(dw.reshape(-1, cols), rdw, F32 * split(reach) + 1e-30, "dweight")
    near(db.reshape(-1, cols), rdb, F32 * split(np.abs(ds)) + 1e-30, "dbias")
    return x, dy, w, b, mean, rstd, dx, dw, db


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "fp32"])
@pytest.mark.parametrize("rows,cols", SHAPES)
def test_shapes(rows, cols, dtype):
    check(rows, cols, dtype, 1)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "fp32"])
@pytest.mark.parametrize("groups,rows,cols,pad", [(0, 12, 320, 8), (2, 14, 1536, 8), (3, 9, 1000, 3),
                                                  (5, 5, 77, 1), (4, 8192 * 2, 64, 0),
                                                  (2, 4 * 1024 + 2, 2056, 0)])
def test_groups_strides_and_long_walks(groups, rows, cols, pad, dtype):
    check(rows, cols, dtype, groups, pad)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "fp32"])
@pytest.mark.parametrize("cols", [1, 7, 8, 9, 64, 125, 700, 1531, 4099, 9001, 12300])
def test_rows_that_start_at_odd_elements(cols, dtype):
    # one column in from an aligned buffer, with strides that keep no row aligned:
    # the same bytes as for the same rows side by side, the columns around untouched
    rows, pad = 70, 3
    g = torch.Generator().manual_seed(cols)
    x, dy = (torch.randn(rows, cols, generator=g).to(dtype).to(DEV) for _ in range(2))
    w, b = (torch.randn(2, cols, generator=g).to(DEV) for _ in range(2))

    def shifted(t):
        buf = torch.full((rows, cols + pad), 7.0, dtype=dtype, device=DEV)
        buf[:, 1:cols + 1] = t
        return buf, buf[:, 1:cols + 1]

    y, mean, rstd = sa.sparse_attn_layer_norm(x, w, b)
    dx, dw, db = sa.sparse_attn_layer_norm_bwd(dy, x, mean, rstd, w)
    xb, xs = shifted(x)
    db_, ds = shifted(dy)
    got = sa.sparse_attn_layer_norm_bwd(ds, xs, mean, rstd, w, dx=ds)        # in place
    for a, c in zip(got, (dx, dw, db)):
        assert torch.equal(a, c)
    out, m, r = sa.sparse_attn_layer_norm(xs, w, b, y=xs)
    assert torch.equal(out, y) and torch.equal(m, mean) and torch.equal(r, rstd)
    for buf in (xb, db_):
        assert bool((buf[:, 0] == 7.0).all()) and bool((buf[:, cols + 1:] == 7.0).all())


def test_large_mean_keeps_the_variance():
    # rows whose mean is far larger than their spread: a difference of squares
    # would lose every digit
    x, *_ = make(8, 5120, torch.float32, 0, shift=0.0)
    x = x + 1000.0
    y, mean, rstd = sa.sparse_attn_layer_norm(x)
    ry, rm, rr = R.layer_norm(x.double().cpu().numpy())
    # the mean is off by at most 64 + 13 half steps of 1000, 5e-3; its square enters
    # the variance relative to 1; measured rows are exact to a few 2^-24
    near(mean, rm, np.full(8, 1000 * 77 * 2.0 ** -24), "mean")
    near(rstd, rr, rr * 1e-4, "rstd")


def test_zero_rows_constant_rows_and_empty_calls():
    x = torch.zeros(4, 100, device=DEV)
    x[1] = 5.0
    y, mean, rstd = sa.sparse_attn_layer_norm(x, eps=0.25)
    assert torch.equal(y, torch.zeros_like(x)) and torch.equal(rstd, torch.full((4,), 2.0, device=DEV))
    assert mean.tolist() == [0.0, 5.0, 0.0, 0.0]
    e = torch.empty(0, 100, device=DEV)
    y, mean, rstd = sa.sparse_attn_layer_norm(e)
    assert y.shape == (0, 100)
    dx, dw, db = sa.sparse_attn_layer_norm_bwd(e, e, mean, rstd, groups=2)
    assert dx.shape == (0, 100) and torch.equal(dw, torch.zeros(2, 100, device=DEV))
    assert torch.equal(db, dw)


def test_in_place_equals_out_of_place_and_repeats_bit_for_bit():
    x, dy, w, b, mean, rstd, dx, dw, db = check(777, 1536, torch.bfloat16, 3)
    y, *_ = sa.sparse_attn_layer_norm(x, w, b)
    again = sa.sparse_attn_layer_norm_bwd(dy, x, mean, rstd, w)
    for a, c in zip(again, (dx, dw, db)):
        assert torch.equal(a, c)
    z = x.clone()
    sa.sparse_attn_layer_norm(z, w, b, y=z)
    assert torch.equal(z, y)
    d = dy.clone()
    sa.sparse_attn_layer_norm_bwd(d, x, mean, rstd, w, dx=d)
    assert torch.equal(d, dx)
    only, none, nope = sa.sparse_attn_layer_norm_bwd(dy, x, mean, rstd, w, with_wgrad=False)
    assert torch.equal(only, dx) and none is None and nope is None


def test_larger_than_the_caches_equals_its_parts():
    # rows that are kept out of the caches (over 512 MB) against the same rows a
    # part at a time; fp32 and bf16, whole and with a padded row, aligned or not
    for dtype, rows, cols, pad in ((torch.bfloat16, 14000, 10240, 0), (torch.float32, 9001, 8200, 8),
                                    (torch.bfloat16, 30000, 5120, 3), (torch.bfloat16, 1200001, 128, 1)):
        g = torch.Generator(device=DEV).manual_seed(rows)
        rnd = lambda *s: torch.randn(*s, generator=g, device=DEV)
        x, dy = (rnd(rows, cols + pad).to(dtype)[:, :cols] for _ in range(2))
        w, b = 1 + 0.3 * rnd(cols), rnd(cols)
        y, mean, rstd = sa.sparse_attn_layer_norm(x, w, b)
        dx, dw, db = sa.sparse_attn_layer_norm_bwd(dy, x, mean, rstd, w)
        sw, sb = torch.zeros(2, cols, dtype=torch.float64, device=DEV)
        for r in range(0, rows, 1500):
            part = slice(r, r + 1500)
            py, pm, pr = sa.sparse_attn_layer_norm(x[part], w, b)
            assert torch.equal(py, y[part]) and torch.equal(pm, mean[part]) and torch.equal(pr, rstd[part])
            pdx, pdw, pdb = sa.sparse_attn_layer_norm_bwd(dy[part], x[part], pm, pr, w)
            assert torch.equal(pdx, dx[part])
            sw += pdw
            sb += pdb
        # sums of `rows` terms of size about 1 (dy xh): two orders of fp32 additions
        # differ by at most 2 F32 of the sum of magnitudes, below 2 F32 rows here
        assert (dw - sw).abs().max() <= 2 * F32 * rows and (db - sb).abs().max() <= 2 * F32 * rows


def test_captured_and_replayed():
    x, dy, w, b, _ = make(300, 2056, torch.bfloat16, 1)
    step = lambda: (lambda y, m, r: (y,) + sa.sparse_attn_layer_norm_bwd(dy, x, m, r, w))(
        *sa.sparse_attn_layer_norm(x, w, b))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = step()
    for k in range(3):
        x.copy_(torch.randn(300, 2056, device=DEV) * (k + 1))
        dy.copy_(torch.randn(300, 2056, device=DEV))
        graph.replay()
        want = step()
        torch.cuda.synchronize()
        for a, c in zip(out, want):
            assert torch.equal(a, c), k
