"""Layer norm on the device against 64 bits: forward with and without a checkpoint, backward from both, sums over rows."""
import numpy as np
import pytest
import torch

import paper_2506_22771_amd as ff
from norm_util import DTYPES, HALF_ULP, TINY, U, Framed, junk_ckpt, padded_ckpt, split_ckpt, typed, values, within
from oracle import norm_oracle as N

pytestmark = pytest.mark.gpu
EPS = 1e-5

# every way that rows are laid out over lanes: 4 to 64 lanes, workgroups of 256 to 1024, rows beyond the registers; widths at both sides of each
SHAPES = [(1, 1), (3, 5), (70, 32), (65, 33), (40, 64), (33, 100), (20, 128), (17, 129), (9, 256), (6, 300), (5, 512), (4, 513), (3, 784), (2, 2000),
          (300, 250), (2, 2049), (5, 4096), (2, 5000), (1, 8192), (3, 8200), (2, 16384), (2, 16390), (1, 32768), (2, 33000)]


def inputs(rows, cols, dtype, seed=0):
    rng = np.random.default_rng(rows * 7 + cols + seed)
    x = (rng.standard_normal((rows, cols)) * np.exp(0.5 * rng.standard_normal((1, cols))) + 0.5 * rng.standard_normal((1, cols))) \
        * np.exp(rng.standard_normal((rows, 1)))
    dy = rng.standard_normal((rows, cols)) * 0.1
    return typed(x, dtype), typed(dy, dtype), 1 + 0.3 * rng.standard_normal(cols), 0.3 * rng.standard_normal(cols)


# Sums: a lane adds up to 32 values (beyond 32768 columns up to cols / 1024), then six levels of lanes and up to sixteen wavefronts, so a sum is off by at
# most D = 32 + cols / 1024 + 24 roundings of the sum of magnitudes.
def depth(cols):
    return 56 + cols // 1024


def forward_bounds(x, w, b, dtype):
    """Bounds of y, mean, rstd (relative) and h."""
    y, h, mean, rstd = N.norm_forward(x, w, b, EPS)
    d = depth(x.shape[1])
    dmean = (d + 2) * U * np.abs(x).mean(1)
    # squares are taken around the rounded mean: that adds dmean^2, and every difference is rounded once
    var = 1 / rstd**2
    drel = 0.5 * ((d + 4) * U + dmean**2 / var) + U * np.abs(x).max(1) ** 2 / var * U + 6 * U
    dh = np.abs(h) * (drel + 3 * U)[:, None] + (rstd * dmean)[:, None] + U * np.abs(x) * rstd[:, None]
    wa, ba = np.abs(1.0 if w is None else w), np.abs(0.0 if b is None else b)
    dyy = wa * dh + 2 * U * (wa * np.abs(h) + ba)
    return (y, h, mean, rstd), (dyy * (1 + HALF_ULP[dtype]) + np.abs(y) * HALF_ULP[dtype] + TINY[dtype], dmean + 2 * U * np.abs(mean), drel * rstd, dh)


def check_kept(q, e, h, dh, cols, stochastic):
    """A checkpoint of h where h itself may be off by dh: the codes' rounding, the exponent's byte one way or the other at its edge."""
    gq, ge = split_ckpt(q, e, cols)
    step = np.repeat(np.exp2(ge.astype(np.float64) - 127), 32, 1)[:, :cols]
    within(N.ckpt_load(gq, ge), h, dh + step * (1.0 if stochastic else 0.5), "kept")
    for b in range(ge.shape[1]):
        at = slice(32 * b, min(cols, 32 * b + 32))
        low = np.maximum(np.abs(h[:, at]) - dh[:, at], 0).max(1)
        high = (np.abs(h[:, at]) + dh[:, at]).max(1)
        for r in range(0, h.shape[0], 1 if h.shape[0] <= 300 else 37):
            assert N.exponent_of(low[r]) <= ge[r, b] <= N.exponent_of(high[r]) or low[r] < 2.0**-100


@pytest.mark.parametrize("dtype", list(DTYPES))
@pytest.mark.parametrize("rows, cols", SHAPES)
def test_forward(rows, cols, dtype):
    x, _, w, b = inputs(rows, cols, dtype)
    odd = cols % 2 == 0    # odd strides and element offsets for the even widths; odd widths bring their own
    for params, left, right, stochastic in [("float32", 0, 0, False), (dtype, 1 if odd else 0, 4 if odd else 0, True)]:
        dw, db = typed(w, params), typed(b, params)
        fx, fy = Framed(rows, cols, dtype, left, right, x), Framed(rows, cols, dtype, right, left)
        (y, h, mean, rstd), (by, bm, br, bh) = forward_bounds(values(x), values(dw), values(db), dtype)
        gm, gr = torch.full((rows,), 7.0, device="cuda"), torch.full((rows,), 7.0, device="cuda")
        q, e = junk_ckpt(rows, cols)
        ff.ff_layer_norm_forward(fx.view, dw, db, EPS, fy.view, gm, gr, q, e, ff.ROUND_STOCHASTIC if stochastic else ff.ROUND_NEAREST, 3, 4)
        within(values(fy.view), y, by, "y")
        within(values(gm), mean, bm, "mean")
        within(values(gr), rstd, br, "rstd")
        check_kept(q, e, h, bh, cols, stochastic)
        assert fx.intact() and fy.intact()
        again = torch.empty((rows, cols), dtype=DTYPES[dtype], device="cuda")       # without the checkpoint: the same bits
        ff.ff_layer_norm_forward(fx.view, dw, db, EPS, again, None, None)
        assert torch.equal(again, fy.view)
        ff.ff_layer_norm_forward(fx.view, dw, db, EPS, fx.view, None, None)          # in place
        assert torch.equal(fx.view, again)


def test_forward_without_parameters_and_with_one():
    x, _, w, b = inputs(20, 300, "bfloat16")
    for pw, pb in [(None, None), (w, None), (None, b)]:
        y = torch.empty_like(x)
        dw, db = (typed(p, "float32") if p is not None else None for p in (pw, pb))
        ff.ff_layer_norm_forward(x, dw, db, EPS, y, None, None)
        (ry, *_), (by, *_) = forward_bounds(values(x), values(dw) if pw is not None else None, values(db) if pb is not None else None, "bfloat16")
        within(values(y), ry, by, "y")


def test_stochastic_checkpoint_is_that_of_the_rows_values():
    """Rows whose normalised values are exact in fp32: the fused checkpoint has the codes of ff_ckpt_store, bit for bit."""
    rows, cols = 40, 256
    x = torch.where(torch.rand((rows, cols), generator=torch.Generator().manual_seed(2)).argsort(1) < cols // 2, 1.0, -1.0).cuda()
    y = torch.empty_like(x)
    for mode in (ff.ROUND_NEAREST, ff.ROUND_STOCHASTIC):
        (q, e), (q2, e2) = junk_ckpt(rows, cols), junk_ckpt(rows, cols)
        ff.ff_layer_norm_forward(x, None, None, 3.0, y, None, None, q, e, mode, 11, 12)      # mean 0, variance 1, eps 3: halves
        assert torch.equal(y, x / 2)
        ff.ff_ckpt_store(y, mode, 11, 12, q2, e2)
        assert torch.equal(q, q2) and torch.equal(e, e2)


def test_a_row_far_from_zero_and_a_constant_row():
    x = np.random.default_rng(0).standard_normal((3, 1000)).astype(np.float32)
    x[0] += 4096
    x[1] = 5.0
    d = typed(x, "float32")
    y, m, r = torch.empty_like(d), torch.empty(3, device="cuda"), torch.empty(3, device="cuda")
    ff.ff_layer_norm_forward(d, None, None, EPS, y, m, r)
    (ry, _, rm, rr), (by, bm, br, _) = forward_bounds(values(d), None, None, "float32")
    within(values(y)[[0, 2]], ry[[0, 2]], by[[0, 2]], "y")
    within(values(r)[[0, 2]], rr[[0, 2]], br[[0, 2]], "rstd")
    assert abs(values(m)[1] - 5) < 5e-6 and np.abs(values(y)[1]).max() < 5e-6 / np.sqrt(EPS)


def test_infinities_and_nan_stay_in_their_rows():
    x, dy, w, b = inputs(6, 700, "float32")
    x[1, 3], x[3, 600], x[4, 0] = float("nan"), float("inf"), -float("inf")
    y, m, r = torch.empty_like(x), torch.empty(6, device="cuda"), torch.empty(6, device="cuda")
    q, e = junk_ckpt(6, 700)
    ff.ff_layer_norm_forward(x, None, None, EPS, y, m, r, q, e)
    bad = np.isnan(values(y)).any(1)
    assert list(bad) == [False, True, False, True, True, False]
    assert (split_ckpt(q, e, 700)[1][[1, 3, 4]] == 255).all() and (split_ckpt(q, e, 700)[1][[0, 2, 5]] != 255).all()
    dx = torch.empty_like(x)
    dw, db = torch.empty(700, device="cuda"), torch.empty(700, device="cuda")
    ws = torch.empty(ff.ff_layer_norm_workspace_bytes(6, 700), dtype=torch.uint8, device="cuda")
    for source in ("x", "kept"):
        ff.ff_layer_norm_backward(dy, x if source == "x" else None, m, q, e, r, None, dx, dw, db, False, ws)
        assert list(np.isnan(values(dx)).all(1)) == [False, True, False, True, True, False]
        assert np.isfinite(values(dx)[[0, 2, 5]]).all() and np.isnan(values(dw)).all() and np.isfinite(values(db)).all()


def backward_bounds(dy, h, dh, rstd, w, dtype):
    """dh: how far h itself may be off."""
    rows, cols = dy.shape
    dx, dw, db = N.norm_backward(dy, h, rstd, w)
    wa = np.abs(1.0 if w is None else w)
    g, d = np.abs(dy) * wa, depth(cols)
    c1, c2 = g.mean(1, keepdims=True), (g * np.abs(h)).mean(1, keepdims=True)
    err = (d + 4) * U * (c1 + np.abs(h) * c2) + dh * c2 + np.abs(h) * (g * dh).mean(1, keepdims=True) + 4 * U * (g + c1 + np.abs(h) * c2)
    err = rstd[:, None] * err + 2 * U * np.abs(dx)
    # column sums: a lane's rows (all of them at worst), the workgroup's groups and the workgroups', 64 + 64 + 16
    n = min(rows, 64 + rows // 64) + 144
    return (dx, dw, db), (err * (1 + HALF_ULP[dtype]) + np.abs(dx) * HALF_ULP[dtype] + TINY[dtype],
                          n * U * (np.abs(dy) * np.abs(h)).sum(0) + (np.abs(dy) * dh).sum(0), n * U * np.abs(dy).sum(0))


def run_backward(dy, x, mean, q, e, rstd, w, dx, accumulate=False, start=0.0):
    rows, cols = dy.shape
    dw, db = torch.full((cols,), start, device="cuda"), torch.full((cols,), start, device="cuda")
    ws = torch.full((ff.ff_layer_norm_workspace_bytes(rows, cols),), 255, dtype=torch.uint8, device="cuda")   # (NaN wherever it is read unwritten)
    ff.ff_layer_norm_backward(dy, x, mean, q, e, rstd, w, dx, dw, db, accumulate, ws)
    return dw, db


@pytest.mark.parametrize("dtype", list(DTYPES))
@pytest.mark.parametrize("rows, cols", SHAPES + [(5000, 40), (3000, 128), (2000, 513)])
def test_backward(rows, cols, dtype):
    x, dy, w, _ = inputs(rows, cols, dtype)
    odd = cols % 2 == 0
    xv = values(x)
    mean32, rstd32 = (a.astype(np.float32) for a in N.norm_forward(xv, None, None, EPS)[2:])
    m, r = torch.from_numpy(mean32).cuda(), torch.from_numpy(rstd32).cuda()
    hv = (xv - mean32[:, None].astype(np.float64)) * rstd32[:, None].astype(np.float64)
    rq, re = N.ckpt_store(hv.astype(np.float32))
    q, e = padded_ckpt(rq, re)
    for source, params, left, right in [("x", "float32", 0, 0), ("kept", dtype, 1 if odd else 0, 4 if odd else 0)]:
        h = hv if source == "x" else N.ckpt_load(rq, re)
        dh = 3 * U * np.abs(h) + (U * np.abs(xv) * rstd32[:, None] if source == "x" else 0)
        dw_ = typed(w, params)
        (rdx, rdw, rdb), (bx, bw, bb) = backward_bounds(values(dy), h, dh, rstd32.astype(np.float64), values(dw_), dtype)
        fdy, fdx = Framed(rows, cols, dtype, left, right, dy), Framed(rows, cols, dtype, right, left)
        fx = Framed(rows, cols, dtype, left, right, x)
        args = (fx.view if source == "x" else None, m if source == "x" else None, None if source == "x" else q, None if source == "x" else e, r)
        dw, db = run_backward(fdy.view, *args, dw_, fdx.view)
        within(values(fdx.view), rdx, bx, f"dx from {source}")
        within(values(dw), rdw, bw, f"dweight from {source}")
        within(values(db), rdb, bb, "dbias")
        assert fdy.intact() and fdx.intact() and fx.intact()
        # added to what is there; only some of the results; in place; the same bits every time
        aw, ab = run_backward(fdy.view, *args, dw_, None, True, 0.5)
        assert torch.equal(aw, dw + 0.5) and torch.equal(ab, db + 0.5)
        only = torch.empty((rows, cols), dtype=DTYPES[dtype], device="cuda")
        ws = torch.empty(ff.ff_layer_norm_workspace_bytes(rows, cols), dtype=torch.uint8, device="cuda")
        ff.ff_layer_norm_backward(fdy.view, *args, dw_, only, None, None, False, ws)
        assert torch.equal(only, fdx.view)
        one = torch.empty(cols, device="cuda")
        ff.ff_layer_norm_backward(fdy.view, *args, dw_, None, None, one, False, ws)
        assert torch.equal(one, db)
        run_backward(fdy.view, *args, dw_, fdy.view)
        assert torch.equal(fdy.view, only)


def test_backward_without_rows_and_without_a_weight():
    for cols in (5, 300, 20000):
        dy = torch.empty((0, cols), device="cuda")
        q, e = ff.ckpt_empty(0, cols)
        none = torch.empty(0, device="cuda")
        dw, db = run_backward(dy, None, None, q, e, none, None, dy, False, 9.0)
        assert not dw.any() and not db.any()
        dw, db = run_backward(dy, None, None, q, e, none, None, dy, True, 9.0)
        assert (dw == 9).all() and (db == 9).all()
    x, dy, _, _ = inputs(10, 70, "float32")
    _, h, mean, rstd = N.norm_forward(values(x), None, None, EPS)
    m, r = torch.from_numpy(mean.astype(np.float32)).cuda(), torch.from_numpy(rstd.astype(np.float32)).cuda()
    dx = torch.empty_like(x)
    run_backward(dy, x, m, None, None, r, None, dx)
    hv = (values(x) - values(m)[:, None]) * values(r)[:, None]
    (ref, *_), (bound, *_) = backward_bounds(values(dy), hv, 4 * U * (np.abs(hv) + np.abs(values(x)) * rstd[:, None]), values(r), None, "float32")
    within(values(dx), ref, bound, "dx")


@pytest.mark.parametrize("cols", [7, 96, 600])
def test_gradients_against_differences(cols):
    """Central differences of sum dy * norm(x) in 64 bits (error 1e-8), where fp32 gives 1e-5."""
    x, dy, w, b = inputs(4, cols, "float32")
    xv, dyv, wv, bv = values(x), values(dy), w.astype(np.float32).astype(np.float64), b.astype(np.float32).astype(np.float64)
    dw_, db_ = typed(w, "float32"), typed(b, "float32")
    y, m, r, dx = torch.empty_like(x), torch.empty(4, device="cuda"), torch.empty(4, device="cuda"), torch.empty_like(x)
    ff.ff_layer_norm_forward(x, dw_, db_, 1e-3, y, m, r)
    gw, gb = run_backward(dy, x, m, None, None, r, dw_, dx)
    loss = lambda x, w, b: float((dyv * N.norm_forward(x, w, b, 1e-3)[0]).sum())  # noqa: E731
    d = 1e-5
    rng = np.random.default_rng(1)
    for _ in range(12):
        at, k = (int(rng.integers(4)), int(rng.integers(cols))), int(rng.integers(cols))
        one, col = np.zeros_like(xv), np.zeros(cols)
        one[at], col[k] = d, d
        size = max(1.0, float(values(r)[at[0]]))
        assert abs((loss(xv + one, wv, bv) - loss(xv - one, wv, bv)) / (2 * d) - values(dx)[at]) < 1e-4 * size
        assert abs((loss(xv, wv + col, bv) - loss(xv, wv - col, bv)) / (2 * d) - values(gw)[k]) < 1e-4
        assert abs((loss(xv, wv, bv + col) - loss(xv, wv, bv - col)) / (2 * d) - values(gb)[k]) < 1e-4


def test_rows_beyond_32_bits_of_offset():
    """Rows that lie more than 2^32 bytes and 2^32 elements apart from the first."""
    rows, cols, ld = 4, 200, (1 << 31) - 37
    buffer = torch.empty(3 * ld + cols, dtype=torch.bfloat16, device="cuda")
    view = buffer.as_strided((rows, cols), (ld, 1))
    x, dy, w, b = inputs(rows, cols, "bfloat16")
    view.copy_(x)
    dw_, db_ = typed(w, "float32"), typed(b, "float32")
    near, m, r = torch.empty_like(x), torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda")
    ff.ff_layer_norm_forward(x, dw_, db_, EPS, near, m, r)
    ff.ff_layer_norm_forward(view, dw_, db_, EPS, view, None, None)
    assert torch.equal(view, near)
    view.copy_(x)
    dx = torch.empty_like(x)
    run_backward(dy, x, m, None, None, r, dw_, dx)
    run_backward(dy, view, m, None, None, r, dw_, view)
    assert torch.equal(view, dx)


def test_calls_in_a_graph():
    """Captured once, replayed over new inputs with eager work between: as eager calls."""
    rows, cols = 50, 900
    x, dy, w, b = inputs(rows, cols, "bfloat16")
    dw_, db_ = typed(w, "float32"), typed(b, "float32")
    y, m, r, dx = torch.empty_like(x), torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda"), torch.empty_like(x)
    q, e = ff.ckpt_empty(rows, cols)
    gw, gb = torch.empty(cols, device="cuda"), torch.empty(cols, device="cuda")
    dW, dB = torch.empty((64, cols), device="cuda"), torch.empty(64, device="cuda")
    ws = torch.empty(ff.ff_layer_norm_workspace_bytes(rows, cols), dtype=torch.uint8, device="cuda")
    wws = torch.empty(ff.ff_ckpt_weight_grad_workspace_bytes(rows, 64, cols), dtype=torch.uint8, device="cuda")
    up = typed(np.random.default_rng(0).standard_normal((rows, 64)), "bfloat16")

    def step():
        ff.ff_layer_norm_forward(x, dw_, db_, EPS, y, m, r, q, e, ff.ROUND_STOCHASTIC, 1, 2)
        ff.ff_layer_norm_backward(dy, None, None, q, e, r, dw_, dx, gw, gb, False, ws)
        ff.ff_ckpt_weight_grad(up, q, e, dw_, db_, dW, dB, False, wws)

    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for i in range(4):
        x.copy_(inputs(rows, cols, "bfloat16", seed=100 + i)[0])
        graph.replay()
        got = [t.clone() for t in (y, dx, gw, gb, dW, dB)]
        torch.cuda.synchronize()
        step()
        assert all(torch.equal(a, b) for a, b in zip(got, (y, dx, gw, gb, dW, dB)))


# More rows than groups run at once, so that they go row after row, at every group that does: 64 lanes (1024 workgroups of four rows), 128 (2048 workgroups) to
# 1024 (256), and the backward pass' few workgroups; whole chunks and rows that end inside one
LONG = [(4400, 784, "float32"), (4200, 1001, "bfloat16"), (2200, 1500, "float16"), (1200, 3001, "float32"), (600, 6002, "bfloat16"), (300, 12001, "float16"),
        (260, 16384, "bfloat16"), (8200, 1030, "bfloat16"), (8200, 1041, "float32"),
        (1030, 6002, "float16"), (520, 12001, "bfloat16"), (520, 16384, "float32")]


@pytest.mark.parametrize("rows, cols, dtype", LONG)
def test_row_after_row(rows, cols, dtype):
    test_forward(rows, cols, dtype)
    test_backward(rows, cols, dtype)


@pytest.mark.parametrize("dtype", list(DTYPES))
@pytest.mark.parametrize("rows, cols", [(70, 6), (65, 33), (33, 100), (9, 500), (4200, 1001), (2200, 1500), (300, 12001), (3, 33001)])
def test_in_place(rows, cols, dtype):
    """A row that ends inside a chunk is read by two lanes in part; all of it before any of it is written."""
    x, dy, w, b = inputs(rows, cols, dtype)
    w, b = typed(w, "float32"), typed(b, "float32")
    m, r, y = torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda"), torch.empty_like(x)
    ff.ff_layer_norm_forward(x, w, b, EPS, y, m, r)
    q, e = ff.ckpt_empty(rows, cols)
    q2, e2 = ff.ckpt_empty(rows, cols)
    ff.ff_layer_norm_forward(x, w, b, EPS, torch.empty_like(x), m, r, q, e, ff.ROUND_STOCHASTIC, 1, 2)
    dx = torch.empty_like(x)
    run_backward(dy, x, m, None, None, r, w, dx)
    over_x, over_dy = x.clone(), dy.clone()
    run_backward(dy, over_x, m, None, None, r, w, over_x)
    run_backward(over_dy, x, m, None, None, r, w, over_dy)
    assert torch.equal(over_x, dx) and torch.equal(over_dy, dx)
    ff.ff_layer_norm_forward(x, w, b, EPS, x, m, r, q2, e2, ff.ROUND_STOCHASTIC, 1, 2)
    assert torch.equal(x, y) and torch.equal(q, q2) and torch.equal(e, e2)
