"""Weight gradients from 8-bit checkpoints against 64 bits."""
import numpy as np
import pytest
import torch

import paper_2506_22771_amd as ff
from norm_util import DTYPES, U, Framed, padded_ckpt, typed, values, within
from oracle import norm_oracle as N

pytestmark = pytest.mark.gpu


def run(dy, q, e, k, gamma=None, beta=None, accumulate=False, start=7.0, with_db=True):
    rows, n = dy.shape
    dw, db = torch.full((n, k), start, device="cuda"), torch.full((n,), start, device="cuda") if with_db else None
    ws = torch.full((ff.ff_ckpt_weight_grad_workspace_bytes(rows, n, k),), 255, dtype=torch.uint8, device="cuda")   # (NaN wherever it is read unwritten)
    ff.ff_ckpt_weight_grad(dy, q, e, gamma, beta, dw, db, accumulate, ws)
    return dw, db


def checkpoint(rows, k, seed):
    rng = np.random.default_rng(seed)
    rq, re = N.ckpt_store((rng.standard_normal((rows, k)) * np.exp(rng.standard_normal((rows, 1)))).astype(np.float32))
    return rq, re, *padded_ckpt(rq, re)


# from one row to several splits of the rows; n and k at both sides of tiles, chunks and blocks (all by the tile of 64 outputs; test_gpu_ckpt_wgrad_tiles.py has the others)
SHAPES = [(1, 1, 1), (1, 5, 33), (2, 300, 7), (31, 8, 32), (32, 64, 64), (33, 65, 63), (64, 100, 257), (100, 129, 40), (128, 500, 784), (65, 640, 650), (1000, 3, 2),
          (777, 17, 1000), (2048, 200, 96), (5000, 70, 130), (40000, 24, 32), (300, 1100, 1030)]


@pytest.mark.parametrize("dtype", list(DTYPES))
@pytest.mark.parametrize("rows, n, k", SHAPES)
def test_against_64_bits(rows, n, k, dtype):
    """Products are exact and sums fp32: off by at most one rounding per row of the sum of magnitudes, and five for gamma, beta and splits."""
    rng = np.random.default_rng(rows + n + k)
    rq, re, q, e = checkpoint(rows, k, rows)
    h = N.ckpt_load(rq, re)
    left, right = (0, 0) if n % 2 else (1, 2)
    dy = Framed(rows, n, dtype, left, right, typed(rng.standard_normal((rows, n)) * np.exp(rng.standard_normal((rows, 1))), dtype))
    dyv = values(dy.view)
    for params in (None, "float32", dtype):
        g, b = (None, None) if params is None else (typed(1 + 0.3 * rng.standard_normal(k), params), typed(0.3 * rng.standard_normal(k), params))
        gv, bv = (None, None) if params is None else (values(g), values(b))
        dw, db = run(dy.view, q, e, k, g, b)
        rw, rb = N.weight_grad(dyv, h, gv, bv)
        size = np.abs(dyv).T @ np.abs(h) * (1 if gv is None else np.abs(gv)) + (0 if bv is None else np.abs(dyv).sum(0)[:, None] * np.abs(bv))
        within(values(dw), rw, (rows + 5) * U * size, "dw")
        within(values(db), rb, (rows + 5) * U * np.abs(dyv).sum(0), "db")
        rms = np.sqrt((rw**2).mean())
        assert np.sqrt(((values(dw) - rw) ** 2).mean()) <= 2e-6 * max(rms, 1e-30) * np.sqrt(max(1.0, rows / 1000))   # (roundings are not all one way)
        assert dy.intact()
    aw, ab = run(dy.view, q, e, k, g, b, True, 0.5)
    assert torch.equal(aw, dw + 0.5) and torch.equal(ab, db + 0.5)
    only, _ = run(dy.view, q, e, k, g, b, with_db=False)
    assert torch.equal(only, dw)


@pytest.mark.parametrize("dtype", list(DTYPES))
@pytest.mark.parametrize("rows, n, k", [(200, 96, 70), (64, 512, 300), (9000, 40, 40)])
def test_whole_numbers_are_exact(rows, n, k, dtype):
    """Small whole numbers, whose sums fp32 holds: every row and column in its place, bit for bit."""
    rng = np.random.default_rng(k)
    rq = rng.integers(-127, 128, (rows, k)).astype(np.int8)
    re = np.full((rows, (k + 31) // 32), 127, np.uint8)
    q, e = padded_ckpt(rq, re)
    dy = rng.integers(-7, 8, (rows, n)).astype(np.float32)
    dw, db = run(typed(dy, dtype), q, e, k)
    np.testing.assert_array_equal(values(dw), dy.T.astype(np.float64) @ rq.astype(np.float64))
    np.testing.assert_array_equal(values(db), dy.astype(np.float64).sum(0))


@pytest.mark.parametrize("dtype", list(DTYPES))
def test_all_bits_of_dy_count(dtype):
    """One row: a product of all of dy's bits with a checkpoint's, formed from up to three exact terms, is off by their two sums' roundings at most."""
    rng = np.random.default_rng(1)
    rq, re, q, e = checkpoint(1, 64, 3)
    size = 20 if dtype == "float16" else 60
    dy = typed(rng.standard_normal((1, 300)) * np.exp2(rng.uniform(-size / 2, size / 4, (1, 300))), dtype)
    dw, _ = run(dy, q, e, 64)
    ref = values(dy).T @ N.ckpt_load(rq, re)
    within(values(dw), ref, 3 * U * np.abs(ref), "dw")
    if dtype == "bfloat16":
        within(values(dw), ref, U * np.abs(ref), "dw")


def test_no_rows():
    q, e = ff.ckpt_empty(0, 40)
    for dtype in DTYPES.values():
        dy = torch.empty((0, 24), dtype=dtype, device="cuda")
        dw, db = run(dy, q, e, 40, None, torch.ones(40, device="cuda"))
        assert not dw.any() and not db.any()
        dw, db = run(dy, q, e, 40, None, None, True)
        assert (dw == 7).all() and (db == 7).all()


@pytest.mark.parametrize("dtype", list(DTYPES))
def test_infinities_and_nan_go_where_the_sums_put_them(dtype):
    """A NaN of dy spoils its row of dw, an infinity leaves infinities or, against a zero, NaN; a block that reads as NaN spoils its columns.  All else is as without."""
    rows, n, k = 150, 70, 100
    rng = np.random.default_rng(5)
    rq, re, _, _ = checkpoint(rows, k, 6)
    re[140, 1] = 255
    rq[140, 32:64] = 0
    q, e = padded_ckpt(rq, re)
    base = rng.standard_normal((rows, n)).astype(np.float32)
    clean = values(run(typed(base, dtype), *padded_ckpt(rq, np.where(re == 255, 127, re)), k)[0])
    base[149, 3], base[7, 9], base[100, 69] = np.nan, np.inf, -np.inf
    dw, db = run(typed(base, dtype), q, e, k)
    got, h = values(dw), N.ckpt_load(rq, re)
    assert np.isnan(got[3]).all() and np.isnan(got[:, 32:64]).all()
    others = [c for c in range(k) if not 32 <= c < 64]
    for row, m in ((9, 7), (69, 100)):
        sign = np.sign(base[m, row]) * np.sign(h[m, others])
        np.testing.assert_array_equal(got[row, others], np.where(sign == 0, np.nan, sign * np.inf))
    fine = [r for r in range(n) if r not in (3, 9, 69)]
    np.testing.assert_array_equal(got[np.ix_(fine, others)], clean[np.ix_(fine, others)])
    sums = values(db)
    assert np.isnan(sums[3]) and sums[9] == np.inf and sums[69] == -np.inf and np.isfinite(sums[fine]).all()


def test_behind_a_norm_it_is_the_layers_gradient():
    """d/dW of sum dy * (W (gamma h + beta)) by differences: linear in W, so exact up to fp32's sums."""
    rng = np.random.default_rng(2)
    rows, n, k = 40, 6, 50
    rq, re, q, e = checkpoint(rows, k, 9)
    h = N.ckpt_load(rq, re)
    g, b, dy = 1 + rng.standard_normal(k), rng.standard_normal(k), rng.standard_normal((rows, n))
    dg, db_, ddy = typed(g, "float32"), typed(b, "float32"), typed(dy, "float32")
    a, W = h * values(dg) + values(db_), rng.standard_normal((n, k))
    loss = lambda W: float((values(ddy) * (a @ W.T)).sum())  # noqa: E731
    dw = values(run(ddy, q, e, k, dg, db_)[0])
    for _ in range(10):
        at = int(rng.integers(n)), int(rng.integers(k))
        one = np.zeros_like(W)
        one[at] = 1.0
        assert abs((loss(W + one) - loss(W - one)) / 2 - dw[at]) < 1e-4


def test_same_bits_every_time():
    rq, re, q, e = checkpoint(3000, 500, 1)
    dy = typed(np.random.default_rng(0).standard_normal((3000, 260)), "float32")
    first = run(dy, q, e, 500)
    for _ in range(3):
        again = run(dy, q, e, 500)
        assert torch.equal(first[0], again[0]) and torch.equal(first[1], again[1])


def test_rows_beyond_32_bits_of_offset():
    rows, n, k, ld = 70, 40, 64, (1 << 26) + 5      # 70 rows: 4.7e9 elements
    rq, re, q, e = checkpoint(rows, k, 2)
    dy = typed(np.random.default_rng(0).standard_normal((rows, n)), "bfloat16")
    far = torch.empty((rows - 1) * ld + n, dtype=torch.bfloat16, device="cuda").as_strided((rows, n), (ld, 1))
    far.copy_(dy)
    assert torch.equal(run(dy, q, e, k)[0], run(far, q, e, k)[0])
