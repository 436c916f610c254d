"""Layer norm of rows that lie far from zero beside their spread: what is lost to the rounding of the mean must not come back scaled up by 1 / sqrt(var + eps)."""
import numpy as np
import pytest
import torch

import paper_2506_22771_amd as ff
from norm_util import DTYPES, HALF_ULP, TINY, U, Framed, junk_ckpt, split_ckpt, typed, values, within
from oracle import norm_oracle as N

pytestmark = pytest.mark.gpu
EPS = 1e-5
# every number of lanes, one chunk and several, whole chunks and ragged rows, rows beyond the registers
WIDTHS = [1, 5, 32, 64, 100, 250, 500, 784, 1000, 2000, 2001, 5000, 8192, 12001, 20000, 33000]


# A sum is off by at most D roundings of the sum of magnitudes: a lane's values in order (up to 32; beyond 32768 columns cols / 1024), six levels of lanes, up
# to sixteen wavefronts; and two for the product with 1 / cols.
def depth(cols):
    return 58 + cols // 1024


def forward(x, stochastic=False):
    rows, cols = x.shape
    y, m, r = torch.empty_like(x), torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda")
    q, e = junk_ckpt(rows, cols)
    ff.ff_layer_norm_forward(x, None, None, EPS, y, m, r, q, e, ff.ROUND_STOCHASTIC if stochastic else ff.ROUND_NEAREST, 5, 6)
    return values(y), values(m), values(r), N.ckpt_load(*split_ckpt(q, e, cols))


@pytest.mark.parametrize("dtype", list(DTYPES))
@pytest.mark.parametrize("cols", WIDTHS)
def test_constant_rows_normalise_to_zero(cols, dtype):
    """The mean of equal values c is off by at most D U |c|, by the same amount d for all of them; of d their mean removes all but (D + 4) U |d|."""
    of = np.array([100.0, 1000.0, 4000.0, -250.0, 0.1015625, 0.0])
    x = typed(np.repeat(of[:, None], cols, 1), dtype)
    assert (values(x)[:, 0] == of).all()
    D = depth(cols)
    left = (D + 4) * U * D * U * np.abs(of)             # of a deviation
    for stochastic in (False, True):
        y, m, r, kept = forward(x, stochastic)
        high = left / np.sqrt(EPS)
        within(m, of, U * np.abs(of) + left, "mean")
        assert (np.abs(r * np.sqrt(EPS) - 1) <= 4 * U + (D * U * of) ** 2 * D * U / EPS).all()
        within(y, np.zeros_like(y), (high * (1 + HALF_ULP[dtype]) + TINY[dtype])[:, None], "y")
        within(kept, np.zeros_like(kept), (high * (1 + (1 / 63 if stochastic else 1 / 127)))[:, None], "kept")


@pytest.mark.parametrize("dtype", list(DTYPES))
@pytest.mark.parametrize("cols", [c for c in WIDTHS if c > 1])
def test_rows_of_small_spread_far_from_zero(cols, dtype):
    """Bounds without the mean's own rounding: dm = D U |mean| is how far the first mean may be off, and dr what is left of that after the deviations'.  Deviations
    from it are exact (values and mean within a factor of two)."""
    rng = np.random.default_rng(cols)
    spread = {"float32": 0.01, "float16": 5.0, "bfloat16": 40.0}[dtype]      # a few steps of the type there
    x = typed(np.array([[4000.0], [-4000.0], [3000.0]]) + spread * rng.standard_normal((3, cols)), dtype)
    xv = values(x)
    assert (np.abs(xv).min(1) * 2 > np.abs(xv).max(1)).all()
    y, h, mean, rstd = (a for a in N.norm_forward(xv, None, None, EPS))
    away = np.abs(xv - mean[:, None])
    var, D = (away**2).mean(1), depth(cols)
    dm = D * U * np.abs(mean)
    dr = (D + 3) * U * (away.mean(1) + dm)
    dvar = (D + 6) * U * (var + dm**2) + 2 * dm * dr + dr**2
    drel = 0.55 * dvar / (var + EPS) + 4 * U
    assert (drel < 0.1).all()
    dh = rstd[:, None] * (dr[:, None] + 3 * U * (away + 2 * dm[:, None])) + np.abs(h) * (drel + 2 * U)[:, None]
    for stochastic in (False, True):
        gy, gm, gr, kept = forward(x, stochastic)
        within(gm, mean, dr + U * np.abs(mean) * 1.01, "mean")
        within(gr, rstd, drel * rstd, "rstd")
        within(gy, y, dh * (1 + HALF_ULP[dtype]) + np.abs(y) * HALF_ULP[dtype] + TINY[dtype], "y")
        block = np.repeat(np.maximum.reduceat(np.abs(h) + dh, np.arange(0, cols, 32), axis=1), 32, 1)[:, :cols]
        within(kept, h, dh + block * (1 / 63 if stochastic else 0.5 / 63), "kept")        # (a block's step is at most its largest value / 63)


def test_no_spread_and_no_eps():
    """1 / sqrt(0) is infinite, and 0 times it is NaN, as the formula has it; a row beside it is as it was."""
    x = typed(np.stack([np.full(300, 4.0), np.random.default_rng(0).standard_normal(300)]), "float32")
    y, r = torch.empty_like(x), torch.empty(2, device="cuda")
    ff.ff_layer_norm_forward(x, None, None, 0.0, y, None, r)
    assert np.isinf(values(r)[0]) and np.isnan(values(y)[0]).all() and np.isfinite(values(y)[1]).all()


def test_views_and_in_place():
    """A view of a wider matrix gives the bits of a matrix of its own, and so does the call in place."""
    x = typed(1000 + 0.1 * np.random.default_rng(1).standard_normal((70, 333)), "float32")
    y, v = torch.empty_like(x), Framed(70, 333, "float32", 1, 2, x)
    ff.ff_layer_norm_forward(x, None, None, EPS, y, None, None)
    ff.ff_layer_norm_forward(v.view, None, None, EPS, v.view, None, None)
    assert torch.equal(v.view, y) and v.intact()
