"""Weight gradients from 8-bit checkpoints by the tiles of 128 and 256 outputs, against 64 bits: rows that end anywhere in a step, n and k inside tiles, chunks
and words, splits, strides, infinities.  Behind every matrix lies what spoils a sum that reads it."""
import os
import shutil
import subprocess

import numpy as np
import pytest
import torch

import paper_2506_22771_amd as ff
from norm_util import DTYPES, U, padded_ckpt, typed, values
from oracle import norm_oracle as N

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

# (rows, n, k) and the tiles that bf16, fp16 and fp32 take there.  Steps are of 32 rows (fp32: 16): one row and 1 to 15 beyond whole steps, where the last step's
# second chunk of a thread has no row, 16 and more; one step, fewer and more than are under way in registers
SHAPES = {(1, 2000, 2000): (128, 128, 128), (33, 2000, 2000): (128, 128, 128), (40, 2000, 2008): (128, 128, 128), (47, 2001, 1999): (128, 128, 128),
          (150, 2000, 2000): (128, 128, 128), (300, 2002, 2001): (128, 128, 128), (250, 2003, 2005): (128, 128, 128),
          (1, 4096, 4096): (256, 256, 256), (41, 3001, 2999): (256, 256, 256), (39, 4002, 4001): (256, 256, 256), (167, 4000, 4000): (256, 256, 256),
          (64, 4096, 4000): (256, 256, 256)}
# and splits of the rows (the last one shorter, and ending inside a step)
SPLIT = {(8195, 1000, 1000): (128, 256, 256), (8199, 1001, 1003): (128, 256, 256)}
ROUND = ("bfloat16", "float16", "float32")


def test_shapes_reach_the_tiles(tmp_path):
    """The plan, built on the host and asked: these shapes are here for their tiles."""
    compiler = shutil.which("g++") or shutil.which("hipcc")
    if compiler is None:
        pytest.skip("no C++ compiler")
    (tmp_path / "plan.cpp").write_text('#include "wgrad_plan.hpp"\n#include <cstdio>\n#include <cstdlib>\nint main(int, char** v)\n{\n'
                                       "    const auto p = ffi::wgrad_plan(atoll(v[1]), atoll(v[2]), atoll(v[3]), atoi(v[4]));\n"
                                       '    printf("%d %d", p.tile, p.splits);\n}\n')
    subprocess.run([compiler, "-std=c++17", "-I" + os.path.join(ROOT, "paper_2506_22771_amd", "csrc"), str(tmp_path / "plan.cpp"), "-o", str(tmp_path / "plan")], check=True)
    for shapes, split in ((SHAPES, False), (SPLIT, True)):
        for shape, tiles in shapes.items():
            for terms, tile in zip((1, 2, 3), tiles):
                out = subprocess.run([str(tmp_path / "plan"), *map(str, shape), str(terms)], check=True, capture_output=True, text=True).stdout.split()
                assert int(out[0]) == tile and (int(out[1]) > 1) == split, (shape, terms, out)


def spoilt(data: np.ndarray, dtype: str, right: int) -> torch.Tensor:
    """A matrix, `right` NaN behind each row and forty rows of NaN behind the last."""
    rows, n = data.shape
    buffer = torch.full((rows + 40, n + right), float("nan"), dtype=DTYPES[dtype], device="cuda")
    view = buffer[:rows, :n]
    view.copy_(typed(data, dtype))
    return view


def spoilt_ckpt(rq: np.ndarray, re: np.ndarray):
    """A checkpoint with forty rows behind it that read as NaN."""
    q, e = padded_ckpt(rq, re)
    bq = torch.full((q.shape[0] + 40, q.shape[1]), 0x5A, dtype=torch.int8, device="cuda")
    be = torch.full((e.shape[0] + 40, e.shape[1]), 255, dtype=torch.uint8, device="cuda")
    bq[:len(q)], be[:len(e)] = q, e
    return bq[:len(q)], be[:len(e)]


def run(dy, q, e, k, gamma=None, beta=None, accumulate=False, start=7.0):
    rows, n = dy.shape
    dw, db = torch.full((n, k), start, device="cuda"), torch.full((n,), start, device="cuda")
    ws = torch.full((ff.ff_ckpt_weight_grad_workspace_bytes(rows, n, k),), 255, dtype=torch.uint8, device="cuda")   # (NaN wherever it is read unwritten)
    ff.ff_ckpt_weight_grad(dy, q, e, gamma, beta, dw, db, accumulate, ws)
    return dw, db


def inputs(rows, n, k):
    rng = np.random.default_rng(rows + n + k)
    rq, re = N.ckpt_store((rng.standard_normal((rows, k)) * np.exp(rng.standard_normal((rows, 1)))).astype(np.float32))
    dy = rng.standard_normal((rows, n)) * np.exp(rng.standard_normal((rows, 1)))
    return rq, re, dy, 1 + 0.3 * rng.standard_normal(k), 0.3 * rng.standard_normal(k)


def close(got, ref, bound, what):
    """On the device, in 64 bits."""
    over = (got.double() - ref).abs() - bound
    assert bool(torch.isfinite(got).all()) and float(over.max()) <= 0, f"{what}: {float(over.max())} beyond its bound"


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ROUND)
@pytest.mark.parametrize("rows, n, k", list(SHAPES) + list(SPLIT))
def test_against_64_bits(rows, n, k, dtype):
    """Products are exact and sums fp32: off by at most one rounding per row of the sum of magnitudes, and five for gamma, beta and splits; in the mean far less,
    as roundings are not all one way."""
    rq, re, dy, g, b = inputs(rows, n, k)
    q, e = spoilt_ckpt(rq, re)
    h = torch.from_numpy(N.ckpt_load(rq, re)).cuda()
    for params, right in ((None, 0), ("float32", 3), (dtype, 2)):
        view = spoilt(dy, dtype, right)
        d = view.double().contiguous()
        dg, db_ = (None, None) if params is None else (typed(g, params), typed(b, params))
        gv, bv = (1.0, 0.0) if params is None else (dg.double(), db_.double())
        dw, db = run(view, q, e, k, dg, db_)
        sums, sizes = d.sum(0), d.abs().sum(0)
        ref, size = torch.mm(d.t().contiguous(), h), torch.mm(d.abs().t().contiguous(), h.abs())
        ref, size = (ref, size) if params is None else (ref * gv + sums[:, None] * bv, size * gv.abs() + sizes[:, None] * bv.abs())
        close(dw, ref, (rows + 5) * U * size, "dw")
        close(db, sums, (rows + 5) * U * sizes, "db")
        off = float(((dw.double() - ref) ** 2).mean().sqrt())
        assert off <= 2e-6 * max(float((ref**2).mean().sqrt()), 1e-30) * np.sqrt(max(1.0, rows / 1000))
    aw, ab = run(view, q, e, k, dg, db_, True, 0.5)
    assert torch.equal(aw, dw + 0.5) and torch.equal(ab, db + 0.5)
    for _ in range(2):
        again = run(view, q, e, k, dg, db_)
        assert torch.equal(again[0], dw) and torch.equal(again[1], db)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ROUND)
@pytest.mark.parametrize("rows, n, k", [(33, 2000, 2000), (47, 2001, 1999), (250, 2003, 2005), (41, 3001, 2999), (167, 4000, 4000), (8199, 1001, 1003)])
def test_whole_numbers_are_exact(rows, n, k, dtype):
    """Small whole numbers, whose sums fp32 holds: every row and column in its place, bit for bit."""
    rng = np.random.default_rng(k)
    rq = rng.integers(-15, 16, (rows, k)).astype(np.int8)
    q, e = spoilt_ckpt(rq, np.full((rows, (k + 31) // 32), 127, np.uint8))
    dy = rng.integers(-7, 8, (rows, n)).astype(np.float32)      # 8199 * 15 * 7 < 2^24
    dw, db = run(spoilt(dy, dtype, 1), q, e, k)
    d = torch.from_numpy(dy).double().cuda()
    assert torch.equal(dw.double(), torch.mm(d.t().contiguous(), torch.from_numpy(rq).double().cuda()))
    assert torch.equal(db.double(), d.sum(0))


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ROUND)
@pytest.mark.parametrize("rows, n, k", [(45, 2000, 2000), (41, 3001, 2999)])
def test_infinities_and_nan_go_where_the_sums_put_them(rows, n, k, dtype):
    """A NaN of dy spoils its row of dw, an infinity leaves infinities or, against a zero, NaN; a block that reads as NaN spoils its columns.  All else is as without."""
    rq, re, dy, _, _ = inputs(rows, n, k)
    dy = dy.astype(np.float32)
    q, e = spoilt_ckpt(rq, re)
    clean = values(run(spoilt(dy, dtype, 0), q, e, k)[0])
    re[rows - 1, 21], rq[rows - 1, 672:704] = 255, 0
    dy[rows - 1, 300], dy[7, 1109], dy[rows - 3, n - 1] = np.nan, np.inf, -np.inf
    q, e = spoilt_ckpt(rq, re)
    dw, db = run(spoilt(dy, dtype, 0), q, e, k)
    got, sums, h = values(dw), values(db), N.ckpt_load(rq, re)
    assert np.isnan(got[300]).all() and np.isnan(got[:, 672:704]).all()
    others = np.r_[0:672, 704:k]
    for row, m in ((1109, 7), (n - 1, rows - 3)):
        with np.errstate(invalid="ignore"):
            np.testing.assert_array_equal(got[row, others], dy[m, row].astype(np.float64) * h[m, others])    # (infinities; against a zero, NaN)
    fine = np.delete(np.arange(n), [300, 1109, n - 1])
    np.testing.assert_array_equal(got[np.ix_(fine, others)], clean[np.ix_(fine, others)])
    assert np.isnan(sums[300]) and sums[1109] == np.inf and sums[n - 1] == -np.inf and np.isfinite(sums[fine]).all()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ROUND)
@pytest.mark.parametrize("rows, n, k", [(37, 2000, 2000), (37, 3001, 2999)])
def test_rows_too_far_apart_for_offsets_of_32_bits(rows, n, k, dtype):
    """A step of rows longer than 2^30 bytes is read another way, and adds up to the same bits."""
    rq, re, dy, g, b = inputs(rows, n, k)
    q, e = spoilt_ckpt(rq, re)
    ld = (1 << 25) + 3
    far = torch.empty((rows - 1) * ld + n, dtype=DTYPES[dtype], device="cuda").as_strided((rows, n), (ld, 1))
    far.copy_(typed(dy, dtype))
    g, b = typed(g, "float32"), typed(b, "float32")
    near, apart = run(spoilt(dy, dtype, 0), q, e, k, g, b), run(far, q, e, k, g, b)
    assert torch.equal(near[0], apart[0]) and torch.equal(near[1], apart[1])


@pytest.mark.gpu
@pytest.mark.parametrize("n", [1, 2, 3, 5, 7, 8])
@pytest.mark.parametrize("rows", [1, 2, 33, 65])
@pytest.mark.parametrize("dtype", ROUND)
def test_last_rows_shorter_than_a_chunk(rows, n, dtype):
    """The small tile: what is left of dy in the last step is less than the two words a thread of fp32 takes, or less than one."""
    rq, re, dy, _, _ = inputs(rows, n, 70)
    q, e = spoilt_ckpt(rq, re)
    d = spoilt(dy, dtype, 0)
    dw, db = run(d, q, e, 70)
    h, dv = torch.from_numpy(N.ckpt_load(rq, re)).cuda(), d.double()
    close(dw, torch.mm(dv.t().contiguous(), h), (rows + 5) * U * torch.mm(dv.abs().t().contiguous(), h.abs()), "dw")
    close(db, dv.sum(0), (rows + 5) * U * dv.abs().sum(0), "db")
