"""Group norm over channels-last maps on the device against 64 bits: forward with and without a checkpoint, backward from both, sums over samples."""
import numpy as np
import pytest
import torch

import paper_2506_22771_amd as ff
from blocks_util import ACTS, act_errors, act_slope
from norm_util import DTYPES, HALF_ULP, TINY, U, Framed, junk_ckpt, padded_ckpt, split_ckpt, typed, values, within
from oracle import blocks_oracle as B
from oracle import norm_oracle as N
from test_gpu_norm import check_kept

pytestmark = pytest.mark.gpu
EPS = 1e-5

# samples, pixels, channels, groups: groups of one channel to all of them, at both sides of a chunk of eight, dividing it or not; one pixel to more than a
# workgroup holds; workgroups of 256 and 1024 threads, slabs that are split; several slices of a row; rows that end inside a chunk
SHAPES = [(1, 1, 1, 1), (2, 1, 8, 2), (3, 4, 5, 1), (2, 7, 9, 3), (1, 24, 12, 4), (2, 16, 32, 8), (2, 9, 40, 5), (3, 30, 24, 2), (2, 64, 64, 64), (2, 49, 100, 4), (1, 100, 130, 13),
          (2, 256, 64, 32), (2, 1024, 64, 32), (1, 1024, 128, 32), (2, 1000, 96, 8), (1, 900, 120, 10), (1, 4097, 16, 4), (2, 3000, 20, 4), (1, 5000, 33, 3), (1, 2500, 200, 2),
          (5, 2, 512, 32), (2, 16, 512, 1), (40, 16, 512, 32), (1, 3, 4104, 1), (2, 1, 20000, 2), (1, 2, 16384, 16384), (3, 300, 1030, 2), (1, 1500, 264, 1), (300, 4, 16, 2)]


def inputs(samples, pixels, channels, dtype, seed=0):
    rng = np.random.default_rng(samples * 7 + pixels * 3 + channels + seed)
    x = (rng.standard_normal((samples * pixels, channels)) * np.exp(0.5 * rng.standard_normal((1, channels))) + 0.5 * rng.standard_normal((1, channels))) \
        * np.repeat(np.exp(rng.standard_normal((samples, 1))), pixels, 0)
    dy = 0.1 * rng.standard_normal(x.shape)
    coeff = (0.05 * rng.standard_normal(samples)).astype(np.float32)
    return typed(x, dtype), typed(dy, dtype), 1 + 0.3 * rng.standard_normal(channels), 0.3 * rng.standard_normal(channels), coeff


# Sums: a thread adds up to 64 values (sixteen pixels of four columns), a sum over the lanes has up to 64 terms and their parts' sums, one over a group's columns up to 64 a lane
# and six levels (groups of up to 4096 columns beside each other; longer ones are joined in 64 bits): D roundings of the sum of magnitudes at most.
D = 170


def forward_bounds(x, samples, groups, w, b, kind, dtype):
    """(y, h, mean, rstd, goodness) and their bounds."""
    y, h, mean, rstd, good = B.group_norm_forward(x, samples, groups, w, b, EPS, kind)
    pixels, per = x.shape[0] // samples, x.shape[1] // groups
    m = pixels * per
    at = lambda v: B.spread(v, pixels, per)  # noqa: E731
    dmean = (D + 2) * U * B.of_groups(np.abs(x), samples, groups) / m
    var = 1 / rstd**2
    top = np.abs(x).reshape(samples, pixels, groups, per).max((1, 3))
    drel = 0.5 * ((D + 4) * U + dmean**2 / var) + U * top**2 / var * U + 6 * U
    dh = np.abs(h) * at(drel + 3 * U) + at(rstd * dmean) + U * np.abs(x) * at(rstd)
    wa, ba = np.abs(1.0 if w is None else w), np.abs(0.0 if b is None else b)
    z = B.affine(h, w, b)
    dz = wa * dh + 2 * U * (wa * np.abs(h) + ba)
    df = act_slope(kind, z, dz)[0] + act_errors(kind, z)[0]
    by = df * (1 + HALF_ULP[dtype]) + np.abs(y) * HALF_ULP[dtype] + TINY[dtype]
    # squares of up to 64 values in a thread, then lanes, wavefronts, parts
    bgood = (2 * np.abs(y) * df + df**2).reshape(samples, -1).sum(1) + (160 + x.shape[0] * x.shape[1] / samples / 2**14) * U * good
    return (y, h, mean, rstd, good), (by, dh, dmean + 2 * U * np.abs(mean), drel * rstd, bgood)


def workspace(samples, pixels, channels, groups):
    return torch.full((ff.ff_group_norm_workspace_bytes(samples, pixels, channels, groups),), 0x5A, dtype=torch.uint8, device="cuda")


@pytest.mark.parametrize("samples, pixels, channels, groups", SHAPES)
def test_forward(samples, pixels, channels, groups):
    rows = samples * pixels
    for i, dtype in enumerate(DTYPES):
        x, _, w, b, _ = inputs(samples, pixels, channels, dtype)
        kind = list(ACTS)[(channels + i) % 4]
        odd = channels % 2 == 0
        for params, left, right, stochastic in [("float32", 0, 0, False), (dtype, 1 if odd else 0, 4 if odd else 0, True)]:
            dw, db = typed(w, params), typed(b, params)
            fx, fy = Framed(rows, channels, dtype, left, right, x), Framed(rows, channels, dtype, right, left)
            (y, h, mean, rstd, good), (by, bh, bm, br, bg) = forward_bounds(values(x), samples, groups, values(dw), values(db), kind, dtype)
            gm, gr, gg = (torch.full(shape, 7.0, device="cuda") for shape in ((samples, groups), (samples, groups), (samples,)))
            q, e = junk_ckpt(rows, channels)
            ws = workspace(samples, pixels, channels, groups)
            ff.ff_group_norm_forward(fx.view, samples, groups, dw, db, EPS, ACTS[kind], fy.view, gm, gr, gg, q, e, int(stochastic), 3, 4, ws)
            what = f"{dtype} {kind} "
            within(values(gm), mean, bm, what + "mean")
            within(values(gr), rstd, br, what + "rstd")
            within(values(fy.view), y, by, what + "y")
            within(values(gg), good, bg, what + "goodness")
            check_kept(q, e, h, bh, channels, stochastic)
            assert fx.intact() and fy.intact()
            plain = Framed(rows, channels, dtype, left, right)
            ff.ff_group_norm_forward(fx.view, samples, groups, dw, db, EPS, ACTS[kind], plain.view, None, None, None, None, None, 0, 0, 0, ws)
            within(values(plain.view), y, by, what + "y without a checkpoint")
            assert plain.intact()
            ff.ff_group_norm_forward(fx.view, samples, groups, dw, db, EPS, ACTS[kind], fx.view, None, None, None, None, None, 0, 0, 0, ws)      # in place
            assert torch.equal(fx.view, plain.view) and fx.intact()


def backward_bounds(dy, coeff, h, dh, rstd, samples, groups, w, b, kind, dtype):
    """(dx, dweight, dbias) and their bounds, where h may be off by dh."""
    dx, dw, db, dz = B.group_norm_backward(dy, coeff, h, rstd, samples, groups, w, b, kind)
    rows, channels = h.shape
    pixels, per = rows // samples, channels // groups
    m = pixels * per
    wa = np.abs(1.0 if w is None else w) + 0 * h
    z = B.affine(h, w, b)
    f, d = N.act(kind, z)
    ez = wa * dh + 2 * U * (wa * np.abs(h) + np.abs(0.0 if b is None else b))
    df, dd = (p + q for p, q in zip(act_errors(kind, z), act_slope(kind, z, ez)))
    c2 = 2 * np.abs(np.repeat(coeff, pixels))[:, None] if coeff is not None else 0.0
    up = np.abs(0 if dy is None else dy) + c2 * np.abs(f)
    edz = up * dd + c2 * df * (np.abs(d) + dd) + 4 * U * up * (np.abs(d) + dd)
    at = lambda v: B.spread(B.of_groups(v, samples, groups) / m, pixels, per)  # noqa: E731
    g, eg = wa * np.abs(dz), wa * edz
    eh = np.abs(dz) * dh + edz * (np.abs(h) + dh)
    c1, c2_ = at(g), at(g * np.abs(h))
    n = D + pixels / 8        # (a thread of the launches that sum takes every eighth pixel at most)
    err = eg + at(eg) + n * U * c1 + dh * c2_ + np.abs(h) * (at(wa * eh) + n * U * c2_) + 6 * U * (g + c1 + np.abs(h) * c2_)
    err = B.spread(rstd, pixels, per) * err + 2 * U * np.abs(dx)
    k = min(rows, D + pixels / 8 + samples)
    return (dx, dw, db), (err * (1 + HALF_ULP[dtype]) + np.abs(dx) * HALF_ULP[dtype] + TINY[dtype], (eh + k * U * np.abs(dz * h)).sum(0) + U * np.abs(dw),
                          (edz + k * U * np.abs(dz)).sum(0) + U * np.abs(db))


@pytest.mark.parametrize("samples, pixels, channels, groups", SHAPES)
def test_backward(samples, pixels, channels, groups):
    rows = samples * pixels
    for i, dtype in enumerate(DTYPES):
        x, dy, w, b, coeff = inputs(samples, pixels, channels, dtype)
        kind = list(ACTS)[(channels // 2 + i) % 4]
        xv = values(x)
        _, h, mean, rstd, _ = B.group_norm_forward(xv, samples, groups, w, b, EPS, kind)
        mean32, rstd32 = mean.astype(np.float32), rstd.astype(np.float32)
        gm, gr = torch.from_numpy(mean32).cuda(), torch.from_numpy(rstd32).cuda()
        per = channels // groups
        for source, params, with_dy, with_coeff, left, right in (("x", "float32", True, False, 0, 0), ("codes", dtype, True, True, 1, 2), ("x", dtype, False, True, 0, 3)):
            dw_, db_ = typed(w, params), typed(b, params)
            if source == "x":
                h = (xv - B.spread(mean32, pixels, per)) * B.spread(rstd32, pixels, per)
                dh, kept = 2 * U * np.abs(h) + U * np.abs(h), (None, None)
            else:
                rq, re = N.ckpt_store(h.astype(np.float32))
                h, dh, kept = N.ckpt_load(rq, re), 0 * h, padded_ckpt(rq, re)
            fx, fd = Framed(rows, channels, dtype, left, right, x), Framed(rows, channels, dtype, right, left, dy)
            to = Framed(rows, channels, dtype, left, left)
            c64, dc = (coeff.astype(np.float64), torch.from_numpy(coeff).cuda()) if with_coeff else (None, None)
            (rx, rw, rb), (bx, bw, bb) = backward_bounds(values(dy) if with_dy else None, c64, h, dh, rstd32.astype(np.float64), samples, groups, values(dw_), values(db_), kind, dtype)
            gw, gb = torch.full((channels,), 7.0, device="cuda"), torch.full((channels,), 7.0, device="cuda")
            ws = workspace(samples, pixels, channels, groups)
            run = lambda dx, gw, gb, acc=False: ff.ff_group_norm_backward(  # noqa: E731
                fd.view if with_dy else None, dc, fx.view if source == "x" else None, gm if source == "x" else None, *kept, gr, samples, groups, dw_, db_, ACTS[kind], dx,
                gw, gb, acc, ws)
            run(to.view, gw, gb)
            what = f"{dtype} {kind} from {source} "
            within(values(to.view), rx, bx, what + "dx")
            within(values(gw), rw, bw, what + "dweight")
            within(values(gb), rb, bb, what + "dbias")
            assert to.intact() and fx.intact() and fd.intact()
            other = torch.full_like(dy, 7)
            run(other, None, None)                                          # what else is asked for changes nothing
            assert torch.equal(other, to.view)
            gw2, gb2 = torch.full((channels,), 3.0, device="cuda"), torch.full((channels,), 7.0, device="cuda")
            run(None, None, gb2)
            assert torch.equal(gb2, gb)
            run(None, gw2, None, True)                                      # added
            within(values(gw2), rw + 3, bw + 2 * U * (np.abs(rw) + 3), what + "dweight added")
            over = fd if with_dy else fx                                    # in place
            if with_dy or source == "x":
                run(over.view, gw2, gb2)
                assert torch.equal(over.view, to.view) and over.intact() and torch.equal(gw2, gw) and torch.equal(gb2, gb)


def test_without_parameters():
    x, dy, _, _, _ = inputs(3, 50, 24, "float32")
    y, dx, gm, gr = torch.empty_like(x), torch.empty_like(x), torch.empty((3, 6), device="cuda"), torch.empty((3, 6), device="cuda")
    ws = workspace(3, 50, 24, 6)
    (ref, h, mean, rstd, _), (by, *_) = forward_bounds(values(x), 3, 6, None, None, "gelu", "float32")
    ff.ff_group_norm_forward(x, 3, 6, None, None, EPS, ff.ACT_GELU, y, gm, gr, None, None, None, 0, 0, 0, ws)
    within(values(y), ref, by, "y")
    ff.ff_group_norm_backward(dy, None, x, gm, None, None, gr, 3, 6, None, None, ff.ACT_GELU, dx, None, None, False, ws)
    h = (values(x) - B.spread(values(gm), 50, 4)) * B.spread(values(gr), 50, 4)
    (rx, *_), (bx, *_) = backward_bounds(values(dy), None, h, 3 * U * np.abs(h), values(gr), 3, 6, None, None, "gelu", "float32")
    within(values(dx), rx, bx, "dx")
    only = torch.full((24,), 0.5, device="cuda")       # a bias alone
    ff.ff_group_norm_forward(x, 3, 6, None, only, EPS, ff.ACT_IDENTITY, y, None, None, None, None, None, 0, 0, 0, ws)
    (ref, *_), (by, *_) = forward_bounds(values(x), 3, 6, None, values(only), "identity", "float32")
    within(values(y), ref, by, "y")


def test_no_samples():
    none = lambda *shape: torch.empty(shape, device="cuda")  # noqa: E731
    x, gw, gb = none(0, 24), torch.full((24,), 7.0, device="cuda"), torch.full((24,), 7.0, device="cuda")
    ws = torch.empty(ff.ff_group_norm_workspace_bytes(0, 1, 24, 4), dtype=torch.uint8, device="cuda")
    ff.ff_group_norm_forward(x, 0, 4, None, None, EPS, ff.ACT_SILU, x, none(0, 4), none(0, 4), none(0), None, None, 0, 0, 0, ws)
    L, P = ff.lib(), __import__("ctypes").c_void_p      # pixels say nothing then
    assert L.ff_group_norm_forward(0, 1 << 20, 24, 4, 0, 0, P(), 0, P(), P(), EPS, 1, P(), 0, P(), P(), P(), P(), P(), 0, 0, 0, P(ws.data_ptr()), ws.numel(), P()) == 0
    for acc, want in ((True, 7.0), (False, 0.0)):
        ff.ff_group_norm_backward(x, None, x, none(0, 4), None, None, none(0, 4), 0, 4, None, None, ff.ACT_SILU, x, gw, gb, acc, ws)
        assert (gw == want).all() and (gb == want).all()


@pytest.mark.parametrize("pixels", [64, 3000])
def test_groups_far_from_zero_and_constant_ones(pixels):
    """Where the mean is far larger than the spread, h is as good as the deviations are: the mean's own rounding is taken out."""
    rng = np.random.default_rng(1)
    dev = rng.standard_normal((2 * pixels, 16)).astype(np.float32)
    x = (1000.0 + dev).astype(np.float32)
    x[:, 12:] = 1000.0
    ws = workspace(2, pixels, 16, 4)
    y, gm, gr = torch.empty((2 * pixels, 16), device="cuda"), torch.empty((2, 4), device="cuda"), torch.empty((2, 4), device="cuda")
    ff.ff_group_norm_forward(torch.from_numpy(x).cuda(), 2, 4, None, None, EPS, ff.ACT_IDENTITY, y, gm, gr, None, None, None, 0, 0, 0, ws)
    ref, *_ = B.group_norm_forward(x, 2, 4, None, None, EPS, "identity")
    # deviations of 1000.0 + x are exact but for the mean, which is off by the roundings of sums of deviations of unit size and, where parts are joined, once
    # by the last place of what is left of a mean of 1000 (2^-24 of 2^-14)
    assert np.abs(values(y) - ref)[:, :12].max() <= 3 * D * U
    assert np.abs(values(y))[:, 12:].max() <= 1e-3 * 316 * 1000 * U       # (1 / sqrt(eps) = 316)


def test_infinities_and_nan_stay_in_their_groups():
    x, _, w, b, _ = inputs(2, 40, 32, "float32")
    x[3, 5], x[45, 20] = float("nan"), float("inf")
    y = torch.empty_like(x)
    q, e = junk_ckpt(80, 32)
    ff.ff_group_norm_forward(x, 2, 4, typed(w, "float32"), typed(b, "float32"), EPS, ff.ACT_SILU, y, None, None, None, q, e, 0, 0, 0, workspace(2, 40, 32, 4))
    bad = np.zeros((80, 32), bool)
    bad[:40, :8], bad[40:, 16:24] = True, True
    np.testing.assert_array_equal(np.isnan(values(y)), bad)
    assert (split_ckpt(q, e, 32)[1] == 255).all()       # (a block of 32 columns holds all four groups)


def test_tiny_arguments_of_gelu():
    """Arguments below the smallest normal number: f = u / 2 and f' = 1/2 there."""
    for dtype in DTYPES:
        x = torch.zeros((8, 8), dtype=DTYPES[dtype], device="cuda")
        bias = torch.full((8,), 2.0**-128, device="cuda")
        dy, dx, gb = torch.ones_like(x), torch.empty_like(x), torch.empty(8, device="cuda")
        ws = workspace(1, 8, 8, 1)
        ff.ff_group_norm_backward(dy, None, x, torch.zeros((1, 1), device="cuda"), None, None, torch.ones((1, 1), device="cuda"), 1, 1, None, bias, ff.ACT_GELU, dx, None, gb,
                                  False, ws)
        assert np.abs(values(gb) - 4).max() < 1e-5


def test_gradients_against_differences():
    """dx, dweight and dbias of sum dy y + c G by central differences of the forward pass in 64 bits."""
    samples, pixels, channels, groups = 2, 6, 12, 3
    x, dy, w, b, coeff = inputs(samples, pixels, channels, "float32")
    w, b = typed(w, "float32"), typed(b, "float32")
    gm, gr, y, dx = torch.empty((2, 3), device="cuda"), torch.empty((2, 3), device="cuda"), torch.empty_like(x), torch.empty_like(x)
    gw, gb, ws = torch.empty(12, device="cuda"), torch.empty(12, device="cuda"), workspace(2, 6, 12, 3)
    for kind in ("silu", "gelu"):
        ff.ff_group_norm_forward(x, 2, 3, w, b, EPS, ACTS[kind], y, gm, gr, None, None, None, 0, 0, 0, ws)
        ff.ff_group_norm_backward(dy, torch.from_numpy(coeff).cuda(), x, gm, None, None, gr, 2, 3, w, b, ACTS[kind], dx, gw, gb, False, ws)

        def loss(xv, wv, bv):
            yv, *_, good = B.group_norm_forward(xv, 2, 3, wv, bv, EPS, kind)
            return (values(dy) * yv).sum() + (coeff * good).sum()

        for i, (got, size) in enumerate(((dx, 72), (gw, 12), (gb, 12))):
            for at in range(0, size, 5):
                hi, lo = [values(t).copy() for t in (x, w, b)], [values(t).copy() for t in (x, w, b)]
                hi[i].flat[at] += 1e-5
                lo[i].flat[at] -= 1e-5
                assert abs((loss(*hi) - loss(*lo)) / 2e-5 - values(got).flat[at]) < 1e-4


@pytest.mark.parametrize("pixels", [16, 900, 4000])
def test_calls_in_a_graph(pixels):
    """Captured once, replayed over new inputs with eager work between: as eager calls.  Two graphs share the workspace, one after the other."""
    x, dy, w, b, coeff = inputs(3, pixels, 40, "bfloat16")
    w, b, c = typed(w, "float32"), typed(b, "float32"), torch.from_numpy(coeff).cuda()
    y, dx, gm, gr, gg = torch.empty_like(x), torch.empty_like(x), torch.empty((3, 5), device="cuda"), torch.empty((3, 5), device="cuda"), torch.empty(3, device="cuda")
    q, e = ff.ckpt_empty(3 * pixels, 40)
    gw, gb, ws = torch.empty(40, device="cuda"), torch.empty(40, device="cuda"), workspace(3, pixels, 40, 5)

    def step():
        ff.ff_group_norm_forward(x, 3, 5, w, b, EPS, ff.ACT_SILU, y, gm, gr, gg, q, e, ff.ROUND_STOCHASTIC, 1, 2, ws)
        ff.ff_group_norm_backward(dy, c, None, None, q, e, gr, 3, 5, w, b, ff.ACT_SILU, dx, gw, gb, False, ws)

    step()
    torch.cuda.synchronize()
    graphs = [torch.cuda.CUDAGraph() for _ in range(2)]
    for g in graphs:
        with torch.cuda.graph(g):
            step()
    for i in range(4):
        x.copy_(inputs(3, pixels, 40, "bfloat16", seed=100 + i)[0])
        graphs[i % 2].replay()
        got = [t.clone() for t in (y, gm, gr, gg, q, e, dx, gw, gb)]
        torch.cuda.synchronize()
        step()
        assert all(torch.equal(a, b) for a, b in zip(got, (y, gm, gr, gg, q, e, dx, gw, gb)))


def test_rows_beyond_32_bits_of_offset():
    """Pixels so far apart that their offsets pass 32 bits."""
    samples, pixels, channels, groups, ld = 2, 2, 24, 3, (1 << 30) + 8
    x, dy, w, b, _ = inputs(samples, pixels, channels, "bfloat16")
    buffer = torch.empty(3 * ld + channels + 64, dtype=torch.bfloat16, device="cuda")
    far = buffer.as_strided((samples * pixels, channels), (ld, 1), 5)
    far.copy_(x)
    w, b = typed(w, "float32"), typed(b, "float32")
    gm, gr, y, dx = torch.empty((2, 3), device="cuda"), torch.empty((2, 3), device="cuda"), torch.empty_like(x), torch.empty_like(x)
    ws = workspace(samples, pixels, channels, groups)
    ff.ff_group_norm_forward(x, 2, 3, w, b, EPS, ff.ACT_SILU, y, gm, gr, None, None, None, 0, 0, 0, ws)
    ff.ff_group_norm_backward(dy, None, x, gm, None, None, gr, 2, 3, w, b, ff.ACT_SILU, dx, None, None, False, ws)
    ff.ff_group_norm_forward(far, 2, 3, w, b, EPS, ff.ACT_SILU, far, None, None, None, None, None, 0, 0, 0, ws)
    assert torch.equal(far, y)
    far.copy_(x)
    ff.ff_group_norm_backward(dy, None, far, gm, None, None, gr, 2, 3, w, b, ff.ACT_SILU, far, None, None, False, ws)
    assert torch.equal(far, dx)


def test_more_samples_than_workgroups():
    """Workgroups take sample after sample."""
    samples, channels = (1 << 20) + 37, 8
    x = torch.randn((samples, channels), device="cuda", generator=torch.Generator("cuda").manual_seed(3))
    y, gm, gr, gg = torch.empty_like(x), torch.empty((samples, 2), device="cuda"), torch.empty((samples, 2), device="cuda"), torch.empty(samples, device="cuda")
    ws = workspace(samples, 1, channels, 2)
    ff.ff_group_norm_forward(x, samples, 2, None, None, EPS, ff.ACT_RELU, y, gm, gr, gg, None, None, 0, 0, 0, ws)
    v = x.double().view(samples, 2, 4)
    ref = torch.relu((v - v.mean(2, keepdim=True)) / torch.sqrt(v.var(2, unbiased=False, keepdim=True) + EPS)).view(samples, channels)
    assert (y - ref).abs().max() < 1e-4 and (gg - (ref**2).sum(1)).abs().max() < 1e-4
    dx, gw, gb = torch.empty_like(x), torch.empty(8, device="cuda"), torch.empty(8, device="cuda")
    ff.ff_group_norm_backward(y, None, x, gm, None, None, gr, samples, 2, None, None, ff.ACT_RELU, dx, gw, gb, False, ws)
    want = (y.double() * (ref > 0)).sum(0)
    assert ((gb - want).abs() <= 1e-4 * want.abs()).all()


def test_work_on_another_stream():
    x, y = torch.zeros((4 * 256, 64), device="cuda"), torch.empty((4 * 256, 64), device="cuda")
    x[::2] = 1.0
    gm, ws = torch.empty((4, 8), device="cuda"), workspace(4, 256, 64, 8)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        for _ in range(20):
            x.add_(1.0)
        ff.ff_group_norm_forward(x, 4, 8, None, None, 0.0, ff.ACT_IDENTITY, y, gm, None, None, None, None, 0, 0, 0, ws)
    side.synchronize()
    assert (gm == 20.5).all() and (y[::2] - 1).abs().max() < 1e-5 and (y[1::2] + 1).abs().max() < 1e-5
