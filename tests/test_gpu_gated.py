"""Gated layers on the device against 64 bits: the forward pass with what it keeps, and the gradient from the checkpoints."""
import numpy as np
import pytest
import torch

import paper_2506_22771_amd as ff
from blocks_util import ACTS, act_errors, act_slope
from norm_util import DTYPES, HALF_ULP, TINY, U, Framed, junk_ckpt, padded_ckpt, split_ckpt, typed, values, within
from oracle import blocks_oracle as B
from oracle import norm_oracle as N

pytestmark = pytest.mark.gpu


def padded_codes(q):
    to = np.zeros((q.shape[0], ff.ff_pitch(q.shape[1])), np.int8)
    to[:, :q.shape[1]] = q
    return torch.from_numpy(to).cuda()


def layer(rows, n, k, seed=0, scale=None):
    """Codes whose projections are of unit size under the scale."""
    rng = np.random.default_rng(rows * 5 + n * 3 + k + seed)
    a = np.clip(np.rint(rng.standard_normal((rows, k)) * 40), -127, 127).astype(np.int8)
    w = rng.integers(-127, 128, (2 * n, k)).astype(np.int8)
    s_a, s_w = np.float32(0.03), np.float32(0.03 / np.sqrt(k) if scale is None else scale)
    return a, w, s_a, s_w


def forward_bounds(a, w, s_a, s_w, kind, dtype):
    """(y, goodness, g, u) and the bounds of the first two and of the errors of g and u.  A projection is a whole number rounded to fp32, times the
    rounded product of the scales: three roundings.  A row's squares are summed by lanes, tiles and columns: fewer than 64 + n / 32 additions on a path."""
    y, good, g, u = B.gated_forward(a, w, np.float64(s_a) * np.float64(s_w), kind)
    n = y.shape[1]
    dg, du = 3 * U * np.abs(g), 3 * U * np.abs(u)
    f, _ = N.act(kind, g)
    df = act_errors(kind, g)[0] + act_slope(kind, g, dg)[0]
    dy = df * np.abs(u) + np.abs(f) * du + 2 * U * np.abs(y)
    dgood = (2 * np.abs(y) * dy + dy**2).sum(1) + (66 + n // 32) * U * good
    return (y, good, g, u), (dy * (1 + HALF_ULP[dtype]) + np.abs(y) * HALF_ULP[dtype] + TINY[dtype], dgood, dg, du)


def check_kept(q, e, v, dv):
    """A checkpoint of v, off by dv at most: the codes' rounding, and exponents one way or the other at their edge."""
    cols = v.shape[1]
    gq, ge = split_ckpt(q, e, cols)
    step = np.repeat(np.exp2(ge.astype(np.float64) - 127), 32, 1)[:, :cols]
    within(N.ckpt_load(gq, ge), v, dv + 0.5 * step, "kept")
    for b in range(ge.shape[1]):
        at = slice(32 * b, min(cols, 32 * b + 32))
        low, high = np.maximum(np.abs(v[:, at]) - dv[:, at], 0).max(1), (np.abs(v[:, at]) + dv[:, at]).max(1)
        for r in range(0, v.shape[0], 1 if v.shape[0] <= 100 else 37):
            assert N.exponent_of(low[r]) <= ge[r, b] <= N.exponent_of(high[r]) or low[r] < 2.0**-100


def run_forward(a, w, s_a, s_w, kind, dtype, left=0, right=0, keep=True):
    rows, k, n = a.shape[0], a.shape[1], w.shape[0] // 2
    y = Framed(rows, n, dtype, left, right)
    good = torch.full((rows,), 7.0, device="cuda")
    g, u = (junk_ckpt(rows, n), junk_ckpt(rows, n)) if keep else ((None, None), (None, None))
    ws = torch.full((ff.ff_gated_workspace_bytes(rows, n, k),), 0x5A, dtype=torch.uint8, device="cuda")
    da, dw = padded_codes(a), padded_codes(w)
    sa, sw = torch.tensor([s_a], device="cuda"), torch.tensor([s_w], device="cuda")
    ff.ff_gated_forward(da, dw, sa, sw, k, ACTS[kind], y.view, good, *g, *u, ws)
    other = torch.full((rows, n), 7, dtype=DTYPES[dtype], device="cuda")
    ff.ff_gated_forward(da, dw, sa, sw, k, ACTS[kind], other, None, None, None, None, None, ws)      # nothing else asked for: the same bits
    assert torch.equal(other, y.view) and y.intact()
    return y.view, good, g, u


# one row to several tiles; outputs and reductions of one, at both sides of a block, a tile, a reduction step and a pitch
SHAPES = [(1, 1, 1), (1, 31, 16), (2, 33, 17), (5, 64, 100), (16, 40, 784), (17, 96, 129), (33, 130, 500), (1, 500, 784), (3, 513, 1000), (64, 500, 784), (100, 96, 2000),
          (130, 260, 300), (256, 128, 512), (257, 129, 640), (300, 257, 96), (700, 1030, 384), (1025, 515, 520), (40, 2000, 784)]


@pytest.mark.parametrize("kind", list(ACTS))
@pytest.mark.parametrize("rows, n, k", SHAPES)
def test_forward(rows, n, k, kind):
    a, w, s_a, s_w = layer(rows, n, k)
    dtype = list(DTYPES)[(rows + n + k) % 3]
    (y, good, g, u), (by, bgood, dg, du) = forward_bounds(a, w, s_a, s_w, kind, dtype)
    gy, ggood, kg, ku = run_forward(a, w, s_a, s_w, kind, dtype, left=n % 3, right=n % 2)
    within(values(gy), y, by, "y")
    within(values(ggood), good, bgood, "goodness")
    check_kept(*kg, g, dg)
    check_kept(*ku, u, du)


@pytest.mark.parametrize("dtype", list(DTYPES))
@pytest.mark.parametrize("rows, n, k", [(1, 300, 600), (20, 70, 333), (300, 200, 129), (513, 384, 256)])
def test_forward_of_every_type(rows, n, k, dtype):
    a, w, s_a, s_w = layer(rows, n, k, seed=4)
    (y, good, g, u), (by, bgood, dg, du) = forward_bounds(a, w, s_a, s_w, "silu", dtype)
    gy, ggood, kg, ku = run_forward(a, w, s_a, s_w, "silu", dtype)
    within(values(gy), y, by, "y")
    within(values(ggood), good, bgood, "goodness")
    check_kept(*kg, g, dg)
    check_kept(*ku, u, du)


# tiles of 128 x 64 and of 256 x 128 outputs, one and several to a workgroup, reductions of one step to several, at both sides of a tile's end
MANY = [(2000, 1500, 90, "float32"), (8200, 2050, 260, "float16"), (8200, 2050, 100, "bfloat16"), (3000, 1500, 130, "float16"), (8150, 2040, 90, "bfloat16"),
        (8192, 2048, 500, "float32"), (70000, 120, 128, "bfloat16"), (40, 32767, 40, "float32")]


@pytest.mark.parametrize("rows, n, k, dtype", MANY)
def test_forward_of_many_tiles(rows, n, k, dtype):
    """Against 64 bits on the device."""
    a, w, s_a, s_w = layer(rows, n, k)
    gy, ggood, kg, ku = run_forward(a, w, s_a, s_w, "silu", dtype, left=3, right=2)
    scale = float(s_a) * float(s_w)
    acc = [torch.from_numpy(a).cuda().double() @ torch.from_numpy(p).cuda().double().t() for p in (w[:n], w[n:])]
    g, u = acc[0] * scale, acc[1] * scale
    sig = torch.sigmoid(g)
    y = g * sig * u
    f = (g * sig).abs()
    # as forward_bounds has it
    dy = (16 * U * (f + 0.2 * g.abs()) + 1.13 * 3 * U * g.abs()) * u.abs() + f * 3 * U * u.abs() + 2 * U * y.abs()
    assert ((gy.double() - y).abs() <= dy * (1 + HALF_ULP[dtype]) + y.abs() * HALF_ULP[dtype] + TINY[dtype]).all()
    assert ((ggood.double() - (y * y).sum(1)).abs() <= (2 * y.abs() * dy + dy**2).sum(1) + (66 + n // 32) * U * (y * y).sum(1)).all()
    for (q, e), v in ((kg, g), (ku, u)):
        nb = (n + 31) // 32
        assert not q[:, n:].any() and not e[:, nb:].any()
        step = torch.exp2(e[:, :nb].double() - 127).repeat_interleave(32, 1)[:, :n]
        assert ((q[:, :n].double() * step - v).abs() <= 3 * U * v.abs() + 0.5 * step).all()
        top = torch.nn.functional.pad(v.abs(), (0, nb * 32 - n)).view(rows, nb, 32).amax(2)
        span = 127 * torch.exp2(e[:, :nb].double() - 127)       # the smallest power of two that covers the block
        assert (top <= span * (1 + 4 * U)).all() and (top * (1 + 4 * U) > span / 2).all()


@pytest.mark.parametrize("rows", [3, 300])
def test_largest_sums_and_extreme_scales(rows):
    """Sums at the end of int32 (all codes alike, the longest reduction), zero codes, and scales that leave fp32's range."""
    k, n = 133144, 33
    a, w = np.full((rows, k), 127, np.int8), np.full((2 * n, k), -127, np.int8)
    w[1] = 127
    a[1] = 0
    da, dw, y = padded_codes(a), padded_codes(w), torch.empty((rows, n), device="cuda")
    ws = torch.empty(ff.ff_gated_workspace_bytes(rows, n, k), dtype=torch.uint8, device="cuda")
    one, g, u = torch.ones(1, device="cuda"), junk_ckpt(rows, n), junk_ckpt(rows, n)
    ff.ff_gated_forward(da, dw, one, one, k, ff.ACT_IDENTITY, y, None, *g, *u, ws)
    top = np.float32(127 * 127 * k)
    want = np.full((rows, n), np.float32(top * top), np.float32)
    want[:, 1] *= -1
    want[1] = 0
    np.testing.assert_array_equal(y.cpu().numpy(), want)
    gq, ge = split_ckpt(*g, n)
    assert (ge[0, 0], gq[0, 0], gq[0, 1]) == (N.exponent_of(float(top)), -gq[0, 1], gq[0, 1]) and not gq[1].any() and (ge[1] == 127).all()
    for scale, status in ((float("inf"), 255), (float("nan"), 255)):
        ff.ff_gated_forward(da, dw, one * scale, one, k, ff.ACT_SILU, y, None, *g, *u, ws)
        gq, ge = split_ckpt(*g, n)
        assert (ge[0, 0] == status) and not gq.any()                              # (the pad bytes are zero: split_ckpt)
        assert torch.isnan(y[1]).all()
    ff.ff_gated_forward(da, dw, one * 2.0**-126, one * 2.0**-20, k, ff.ACT_IDENTITY, y, None, *g, *u, ws)
    assert not y.any() and not split_ckpt(*u, n)[0].any()


def test_rows_behind_the_last_are_left_alone():
    """Outputs that are the first rows of larger buffers."""
    rows, n, k = 37, 70, 90
    a, w, s_a, s_w = layer(rows, n, k)
    y = torch.full((rows + 40, n), 7.0, device="cuda")
    (g, e), (u, f) = junk_ckpt(rows + 40, n), junk_ckpt(rows + 40, n)
    good = torch.full((rows + 40,), 7.0, device="cuda")
    ws = torch.empty(ff.ff_gated_workspace_bytes(rows, n, k), dtype=torch.uint8, device="cuda")
    ff.ff_gated_forward(padded_codes(a), padded_codes(w), torch.tensor([s_a], device="cuda"), torch.tensor([s_w], device="cuda"), k, ff.ACT_RELU, y[:rows], good[:rows],
                        g[:rows], e[:rows], u[:rows], f[:rows], ws)
    assert (y[rows:] == 7).all() and (good[rows:] == 7).all()
    for t in (g, e, u, f):
        assert (t[rows:] == 0x5A).all()


# t = dy + 2 c f u, dg = t u f', du = t f
def backward_bounds(g, u, kind, coeff, dy, dtype):
    f, d = N.act(kind, g)
    df, dd = act_errors(kind, g)
    c2 = 2 * np.abs(coeff[:, None]) if coeff is not None else 0.0
    t = (0 if dy is None else dy) + (0 if coeff is None else 2 * coeff[:, None] * f * u)
    size = np.abs(0 if dy is None else dy) + c2 * np.abs(f * u)
    dt = c2 * np.abs(u) * df + 4 * U * size
    refs = B.gated_backward(g, u, kind, coeff, dy)
    errs = (dt * np.abs(u * d) + np.abs(t * u) * dd + 3 * U * size * np.abs(u * d), dt * np.abs(f) + np.abs(t) * df + 2 * U * size * np.abs(f))
    return refs, [e * (1 + HALF_ULP[dtype]) + np.abs(r) * HALF_ULP[dtype] + TINY[dtype] for e, r in zip(errs, refs)]


@pytest.mark.parametrize("with_dy, with_coeff", [(True, False), (True, True), (False, True)])
@pytest.mark.parametrize("dtype", list(DTYPES))
@pytest.mark.parametrize("kind", list(ACTS))
def test_backward(kind, dtype, with_dy, with_coeff):
    for rows, n, left, right in [(1, 1, 0, 0), (5, 37, 1, 0), (64, 500, 0, 0), (130, 96, 3, 5), (3, 2050, 0, 2)]:
        rng = np.random.default_rng(rows + n)
        raw = [(rng.standard_normal((rows, n)) * rng.choice([0.01, 1, 5], (rows, 1))).astype(np.float32) for _ in range(2)]
        raw[0][rng.random((rows, n)) < 0.05] = 0
        (gq, ge), (uq, ue) = N.ckpt_store(raw[0]), N.ckpt_store(raw[1])
        g, u = N.ckpt_load(gq, ge), N.ckpt_load(uq, ue)
        coeff = (rng.standard_normal(rows) * 0.05).astype(np.float32) if with_coeff else None
        dy = Framed(rows, n, dtype, left, right, typed(rng.standard_normal((rows, n)), dtype)) if with_dy else None
        dc = torch.from_numpy(coeff).cuda() if with_coeff else None
        kept = (*padded_ckpt(gq, ge), *padded_ckpt(uq, ue))
        both = Framed(rows, 2 * n, dtype, left, right)      # halves of one matrix
        ff.ff_gated_backward(*kept, ACTS[kind], dc, dy.view if with_dy else None, both.view[:, :n], both.view[:, n:])
        refs, bounds = backward_bounds(g, u, kind, None if coeff is None else coeff.astype(np.float64), values(dy.view) if with_dy else None, dtype)
        within(values(both.view[:, :n]), refs[0], bounds[0], f"dg {kind} {rows}x{n}")
        within(values(both.view[:, n:]), refs[1], bounds[1], f"du {kind} {rows}x{n}")
        assert both.intact()
        if with_dy:
            assert dy.intact()
            du = torch.full((rows, n), 7, dtype=DTYPES[dtype], device="cuda")
            ff.ff_gated_backward(*kept, ACTS[kind], dc, dy.view, dy.view, du)        # in place
            assert torch.equal(dy.view, both.view[:, :n]) and torch.equal(du, both.view[:, n:]) and dy.intact()


@pytest.mark.parametrize("kind", ["gelu", "silu"])
def test_backward_against_differences(kind):
    """By central differences in 64 bits (error 1e-9), where fp32 gives 1e-5."""
    rng = np.random.default_rng(8)
    (gq, ge), (uq, ue) = (N.ckpt_store(rng.standard_normal((16, 64)).astype(np.float32)) for _ in range(2))
    g, u = N.ckpt_load(gq, ge), N.ckpt_load(uq, ue)
    dy, c = rng.standard_normal((16, 64)).astype(np.float32), rng.standard_normal(16).astype(np.float32)
    loss = lambda g, u: dy * N.act(kind, g)[0] * u + c[:, None] * (N.act(kind, g)[0] * u) ** 2  # noqa: E731
    d = torch.empty((16, 128), device="cuda")
    ff.ff_gated_backward(*padded_ckpt(gq, ge), *padded_ckpt(uq, ue), ACTS[kind], torch.from_numpy(c).cuda(), torch.from_numpy(dy).cuda(), d[:, :64], d[:, 64:])
    assert np.abs((loss(g + 1e-5, u) - loss(g - 1e-5, u)) / 2e-5 - values(d[:, :64])).max() < 1e-4
    assert np.abs((loss(g, u + 1e-5) - loss(g, u - 1e-5)) / 2e-5 - values(d[:, 64:])).max() < 1e-4


def test_forward_backward_and_the_products_behind_them():
    """A gated layer's whole gradient from the calls there are: [dg | du] to the weights' gradient from the input's checkpoint and, in int8, to the input's."""
    rows, n, k = 70, 45, 100
    rng = np.random.default_rng(5)
    x = rng.standard_normal((rows, k)).astype(np.float32)
    w = (rng.standard_normal((2 * n, k)) / np.sqrt(k)).astype(np.float32)
    new = lambda *shape, of=torch.float32: torch.empty(shape, dtype=of, device="cuda")  # noqa: E731
    ws = new(1 << 20, of=torch.uint8)
    dx_, dw_ = torch.from_numpy(x).cuda(), torch.from_numpy(w).cuda()
    a_q, s_a, w_q, w_qt, s_w = new(rows, ff.ff_pitch(k), of=torch.int8), new(1), new(2 * n, ff.ff_pitch(k), of=torch.int8), new(k, ff.ff_pitch(2 * n), of=torch.int8), new(1)
    ff.ff_quantize(dx_, rows, k, ff.ROUND_NEAREST, 0, 0, a_q, None, s_a, ws)
    ff.ff_quantize(dw_, 2 * n, k, ff.ROUND_NEAREST, 0, 0, w_q, w_qt, s_w, ws)
    y, g, u, h = new(rows, n), ff.ckpt_empty(rows, n), ff.ckpt_empty(rows, n), ff.ckpt_empty(rows, k)
    ff.ff_ckpt_store(dx_, ff.ROUND_NEAREST, 0, 0, *h)
    ff.ff_gated_forward(a_q, w_q, s_a, s_w, k, ff.ACT_SILU, y, None, *g, *u, ws)
    dy = torch.from_numpy(rng.standard_normal((rows, n)).astype(np.float32)).cuda()
    d = new(rows, 2 * n)
    ff.ff_gated_backward(*g, *u, ff.ACT_SILU, None, dy, d[:, :n], d[:, n:])
    dW = new(2 * n, k)
    ff.ff_ckpt_weight_grad(d, *h, None, None, dW, None, False, new(ff.ff_ckpt_weight_grad_workspace_bytes(rows, 2 * n, k), of=torch.uint8))
    hv = N.ckpt_load(*split_ckpt(*h, k))
    within(values(dW), values(d).T @ hv, (rows + 12) * U * (np.abs(values(d)).T @ np.abs(hv)), "dW")
    from paper_2506_22771_amd.normed import _Dense
    d_q, s_d, e_acc = new(rows, ff.ff_pitch(2 * n), of=torch.int8), new(1), new(rows, ff.ff_pitch32(k), of=torch.int32)
    ff.ff_quantize(d, rows, 2 * n, ff.ROUND_NEAREST, 0, 0, d_q, None, s_d, ws)
    ff.ff_layer_input_grad(ff.layer_desc(_Dense(k, 2 * n), rows), d_q, w_qt, e_acc, ws)
    want = d_q[:, :2 * n].cpu().numpy().astype(np.int64) @ w_q[:, :k].cpu().numpy().astype(np.int64)
    np.testing.assert_array_equal(e_acc[:, :k].cpu().numpy(), want)
    # and all of it is the gradient of the layer in real numbers, but for eight bits: half a step of x, of w, of what was kept and of d, at random over sums of 90 terms
    gr, ur = x.astype(np.float64) @ w[:n].T.astype(np.float64), x.astype(np.float64) @ w[n:].T.astype(np.float64)
    dg, du = B.gated_backward(gr, ur, "silu", None, values(dy))
    ref = np.concatenate([dg, du], 1) @ w.astype(np.float64)
    got = e_acc[:, :k].cpu().numpy() * float(s_d) * float(s_w)
    assert np.linalg.norm(got - ref) < 0.05 * np.linalg.norm(ref)


@pytest.mark.parametrize("rows", [1, 48, 600])
def test_calls_in_a_graph(rows):
    """Captured once, replayed over new inputs with eager work between: as eager calls.  Two graphs share the workspace, one after the other."""
    n, k = 200, 333
    a, w, s_a, s_w = layer(rows, n, k)
    aq, wq, sa, sw = padded_codes(a), padded_codes(w), torch.tensor([s_a], device="cuda"), torch.tensor([s_w], device="cuda")
    y, good, g, u = torch.empty((rows, n), device="cuda"), torch.empty(rows, device="cuda"), ff.ckpt_empty(rows, n), ff.ckpt_empty(rows, n)
    c, d = torch.full((rows,), 0.1, device="cuda"), torch.empty((rows, 2 * n), device="cuda")
    ws = torch.empty(ff.ff_gated_workspace_bytes(rows, n, k), dtype=torch.uint8, device="cuda")

    def step():
        ff.ff_gated_forward(aq, wq, sa, sw, k, ff.ACT_GELU, y, good, *g, *u, ws)
        ff.ff_gated_backward(*g, *u, ff.ACT_GELU, c, y, d[:, :n], d[:, n:])

    step()
    torch.cuda.synchronize()
    graphs = [torch.cuda.CUDAGraph() for _ in range(2)]
    for gr in graphs:
        with torch.cuda.graph(gr):
            step()
    for i in range(4):
        aq.copy_(padded_codes(layer(rows, n, k, seed=100 + i)[0]))
        graphs[i % 2].replay()
        got = [t.clone() for t in (y, good, *g, *u, d)]
        torch.cuda.synchronize()
        step()
        assert all(torch.equal(p, q) for p, q in zip(got, (y, good, *g, *u, d)))


def test_backward_beyond_32_bits_of_offset():
    """Rows so far apart that their offsets pass 32 bits."""
    rows, n, ld = 3, 40, (1 << 31) - 8
    rng = np.random.default_rng(0)
    (gq, ge), (uq, ue) = (N.ckpt_store(rng.standard_normal((rows, n)).astype(np.float32)) for _ in range(2))
    buffer = torch.empty(2 * ld + n + 64, dtype=torch.bfloat16, device="cuda")
    far = buffer.as_strided((rows, n), (ld, 1), 3)
    dy = typed(rng.standard_normal((rows, n)), "bfloat16")
    far.copy_(dy)
    kept = (*padded_ckpt(gq, ge), *padded_ckpt(uq, ue))
    dg, du, du2 = (torch.empty((rows, n), dtype=torch.bfloat16, device="cuda") for _ in range(3))
    ff.ff_gated_backward(*kept, ff.ACT_SILU, None, dy, dg, du)
    ff.ff_gated_backward(*kept, ff.ACT_SILU, None, far, far, du2)
    assert torch.equal(far, dg) and torch.equal(du, du2)
    a, w, s_a, s_w = layer(rows, n, 50)
    ws = torch.empty(ff.ff_gated_workspace_bytes(rows, n, 50), dtype=torch.uint8, device="cuda")
    args = padded_codes(a), padded_codes(w), torch.tensor([s_a], device="cuda"), torch.tensor([s_w], device="cuda"), 50, ff.ACT_SILU
    ff.ff_gated_forward(*args, dg, None, None, None, None, None, ws)
    ff.ff_gated_forward(*args, far, None, None, None, None, None, ws)
    assert torch.equal(far, dg)


def test_work_on_another_stream():
    rows, n, k = 64, 96, 128
    aq, wq = torch.zeros((rows, k), dtype=torch.int8, device="cuda"), torch.ones((2 * n, k), dtype=torch.int8, device="cuda")
    one, y = torch.ones(1, device="cuda"), torch.empty((rows, n), device="cuda")
    ws = torch.empty(ff.ff_gated_workspace_bytes(rows, n, k), dtype=torch.uint8, device="cuda")
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        for _ in range(20):
            aq.add_(1)
        ff.ff_gated_forward(aq, wq, one, one, k, ff.ACT_IDENTITY, y, None, None, None, None, None, ws)
    side.synchronize()
    assert (y == (20 * k) ** 2).all()
