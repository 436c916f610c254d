"""8-bit checkpoints on the device: codes and exponent bytes bit for bit, values read back, gradients through activations."""
import numpy as np
import pytest
import torch

import paper_2506_22771_amd as ff
from norm_util import DTYPES, HALF_ULP, TINY, U, Framed, junk_ckpt, padded_ckpt, split_ckpt, typed, values, within
from oracle import norm_oracle as N

pytestmark = pytest.mark.gpu
ACTS = {"identity": ff.ACT_IDENTITY, "relu": ff.ACT_RELU, "gelu": ff.ACT_GELU, "silu": ff.ACT_SILU}


def hard_values(rows, cols, seed, dtype="float32"):
    """Blocks of very different sizes, at the edges of exponents and codes; zeros, subnormals, the type's largest values."""
    rng = np.random.default_rng(seed)
    x = rng.standard_normal((rows, cols)) * np.exp(rng.standard_normal((rows, 1)))
    nb = (cols + 31) // 32
    for b in range(nb):
        r, at = rng.integers(rows), slice(32 * b, min(cols, 32 * b + 32))
        kind = int(rng.integers(8))
        n = x[r, at].size
        if kind == 0:
            x[r, at] = 0
        elif kind == 1:
            x[r, at] = rng.integers(-254, 255, n) / 2      # halves: ties of codes of scale 1
            x[r, at][0] = 127
        elif kind == 2:
            x[r, at] = rng.choice([127, 127.5, -127, 126.5, 0.5, -0.5], n)
        elif kind == 3:
            x[r, at] *= 1e-4 if dtype == "float16" else 2.0**-101
        elif kind == 4:
            x[r, at] *= 1e-6 if dtype == "float16" else 1e-40
        elif kind == 5:
            x[r, at] = float(torch.finfo(DTYPES[dtype]).max) * rng.choice([1, -1, 0.5, 0.3], n)
        elif kind == 6:
            x[r, at] = -0.0
    with np.errstate(over="ignore"):
        return torch.from_numpy(x).to(DTYPES[dtype]).float().numpy()


SHAPES = [(1, 1), (3, 7), (5, 31), (4, 32), (6, 33), (2, 64), (7, 100), (3, 512), (5, 513), (9, 784), (33, 500), (2, 2000), (1, 16500), (70, 36)]


@pytest.mark.parametrize("stochastic", [False, True])
@pytest.mark.parametrize("dtype", list(DTYPES))
@pytest.mark.parametrize("rows, cols", SHAPES)
def test_codes_bit_for_bit_and_values_read_back(rows, cols, dtype, stochastic):
    x = hard_values(rows, cols, rows * 1000 + cols, dtype)
    seed, tag = 31 + rows, ff.ff_stream_tag(3, 1, 0, 0)
    rq, re = N.ckpt_store(x, N.uniforms(rows, cols, seed, tag) if stochastic else None)
    left, right = (0, 0) if cols % 2 else (1, 2)   # (odd element offsets and strides for half of the shapes)
    frame = Framed(rows, cols, dtype, left, right, torch.from_numpy(x).to(DTYPES[dtype]))
    q, e = junk_ckpt(rows, cols)
    ff.ff_ckpt_store(frame.view, ff.ROUND_STOCHASTIC if stochastic else ff.ROUND_NEAREST, seed, tag, q, e)
    gq, ge = split_ckpt(q, e, cols)
    np.testing.assert_array_equal(ge, re)
    np.testing.assert_array_equal(gq, rq)
    assert frame.intact()
    ref = N.ckpt_load(rq, re)
    for out in DTYPES:
        to = Framed(rows, cols, out, left, right)
        ff.ff_ckpt_load(q, e, to.view)
        want = np.clip(ref, -65504, 65504) if out == "float16" else ref
        if out != "float16":
            np.testing.assert_array_equal(values(to.view), want)        # exact
        else:
            within(values(to.view), want, np.abs(want) * HALF_ULP[out] + TINY[out], out)
        assert to.intact()


def test_blocks_with_infinities_and_nan_read_as_nan_and_leave_others_alone():
    x = np.random.default_rng(0).standard_normal((4, 100)).astype(np.float32)
    x[0, 5], x[1, 40], x[2, 99] = np.inf, np.nan, -np.inf
    rq, re = N.ckpt_store(x)
    for mode in (ff.ROUND_NEAREST, ff.ROUND_STOCHASTIC):
        q, e = junk_ckpt(4, 100)
        ff.ff_ckpt_store(typed(x, "float32"), mode, 1, 2, q, e)
        gq, ge = split_ckpt(q, e, 100)
        np.testing.assert_array_equal(ge, re)
        assert not gq[ge.repeat(32, 1)[:, :100] == 255].any()
        for dtype, of in DTYPES.items():
            to = torch.empty((4, 100), dtype=of, device="cuda")
            ff.ff_ckpt_load(q, e, to)
            np.testing.assert_array_equal(np.isnan(values(to)), re.repeat(32, 1)[:, :100] == 255)


def test_no_rows():
    for dtype in DTYPES.values():
        x = torch.empty((0, 40), dtype=dtype, device="cuda")
        q, e = ff.ckpt_empty(0, 40)
        ff.ff_ckpt_store(x, ff.ROUND_NEAREST, 0, 0, q, e)
        ff.ff_ckpt_load(q, e, x)
        ff.ff_ckpt_act_backward(q, e, ff.ACT_GELU, None, x, x)


def test_elements_beyond_32_bits_of_index():
    """A matrix of more than 2^32 elements: offsets, and the random words of the last row, whose index has a high word."""
    rows, cols = (1 << 17) + 3, 32775
    x = torch.zeros((rows, cols), dtype=torch.bfloat16, device="cuda")
    tail = torch.randn((2, cols), device="cuda", generator=torch.Generator("cuda").manual_seed(1)).bfloat16()
    x[-2:] = tail
    q, e = ff.ckpt_empty(rows, cols)
    ff.ff_ckpt_store(x, ff.ROUND_STOCHASTIC, 9, 4, q, e)
    first = (rows - 2) * cols
    assert first > 1 << 32
    m64, m32 = (1 << 64) - 1, 0xFFFFFFFF
    z = (9 + 0x9E3779B97F4A7C15 * 5) & m64
    z = ((z ^ (z >> 30)) * 0xBF58476D1CE4E5B9) & m64
    z = ((z ^ (z >> 27)) * 0x94D049BB133111EB) & m64
    z ^= z >> 31
    idx = np.arange(first, first + 2 * cols, dtype=np.uint64)
    v = (idx & np.uint64(m32)) ^ ((np.uint64(z & m32) + (idx >> np.uint64(32)) * np.uint64((z >> 32) | 1)) & np.uint64(m32))
    v ^= v >> np.uint64(16)
    v = (v * np.uint64(0x7FEB352D)) & np.uint64(m32)
    v ^= v >> np.uint64(15)
    v = (v * np.uint64(0x846CA68B)) & np.uint64(m32)
    v ^= v >> np.uint64(16)
    u = (v >> np.uint64(8)).astype(np.float64).reshape(2, cols) * 2.0**-24
    rq, re = N.ckpt_store(tail.float().cpu().numpy(), u)
    gq, ge = split_ckpt(q[-2:], e[-2:], cols)
    np.testing.assert_array_equal(ge, re)
    np.testing.assert_array_equal(gq, rq)
    del x
    back = torch.full((rows, cols), 7.0, dtype=torch.bfloat16, device="cuda")
    ff.ff_ckpt_load(q, e, back)
    np.testing.assert_array_equal(values(back[-2:]), N.ckpt_load(rq, re))
    assert not back[:-2].any()
    dx = back
    ff.ff_ckpt_act_backward(q, e, ff.ACT_IDENTITY, None, back, dx)
    np.testing.assert_array_equal(values(dx[-2:]), N.ckpt_load(rq, re))


# dx = (dy + 2 c f) f': f and f' are fp32 functions, good to a few units in the last place of the largest term they are made of: 1 for sigma and Phi,
# |u| for f.  Phi is off by 1.3 U for 16-bit values and U / 14 for fp32 by its approximation, exp2 and rcp by a unit each; twelve roundings follow at most.
def act_bound(kind, u, coeff, dy, dtype):
    f, d = N.act(kind, u)
    up = np.abs(dy if dy is not None else 0.0) + (2 * np.abs(coeff[:, None] * f) if coeff is not None else 0.0)
    df = 16 * U * (np.abs(f) + np.abs(u) * 0.2) if kind in ("gelu", "silu") else 0 * u
    dd = 16 * U * (1.2 + 0 * u) if kind in ("gelu", "silu") else 0 * u
    ref = N.act_backward(kind, u, coeff, dy)
    err = up * dd + (2 * np.abs(coeff[:, None]) * df * np.abs(d) if coeff is not None else 0) + 4 * U * up * np.abs(d)
    return err * (1 + HALF_ULP[dtype]) + np.abs(ref) * HALF_ULP[dtype] + TINY[dtype]


@pytest.mark.parametrize("with_dy, with_coeff", [(True, False), (True, True), (False, True)])
@pytest.mark.parametrize("dtype", list(DTYPES))
@pytest.mark.parametrize("kind", list(ACTS))
def test_activation_gradient(kind, dtype, with_dy, with_coeff):
    for rows, cols, left, right in [(1, 1, 0, 0), (5, 37, 1, 0), (64, 500, 0, 0), (130, 96, 3, 5)]:
        rng = np.random.default_rng(rows + cols)
        u = (rng.standard_normal((rows, cols)) * rng.choice([0.01, 1, 5, 40], (rows, 1))).astype(np.float32)
        u[rng.random((rows, cols)) < 0.05] = 0
        rq, re = N.ckpt_store(u)
        q, e = padded_ckpt(rq, re)
        uv = N.ckpt_load(rq, re)
        coeff = rng.standard_normal(rows).astype(np.float32) * 0.05 if with_coeff else None
        dy = Framed(rows, cols, dtype, left, right, typed(rng.standard_normal((rows, cols)), dtype)) if with_dy else None
        to = Framed(rows, cols, dtype, right, left)
        dc = torch.from_numpy(coeff).cuda() if with_coeff else None
        ff.ff_ckpt_act_backward(q, e, ACTS[kind], dc, dy.view if with_dy else None, to.view)
        dyv = values(dy.view) if with_dy else None
        c64 = coeff.astype(np.float64) if with_coeff else None
        within(values(to.view), N.act_backward(kind, uv, c64, dyv), act_bound(kind, uv, c64, dyv, dtype), f"{kind} {rows}x{cols}")
        assert to.intact()
        if with_dy:
            assert dy.intact()
            ref = values(to.view)
            ff.ff_ckpt_act_backward(q, e, ACTS[kind], dc, dy.view, dy.view)     # in place
            np.testing.assert_array_equal(values(dy.view), ref)


@pytest.mark.parametrize("kind", list(ACTS))
def test_activation_gradient_at_extreme_arguments(kind):
    """Arguments where exp under- or overflows, and blocks that read as NaN."""
    u = np.zeros((6, 32), np.float32)
    for r, v in enumerate([1e30, -1e30, 100.0, -100.0, 3e38, 0.0]):
        u[r] = v
    rq, re = N.ckpt_store(u)
    re[5] = 255
    q, e = padded_ckpt(rq, re)
    dy = torch.ones((6, 32), device="cuda")
    dx = torch.empty_like(dy)
    ff.ff_ckpt_act_backward(q, e, ACTS[kind], None, dy, dx)
    got = values(dx)
    if kind == "identity":
        assert (got == 1).all()
    else:
        assert (got[[0, 2, 4]] == 1).all() and (got[[1, 3]] == 0).all() and np.isnan(got[5]).all()


@pytest.mark.parametrize("kind", ["gelu", "silu"])
def test_activation_gradient_against_differences(kind):
    """d/du of dy f(u) + c f(u)^2 by central differences in 64 bits (error 1e-9), where fp32 gives 1e-5."""
    rng = np.random.default_rng(8)
    rq, re = N.ckpt_store((rng.standard_normal((16, 64)) * 2).astype(np.float32))
    q, e = padded_ckpt(rq, re)
    u, dy, c = N.ckpt_load(rq, re), rng.standard_normal((16, 64)).astype(np.float32), rng.standard_normal(16).astype(np.float32)
    loss = lambda u: dy * N.act(kind, u)[0] + c[:, None] * N.act(kind, u)[0] ** 2  # noqa: E731
    dx = torch.empty((16, 64), device="cuda")
    ff.ff_ckpt_act_backward(q, e, ACTS[kind], torch.from_numpy(c).cuda(), torch.from_numpy(dy).cuda(), dx)
    assert np.abs((loss(u + 1e-5) - loss(u - 1e-5)) / 2e-5 - values(dx)).max() < 1e-4


def test_work_on_another_stream():
    """The calls run on the current stream, behind what it already holds."""
    x = torch.zeros((512, 4096), device="cuda")
    q, e = ff.ckpt_empty(512, 4096)
    back = torch.empty_like(x)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        for _ in range(20):
            x.add_(1.0)
        ff.ff_ckpt_store(x, ff.ROUND_NEAREST, 0, 0, q, e)
        ff.ff_ckpt_load(q, e, back)
    side.synchronize()
    assert (back == 20).all()


@pytest.mark.parametrize("dtype", list(DTYPES))
@pytest.mark.parametrize("rows, cols", [(3000, 101), (999, 13), (2000, 3), (40, 4097)])
def test_activation_gradient_in_place_of_many_ragged_rows(rows, cols, dtype):
    """Rows end inside chunks that other wavefronts share with their neighbours: none may read what another has written."""
    g = torch.Generator("cuda").manual_seed(rows)
    q, e = ff.ckpt_empty(rows, cols)
    ff.ff_ckpt_store(torch.randn((rows, cols), device="cuda", generator=g), ff.ROUND_NEAREST, 0, 0, q, e)
    c = torch.randn(rows, device="cuda", generator=g)
    dy = torch.randn((rows, cols), device="cuda", generator=g).to(DTYPES[dtype])
    for kind in ("gelu", "identity"):
        for coeff in (c, None):
            dx = torch.empty_like(dy)
            ff.ff_ckpt_act_backward(q, e, ACTS[kind], coeff, dy, dx)
            over = dy.clone()
            ff.ff_ckpt_act_backward(q, e, ACTS[kind], coeff, over, over)
            assert torch.equal(over, dx)
