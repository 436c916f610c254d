"""Dropout on the device against 64 bits: which elements are dropped is exact, what is kept is rounded."""
import numpy as np
import pytest
import torch

import paper_2506_22771_amd as ff
from norm_util import DTYPES, HALF_ULP, TINY, U, Framed, typed, values, within
from oracle import blocks_oracle as B
from oracle import norm_oracle as N

pytestmark = pytest.mark.gpu

# rows of one element to several workgroups' chunks; at both sides of a chunk, odd, and of 4096 chunks and more
SHAPES = [(1, 1), (3, 5), (2, 7), (7, 8), (5, 9), (64, 500), (33, 100), (130, 96), (1001, 87), (3, 4097), (2, 32768), (1, 40001)]


def bound(x, r, y, p, dtype):
    """The scale is rounded once, the product, the sum and the result once each."""
    kept = np.abs(x) / max(1 - p, 1e-30) if p < 1 else 0 * np.abs(x)
    return (2 * U * kept + U * np.abs(y)) * (1 + HALF_ULP[dtype]) + np.abs(y) * HALF_ULP[dtype] + TINY[dtype]


@pytest.mark.parametrize("dtype", list(DTYPES))
@pytest.mark.parametrize("rows, cols", SHAPES)
def test_forward_and_backward(rows, cols, dtype):
    rng = np.random.default_rng(rows + 3 * cols)
    x, r, dy = (typed(rng.standard_normal((rows, cols)), dtype) for _ in range(3))
    for p, residual, left, right in ((0.1, True, 0, 0), (0.5, False, 1, 2), (0.875, True, 3, 0)):
        p32 = float(np.float32(p))
        fx, fr, fy = Framed(rows, cols, dtype, left, right, x), Framed(rows, cols, dtype, right, left, r), Framed(rows, cols, dtype, right, right)
        ff.ff_dropout(fx.view, fr.view if residual else None, p, 11, 5 << 20, None, fy.view)
        ref, kept = B.dropout(values(x), values(r) if residual else None, p, 11, 5 << 20)
        within(values(fy.view), ref, bound(values(x), values(r), ref, p32, dtype), "y")
        if not residual:
            assert ((values(fy.view) == 0) == ~kept)[values(x) != 0].all()
        assert fx.intact() and fr.intact() and fy.intact()
        dx = torch.full_like(dy, 7)
        ff.ff_dropout(dy, None, p, 11, 5 << 20, None, dx)     # the gradient: the same elements
        ref, again = B.dropout(values(dy), None, p, 11, 5 << 20)
        assert (again == kept).all()
        within(values(dx), ref, bound(values(dy), 0, ref, p32, dtype), "dx")
        for to in (fx, fr):                                    # in place, over either input
            other = torch.full_like(x, 7)
            ff.ff_dropout(fx.view, fr.view if residual else None, p, 11, 5 << 20, None, other)
            if to is fr and not residual:
                continue
            ff.ff_dropout(fx.view, fr.view if residual else None, p, 11, 5 << 20, None, to.view)
            assert torch.equal(to.view, other) and to.intact()
            fx.view.copy_(x)


def test_borders_of_p():
    x = torch.randn((50, 333), device="cuda", generator=torch.Generator("cuda").manual_seed(1))
    y = torch.empty_like(x)
    ff.ff_dropout(x, None, 0.0, 1, 2, None, y)
    assert torch.equal(x, y)
    ff.ff_dropout(x, None, 1.0, 1, 2, None, y)
    assert not y.any()
    ff.ff_dropout(x, x, 1.0, 1, 2, None, y)
    assert torch.equal(x, y)
    u = N.uniforms(50, 333, 1, 2)
    for at in ((0, 0), (49, 332), (7, 100)):
        p = float(u[at])                        # (a multiple of 2^-24: exact in fp32) its own element is kept, the next p up drops it
        ff.ff_dropout(x, None, p, 1, 2, None, y)
        assert ((y != 0).cpu().numpy() == (u >= p)).all() and y[at] != 0
        up = float(np.nextafter(np.float32(p), np.float32(1)))
        ff.ff_dropout(x, None, up, 1, 2, None, y)
        assert ((y != 0).cpu().numpy() == (u >= up)).all() and y[at] == 0
    ff.ff_dropout(x, None, 1 - 2.0**-24, 1, 2, None, y)
    assert ((y != 0).cpu().numpy() == (u >= 1 - 2.0**-24)).all()


def test_what_is_dropped_is_zero_whatever_it_was():
    x = torch.full((40, 65), float("nan"), device="cuda")
    x[:, ::2] = float("inf")
    y = torch.empty_like(x)
    ff.ff_dropout(x, None, 0.5, 3, 4, None, y)
    _, kept = B.dropout(np.zeros((40, 65)), None, 0.5, 3, 4)
    y = y.cpu().numpy()
    assert (y[~kept] == 0).all() and not np.isfinite(y[kept]).any()
    x.fill_(float("nan"))
    ff.ff_dropout(x, None, 1.0, 3, 4, None, x)
    assert (x == 0).all()


def test_seeds_tags_and_steps():
    x = torch.ones((100, 100), device="cuda")
    def of(seed, tag, step=None):
        y = torch.empty_like(x)
        ff.ff_dropout(x, None, 0.5, seed, tag, None if step is None else torch.tensor([step], device="cuda"), y)
        return y.cpu().numpy()
    base = of(1, ff.ff_stream_tag(0, 3, 1, 2))
    for other in (of(2, ff.ff_stream_tag(0, 3, 1, 2)), of(1, ff.ff_stream_tag(0, 4, 1, 2)), of(1, ff.ff_stream_tag(1, 3, 1, 2))):
        assert 0.4 < (base == other).mean() < 0.6     # independent: a half agree, by 100 standard deviations of 0.005 / 5
    for step in (0, 1, 9):
        assert (of(1, ff.ff_stream_tag(0, 3, 1, 2), step) == of(1, ff.ff_stream_tag(step, 3, 1, 2))).all()


def test_graph_of_a_step_in_device_memory():
    """Every replay drops what an eager call of its step drops, with eager calls and synchronisation between them; a second graph over the same buffers."""
    x = torch.randn((300, 77), device="cuda", generator=torch.Generator("cuda").manual_seed(2)).half()
    r, y, step = x * 2, torch.empty_like(x), torch.zeros(1, dtype=torch.int64, device="cuda")
    call = lambda to, at: ff.ff_dropout(x, r, 0.3, 5, ff.ff_stream_tag(0, 1, 0, 0), at, to)  # noqa: E731
    call(y, step)
    torch.cuda.synchronize()
    graphs = [torch.cuda.CUDAGraph() for _ in range(2)]
    for g in graphs:
        with torch.cuda.graph(g):
            call(y, step)
            step.add_(1)
    assert int(step) == 0
    for i in range(5):
        graphs[i % 2].replay()
        torch.cuda.synchronize()
        eager = torch.empty_like(x)
        call(eager, torch.tensor([i], device="cuda"))
        assert torch.equal(y, eager) and int(step) == i + 1


def test_elements_beyond_32_bits_of_index():
    rows, cols = (1 << 17) + 3, 32775
    x = torch.zeros((rows, cols), dtype=torch.bfloat16, device="cuda")
    x[-2:] = 1
    ff.ff_dropout(x, None, 0.5, 9, 4, None, x)
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
    kept = (v >> np.uint64(31)).reshape(2, cols) == 1      # u >= 1/2: the top bit
    np.testing.assert_array_equal(values(x[-2:]), 2.0 * kept)
    assert not x[:-2].any()


def test_work_on_another_stream():
    x, y = torch.zeros((512, 4096), device="cuda"), torch.empty((512, 4096), device="cuda")
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        for _ in range(20):
            x.add_(1.0)
        ff.ff_dropout(x, x, 0.0, 0, 0, None, y)
    side.synchronize()
    assert (y == 40).all()
