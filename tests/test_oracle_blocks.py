"""The oracle of gated layers, group norm and dropout against definitions and differences, on the CPU."""
import numpy as np
import pytest

from oracle import blocks_oracle as B
from oracle import norm_oracle as N


@pytest.mark.parametrize("kind", ["identity", "relu", "gelu", "silu"])
def test_gated_gradient_against_differences(kind):
    rng = np.random.default_rng(1)
    g, u, dy, c = rng.standard_normal((5, 7)), rng.standard_normal((5, 7)), rng.standard_normal((5, 7)), rng.standard_normal(5)
    loss = lambda g, u: (dy * N.act(kind, g)[0] * u).sum() + (c[:, None] * (N.act(kind, g)[0] * u) ** 2).sum()  # noqa: E731
    dg, du = B.gated_backward(g, u, kind, c, dy)
    for i in range(5):
        for j in range(7):
            e = np.zeros_like(g)
            e[i, j] = 1e-5
            assert abs((loss(g + e, u) - loss(g - e, u)) / 2e-5 - dg[i, j]) < 1e-7
            assert abs((loss(g, u + e) - loss(g, u - e)) / 2e-5 - du[i, j]) < 1e-7


def test_gated_forward_is_two_products():
    rng = np.random.default_rng(2)
    a, w = rng.integers(-127, 128, (3, 9), dtype=np.int8), rng.integers(-127, 128, (8, 9), dtype=np.int8)
    y, good, g, u = B.gated_forward(a, w, 0.01, "silu")
    for m in range(3):
        for j in range(4):
            gv = 0.01 * sum(int(a[m, k]) * int(w[j, k]) for k in range(9))
            uv = 0.01 * sum(int(a[m, k]) * int(w[4 + j, k]) for k in range(9))
            assert abs(g[m, j] - gv) < 1e-12 and abs(u[m, j] - uv) < 1e-12
            assert abs(y[m, j] - gv / (1 + np.exp(-gv)) * uv) < 1e-9
    np.testing.assert_allclose(good, [(r**2).sum() for r in y])


@pytest.mark.parametrize("kind", ["identity", "gelu", "silu", "relu"])
@pytest.mark.parametrize("samples, pixels, channels, groups", [(2, 3, 6, 3), (1, 5, 4, 1), (3, 4, 4, 4)])
def test_group_norm_gradients_against_differences(kind, samples, pixels, channels, groups):
    rng = np.random.default_rng(3)
    x, dy = rng.standard_normal((samples * pixels, channels)), rng.standard_normal((samples * pixels, channels))
    w, b, c = 1 + 0.3 * rng.standard_normal(channels), 0.3 * rng.standard_normal(channels), rng.standard_normal(samples)

    def loss(x, w, b):
        y, *_, good = B.group_norm_forward(x, samples, groups, w, b, 1e-5, kind)
        return (dy * y).sum() + (c * good).sum()

    y, h, mean, rstd, _ = B.group_norm_forward(x, samples, groups, w, b, 1e-5, kind)
    part = x.reshape(samples, pixels, groups, -1)[0, :, 0]
    assert abs(mean[0, 0] - part.mean()) < 1e-12 and abs(rstd[0, 0] - (part.var() + 1e-5) ** -0.5) < 1e-9
    dx, dw, db, _ = B.group_norm_backward(dy, c, h, rstd, samples, groups, w, b, kind)
    for args, grad in ((0, dx), (1, dw), (2, db)):
        for at in np.ndindex(grad.shape):
            v = [x, w, b]
            e = np.zeros_like(v[args])
            e[at] = 1e-6
            hi, lo = list(v), list(v)
            hi[args], lo[args] = v[args] + e, v[args] - e
            assert abs((loss(*hi) - loss(*lo)) / 2e-6 - grad[at]) < 2e-6 * max(1, np.abs(grad).max())


def test_dropout_keeps_its_share_and_its_mean():
    x = np.ones((200, 300))
    for p in (0.0, 0.1, 0.5, 0.9):
        y, kept = B.dropout(x, None, p, 3, 4)
        n = x.size
        assert abs(kept.mean() - (1 - p)) <= 5 * np.sqrt(p * (1 - p) / n)      # five standard deviations of a share
        assert abs(y.mean() - 1) <= 5 * np.sqrt(p / (1 - p) / n) + 1e-7
    assert not B.dropout(x, None, 1.0, 3, 4)[0].any()
    assert (B.dropout(x, 2 * x, 1.0, 3, 4)[0] == 2).all()
