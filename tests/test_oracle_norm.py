"""The 64-bit restatements that the GPU tests compare with: against hand-worked cases, brute force and differences."""
import numpy as np
import pytest

from oracle import ff_oracle as O
from oracle import norm_oracle as N


def test_uniforms_are_the_librarys():
    for seed, tag, rows, cols in [(0, 0, 2, 5), (12345, 1 << 20, 3, 7), (2**40 + 3, 77, 1, 64)]:
        u = N.uniforms(rows, cols, seed, tag)
        assert [O.uniform(seed, tag, i) for i in range(rows * cols)] == list(u.reshape(-1))


def test_exponents_by_hand():
    up = lambda v: float(np.nextafter(np.float32(v), np.float32(np.inf)))  # noqa: E731
    for amax, s in [(127.0, 0), (up(127.0), 1), (254.0, 1), (1.0, -6), (127 / 64, -6), (up(127 / 64), -5), (2.0**-100, -106),
                    (127 * 2.0**121, 121), (float(np.finfo(np.float32).max), 121)]:
        assert N.exponent_of(amax) == s + 127
    assert N.exponent_of(0.0) == 127 and N.exponent_of(2.0**-101) == 127
    assert N.exponent_of(float("inf")) == 255 and N.exponent_of(float("nan")) == 255


def test_codes_by_hand():
    x = np.zeros((1, 40), np.float32)
    x[0, :6] = [127, -127, 0.5, 1.5, 2.5, -0.49]      # scale 1: ties to even
    x[0, 32:35] = [1.0, -1.0, 1 / 64]                 # scale 2^-6
    q, e = N.ckpt_store(x)
    assert list(q[0, :6]) == [127, -127, 0, 2, 2, 0] and list(q[0, 32:35]) == [64, -64, 1] and list(e[0]) == [127, 121]
    np.testing.assert_array_equal(N.ckpt_load(q, e)[0, 32:35], [1.0, -1.0, 1 / 64])
    x[0, 33] = np.inf
    q, e = N.ckpt_store(x)
    assert e[0, 1] == 255 and not q[0, 32:].any() and np.isnan(N.ckpt_load(q, e)[0, 32:]).all()


def test_stochastic_codes_are_unbiased_and_near():
    rng = np.random.default_rng(0)
    x = np.tile(rng.standard_normal((1, 64)).astype(np.float32), (4000, 1))
    q, e = N.ckpt_store(x, N.uniforms(4000, 64, 5, 9))
    step = np.repeat(np.exp2(e.astype(float) - 127), 32, 1)
    err = (N.ckpt_load(q, e) - x) / step
    assert np.abs(err).max() < 1 and np.abs(err.mean(0)).max() < 5 * 0.5 / np.sqrt(4000)


@pytest.mark.parametrize("cols", [1, 2, 33])
def test_norm_gradients_against_differences(cols):
    rng = np.random.default_rng(cols)
    x, w, b, dy = rng.standard_normal((3, cols)), rng.standard_normal(cols), rng.standard_normal(cols), rng.standard_normal((3, cols))
    y, h, mean, rstd = N.norm_forward(x, w, b, 1e-3)
    loss = lambda x, w, b: float((dy * N.norm_forward(x, w, b, 1e-3)[0]).sum())  # noqa: E731
    dx, dw, db = N.norm_backward(dy, h, rstd, w)
    d = 1e-6
    for c in range(cols):
        one = np.zeros(cols)
        one[c] = d
        assert abs((loss(x, w + one, b) - loss(x, w - one, b)) / (2 * d) - dw[c]) < 1e-7
        assert abs((loss(x, w, b + one) - loss(x, w, b - one)) / (2 * d) - db[c]) < 1e-7
        for r in range(3):
            at = np.zeros_like(x)
            at[r, c] = d
            assert abs((loss(x + at, w, b) - loss(x - at, w, b)) / (2 * d) - dx[r, c]) < 1e-5


@pytest.mark.parametrize("kind", ["identity", "relu", "gelu", "silu"])
def test_activation_gradient_against_differences(kind):
    rng = np.random.default_rng(3)
    u, dy, c = rng.standard_normal((4, 50)) * 2, rng.standard_normal((4, 50)), rng.standard_normal(4)
    got = N.act_backward(kind, u, c, dy)
    loss = lambda u: dy * N.act(kind, u)[0] + c[:, None] * N.act(kind, u)[0] ** 2  # noqa: E731
    d = 1e-6
    assert np.abs((loss(u + d) - loss(u - d)) / (2 * d) - got).max() < 1e-7
    assert np.array_equal(N.act_backward(kind, u, None, dy), dy * N.act(kind, u)[1])


def test_weight_gradient_is_that_of_the_affine_input():
    rng = np.random.default_rng(4)
    h, dy, g, b = rng.standard_normal((9, 5)), rng.standard_normal((9, 4)), rng.standard_normal(5), rng.standard_normal(5)
    dw, db = N.weight_grad(dy, h, g, b)
    np.testing.assert_allclose(dw, dy.T @ (h * g + b), rtol=1e-12)
    np.testing.assert_allclose(db, dy.sum(0), rtol=1e-12)
