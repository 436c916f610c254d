"""Gated layers, group norm over channels-last maps and dropout, in numpy and 64 bits.  Test infrastructure only."""
from __future__ import annotations

import numpy as np

from .norm_oracle import act, uniforms


def gated_forward(a_q, w_q, scale, kind):
    """(y, goodness, g, u) in fp64 from int8 codes without pad columns; w_q [2n, k], the gate's rows first."""
    acc = a_q.astype(np.float64) @ w_q.astype(np.float64).T    # (whole numbers below 2^53: exact)
    n = w_q.shape[0] // 2
    g, u = acc[:, :n] * float(scale), acc[:, n:] * float(scale)
    y = act(kind, g)[0] * u
    return y, (y * y).sum(1), g, u


def gated_backward(g, u, kind, coeff, dy):
    """(dg, du) in fp64."""
    f, d = act(kind, g)
    t = np.zeros_like(g) if dy is None else np.asarray(dy, np.float64)
    if coeff is not None:
        t = t + 2.0 * np.asarray(coeff, np.float64)[:, None] * f * u
    return t * u * d, t * f


def spread(v, pixels, per):
    """Values of [samples, groups] at every place of the map [samples * pixels, groups * per]."""
    return np.repeat(np.repeat(np.asarray(v, np.float64), per, 1), pixels, 0)


def of_groups(v, samples, groups):
    """Sums of a map over every sample's groups, [samples, groups]."""
    rows, channels = v.shape
    return v.reshape(samples, rows // samples, groups, channels // groups).sum((1, 3))


def group_norm_forward(x, samples, groups, weight, bias, eps, kind):
    """(y, h, mean, rstd, goodness) in fp64."""
    x = np.asarray(x, np.float64)
    pixels, per = x.shape[0] // max(1, samples), x.shape[1] // groups
    m = pixels * per
    mean = of_groups(x, samples, groups) / m
    dev = x - spread(mean, pixels, per)
    rstd = 1.0 / np.sqrt(of_groups(dev**2, samples, groups) / m + eps)
    h = dev * spread(rstd, pixels, per)
    y = act(kind, affine(h, weight, bias))[0]
    return y, h, mean, rstd, (y**2).reshape(samples, -1).sum(1)


def affine(h, weight, bias):
    return h * (1.0 if weight is None else np.asarray(weight, np.float64)) + (0.0 if bias is None else np.asarray(bias, np.float64))


def group_norm_backward(dy, coeff, h, rstd, samples, groups, weight, bias, kind):
    """(dx, dweight, dbias, dz) in fp64."""
    h = np.asarray(h, np.float64)
    pixels, per = h.shape[0] // max(1, samples), h.shape[1] // groups
    f, d = act(kind, affine(h, weight, bias))
    dz = np.zeros_like(h) if dy is None else np.asarray(dy, np.float64)
    if coeff is not None:
        dz = dz + 2.0 * np.repeat(np.asarray(coeff, np.float64), pixels)[:, None] * f
    dz = dz * d
    g = dz * (1.0 if weight is None else np.asarray(weight, np.float64))
    mean = lambda v: spread(of_groups(v, samples, groups) / (pixels * per), pixels, per)  # noqa: E731
    dx = spread(rstd, pixels, per) * (g - mean(g) - h * mean(g * h))
    return dx, (dz * h).sum(0), dz.sum(0), dz


def dropout(x, r, p, seed, tag):
    """(y, kept) in fp64; p as fp32 holds it."""
    x = np.asarray(x, np.float64)
    p = float(np.float32(p))
    kept = uniforms(*x.shape, seed, tag) >= p
    y = np.where(kept, x / (1.0 - p) if p < 1 else 0.0, 0.0)
    return y if r is None else y + np.asarray(r, np.float64), kept
