"""Layer norm, 8-bit checkpoints and the gradients read from them, in numpy and 64 bits.  Test infrastructure only."""
from __future__ import annotations

import math

import numpy as np

BLOCK = 32


def uniforms(rows: int, cols: int, seed: int, tag: int) -> np.ndarray:
    """The uniform of every element (fp64, multiples of 2^-24): a splitmix64 finaliser of the key, a two-multiply mixer per element."""
    m64 = (1 << 64) - 1
    z = (seed + 0x9E3779B97F4A7C15 * (tag + 1)) & m64
    z = ((z ^ (z >> 30)) * 0xBF58476D1CE4E5B9) & m64
    z = ((z ^ (z >> 27)) * 0x94D049BB133111EB) & m64
    z ^= z >> 31
    idx = np.arange(rows * cols, dtype=np.uint64)
    m32 = np.uint64(0xFFFFFFFF)
    k = (np.uint64(z & 0xFFFFFFFF) + (idx >> np.uint64(32)) * np.uint64((z >> 32) | 1)) & m32
    v = (idx & m32) ^ k
    v ^= v >> np.uint64(16)
    v = (v * np.uint64(0x7FEB352D)) & m32
    v ^= v >> np.uint64(15)
    v = (v * np.uint64(0x846CA68B)) & m32
    v ^= v >> np.uint64(16)
    return (v >> np.uint64(8)).astype(np.float64).reshape(rows, cols) * 2.0**-24


def exponent_of(amax: float) -> int:
    """The exponent byte of a block of this absmax."""
    if not math.isfinite(amax):
        return 255
    if amax < 2.0**-100:
        return 127
    s = -200
    while amax > 127 * 2.0**s:   # the definition as it is said
        s += 1
    return min(s, 121) + 127


def ckpt_store(x: np.ndarray, u=None):
    """(codes int8 [rows, cols], exponent bytes [rows, blocks]) of an fp32 matrix; u: uniforms, or None for nearest-even."""
    x = np.asarray(x, np.float32)
    rows, cols = x.shape
    nb = -(-cols // BLOCK)
    q, e = np.zeros((rows, cols), np.int8), np.zeros((rows, nb), np.uint8)
    for b in range(nb):
        at = slice(b * BLOCK, min(cols, (b + 1) * BLOCK))
        part = x[:, at].astype(np.float64)
        for r in range(rows):
            a = np.abs(part[r])
            e[r, b] = exponent_of(float("nan") if np.isnan(a).any() else float(a.max()))
        fine = (e[:, b] != 255) & (np.abs(np.nan_to_num(part, nan=0, posinf=0, neginf=0)).max(1) >= 2.0**-100)
        t = np.where(fine[:, None], part, 0.0) * np.exp2(127.0 - e[:, b].astype(np.float64))[:, None]
        if u is None:
            code = np.rint(t)
        else:
            low = np.floor(t)
            frac = (t.astype(np.float32) - low.astype(np.float32)).astype(np.float64)   # (rounded to fp32, as the quantiser's definition has it)
            code = low + (u[:, at] < frac)
        q[:, at] = np.clip(np.where(fine[:, None], code, 0), -127, 127).astype(np.int8)
    return q, e


def ckpt_load(q: np.ndarray, e: np.ndarray) -> np.ndarray:
    """fp64 values of a checkpoint without pad columns."""
    s = np.repeat(np.exp2(e.astype(np.float64) - 127.0), BLOCK, axis=1)[:, :q.shape[1]]
    v = q.astype(np.float64) * s
    return np.where(np.repeat(e == 255, BLOCK, axis=1)[:, :q.shape[1]], np.nan, v)


def norm_forward(x, weight, bias, eps):
    """(y, h, mean, rstd) in fp64."""
    x = np.asarray(x, np.float64)
    mean = x.mean(1)
    rstd = 1.0 / np.sqrt(((x - mean[:, None]) ** 2).mean(1) + eps)
    h = (x - mean[:, None]) * rstd[:, None]
    return h * (1.0 if weight is None else np.asarray(weight, np.float64)) + (0.0 if bias is None else np.asarray(bias, np.float64)), h, mean, rstd


def norm_backward(dy, h, rstd, weight):
    """(dx, dweight, dbias) in fp64."""
    dy, h, rstd = (np.asarray(a, np.float64) for a in (dy, h, rstd))
    g = dy * (1.0 if weight is None else np.asarray(weight, np.float64))
    dx = rstd[:, None] * (g - g.mean(1, keepdims=True) - h * (g * h).mean(1, keepdims=True))
    return dx, (dy * h).sum(0), dy.sum(0)


def act(kind: str, u):
    """(f(u), f'(u)) in fp64."""
    u = np.asarray(u, np.float64)
    if kind == "relu":
        return np.maximum(u, 0), np.where(np.isnan(u), np.nan, (u > 0).astype(np.float64))
    if kind == "gelu":
        phi = 0.5 * np.vectorize(math.erfc, otypes=[float])(-u / math.sqrt(2.0)) if u.size else u
        return u * phi, phi + u * np.exp(-0.5 * u * u) / math.sqrt(2 * math.pi)
    if kind == "silu":
        s = 1.0 / (1.0 + np.exp(-u))
        return u * s, s * (1 + u * (1 - s))
    return u, np.ones_like(u)


def act_backward(kind, u, coeff, dy):
    f, d = act(kind, u)
    up = 0.0 if dy is None else np.asarray(dy, np.float64)
    if coeff is not None:
        up = up + 2.0 * np.asarray(coeff, np.float64)[:, None] * f
    return up * d


def weight_grad(dy, h, gamma, beta):
    """(dw, db) in fp64."""
    dy = np.asarray(dy, np.float64)
    db = dy.sum(0)
    dw = dy.T @ np.asarray(h, np.float64)
    if gamma is not None:
        dw = dw * np.asarray(gamma, np.float64)
    if beta is not None:
        dw = dw + db[:, None] * np.asarray(beta, np.float64)
    return dw, db
