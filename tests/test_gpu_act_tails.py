"""Activations far below zero, where their values are small: outputs of the group norm and of gated layers, forward and backward, are as good relative to themselves as their type's
rounding asks for."""
import numpy as np
import pytest
import torch

import paper_2506_22771_amd as ff
from blocks_util import ACTS
from norm_util import DTYPES, HALF_ULP, TINY, U, padded_ckpt, typed, values, within
from oracle import norm_oracle as N
from test_gpu_gated import padded_codes

pytestmark = pytest.mark.gpu


def of_norm(kind, dtype, most):
    """f of a bias: the groups are constant, so that h is zero."""
    u = np.linspace(-most, most, 40001, dtype=np.float32)
    x, bias = torch.zeros((1, u.size), dtype=DTYPES[dtype], device="cuda"), typed(u, "float32")
    y, ws = torch.empty_like(x), torch.empty(ff.ff_group_norm_workspace_bytes(1, 1, u.size, 1), dtype=torch.uint8, device="cuda")
    ff.ff_group_norm_forward(x, 1, 1, None, bias, 1e-5, ACTS[kind], y, None, None, None, None, None, 0, 0, 0, ws)
    return u.astype(np.float64)[None], values(y), 1.0


def of_gated(kind, dtype, most):
    """f of a gate, whole numbers times a power of two, against 63 other inputs' sum, a value of 127 * 127 * 63 of them: both exact."""
    scale = 2.0 ** np.floor(np.log2(most / 16129))
    a, w = np.full((127, 64), 127, np.int8), np.zeros((2 * 255, 64), np.int8)
    a[:, 0] = np.arange(1, 128)
    w[:255, 0] = np.arange(-127, 128)
    w[255:, 1:] = 127
    y, ws = torch.empty((127, 255), dtype=DTYPES[dtype], device="cuda"), torch.empty(ff.ff_gated_workspace_bytes(127, 255, 64), dtype=torch.uint8, device="cuda")
    ff.ff_gated_forward(padded_codes(a), padded_codes(w), torch.full((1,), scale, device="cuda"), torch.ones(1, device="cuda"), 64, ACTS[kind], y, None, None, None, None, None, ws)
    g = a[:, :1].astype(np.float64) * np.arange(-127, 128) * scale
    u = 127 * 127 * 63 * scale
    return g, values(y) / u, u


def of_gradient(kind, dtype, most):
    """du = f(g) where dy is one, of every code at several scales."""
    e = np.arange(5)[:, None] + int(np.floor(np.log2(most / 127))) - 4
    q = np.tile(np.arange(-127, 129).clip(max=127).astype(np.int8), (5, 1))
    g = q.astype(np.float64) * np.exp2(e)
    ckpt = padded_ckpt(q, np.repeat(e + 127, 8, 1).astype(np.uint8))
    one = padded_ckpt(np.ones_like(q), np.full((5, 8), 127, np.uint8))
    dy = torch.ones(q.shape, dtype=DTYPES[dtype], device="cuda")
    dg, du = torch.empty_like(dy), torch.empty_like(dy)
    ff.ff_gated_backward(*ckpt, *one, ACTS[kind], None, dy, dg, du)
    return g, values(du), 1.0


ROUTES = {"norm": of_norm, "gated": of_gated, "gradient": of_gradient}


# 16-bit GELU: Phi by a fit that is off by 2.8e-5 of itself down to -6 and by 6.1e-4 down to -9.  Its exponential's argument is rounded twice: u^2/2 times 2^-23 in the exponent,
# half of that from each.  Then: exp2 and rcp a unit (2 U) each, the reciprocal's argument U, which tell in the sum by twice their size at most, six roundings of the sum whose terms
# are up to 2.3 times what they add up to, and four products: below 32 U.  f times the value once more, and the output's rounding (of y, before it is divided by the value).
@pytest.mark.parametrize("route", list(ROUTES))
@pytest.mark.parametrize("dtype", ["bfloat16", "float16"])
def test_gelu_of_16_bits(dtype, route):
    u, got, size = ROUTES[route]("gelu", dtype, 9.0)
    ref, _ = N.act("gelu", u)
    off = np.where(u < -6, 6.1e-4, 2.8e-5) + u**2 * U + 34 * U
    within(got, ref, np.abs(ref) * (off + HALF_ULP[dtype] * (1 + off)) + TINY[dtype] / size, f"{dtype} {route}")


# fp32 SiLU: exp2 and rcp a unit (2 U) each; the exponential's second factor, its sum with one, f = u sigma and f times the value half a unit (U) each.  The argument's rounding is put right to
# below 2^-40, but for the last place of ln 2 in it: 1.91e-9 of |x| = 1.4427 |u|, 0.047 U for each of |u|.  Where sigma is a normal number.
@pytest.mark.parametrize("route", list(ROUTES))
def test_silu_of_32_bits(route):
    u, got, _ = ROUTES[route]("silu", "float32", 86.0)
    ref, _ = N.act("silu", u)
    within(got, ref, np.abs(ref) * (8 + 0.047 * np.abs(u)) * U, route)


@pytest.mark.parametrize("dtype", list(DTYPES))
@pytest.mark.parametrize("kind", ["gelu", "silu"])
def test_the_largest_arguments(kind, dtype):
    """f(u) = u far above zero, up to infinity, and 0 far below."""
    u = torch.tensor([3.0e38, 1.0e30, 200.0, float("inf"), -3.0e38, -1.0e30, -200.0, 0.0], device="cuda")
    x = torch.zeros((1, 8), dtype=DTYPES[dtype], device="cuda")
    y, ws = torch.empty_like(x), torch.empty(ff.ff_group_norm_workspace_bytes(1, 1, 8, 1), dtype=torch.uint8, device="cuda")
    ff.ff_group_norm_forward(x, 1, 1, None, u, 1e-5, ACTS[kind], y, None, None, None, None, None, 0, 0, 0, ws)
    assert torch.equal(y, u.clamp(min=0).to(DTYPES[dtype])[None])
