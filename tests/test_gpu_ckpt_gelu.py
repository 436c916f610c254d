"""The gradient through GELU in fp32 is as good as fp32 arithmetic on the formula: Phi's error is that of its roundings."""
import numpy as np
import pytest
import torch

import paper_2506_22771_amd as ff
from norm_util import U, padded_ckpt, values
from oracle import norm_oracle as N

pytestmark = pytest.mark.gpu


def arguments(scale):
    u = (np.random.default_rng(3).standard_normal((512, 1000)) * scale).astype(np.float32)
    rq, re = N.ckpt_store(u)
    return N.ckpt_load(rq, re), *padded_ckpt(rq, re)


def rms(a):
    return float(np.sqrt((a**2).mean()))


# f' = Phi + u phi: the roundings of Phi, of its argument, of the density and of the sum are each U / sqrt 3 of their terms at worst (a rounding is uniform within
# U of a value's power of two), terms that are no larger than f' over most arguments: four of them, 4^(1/2) / sqrt 3 U = 1.15 U if all were of the whole size, and less than
# U as they are not.  f adds a product of Phi's error alone, so that f f' has sqrt 2 U.
@pytest.mark.parametrize("scale", [0.3, 1.0, 4.0])
def test_as_close_as_fp32_arithmetic(scale):
    u, q, e = arguments(scale)
    f, d = N.act("gelu", u)
    dx, one, half = torch.empty(u.shape, device="cuda"), torch.ones(u.shape, device="cuda"), torch.full((len(u),), 0.5, device="cuda")
    ff.ff_ckpt_act_backward(q, e, ff.ACT_GELU, None, one, dx)
    assert rms(values(dx) - d) <= U * rms(d)
    assert np.abs(values(dx) - d).max() <= 8 * U
    ff.ff_ckpt_act_backward(q, e, ff.ACT_GELU, half, None, dx)
    assert rms(values(dx) - f * d) <= np.sqrt(2) * U * rms(f * d)
