"""Shared by the tests of gated layers, group norm and dropout: bounds on an activation's roundings."""
import numpy as np

import paper_2506_22771_amd as ff
from norm_util import U
from oracle import norm_oracle as N

ACTS = {"identity": ff.ACT_IDENTITY, "relu": ff.ACT_RELU, "gelu": ff.ACT_GELU, "silu": ff.ACT_SILU}


# f and f' are fp32 functions, good to a few units in the last place of the largest term they are made of: 1 for sigma and Phi, |u| for f.  Phi is off by 1.3 U for
# 16-bit values and U / 14 for fp32 by its approximation, exp2 and rcp by a unit each; twelve roundings follow at most.
def act_errors(kind, u):
    """(error of f, error of f') at fp32 arguments u."""
    f, _ = N.act(kind, u)
    smooth = kind in ("gelu", "silu")
    return 16 * U * (np.abs(f) + 0.2 * np.abs(u)) if smooth else 0 * u, 16 * U * (1.2 + 0 * u) if smooth else 0 * u


def act_slope(kind, u, du):
    """How far f and f' are where the argument is off by du: by their largest slopes (f' at most 1.13, f'' at most 0.8), or across ReLU's border."""
    if kind == "identity":
        return du, 0 * du
    if kind == "relu":
        return du, (np.abs(u) <= du).astype(np.float64)
    return 1.13 * du, 0.8 * du
