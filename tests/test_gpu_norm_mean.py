"""The mean of a row, where its values' sum is exact: what is done for rows far from zero takes nothing from others."""
import numpy as np
import pytest
import torch

import paper_2506_22771_amd as ff
from norm_util import DTYPES, U, typed, values, within

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", list(DTYPES))
@pytest.mark.parametrize("cols", [3, 30, 100, 500, 784, 1000, 2000, 4096, 12001, 33000])
@pytest.mark.parametrize("offset", [0, 1, 60])
def test_mean_of_whole_numbers(cols, offset, dtype):
    """Sums of whole numbers below 2^24 are exact, so the mean has the roundings of 1 / cols and of the product, and one more where the deviations' mean is added, whose
    own error is U / cols of the sum of their magnitudes, with two roundings for the sum of each of two dozen levels and of a lane's values at worst: next to nothing
    beside a mean that is larger than the spread."""
    rng = np.random.default_rng(cols + offset)
    x = rng.integers(-60, 61, (5, cols)) + offset
    m = torch.empty(5, device="cuda")
    t = typed(x, dtype)
    ff.ff_layer_norm_forward(t, None, None, 1e-5, torch.empty_like(t), m, None)
    mean, spread = x.mean(1), x.std(1)
    near = np.abs(mean) < 0.9 * spread
    deviations = (64 + cols // 1024) * U * np.abs(x - mean[:, None]).mean(1)
    within(values(m), mean, 2.01 * U * np.abs(mean) + np.where(near, 0, U * np.abs(mean) + deviations), "mean")
