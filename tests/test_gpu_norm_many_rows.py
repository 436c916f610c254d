"""The norm's backward pass over more rows than one launch makes column sums of: every lane group's sums, through the workspace and the launch that adds them."""
import pytest

import test_gpu_norm
from norm_util import DTYPES

pytestmark = pytest.mark.gpu

# 4, 8, 16, 32 and 64 lanes, 64 with two and three chunks, 256 with one and two, 512 with two and four; whole chunks and ragged rows
SHAPES = [(5000, 24), (2000, 7), (3000, 60), (3000, 64), (2500, 120), (2500, 127), (1500, 250), (1500, 256), (1500, 400), (1500, 501), (1500, 784), (1500, 783),
          (8200, 1104), (1500, 2000), (1500, 2001), (1200, 4096), (1200, 4001), (1100, 8192), (1100, 8191), (1050, 10240), (1050, 9001)]


@pytest.mark.parametrize("dtype", list(DTYPES))
@pytest.mark.parametrize("rows, cols", SHAPES)
def test_sums_through_the_workspace(rows, cols, dtype):
    test_gpu_norm.test_backward(rows, cols, dtype)
