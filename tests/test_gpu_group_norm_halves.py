"""Group norm of rows that end in the middle of a chunk of eight columns, in groups of whole fours: the kernels of any row, forward and backward, from a few channels to rows that no
workgroup holds.  Bounds as in test_gpu_group_norm.py."""
import pytest

import paper_2506_22771_amd as ff
import test_gpu_group_norm as G

pytestmark = pytest.mark.gpu

# samples, pixels, channels, groups; of the wide ones 2 x 1 x 4804 fits a workgroup forward, 6004 and 8188 in one group do not
SHAPES = [(2, 9, 12, 1), (2, 16, 20, 5), (3, 33, 28, 7), (1, 200, 60, 3), (2, 1000, 12, 3), (2, 3000, 36, 1), (2, 1, 4804, 1), (1, 1, 6004, 1501), (1, 4, 6004, 1), (3, 2, 6004, 1),
          (4, 1, 6004, 19), (64, 1, 6004, 1), (1, 4, 8188, 1), (1, 16, 7996, 1)]


@pytest.mark.parametrize("samples, pixels, channels, groups", SHAPES)
def test_forward(samples, pixels, channels, groups):
    assert channels % 8 == 4 and channels // groups % 4 == 0 and ff.ff_group_norm_workspace_bytes(samples, pixels, channels, groups) > 0
    G.test_forward(samples, pixels, channels, groups)


@pytest.mark.parametrize("samples, pixels, channels, groups", SHAPES)
def test_backward(samples, pixels, channels, groups):
    G.test_backward(samples, pixels, channels, groups)
