"""Gated layers in many tiles, the last of every row of which leave wavefronts without columns: such a wavefront goes on to the next tile at once, whose steps are copied to where the
others' outputs were staged."""
import pytest

import test_gpu_gated as G

pytestmark = pytest.mark.gpu


# reductions of one step of 128 bytes to three; 32 columns of 64, and 32 and 64 of 128
@pytest.mark.parametrize("rows, n, k, dtype", [(2000, 1568, 200, "float32"), (3000, 1504, 100, "bfloat16"), (8200, 2080, 200, "float32"), (8200, 2112, 250, "bfloat16"),
                                               (8200, 2080, 380, "float16"), (16390, 1056, 256, "float32")])
def test_wavefronts_without_columns(rows, n, k, dtype):
    G.test_forward_of_many_tiles(rows, n, k, dtype)
