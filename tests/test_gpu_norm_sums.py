"""The column sums of the norm's backward pass: the same bits whatever else the call is asked for."""
import pytest
import torch

import paper_2506_22771_amd as ff
from norm_util import DTYPES
from test_gpu_norm import EPS, inputs, run_backward

pytestmark = pytest.mark.gpu

# few rows, whose column sums other workgroups of the launch may make, and more; whole chunks and ragged rows; rows beyond the registers
SHAPES = [(1, 784), (7, 5), (70, 24), (128, 784), (200, 500), (256, 1001), (300, 783), (512, 784), (512, 2001), (900, 2000), (1000, 4096), (700, 12001), (1100, 300), (2100, 2000),
          (5, 20000)]


@pytest.mark.parametrize("dtype", list(DTYPES))
@pytest.mark.parametrize("rows, cols", SHAPES)
def test_equal_inputs_give_equal_bits(rows, cols, dtype):
    """In place and not, with dx and without, both sums and one, in a view and not."""
    x, dy, w, b = inputs(rows, cols, dtype)
    w = torch.from_numpy(w).float().cuda()
    m, r, q_e = torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda"), ff.ckpt_empty(rows, cols)
    ff.ff_layer_norm_forward(x, None, None, EPS, torch.empty_like(x), m, r, *q_e)
    wide = torch.empty((rows, cols + 3), dtype=DTYPES[dtype], device="cuda")
    for source in ("x", "kept"):
        tail = (m, None, None, r, w) if source == "x" else (None, *q_e, r, w)
        of = x if source == "x" else None
        dx = torch.empty_like(dy)
        first = run_backward(dy, of, *tail, dx)
        over = dy.clone()
        forms = {"over dy": (run_backward(over, of, *tail, over), over), "without dx": (run_backward(dy, of, *tail, None), dx)}
        view = wide[:, 1:cols + 1]
        view.copy_(dy)
        forms["over a view of dy"] = (run_backward(view, of, *tail, view), view)
        if source == "x":
            over_x = x.clone()
            forms["over x"] = (run_backward(dy, over_x, *tail, over_x), over_x)
        for what, (sums, got) in forms.items():
            assert torch.equal(got, dx) and torch.equal(sums[0], first[0]) and torch.equal(sums[1], first[1]), (source, what)
        over = dy.clone()
        aw, ab = run_backward(over, of, *tail, over, True, 0.5)
        assert torch.equal(aw, first[0] + 0.5) and torch.equal(ab, first[1] + 0.5) and torch.equal(over, dx)
        ws, one = torch.empty(ff.ff_layer_norm_workspace_bytes(rows, cols), dtype=torch.uint8, device="cuda"), torch.empty(cols, device="cuda")
        over = dy.clone()
        ff.ff_layer_norm_backward(over, of, *tail, over, one, None, False, ws)
        assert torch.equal(one, first[0]) and torch.equal(over, dx)
