"""The calls of gated layers, group norm and dropout take tensors of one device, the current one; as in test_norm_devices.py, tensors without memory stand for those
of a GPU's."""
import pytest
import torch
from torch._subclasses.fake_tensor import FakeTensorMode

import paper_2506_22771_amd as ff


def calls(on):
    """Every call, with the device of each tensor from on(name)."""
    B = ff.binding._native()

    def new(name, *shape, of=torch.float32):
        return torch.empty(shape, dtype=of, device=on(name))

    x, r, y, dy, dx, du = (new(n, 4, 40) for n in ("x", "r", "y", "dy", "dx", "du"))
    w, b, dw, db = (new(n, 40) for n in ("w", "b", "dw", "db"))
    good, coeff, mean, rstd = new("good", 4), new("coeff", 4), new("mean", 4, 5), new("rstd", 4, 5)
    a_q, w_q, s_a, s_w = new("a_q", 4, 48, of=torch.int8), new("w_q", 80, 48, of=torch.int8), new("s_a", 1), new("s_w", 1)
    q, e, qu, eu = (new(n, 4, 48 if n[0] == "q" else 16, of=torch.int8 if n[0] == "q" else torch.uint8) for n in ("q", "e", "qu", "eu"))
    step, ws = new("step", 1, of=torch.int64), new("ws", 1 << 16, of=torch.uint8)
    return [("a_q w_q s_a s_w y good q e qu eu ws", lambda: B.gated_forward(a_q, w_q, s_a, s_w, 40, 3, y, good, q, e, qu, eu, ws, 0)),
            ("q e qu eu coeff dy dx du", lambda: B.gated_backward(q, e, qu, eu, 3, coeff, dy, dx, du, 0)),
            ("x w b y mean rstd good q e ws", lambda: B.group_norm_forward(x, 4, 5, w, b, 1e-5, 3, y, mean, rstd, good, q, e, 0, 0, 0, ws, 0)),
            ("dy coeff x mean rstd w b dx dw db ws", lambda: B.group_norm_backward(dy, coeff, x, mean, None, None, rstd, 4, 5, w, b, 3, dx, dw, db, False, ws, 0)),
            ("dy coeff q e rstd w b dx dw db ws", lambda: B.group_norm_backward(dy, coeff, None, None, q, e, rstd, 4, 5, w, b, 3, dx, dw, db, False, ws, 0)),
            ("x r step y", lambda: B.dropout(x, r, 0.5, 0, 0, step, y, 0))]


@pytest.mark.skipif(torch.cuda.device_count() == 1, reason="tensors without memory on a second device ask the runtime for it where there is one device")
def test_tensors_of_two_devices():
    with FakeTensorMode():
        for i, (names, _) in enumerate(calls(lambda name: "cuda:0")):
            for other in names.split():
                with pytest.raises(ValueError, match="tensors on one device expected, got cuda:. and cuda:."):
                    calls(lambda name: "cuda:1" if name == other else "cuda:0")[i][1]()


@pytest.mark.gpu
@pytest.mark.skipif(torch.cuda.device_count() < 2, reason="one device")
def test_tensors_of_another_device_than_the_current_one():
    for _, call in calls(lambda name: "cuda:1"):
        with pytest.raises(ValueError, match="tensors on the current device, cuda:0, expected, got cuda:1"):
            call()
