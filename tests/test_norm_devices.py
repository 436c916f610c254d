"""The layer norm and checkpoint calls take tensors of one device, the current one.  Without a GPU, tensors without memory stand for those of its devices: what is
not refused for where it lies reaches the library with null addresses, which it refuses by its status."""
import pytest
import torch
from torch._subclasses.fake_tensor import FakeTensorMode

import paper_2506_22771_amd as ff


def calls(on):
    """Every call, with the device of each tensor from on(name)."""
    B = ff.binding._native()

    def new(name, *shape, of=torch.float32):
        return torch.empty(shape, dtype=of, device=on(name))

    x, y, dy, dx = (new(n, 4, 40) for n in ("x", "y", "dy", "dx"))
    w, b, dw, db = (new(n, 40) for n in ("w", "b", "dw", "db"))
    m, r = new("mean", 4), new("rstd", 4)
    q, e = new("q", 4, 48, of=torch.int8), new("e", 4, 16, of=torch.uint8)
    W, ws = new("dw", 40, 40), new("ws", 1 << 16, of=torch.uint8)
    return [("x w b y mean rstd q e", lambda: B.layer_norm_forward(x, w, b, 1e-5, y, m, r, q, e, 0, 0, 0, 0)),
            ("dy x mean rstd w dx dw db ws", lambda: B.layer_norm_backward(dy, x, m, None, None, r, w, dx, dw, db, False, ws, 0)),
            ("dy q e rstd w dx dw db ws", lambda: B.layer_norm_backward(dy, None, None, q, e, r, w, dx, dw, db, False, ws, 0)),
            ("x q e", lambda: B.ckpt_store(x, 0, 0, 0, q, e, 0)),
            ("q e x", lambda: B.ckpt_load(q, e, x, 0)),
            ("q e mean dy dx", lambda: B.ckpt_act_backward(q, e, 1, m, dy, dx, 0)),
            ("dy q e w b dw db ws", lambda: B.ckpt_weight_grad(dy, q, e, w, b, W, db, False, ws, 0))]


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
