"""One row of a matrix whatever the distance to its next: a stride that no second row follows counts for nothing."""
import pytest
import torch

import paper_2506_22771_amd as ff

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("stride", [0, 1, 39, 1 << 31, (1 << 31) + 1, 1 << 40])
def test_any_stride(stride):
    g = torch.Generator("cuda").manual_seed(1)
    x, dy, w = torch.randn((1, 40), device="cuda", generator=g), torch.randn((1, 40), device="cuda", generator=g), torch.randn(40, device="cuda", generator=g)
    ws = torch.empty(max(ff.ff_layer_norm_workspace_bytes(1, 40), ff.ff_ckpt_weight_grad_workspace_bytes(1, 40, 40)), dtype=torch.uint8, device="cuda")

    def all_of(of):
        m, r, ckpt = torch.empty(1, device="cuda"), torch.empty(1, device="cuda"), ff.ckpt_empty(1, 40)
        y, dx, back, da = (of(torch.empty((1, 40), device="cuda")) for _ in range(4))
        dw, db, dW = torch.empty(40, device="cuda"), torch.empty(40, device="cuda"), torch.empty((40, 40), device="cuda")
        ff.ff_layer_norm_forward(of(x), w, w, 1e-5, y, m, r, *ckpt)
        ff.ff_layer_norm_backward(of(dy), of(x), m, None, None, r, w, dx, dw, db, False, ws)
        ff.ff_ckpt_store(of(x), ff.ROUND_NEAREST, 0, 0, *ckpt)
        ff.ff_ckpt_load(*ckpt, back)
        ff.ff_ckpt_act_backward(*ckpt, ff.ACT_SILU, None, of(dy), da)
        ff.ff_ckpt_weight_grad(of(dy), *ckpt, None, None, dW, None, False, ws)
        return y, m, r, dx, dw, db, back, da, dW, *ckpt

    for got, ref in zip(all_of(lambda t: t.as_strided((1, 40), (stride, 1))), all_of(lambda t: t)):
        assert torch.equal(got, ref)
