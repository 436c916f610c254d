"""The calls on int8 codes and fp32 tensors compare types before the library, which sees addresses only, reads a tensor as what it is not (and a 16-bit one beyond its end).  Host tensors:
types are looked at before where they lie, and nothing is launched."""
import types

import pytest
import torch

import paper_2506_22771_amd as ff

F, B, C, A, W = torch.float32, torch.bfloat16, torch.int8, torch.int32, torch.int64
DENSE = ff.layer_desc(types.SimpleNamespace(kind="dense", in_features=40, out_features=24, H=0, W=0, C_in=0, C_out=0, ksize=0, stride=0, pad=0, relu=1, l2norm_out=1), 4)
NET = ff.Net([], 0, [], [], [])

# every call with its tensors' types in their order; _: the other arguments
CALLS = {
    "ff_quantize": ((F, C, C, F), lambda x, q, q_t, s: ff.ff_quantize(x, 4, 40, 0, 0, 0, q, q_t, s, None)),
    "ff_layer_forward": ((C, C, A, W, A), lambda a, w, acc, g, v: ff.ff_layer_forward(DENSE, a, w, acc, g, v, None)),
    "ff_goodness_loss": ((W, A, F, F, F, F, F, F), lambda g, v, *f: ff.ff_goodness_loss(DENSE, g, v, f[0], f[1], 1, 2.0, *f[2:])),
    "ff_layer_handoff": ((A, F, F, F, F, C, C, F), lambda acc, s_a, s_w, g, m, q, q_t, s: ff.ff_layer_handoff(DENSE, acc, s_a, s_w, g, m, 0, 0, 0, q, q_t, s)),
    "ff_lookahead": ((F, F), lambda c, t: ff.ff_lookahead(c, 2, 4, 0.1, t)),
    "ff_layer_backward_local": ((A, A, F, F, F, C, C, F, A), lambda acc, v, s_a, s_w, c, a, g, s, dw: ff.ff_layer_backward_local(DENSE, acc, v, s_a, s_w, c, 0, 0, 0, a, g, s, dw, None)),
    "ff_layer_backward_local_noalloc": ((A, A, F, F, F, C, C, F, A), lambda acc, v, s_a, s_w, c, a, g, s, dw: ff.ff_layer_backward_local_noalloc(
        DENSE, acc, v, s_a, s_w, c, 0, 0, 0, a, g, s, dw)),
    "ff_chain_gradients": ((A, F, F, F, A, F, F, F, F, F, F), lambda acc, s_a, s_w, c, e, s_h, s_u, h, g, hm, gm: ff.ff_chain_gradients(DENSE, acc, s_a, s_w, c, e, s_h, s_u, 0.1, h, g, hm, gm)),
    "ff_layer_input_grad": ((C, C, A), lambda h, w, e: ff.ff_layer_input_grad(DENSE, h, w, e, None)),
    "ff_layer_update": ((F, A, F, F, A, F, F, C, F), lambda w, dp, sg, sa, dn, sn, an, q, s: ff.ff_layer_update(DENSE, w, dp, sg, sa, dn, sn, an, 0.1, 8, q, s, None)),
    "ff_train_step": ((F, F, F, F), lambda p, n, loss, good: ff.ff_train_step(NET, p, n, 2.0, 0.1, 0.1, 0, 0, loss, good, None)),
    "ff_train_step_at": ((F, F, W, F, F), lambda p, n, at, loss, good: ff.ff_train_step_at(NET, p, n, 2.0, 0.1, 0.1, 0, at, 1, loss, good, None)),
}


@pytest.mark.parametrize("name", list(CALLS))
def test_types(name):
    of, call = CALLS[name]
    right = [torch.zeros(160, dtype=t) for t in of]
    with pytest.raises(ValueError, match="device tensor expected"):     # the right types get as far as where they lie
        call(*right)
    for i, t in enumerate(of):
        for other in {B, torch.float16, torch.float64, F, C, A} - {t}:
            # those before it are absent, as an absent tensor is passed on; nothing behind it has been looked at
            with pytest.raises(ValueError, match=f"{t} tensor expected, got {other}"):
                call(*[None] * i, torch.zeros(160, dtype=other), *right[i + 1:])


def test_words_without_a_sign():
    _, call = CALLS["ff_layer_forward"]
    with pytest.raises(ValueError, match="device tensor expected"):
        call(None, None, None, torch.zeros(4, dtype=torch.uint64), torch.zeros(4, dtype=A))


def test_weights_of_a_net():
    layer = types.SimpleNamespace(kind="dense", in_features=40, out_features=24, H=0, W=0, C_in=0, C_out=0, ksize=0, stride=0, pad=0, relu=1, l2norm_out=1)
    w, q, s = torch.zeros(24, 40), torch.zeros((24, 48), dtype=C), torch.zeros(1)
    ff.Net([layer], 4, [w], [q], [s])
    for bad in (([w.bfloat16()], [q], [s]), ([w], [q.float()], [s]), ([w], [q], [s.double()])):
        with pytest.raises(ValueError, match="tensor expected, got"):
            ff.Net([layer], 4, *bad)
