"""What the layer norm and checkpoint calls refuse, on the host, before anything is launched (this runs without a GPU)."""
import ctypes as C

import pytest
import torch

INVALID, SHAPE, ALIGN, WORKSPACE, UNSUPPORTED = -1, -2, -3, -4, -6
P = C.c_void_p
A = P(0x1000)        # never dereferenced: validation fails first
NULL = P(0)


@pytest.fixture(scope="module")
def ff():
    import paper_2506_22771_amd as m
    try:
        m.lib()
    except FileNotFoundError:
        import __graft_entry__ as g
        g.build()
        m.lib()
    return m


def call(fn, args, **changes):
    values = dict(args)
    assert set(changes) <= set(values)
    values.update(changes)
    return fn(*values.values())


FORWARD = dict(rows=4, cols=40, dtype=0, param=0, x=A, ldx=40, w=A, b=A, eps=1e-5, y=A, ldy=40, mean=A, rstd=A, q=A, e=A, mode=0, seed=0, tag=0, s=NULL)
BACKWARD = dict(rows=4, cols=40, dtype=0, param=0, dy=A, lddy=40, x=NULL, ldx=0, mean=NULL, q=A, e=A, rstd=A, w=A, dx=A, lddx=40, dw=A, db=A, acc=0, ws=A,
                wsb=1 << 30, s=NULL)
STORE = dict(x=A, dtype=1, ldx=40, rows=4, cols=40, mode=0, seed=0, tag=0, q=A, e=A, s=NULL)
LOAD = dict(q=A, e=A, rows=4, cols=40, x=A, dtype=2, ldx=40, s=NULL)
ACT = dict(q=A, e=A, rows=4, cols=40, act=2, coeff=A, dy=A, lddy=40, dx=A, lddx=40, dtype=0, s=NULL)
WGRAD = dict(dy=A, dtype=0, lddy=24, q=A, e=A, rows=4, n=24, k=40, g=A, b=A, param=0, dw=A, db=A, acc=0, ws=A, wsb=1 << 30, s=NULL)


def test_sizes_types_and_modes(ff):
    L = ff.lib()
    for fn, args in ((L.ff_layer_norm_forward, FORWARD), (L.ff_layer_norm_backward, BACKWARD), (L.ff_ckpt_store, STORE), (L.ff_ckpt_load, LOAD),
                     (L.ff_ckpt_act_backward, ACT)):
        assert call(fn, args, rows=-1) == INVALID and call(fn, args, cols=-1) == INVALID
        assert call(fn, args, cols=0) == SHAPE
        assert call(fn, args, cols=(1 << 24) + 1) == UNSUPPORTED and call(fn, args, rows=1 << 31) == UNSUPPORTED
        assert call(fn, args, rows=(1 << 31) - 1, cols=1 << 20) == UNSUPPORTED
        assert call(fn, args, dtype=3) == INVALID and call(fn, args, dtype=-1) == INVALID
    for fn, args in ((L.ff_layer_norm_forward, FORWARD), (L.ff_ckpt_store, STORE)):
        assert call(fn, args, mode=2) == INVALID
    for fn, args in ((L.ff_layer_norm_forward, FORWARD), (L.ff_layer_norm_backward, BACKWARD), (L.ff_ckpt_weight_grad, WGRAD)):
        assert call(fn, args, param=1) == INVALID       # neither fp32 nor the matrix's type
    for eps in (-1.0, float("nan")):
        assert call(L.ff_layer_norm_forward, FORWARD, eps=eps) == INVALID
    assert call(L.ff_ckpt_act_backward, ACT, act=4) == INVALID and call(L.ff_ckpt_act_backward, ACT, act=-1) == INVALID
    for fn, args in ((L.ff_layer_norm_backward, BACKWARD), (L.ff_ckpt_weight_grad, WGRAD)):
        assert call(fn, args, acc=2) == INVALID
    assert call(L.ff_ckpt_weight_grad, WGRAD, n=0) == SHAPE and call(L.ff_ckpt_weight_grad, WGRAD, k=0) == SHAPE
    assert call(L.ff_ckpt_weight_grad, WGRAD, n=65536, lddy=65536) == UNSUPPORTED
    assert call(L.ff_ckpt_weight_grad, WGRAD, rows=-1) == INVALID


def test_addresses_strides_and_workspace(ff):
    L = ff.lib()
    off1, off2, off8 = P(0x1001), P(0x1002), P(0x1008)
    for name in ("x", "y", "q", "e"):
        assert call(L.ff_layer_norm_forward, FORWARD, **{name: NULL}) == INVALID
    assert call(L.ff_layer_norm_forward, FORWARD, ldx=39) == SHAPE and call(L.ff_layer_norm_forward, FORWARD, ldy=39) == SHAPE
    assert call(L.ff_layer_norm_forward, FORWARD, ldx=(1 << 31) + 1) == UNSUPPORTED
    for name in ("x", "y", "w", "b", "mean", "rstd"):
        assert call(L.ff_layer_norm_forward, FORWARD, **{name: off2}) == ALIGN
    assert call(L.ff_layer_norm_forward, FORWARD, dtype=1, x=off1) == ALIGN
    for name in ("q", "e"):
        assert call(L.ff_layer_norm_forward, FORWARD, **{name: off8}) == ALIGN

    for name in ("dy", "q", "e", "rstd", "ws"):
        assert call(L.ff_layer_norm_backward, BACKWARD, **{name: NULL}) == INVALID
    assert call(L.ff_layer_norm_backward, BACKWARD, x=A, ldx=40) == INVALID                    # x without mean
    assert call(L.ff_layer_norm_backward, BACKWARD, x=A, ldx=39, mean=A) == SHAPE
    assert call(L.ff_layer_norm_backward, BACKWARD, dx=NULL, dw=NULL, db=NULL) == INVALID
    assert call(L.ff_layer_norm_backward, BACKWARD, wsb=ff.ff_layer_norm_workspace_bytes(4, 40) - 1) == WORKSPACE
    assert call(L.ff_layer_norm_backward, BACKWARD, ws=off8) == ALIGN
    assert call(L.ff_layer_norm_backward, BACKWARD, lddx=39) == SHAPE

    for name in ("x", "q", "e"):
        assert call(L.ff_ckpt_store, STORE, **{name: NULL}) == INVALID and call(L.ff_ckpt_load, LOAD, **{name: NULL}) == INVALID
    assert call(L.ff_ckpt_store, STORE, ldx=39) == SHAPE and call(L.ff_ckpt_load, LOAD, ldx=39) == SHAPE
    assert call(L.ff_ckpt_load, LOAD, x=off1) == ALIGN and call(L.ff_ckpt_store, STORE, q=off8) == ALIGN

    assert call(L.ff_ckpt_act_backward, ACT, coeff=NULL, dy=NULL) == INVALID and call(L.ff_ckpt_act_backward, ACT, dx=NULL) == INVALID
    assert call(L.ff_ckpt_act_backward, ACT, coeff=off2) == ALIGN and call(L.ff_ckpt_act_backward, ACT, lddy=39) == SHAPE

    for name in ("dy", "q", "e", "dw", "ws"):
        assert call(L.ff_ckpt_weight_grad, WGRAD, **{name: NULL}) == INVALID
    assert call(L.ff_ckpt_weight_grad, WGRAD, lddy=23) == SHAPE and call(L.ff_ckpt_weight_grad, WGRAD, dw=off2) == ALIGN
    assert call(L.ff_ckpt_weight_grad, WGRAD, wsb=ff.ff_ckpt_weight_grad_workspace_bytes(4, 24, 40) - 1) == WORKSPACE


def test_no_rows_ask_for_no_matrices(ff):
    L = ff.lib()
    assert call(L.ff_layer_norm_forward, FORWARD, rows=0, x=NULL, y=NULL, q=NULL, e=NULL) == 0
    assert call(L.ff_ckpt_store, STORE, rows=0, x=NULL, q=NULL, e=NULL) == 0
    assert call(L.ff_ckpt_load, LOAD, rows=0, x=NULL, q=NULL, e=NULL) == 0
    assert call(L.ff_ckpt_act_backward, ACT, rows=0, q=NULL, e=NULL, coeff=NULL, dy=NULL, dx=NULL) == 0


def test_sizes_of_layouts_and_workspaces(ff):
    assert [ff.ff_ckpt_blocks(c) for c in (-1, 0, 1, 32, 33, 784)] == [0, 0, 1, 1, 2, 25]
    assert ff.ff_layer_norm_workspace_bytes(-1, 4) == 0 and ff.ff_layer_norm_workspace_bytes(4, 0) == 0
    assert ff.ff_layer_norm_workspace_bytes(0, 4) >= ff.WS_MIN_BYTES
    assert ff.ff_ckpt_weight_grad_workspace_bytes(4, 0, 4) == 0 and ff.ff_ckpt_weight_grad_workspace_bytes(4, 65536, 4) == 0
    assert ff.ff_ckpt_weight_grad_workspace_bytes(1, 4, 4) >= ff.WS_MIN_BYTES
    for cols in (1, 16, 500, 513, 784, 4096, 20000):
        assert ff.binding._pitch(cols) == ff.ff_pitch(cols)


def test_the_binding_compares_shapes_and_types(ff):
    """Host tensors: every one of these is refused before the address is asked for, or because of where the tensor lies."""
    x, q, e = torch.zeros(4, 40), torch.zeros((4, 48), dtype=torch.int8), torch.zeros((4, 16), dtype=torch.uint8)
    w = torch.zeros(40)
    for bad in (lambda: ff.ff_layer_norm_forward(x, w, w, 1e-5, x[:3], None, None), lambda: ff.ff_layer_norm_forward(x.double(), w, w, 1e-5, x, None, None),
                lambda: ff.ff_layer_norm_forward(x, w, w, 1e-5, x, None, None), lambda: ff.ff_layer_norm_forward(x[0], w, w, 1e-5, x, None, None),
                lambda: ff.ff_ckpt_store(x, 0, 0, 0, q, e), lambda: ff.ff_ckpt_load(q, e, x.bool()),
                lambda: ff.ff_ckpt_weight_grad(x, q, e, None, None, torch.zeros(39, 40), None, False, None),
                lambda: ff.ff_ckpt_act_backward(q, e, 0, None, x.half(), x),
                lambda: ff.binding._ckpt(q[:, :47], e, 4, 40), lambda: ff.binding._ckpt(q, e[:3], 4, 40), lambda: ff.binding._ckpt(q, None, 4, 40),
                lambda: ff.binding._ckpt(q.to(torch.uint8), e, 4, 40), lambda: ff.binding._params(w.half(), None, "w", 40, torch.bfloat16),
                lambda: ff.binding._params(w, w.half(), "w", 40, torch.float16), lambda: ff.binding._vec(w, "v", 39, torch.float32)):
        with pytest.raises(ValueError):
            bad()
