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


def test_the_binding_compares_shapes_and_types(ff):
    """Every one of these is refused before the library is called.  Host tensors of the right shapes and types are refused for where they lie."""
    x, q, e = torch.zeros(4, 40), torch.zeros((4, 48), dtype=torch.int8), torch.zeros((4, 16), dtype=torch.uint8)
    w, r, none = torch.zeros(40), torch.zeros(4), None
    ws = torch.zeros(1 << 16, dtype=torch.uint8)
    matrix, device = "float32, bfloat16 or float16 matrix", "device tensor"
    B = ff.binding._native()    # (the functions that take the stream as a number: there is none to ask for here)
    for expected, bad in (
            (matrix, lambda: B.layer_norm_forward(x.double(), w, w, 1e-5, x, r, r, none, none, 0, 0, 0, 0)),
            (matrix, lambda: B.layer_norm_forward(x[0], w, w, 1e-5, x, r, r, none, none, 0, 0, 0, 0)),
            ("x: a tensor", lambda: B.layer_norm_forward([1.0], w, w, 1e-5, x, r, r, none, none, 0, 0, 0, 0)),
            ("x: a dense tensor", lambda: B.ckpt_store(x.to_sparse(), 0, 0, 0, q, e, 0)),
            (device, lambda: B.layer_norm_forward(x, w, w, 1e-5, x, r, r, none, none, 0, 0, 0, 0)),
            (matrix, lambda: B.ckpt_load(q, e, x.bool(), 0)),
            (device, lambda: B.ckpt_store(x, 0, 0, 0, q, e, 0)),
            (device, lambda: B.ckpt_act_backward(q, e, 0, none, none, x, 0)),
            (device, lambda: B.layer_norm_backward(x, none, none, q, e, r, w, none, w, w, False, ws, 0)),
            (device, lambda: B.ckpt_weight_grad(x, q, e, none, none, torch.zeros(40, 40), none, False, ws, 0))):
        with pytest.raises(ValueError, match=expected):
            bad()
    with pytest.raises(TypeError):
        B.ckpt_load(q, e)


@pytest.mark.gpu
def test_the_binding_compares_device_tensors_with_each_other(ff):
    new = lambda *shape, of=torch.float32: torch.zeros(shape, dtype=of, device="cuda")  # noqa: E731
    x, w, r, none = new(4, 40), new(40), new(4), None
    q, e = new(4, 48, of=torch.int8), new(4, 16, of=torch.uint8)
    ws = new(1 << 20, of=torch.uint8)
    forward = lambda x=x, w=w, b=w, y=x, m=r, r=r, q=none, e=none: ff.ff_layer_norm_forward(x, w, b, 1e-5, y, m, r, q, e)  # noqa: E731
    wgrad = lambda dy=x, q=q, e=e, g=none, b=none, dw=new(40, 40), db=none, ws=ws: ff.ff_ckpt_weight_grad(dy, q, e, g, b, dw, db, False, ws)  # noqa: E731
    backward = lambda dy=x, x=none, m=none, q=q, e=e, dx=none, dw=w: ff.ff_layer_norm_backward(dy, x, m, q, e, r, w, dx, dw, none, False, ws)  # noqa: E731
    for expected, bad in (
            (r"y: float32 \[4, 40\]", lambda: forward(y=x[:3])), (r"y: float32 \[4, 40\]", lambda: forward(y=x.half())),
            ("consecutive columns", lambda: forward(x=new(40, 4).t(), y=x)), ("consecutive columns", lambda: forward(x=new(1, 40).expand(4, 40))),
            (r"weight: float32 \[40\]", lambda: forward(w=new(39))), ("weight: float32", lambda: forward(w=w.half())),
            (r"bias: float32 \[40\]", lambda: forward(b=w.bfloat16())), ("contiguous", lambda: forward(w=new(80)[::2])),
            (r"mean: float32 \[4\]", lambda: forward(m=new(5))), (r"rstd: float32 \[4\]", lambda: forward(r=r.double())),
            ("both codes and exponent bytes", lambda: forward(q=q)), (r"codes: contiguous int8 \[4, 48\]", lambda: forward(q=q[:, :47], e=e)),
            (r"codes: contiguous int8 \[4, 48\]", lambda: forward(q=e, e=e)), (r"exponent bytes: contiguous uint8 \[4, 16\]", lambda: forward(q=q, e=e[:3])),
            ("device tensor", lambda: forward(w=w.cpu())), ("device tensor", lambda: forward(q=q.cpu(), e=e)),
            (r"x: float32 \[4, 40\]", lambda: backward(x=x[:, :39])), (r"dx: float32 \[4, 40\]", lambda: backward(dx=x.half())),
            (r"dweight: float32 \[40\]", lambda: backward(dw=r)),
            (r"dw: contiguous float32 \[40, 40\]", lambda: wgrad(dw=new(40, 40, of=torch.float16))), ("dw: contiguous", lambda: wgrad(dw=new(40, 80)[:, :40])),
            ("dw: contiguous float32", lambda: wgrad(dw=new(39, 40))), (r"db: float32 \[40\]", lambda: wgrad(db=r)), ("gamma: float32", lambda: wgrad(g=w.half())),
            ("ws: contiguous", lambda: wgrad(ws=ws[::2])), (r"codes: contiguous int8 \[4, 16\]", lambda: wgrad(dw=new(40, 9))),
            (r"dy: float32 \[4, 40\]", lambda: ff.ff_ckpt_act_backward(q, e, 1, none, x.half(), x)),
            (r"coeff: float32 \[4\]", lambda: ff.ff_ckpt_act_backward(q, e, 1, w, x, x))):
        with pytest.raises(ValueError, match=expected):
            bad()
    # and the library's own refusals come back as its status
    for status, bad in ((-1, lambda: ff.ff_ckpt_act_backward(q, e, 9, none, x, x)), (-1, lambda: ff.ff_ckpt_act_backward(q, e, 1, none, none, x)),
                        (-4, lambda: wgrad(ws=ws[:16])), (-1, lambda: wgrad(ws=none)), (-1, lambda: backward(x=x)),
                        (-1, lambda: ff.ff_ckpt_store(x, 7, 0, 0, q, e)), (-1, lambda: ff.ff_layer_norm_forward(x, w, w, -1.0, x, r, r)),
                        (-2, lambda: ff.ff_layer_norm_forward(new(4, 0), none, none, 1e-5, new(4, 0), r, r))):
        with pytest.raises(ff.FFError) as err:
            bad()
        assert err.value.status == status


@pytest.mark.parametrize("rows, cols", [(1 << 27, 1024), ((1 << 26) - 1, 257), (1 << 29, 1)])
def test_more_elements_than_a_launch_has_lanes_for(ff, rows, cols):
    """Refused, not handed to a launch that fails: 2^34 elements of rows of codes and more (257 columns: rows of 272 codes, 288 with whole blocks)."""
    L = ff.lib()
    for fn, args in ((L.ff_layer_norm_forward, FORWARD), (L.ff_layer_norm_backward, BACKWARD), (L.ff_ckpt_store, STORE), (L.ff_ckpt_load, LOAD),
                     (L.ff_ckpt_act_backward, ACT)):
        assert call(fn, args, rows=rows, cols=cols) == UNSUPPORTED
    assert ff.ff_layer_norm_workspace_bytes(rows, cols) == 0
    assert ff.ff_layer_norm_workspace_bytes((1 << 24) - 1, 1000) > 0
