"""What the gated, group norm and dropout calls refuse, on the host, before anything is launched (this runs without a GPU)."""
import ctypes as C

import pytest
import torch

from test_norm_abi import ALIGN, INVALID, NULL, SHAPE, UNSUPPORTED, WORKSPACE, A, P, call, ff  # noqa: F401  (ff: the fixture)

OVERFLOW = -5
OFF1, OFF2, OFF4, OFF8 = P(0x1001), P(0x1002), P(0x1004), P(0x1008)
BIG = 1 << 40

GATED = dict(rows=4, n=40, k=50, a=A, w=A, sa=A, sw=A, act=3, y=A, dtype=0, ldy=40, good=A, qg=A, eg=A, qu=A, eu=A, ws=A, wsb=BIG, s=NULL)
GATED_B = dict(qg=A, eg=A, qu=A, eu=A, rows=4, n=40, act=2, coeff=A, dy=A, lddy=40, dg=A, lddg=80, du=A, lddu=80, dtype=1, s=NULL)
GROUP = dict(samples=2, pixels=3, channels=40, groups=8, dtype=0, param=0, x=A, ldx=40, w=A, b=A, eps=1e-5, act=1, y=A, ldy=40, mean=A, rstd=A, good=A, q=A, e=A,
             mode=0, seed=0, tag=0, ws=A, wsb=BIG, s=NULL)
GROUP_B = dict(samples=2, pixels=3, channels=40, groups=8, dtype=0, param=0, dy=A, lddy=40, coeff=A, x=NULL, ldx=0, mean=NULL, q=A, e=A, rstd=A, w=A, b=A, act=1, dx=A,
               lddx=40, dw=A, db=A, acc=0, ws=A, wsb=BIG, s=NULL)
DROP = dict(rows=4, cols=40, dtype=0, x=A, ldx=40, r=A, ldr=40, p=0.5, seed=1, tag=2, step=NULL, y=A, ldy=40, s=NULL)


def test_sizes(ff):  # noqa: F811
    L = ff.lib()
    for fn, args, names in ((L.ff_gated_forward, GATED, ("rows", "n", "k")), (L.ff_gated_backward, GATED_B, ("rows", "n")), (L.ff_dropout, DROP, ("rows", "cols")),
                            (L.ff_group_norm_forward, GROUP, ("samples", "pixels", "channels", "groups")),
                            (L.ff_group_norm_backward, GROUP_B, ("samples", "pixels", "channels", "groups"))):
        for name in names:
            assert call(fn, args, **{name: -1}) == INVALID, name
        for name in names[1:]:
            assert call(fn, args, **{name: 0}) == SHAPE, name
    assert call(L.ff_gated_forward, GATED, n=32768, ldy=32768) == UNSUPPORTED and call(L.ff_gated_forward, GATED, rows=8388481) == UNSUPPORTED
    assert call(L.ff_gated_forward, GATED, k=133145) == OVERFLOW
    assert call(L.ff_gated_forward, GATED, rows=8388480, n=32767, ldy=32767) == UNSUPPORTED
    assert call(L.ff_gated_backward, GATED_B, rows=1 << 31) == UNSUPPORTED and call(L.ff_gated_backward, GATED_B, rows=1 << 27, n=1024) == UNSUPPORTED
    for fn, args in ((L.ff_group_norm_forward, GROUP), (L.ff_group_norm_backward, GROUP_B)):
        assert call(fn, args, groups=7) == SHAPE and call(fn, args, groups=80) == SHAPE
        assert call(fn, args, channels=65536) == UNSUPPORTED and call(fn, args, samples=1 << 20, pixels=1 << 11) == UNSUPPORTED
        assert call(fn, args, samples=1 << 16, pixels=1 << 11, channels=1024) == UNSUPPORTED
        assert call(fn, args, samples=1 << 40, pixels=1 << 40) == UNSUPPORTED      # (their product has no 64 bits)
    assert call(L.ff_dropout, DROP, rows=1 << 27, cols=1024) == UNSUPPORTED and call(L.ff_dropout, DROP, cols=(1 << 24) + 1) == UNSUPPORTED


def test_types_and_numbers(ff):  # noqa: F811
    L = ff.lib()
    for fn, args in ((L.ff_gated_forward, GATED), (L.ff_gated_backward, GATED_B), (L.ff_group_norm_forward, GROUP), (L.ff_group_norm_backward, GROUP_B), (L.ff_dropout, DROP)):
        assert call(fn, args, dtype=3) == INVALID and call(fn, args, dtype=-1) == INVALID
        if "act" in args:
            assert call(fn, args, act=4) == INVALID and call(fn, args, act=-1) == INVALID
        if "param" in args:
            assert call(fn, args, param=1) == INVALID
    for eps in (-1.0, float("nan")):
        assert call(L.ff_group_norm_forward, GROUP, eps=eps) == INVALID
    assert call(L.ff_group_norm_forward, GROUP, mode=2) == INVALID and call(L.ff_group_norm_backward, GROUP_B, acc=2) == INVALID
    for p in (-0.1, 1.0001, float("nan"), float("inf")):
        assert call(L.ff_dropout, DROP, p=p) == INVALID


def test_addresses_strides_and_workspaces(ff):  # noqa: F811
    L = ff.lib()
    for name in ("a", "w", "sa", "sw", "y", "ws", "eg", "qu", "eu", "qg"):
        assert call(L.ff_gated_forward, GATED, **{name: NULL}) == INVALID, name
    for name, off in (("a", OFF8), ("w", OFF8), ("sa", OFF2), ("sw", OFF2), ("good", OFF2), ("qg", OFF8), ("eg", OFF8), ("qu", OFF8), ("eu", OFF8), ("ws", OFF8), ("y", OFF2)):
        assert call(L.ff_gated_forward, GATED, **{name: off}) == ALIGN, name
    assert call(L.ff_gated_forward, GATED, dtype=1, y=OFF1) == ALIGN
    assert call(L.ff_gated_forward, GATED, ldy=39) == SHAPE and call(L.ff_gated_forward, GATED, ldy=(1 << 31) + 1) == UNSUPPORTED
    assert call(L.ff_gated_forward, GATED, wsb=ff.ff_gated_workspace_bytes(4, 40, 50) - 1) == WORKSPACE

    for name in ("qg", "eg", "qu", "eu", "dg", "du"):
        assert call(L.ff_gated_backward, GATED_B, **{name: NULL}) == INVALID, name
    assert call(L.ff_gated_backward, GATED_B, coeff=NULL, dy=NULL) == INVALID
    for name, off in (("qg", OFF8), ("eu", OFF8), ("coeff", OFF2), ("dy", OFF1), ("dg", OFF1), ("du", OFF1)):
        assert call(L.ff_gated_backward, GATED_B, **{name: off}) == ALIGN, name
    for name in ("lddy", "lddg", "lddu"):
        assert call(L.ff_gated_backward, GATED_B, **{name: 39}) == SHAPE, name

    for name in ("x", "y", "q", "e", "ws"):
        assert call(L.ff_group_norm_forward, GROUP, **{name: NULL}) == INVALID, name
    for name, off in (("x", OFF2), ("y", OFF2), ("w", OFF2), ("b", OFF2), ("mean", OFF2), ("rstd", OFF2), ("good", OFF2), ("q", OFF8), ("e", OFF8), ("ws", OFF8)):
        assert call(L.ff_group_norm_forward, GROUP, **{name: off}) == ALIGN, name
    assert call(L.ff_group_norm_forward, GROUP, ldx=39) == SHAPE and call(L.ff_group_norm_forward, GROUP, ldy=39) == SHAPE
    need = ff.ff_group_norm_workspace_bytes(2, 3, 40, 8)
    assert call(L.ff_group_norm_forward, GROUP, wsb=need - 1) == WORKSPACE and call(L.ff_group_norm_backward, GROUP_B, wsb=need - 1) == WORKSPACE

    for name in ("q", "e", "rstd", "ws"):
        assert call(L.ff_group_norm_backward, GROUP_B, **{name: NULL}) == INVALID, name
    assert call(L.ff_group_norm_backward, GROUP_B, dy=NULL, coeff=NULL) == INVALID
    assert call(L.ff_group_norm_backward, GROUP_B, x=A, ldx=40) == INVALID                     # x without mean
    assert call(L.ff_group_norm_backward, GROUP_B, x=A, ldx=39, mean=A) == SHAPE
    assert call(L.ff_group_norm_backward, GROUP_B, dx=NULL, dw=NULL, db=NULL) == INVALID
    for name, off in (("dy", OFF2), ("coeff", OFF2), ("rstd", OFF2), ("dx", OFF2), ("dw", OFF2), ("db", OFF2), ("q", OFF8)):
        assert call(L.ff_group_norm_backward, GROUP_B, **{name: off}) == ALIGN, name
    for name in ("lddy", "lddx"):
        assert call(L.ff_group_norm_backward, GROUP_B, **{name: 39}) == SHAPE, name

    for name in ("x", "y"):
        assert call(L.ff_dropout, DROP, **{name: NULL}) == INVALID, name
    for name, off in (("x", OFF2), ("r", OFF2), ("y", OFF2), ("step", OFF4)):
        assert call(L.ff_dropout, DROP, **{name: off}) == ALIGN, name
    for name in ("ldx", "ldr", "ldy"):
        assert call(L.ff_dropout, DROP, **{name: 39}) == SHAPE, name


def test_no_rows_ask_for_no_matrices(ff):  # noqa: F811
    L = ff.lib()
    assert call(L.ff_gated_forward, GATED, rows=0, a=NULL, y=NULL, qg=NULL, eg=NULL, qu=NULL, eu=NULL) == 0
    assert call(L.ff_gated_backward, GATED_B, rows=0, qg=NULL, eg=NULL, qu=NULL, eu=NULL, dy=NULL, coeff=NULL, dg=NULL, du=NULL) == 0
    assert call(L.ff_group_norm_forward, GROUP, samples=0, x=NULL, y=NULL, q=NULL, e=NULL) == 0
    assert call(L.ff_dropout, DROP, rows=0, x=NULL, r=NULL, y=NULL) == 0


def test_workspaces(ff):  # noqa: F811
    assert ff.ff_gated_workspace_bytes(-1, 4, 4) == 0 and ff.ff_gated_workspace_bytes(4, 0, 4) == 0 and ff.ff_gated_workspace_bytes(4, 4, 1 << 20) == 0
    assert ff.ff_gated_workspace_bytes(0, 4, 4) >= ff.WS_MIN_BYTES
    assert ff.ff_group_norm_workspace_bytes(2, 0, 4, 2) == 0 and ff.ff_group_norm_workspace_bytes(2, 3, 4, 3) == 0
    assert ff.ff_group_norm_workspace_bytes(0, 3, 4, 2) >= ff.WS_MIN_BYTES and ff.ff_group_norm_workspace_bytes(0, 1 << 20, 4, 2) >= ff.WS_MIN_BYTES


def test_the_binding_compares_shapes_and_types(ff):  # noqa: F811
    """Refused before the library is called; host tensors of the right shapes and types for where they lie."""
    B = ff.binding._native()
    x, w, none = torch.zeros(6, 40), torch.zeros(40), None
    q, e = torch.zeros((6, 48), dtype=torch.int8), torch.zeros((6, 16), dtype=torch.uint8)
    aq, wq, s = torch.zeros((6, 64), dtype=torch.int8), torch.zeros((80, 64), dtype=torch.int8), torch.zeros(1)
    ws = torch.zeros(1 << 16, dtype=torch.uint8)
    matrix, device = "float32, bfloat16 or float16 matrix", "device tensor"
    for expected, bad in (
            (matrix, lambda: B.dropout(x.double(), none, 0.5, 0, 0, none, x, 0)), (device, lambda: B.dropout(x, none, 0.5, 0, 0, none, x, 0)),
            (matrix, lambda: B.gated_forward(aq, wq, s, s, 50, 1, x[0], none, none, none, none, none, ws, 0)),
            (device, lambda: B.gated_forward(aq, wq, s, s, 50, 1, x, none, none, none, none, none, ws, 0)),
            (device, lambda: B.gated_backward(q, e, q, e, 1, none, x, x, x, 0)),
            (device, lambda: B.group_norm_forward(x, 2, 8, w, w, 1e-5, 1, x, none, none, none, none, none, 0, 0, 0, ws, 0)),
            ("dy, x or dx: a matrix", lambda: B.group_norm_backward(none, s, none, none, q, e, s, 2, 8, w, w, 1, none, w, w, False, ws, 0)),
            (device, lambda: B.group_norm_backward(x, none, none, none, q, e, s, 2, 8, w, w, 1, x, w, w, False, ws, 0))):
        with pytest.raises(ValueError, match=expected):
            bad()
    with pytest.raises(TypeError):
        B.dropout(x, none)


@pytest.mark.gpu
def test_the_binding_compares_device_tensors_with_each_other(ff):  # noqa: F811
    new = lambda *shape, of=torch.float32: torch.zeros(shape, dtype=of, device="cuda")  # noqa: E731
    x, w, none, s = new(6, 40), new(40), None, new(1)
    q, e, aq, wq = new(6, 48, of=torch.int8), new(6, 16, of=torch.uint8), new(6, 64, of=torch.int8), new(80, 64, of=torch.int8)
    st, ws = new(2, 8), new(1 << 20, of=torch.uint8)
    gated = lambda a=aq, w=wq, sa=s, sw=s, k=50, y=x, good=none, g=(none, none), u=(none, none), ws=ws: ff.ff_gated_forward(a, w, sa, sw, k, 1, y, good, *g, *u, ws)  # noqa: E731
    group = lambda x=x, n=2, g=8, w=w, b=w, y=x, m=st, r=st, good=none, q=none, e=none, ws=ws: ff.ff_group_norm_forward(  # noqa: E731
        x, n, g, w, b, 1e-5, 1, y, m, r, good, q, e, 0, 0, 0, ws)
    back = lambda dy=x, c=none, x=none, m=none, q=q, e=e, r=st, n=2, w=w, dx=x, dw=w, ws=ws: ff.ff_group_norm_backward(  # noqa: E731
        dy, c, x, m, q, e, r, n, 8, w, w, 1, dx, dw, none, False, ws)
    for expected, bad in (
            (r"a_q: contiguous int8 \[6, 64\]", lambda: gated(a=aq[:, :63])), (r"a_q: contiguous int8 \[6, 80\]", lambda: gated(k=80)),
            (r"w_q: contiguous int8 \[80, 64\]", lambda: gated(w=wq[:79])), ("s_a: one float32", lambda: gated(sa=new(2))), ("s_w: one float32", lambda: gated(sw=s.half())),
            (r"goodness: float32 \[6\]", lambda: gated(good=w)), (r"codes: contiguous int8 \[6, 48\]", lambda: gated(g=(aq, e), u=(q, e))),
            (r"dg|du: float32 \[6, 40\]", lambda: ff.ff_gated_backward(q, e, q, e, 1, none, x, x, x.half())),
            (r"dy: float32 \[6, 40\]", lambda: ff.ff_gated_backward(q, e, q, e, 1, none, x.half(), x, x)),
            ("samples: a number of equal parts of 6 rows", lambda: group(n=4)), ("samples: a number", lambda: group(n=-2)), ("samples: a number", lambda: group(n=0)),
            (r"mean: contiguous float32 \[2, 8\]", lambda: group(m=new(8, 2))), (r"rstd: contiguous float32 \[2, 8\]", lambda: group(r=new(16))),
            (r"(mean|rstd): contiguous float32 \[3, 8\]", lambda: group(n=3)), (r"goodness: float32 \[2\]", lambda: group(good=new(6))),
            (r"weight: float32 \[40\]", lambda: group(w=new(8))), (r"y: float32 \[6, 40\]", lambda: group(y=x.half())), ("both codes", lambda: group(q=q)),
            (r"coeff: float32 \[2\]", lambda: back(c=new(6))), (r"rstd: contiguous float32 \[2, 8\]", lambda: back(r=new(2, 40))), (r"dx: float32", lambda: back(dx=x.half())),
            (r"r: float32 \[6, 40\]", lambda: ff.ff_dropout(x, x[:5], 0.5, 0, 0, none, x)), ("step: one int64", lambda: ff.ff_dropout(x, none, 0.5, 0, 0, s, x)),
            ("device tensor", lambda: ff.ff_dropout(x, x.cpu(), 0.5, 0, 0, none, x)), ("device tensor", lambda: gated(sa=s.cpu()))):
        with pytest.raises(ValueError, match=expected):
            bad()
    for status, bad in ((INVALID, lambda: ff.ff_dropout(x, none, 1.5, 0, 0, none, x)), (WORKSPACE, lambda: gated(ws=ws[:16])), (INVALID, lambda: gated(g=(q, e))),
                        (SHAPE, lambda: group(g=7, m=none, r=none)), (INVALID, lambda: back(dy=none, dx=x)), (INVALID, lambda: back(x=x)), (WORKSPACE, lambda: back(ws=ws[:16])),
                        (INVALID, lambda: ff.ff_gated_backward(q, e, q, e, 1, none, none, x, new(6, 40))), (INVALID, lambda: group(ws=none))):
        with pytest.raises(ff.FFError) as err:
            bad()
        assert err.value.status == status
