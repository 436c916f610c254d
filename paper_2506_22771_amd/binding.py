"""ctypes binding of include/ffint8.h.  Argument marshalling only.

Functions mirror the C-ABI names.  Tensor arguments are torch CUDA tensors (or None where the
header allows NULL); their data_ptr() is handed to the library together with the current
torch stream, its type compared with the header's.  The calls on matrices of floating-point values (norms, checkpoints, gated layers, dropout) take the compiled way (csrc/bind.cpp).  Nothing here computes."""
from __future__ import annotations

import ctypes as C
import os
from typing import List, Optional, Sequence

import torch

ROUND_NEAREST, ROUND_STOCHASTIC = 0, 1
PASS_POS, PASS_NEG = 1, -1
KIND_ACT, KIND_GRAD, KIND_CHAIN = 0, 1, 2
ACT_IDENTITY, ACT_RELU, ACT_GELU, ACT_SILU = 0, 1, 2, 3
CKPT_BLOCK = 32
WS_MIN_BYTES = 1024

_LIB_PATH = os.path.join(os.path.dirname(os.path.abspath(__file__)), "libffint8.so")
_lib = None


class FFError(RuntimeError):
    def __init__(self, status: int, what: str):
        self.status = status
        super().__init__(f"{what}: {ff_status_string(status)} ({status})")


class LayerDesc(C.Structure):
    _fields_ = [(n, C.c_int32) for n in ("kind", "batch", "in_features", "out_features", "H", "W", "C_in", "C_out",
                                         "ksize", "stride", "pad", "relu", "l2norm_out", "input_back", "role", "skip")]


class NetDesc(C.Structure):
    _fields_ = [("n_layers", C.c_int32), ("batch", C.c_int32), ("layers", C.POINTER(LayerDesc)),
                ("train_layer", C.POINTER(C.c_int32)), ("lookahead", C.c_int32),
                ("theta_layer", C.POINTER(C.c_float)), ("launch_mode", C.c_int32)]


class NetState(C.Structure):
    _fields_ = [("w_master", C.POINTER(C.c_void_p)), ("w_q", C.POINTER(C.c_void_p)), ("s_w", C.POINTER(C.c_void_p))]


def lib() -> C.CDLL:
    """Loads the built HIP library; raises if it has not been built (python -m paper_2506_22771_amd.build)."""
    global _lib
    if _lib is None:
        if not os.path.exists(_LIB_PATH):
            raise FileNotFoundError(f"{_LIB_PATH} is missing: build it with `python -m paper_2506_22771_amd.build`")
        L = C.CDLL(_LIB_PATH)
        P, i32, i64, u64, f32, sz = C.c_void_p, C.c_int32, C.c_int64, C.c_uint64, C.c_float, C.c_size_t
        LD = C.POINTER(LayerDesc)
        L.ff_pitch.restype = i64
        L.ff_pitch.argtypes = [i64]
        L.ff_pitch32.restype = i64
        L.ff_pitch32.argtypes = [i64]
        L.ff_stream_tag.restype = u64
        L.ff_stream_tag.argtypes = [u64, C.c_uint32, C.c_uint32, C.c_uint32]
        L.ff_status_string.restype = C.c_char_p
        L.ff_status_string.argtypes = [i32]
        L.ff_version.restype = C.c_char_p
        L.ff_goodness_shift.restype = i32
        L.ff_goodness_shift.argtypes = [LD]
        L.ff_layer_dw_chunks.restype = i32
        L.ff_layer_dw_chunks.argtypes = [LD]
        L.ff_layer_workspace_bytes.restype = sz
        L.ff_layer_workspace_bytes.argtypes = [LD]
        L.ff_quantize.restype = i32
        L.ff_quantize.argtypes = [P, i64, i64, i32, u64, u64, P, P, P, P, sz, P]
        L.ff_layer_forward.restype = i32
        L.ff_layer_forward.argtypes = [LD, P, P, P, P, P, P, sz, P]
        L.ff_goodness_loss.restype = i32
        L.ff_goodness_loss.argtypes = [LD, P, P, P, P, i32, f32, P, P, P, P, P]
        L.ff_layer_handoff.restype = i32
        L.ff_layer_handoff.argtypes = [LD, P, P, P, P, P, i32, u64, u64, P, P, P, P]
        L.ff_lookahead.restype = i32
        L.ff_lookahead.argtypes = [P, i32, i64, f32, P, P]
        L.ff_layer_backward_local.restype = i32
        L.ff_layer_backward_local.argtypes = [LD, P, P, P, P, P, i32, u64, u64, P, P, P, P, P, sz, P]
        L.ff_layer_backward_local_noalloc.restype = i32
        L.ff_layer_backward_local_noalloc.argtypes = [LD, P, P, P, P, P, i32, u64, u64, P, P, P, P, P]
        L.ff_noalloc_scratch_bytes.restype = sz
        L.ff_chain_gradients.restype = i32
        L.ff_chain_gradients.argtypes = [LD, P, P, P, P, P, P, P, f32, P, P, P, P, P]
        L.ff_layer_input_grad.restype = i32
        L.ff_layer_input_grad.argtypes = [LD, P, P, P, P, sz, P]
        L.ff_layer_update.restype = i32
        L.ff_layer_update.argtypes = [LD, P, P, P, P, P, P, P, f32, i32, P, P, P, sz, P]
        L.ff_train_step.restype = i32
        L.ff_train_step.argtypes = [C.POINTER(NetDesc), C.POINTER(NetState), P, P, f32, f32, f32, u64, u64, P, P, P,
                                    sz, P]
        L.ff_train_step_at.restype = i32
        L.ff_train_step_at.argtypes = [C.POINTER(NetDesc), C.POINTER(NetState), P, P, f32, f32, f32, u64, P, i32, P, P,
                                       P, sz, P]
        L.ff_workspace_bytes.restype = sz
        L.ff_workspace_bytes.argtypes = [C.POINTER(NetDesc)]
        L.ff_ckpt_blocks.restype = i64
        L.ff_ckpt_blocks.argtypes = [i64]
        L.ff_layer_norm_forward.restype = i32
        L.ff_layer_norm_forward.argtypes = [i64, i64, i32, i32, P, i64, P, P, f32, P, i64, P, P, P, P, i32, u64, u64, P]
        L.ff_layer_norm_workspace_bytes.restype = sz
        L.ff_layer_norm_workspace_bytes.argtypes = [i64, i64]
        L.ff_layer_norm_backward.restype = i32
        L.ff_layer_norm_backward.argtypes = [i64, i64, i32, i32, P, i64, P, i64, P, P, P, P, P, P, i64, P, P, i32, P, sz, P]
        L.ff_ckpt_store.restype = i32
        L.ff_ckpt_store.argtypes = [P, i32, i64, i64, i64, i32, u64, u64, P, P, P]
        L.ff_ckpt_load.restype = i32
        L.ff_ckpt_load.argtypes = [P, P, i64, i64, P, i32, i64, P]
        L.ff_ckpt_act_backward.restype = i32
        L.ff_ckpt_act_backward.argtypes = [P, P, i64, i64, i32, P, P, i64, P, i64, i32, P]
        L.ff_ckpt_weight_grad_workspace_bytes.restype = sz
        L.ff_ckpt_weight_grad_workspace_bytes.argtypes = [i64, i64, i64]
        L.ff_ckpt_weight_grad.restype = i32
        L.ff_ckpt_weight_grad.argtypes = [P, i32, i64, P, P, i64, i64, i64, P, P, i32, P, P, i32, P, sz, P]
        L.ff_gated_workspace_bytes.restype = sz
        L.ff_gated_workspace_bytes.argtypes = [i64, i64, i64]
        L.ff_gated_forward.restype = i32
        L.ff_gated_forward.argtypes = [i64, i64, i64, P, P, P, P, i32, P, i32, i64, P, P, P, P, P, P, sz, P]
        L.ff_gated_backward.restype = i32
        L.ff_gated_backward.argtypes = [P, P, P, P, i64, i64, i32, P, P, i64, P, i64, P, i64, i32, P]
        L.ff_group_norm_workspace_bytes.restype = sz
        L.ff_group_norm_workspace_bytes.argtypes = [i64, i64, i64, i64]
        L.ff_group_norm_forward.restype = i32
        L.ff_group_norm_forward.argtypes = [i64, i64, i64, i64, i32, i32, P, i64, P, P, f32, i32, P, i64, P, P, P, P, P, i32, u64, u64, P, sz, P]
        L.ff_group_norm_backward.restype = i32
        L.ff_group_norm_backward.argtypes = [i64, i64, i64, i64, i32, i32, P, i64, P, P, i64, P, P, P, P, P, P, i32, P, i64, P, P, i32, P, sz, P]
        L.ff_dropout.restype = i32
        L.ff_dropout.argtypes = [i64, i64, i32, P, i64, P, i64, f32, u64, u64, P, P, i64, P]
        L.ff_timing_enable.restype = i32
        L.ff_timing_enable.argtypes = [i32]
        L.ff_timing_clock_probe.restype = i32
        L.ff_timing_clock_probe.argtypes = [P]
        L.ff_probe_mfma_ceiling.restype = i32
        L.ff_probe_mfma_ceiling.argtypes = [i32, i32, P, sz, P, C.POINTER(C.c_double), P]
        L.ff_timing_fused_stamps.restype = i32
        L.ff_timing_fused_stamps.argtypes = [P]
        L.ff_timing_reset.restype = i32
        L.ff_timing_read.restype = i32
        L.ff_timing_read.argtypes = [i32, C.POINTER(C.c_double), C.POINTER(C.c_int64)]
        _lib = L
    return _lib


# Addresses go to the library as plain integers (the argument types say void*), and the current stream's is asked for without
# building a stream object: the single operations of a small layer are issued by the host, which took 44.5 us for the six launches of a
# dense layer's forward pass (784 -> 1201, 1000 samples) and takes 32 this way.
def _ptr(t: Optional[torch.Tensor]) -> Optional[int]:
    if t is None:
        return None
    if not t.is_cuda:
        raise ValueError("device tensor expected")
    if not t.is_contiguous():
        raise ValueError("contiguous tensor expected")
    return t.data_ptr()


def _refuse_type(t: torch.Tensor, of: torch.dtype) -> None:
    raise ValueError(f"{of} tensor expected, got {t.dtype}")


def _typed(*of: torch.dtype):
    """_ptr for tensors of these types: the library takes what lies at an address for what its header names."""
    def ptr(t: Optional[torch.Tensor]) -> Optional[int]:
        if t is None:
            return None
        if t.dtype not in of:
            _refuse_type(t, of[0])
        if not t.is_cuda or not t.is_contiguous():
            return _ptr(t)   # (which says so)
        return t.data_ptr()
    return ptr


_f32, _i8, _i32, _i64 = _typed(torch.float32), _typed(torch.int8), _typed(torch.int32), _typed(torch.int64, torch.uint64)


def _stream() -> int:
    if not torch.cuda.is_initialized():
        return torch.cuda.current_stream().cuda_stream
    return torch._C._cuda_getCurrentRawStream(torch._C._cuda_getDevice())


def _chk(st: int, what: str) -> None:
    if st != 0:
        raise FFError(st, what)


def layer_desc(layer, batch: int) -> LayerDesc:
    """From a workloads.Layer (or any object with the same attributes)."""
    kind = {"dense": 0, "conv": 1, "dwconv": 2}[layer.kind]
    return LayerDesc(kind, batch, layer.in_features, layer.out_features, layer.H, layer.W, layer.C_in, layer.C_out,
                     layer.ksize, layer.stride, layer.pad, layer.relu, layer.l2norm_out,
                     getattr(layer, "input_back", 0), {"ff": 0, "proj": 1}[getattr(layer, "role", "ff")],
                     {"none": 0, "identity": 1, "projection": 2}[getattr(layer, "skip", "none")])


def ff_pitch(cols: int) -> int:
    return int(lib().ff_pitch(cols))


def ff_pitch32(cols: int) -> int:
    return int(lib().ff_pitch32(cols))


def ff_stream_tag(step: int, layer: int, pass_idx: int, kind: int) -> int:
    return int(lib().ff_stream_tag(step, layer, pass_idx, kind))


def ff_status_string(st: int) -> str:
    return lib().ff_status_string(st).decode()


def ff_version() -> str:
    return lib().ff_version().decode()


def ff_goodness_shift(desc: LayerDesc) -> int:
    return int(lib().ff_goodness_shift(C.byref(desc)))


def ff_layer_dw_chunks(desc: LayerDesc) -> int:
    return int(lib().ff_layer_dw_chunks(C.byref(desc)))


def ff_layer_workspace_bytes(desc: LayerDesc) -> int:
    return int(lib().ff_layer_workspace_bytes(C.byref(desc)))


def ff_quantize(x, rows, cols, round_mode, seed, stream_tag, q, q_t, scale, ws) -> None:
    _chk(lib().ff_quantize(_f32(x), rows, cols, round_mode, seed, stream_tag, _i8(q), _i8(q_t), _f32(scale),
                           _ptr(ws), ws.numel() * ws.element_size() if ws is not None else 0, _stream()), "ff_quantize")


def ff_layer_forward(desc, a_q, w_q, acc, gsum_int, vmax, ws) -> None:
    _chk(lib().ff_layer_forward(C.byref(desc), _i8(a_q), _i8(w_q), _i32(acc), _i64(gsum_int), _i32(vmax), _ptr(ws),
                                ws.numel() * ws.element_size() if ws is not None else 0, _stream()), "ff_layer_forward")


def ff_goodness_loss(desc, gsum_int, vmax, s_a, s_w, pass_sign, theta, goodness, coeff, loss_mean, next_amax) -> None:
    _chk(lib().ff_goodness_loss(C.byref(desc), _i64(gsum_int), _i32(vmax), _f32(s_a), _f32(s_w), pass_sign, theta,
                                _f32(goodness), _f32(coeff), _f32(loss_mean), _f32(next_amax), _stream()),
         "ff_goodness_loss")


def ff_layer_handoff(desc, acc, s_a, s_w, goodness, amax, round_mode, seed, stream_tag, q, q_t, scale) -> None:
    _chk(lib().ff_layer_handoff(C.byref(desc), _i32(acc), _f32(s_a), _f32(s_w), _f32(goodness), _f32(amax), round_mode,
                                seed, stream_tag, _i8(q), _i8(q_t), _f32(scale), _stream()), "ff_layer_handoff")


def ff_lookahead(coeff, n_layers, batch, lam, coeff_total) -> None:
    _chk(lib().ff_lookahead(_f32(coeff), n_layers, batch, lam, _f32(coeff_total), _stream()), "ff_lookahead")


def ff_layer_backward_local(desc, acc, vmax, s_a, s_w, coeff_total, round_mode, seed, stream_tag, a_q_t, gy_q_t, s_g,
                            dw_acc, ws) -> None:
    _chk(lib().ff_layer_backward_local(C.byref(desc), _i32(acc), _i32(vmax), _f32(s_a), _f32(s_w), _f32(coeff_total),
                                       round_mode, seed, stream_tag, _i8(a_q_t), _i8(gy_q_t), _f32(s_g), _i32(dw_acc),
                                       _ptr(ws), ws.numel() * ws.element_size() if ws is not None else 0, _stream()),
         "ff_layer_backward_local")


def ff_layer_backward_local_noalloc(desc, acc, vmax, s_a, s_w, coeff_total, round_mode, seed, stream_tag, a_q_t,
                                    gy_q_t, s_g, dw_acc) -> None:
    _chk(lib().ff_layer_backward_local_noalloc(C.byref(desc), _i32(acc), _i32(vmax), _f32(s_a), _f32(s_w),
                                               _f32(coeff_total), round_mode, seed, stream_tag, _i8(a_q_t),
                                               _i8(gy_q_t), _f32(s_g), _i32(dw_acc), _stream()),
         "ff_layer_backward_local_noalloc")


def ff_noalloc_scratch_bytes() -> int:
    return int(lib().ff_noalloc_scratch_bytes())


def ff_chain_gradients(desc, acc, s_a, s_w, coeff, e_acc, s_h, s_w_up, lam, h, g, h_amax, g_amax) -> None:
    _chk(lib().ff_chain_gradients(C.byref(desc), _i32(acc), _f32(s_a), _f32(s_w), _f32(coeff), _i32(e_acc), _f32(s_h),
                                  _f32(s_w_up), lam, _f32(h), _f32(g), _f32(h_amax), _f32(g_amax), _stream()),
         "ff_chain_gradients")


def ff_layer_input_grad(desc, h_q, w_q_t, e_acc, ws) -> None:
    _chk(lib().ff_layer_input_grad(C.byref(desc), _i8(h_q), _i8(w_q_t), _i32(e_acc), _ptr(ws),
                                   ws.numel() * ws.element_size() if ws is not None else 0, _stream()),
         "ff_layer_input_grad")


def ff_layer_update(desc, w_master, dw_pos, s_g_pos, s_a_pos, dw_neg, s_g_neg, s_a_neg, lr, total_samples, w_q, s_w,
                    ws) -> None:
    _chk(lib().ff_layer_update(C.byref(desc), _f32(w_master), _i32(dw_pos), _f32(s_g_pos), _f32(s_a_pos), _i32(dw_neg),
                               _f32(s_g_neg), _f32(s_a_neg), lr, total_samples, _i8(w_q), _f32(s_w), _ptr(ws),
                               ws.numel() * ws.element_size() if ws is not None else 0, _stream()), "ff_layer_update")


class Net:
    """Host-side descriptors of a layer stack plus the device pointers of its trainable state.
    Holds references to the tensors so that the pointer arrays stay valid."""

    def __init__(self, layers: Sequence, batch: int, w_master: List[torch.Tensor], w_q: List[torch.Tensor],
                 s_w: List[torch.Tensor], train_layer: Optional[Sequence[int]] = None, lookahead: str = "coeff",
                 theta_layer: Optional[Sequence[float]] = None, launch_mode: str = "auto"):
        self.k = len(layers)
        self.batch = batch
        self._descs = (LayerDesc * self.k)(*[layer_desc(l, batch) for l in layers])
        self._mask = (C.c_int32 * self.k)(*[int(bool(f)) for f in train_layer]) if train_layer is not None else None
        self._theta = (C.c_float * self.k)(*[float(t) for t in theta_layer]) if theta_layer is not None else None
        if theta_layer is not None and len(theta_layer) != self.k:
            raise ValueError("theta_layer needs one threshold per layer")
        self.desc = NetDesc(self.k, batch, self._descs, self._mask, {"coeff": 0, "chain": 1}[lookahead], self._theta,
                            {"auto": 0, "kernels": 1, "fused": 2, "lanes": 3}[launch_mode])
        self.w_master, self.w_q, self.s_w = list(w_master), list(w_q), list(s_w)
        for of, tensors in ((torch.float32, self.w_master), (torch.int8, self.w_q), (torch.float32, self.s_w)):
            for t in tensors:
                if t.dtype is not of:
                    _refuse_type(t, of)
        self._pm = (C.c_void_p * self.k)(*[t.data_ptr() for t in self.w_master])
        self._pq = (C.c_void_p * self.k)(*[t.data_ptr() for t in self.w_q])
        self._ps = (C.c_void_p * self.k)(*[t.data_ptr() for t in self.s_w])
        self.state = NetState(self._pm, self._pq, self._ps)

    def workspace_bytes(self) -> int:
        return ff_workspace_bytes(self)


def ff_workspace_bytes(net: Net) -> int:
    return int(lib().ff_workspace_bytes(C.byref(net.desc)))


def ff_train_step(net: Net, x_pos, x_neg, theta, lam, lr, seed, step, loss, goodness, ws) -> None:
    _chk(lib().ff_train_step(C.byref(net.desc), C.byref(net.state), _f32(x_pos), _f32(x_neg), theta, lam, lr, seed,
                             step, _f32(loss), _f32(goodness), _ptr(ws),
                             ws.numel() * ws.element_size() if ws is not None else 0, _stream()), "ff_train_step")


def ff_train_step_at(net: Net, x_pos, x_neg, theta, lam, lr, seed, step_dev, advance, loss, goodness, ws) -> None:
    _chk(lib().ff_train_step_at(C.byref(net.desc), C.byref(net.state), _f32(x_pos), _f32(x_neg), theta, lam, lr, seed,
                                _i64(step_dev), int(advance), _f32(loss), _f32(goodness), _ptr(ws),
                                ws.numel() * ws.element_size() if ws is not None else 0, _stream()), "ff_train_step_at")


# --- layer norm and 8-bit checkpoints.  Matrices are 2-D tensors of float32, bfloat16 or float16 with consecutive columns and any row
# stride (a view of some columns of a wider tensor will do).  Shapes, types, strides and devices are compared with each other, and the device with the
# current one, whose stream is used (ValueError), because the library sees addresses and sizes only; that and the marshalling are compiled (csrc/bind.cpp).
_bind = None


def _native():
    """The built marshalling module; raises if it has not been built (python -m paper_2506_22771_amd.build)."""
    global _bind
    if _bind is None:
        lib()
        try:
            from . import _bind as module
        except ImportError as e:
            raise FileNotFoundError(f"paper_2506_22771_amd/_bind.so: {e}: build it with `python -m paper_2506_22771_amd.build`") from e
        _bind = module
    return _bind


def ff_ckpt_blocks(cols: int) -> int:
    return int(lib().ff_ckpt_blocks(cols))


def ckpt_empty(rows: int, cols: int, device="cuda"):
    """Codes and exponent bytes for a checkpoint of a [rows, cols] matrix, not filled in."""
    return (torch.empty((rows, ff_pitch(cols)), dtype=torch.int8, device=device),
            torch.empty((rows, ff_pitch(ff_ckpt_blocks(cols))), dtype=torch.uint8, device=device))


def ff_layer_norm_forward(x, weight, bias, eps, y, mean, rstd, q=None, e=None, round_mode=ROUND_NEAREST, seed=0,
                          stream_tag=0) -> None:
    _chk(_native().layer_norm_forward(x, weight, bias, eps, y, mean, rstd, q, e, round_mode, seed, stream_tag, _stream()),
         "ff_layer_norm_forward")


def ff_layer_norm_workspace_bytes(rows: int, cols: int) -> int:
    return int(lib().ff_layer_norm_workspace_bytes(rows, cols))


def ff_layer_norm_backward(dy, x, mean, q, e, rstd, weight, dx, dweight, dbias, accumulate, ws) -> None:
    """h comes from x, mean and rstd, or, with x = None, from the checkpoint q, e and rstd."""
    _chk(_native().layer_norm_backward(dy, x, mean, q, e, rstd, weight, dx, dweight, dbias, accumulate, ws, _stream()),
         "ff_layer_norm_backward")


def ff_ckpt_store(x, round_mode, seed, stream_tag, q, e) -> None:
    _chk(_native().ckpt_store(x, round_mode, seed, stream_tag, q, e, _stream()), "ff_ckpt_store")


def ff_ckpt_load(q, e, x) -> None:
    _chk(_native().ckpt_load(q, e, x, _stream()), "ff_ckpt_load")


def ff_ckpt_act_backward(q, e, act, coeff, dy, dx) -> None:
    _chk(_native().ckpt_act_backward(q, e, act, coeff, dy, dx, _stream()), "ff_ckpt_act_backward")


def ff_ckpt_weight_grad_workspace_bytes(rows: int, n: int, k: int) -> int:
    return int(lib().ff_ckpt_weight_grad_workspace_bytes(rows, n, k))


def ff_ckpt_weight_grad(dy, q, e, gamma, beta, dw, db, accumulate, ws) -> None:
    _chk(_native().ckpt_weight_grad(dy, q, e, gamma, beta, dw, db, accumulate, ws, _stream()), "ff_ckpt_weight_grad")


# --- gated layers, group norm, dropout: tensors as above.  Maps are matrices [samples * pixels, channels].
def ff_gated_workspace_bytes(rows: int, n: int, k: int) -> int:
    return int(lib().ff_gated_workspace_bytes(rows, n, k))


def ff_gated_forward(a_q, w_q, s_a, s_w, k, act, y, goodness, qg, eg, qu, eu, ws) -> None:
    """a_q int8 [rows, ff_pitch(k)], w_q int8 [2n, ff_pitch(k)] with the gate's rows first, y [rows, n]."""
    _chk(_native().gated_forward(a_q, w_q, s_a, s_w, k, act, y, goodness, qg, eg, qu, eu, ws, _stream()), "ff_gated_forward")


def ff_gated_backward(qg, eg, qu, eu, act, coeff, dy, dg, du) -> None:
    _chk(_native().gated_backward(qg, eg, qu, eu, act, coeff, dy, dg, du, _stream()), "ff_gated_backward")


def ff_group_norm_workspace_bytes(samples: int, pixels: int, channels: int, groups: int) -> int:
    return int(lib().ff_group_norm_workspace_bytes(samples, pixels, channels, groups))


def ff_group_norm_forward(x, samples, groups, weight, bias, eps, act, y, mean, rstd, goodness, q, e, round_mode, seed, stream_tag, ws) -> None:
    _chk(_native().group_norm_forward(x, samples, groups, weight, bias, eps, act, y, mean, rstd, goodness, q, e, round_mode, seed, stream_tag, ws,
                                      _stream()), "ff_group_norm_forward")


def ff_group_norm_backward(dy, coeff, x, mean, q, e, rstd, samples, groups, weight, bias, act, dx, dweight, dbias, accumulate, ws) -> None:
    """h comes from x, mean and rstd, or, with x = None, from the checkpoint q, e and rstd.  One of dy, x and dx is given: it says how many rows there are, and their type."""
    _chk(_native().group_norm_backward(dy, coeff, x, mean, q, e, rstd, samples, groups, weight, bias, act, dx, dweight, dbias, accumulate, ws, _stream()),
         "ff_group_norm_backward")


def ff_dropout(x, r, p, seed, stream_tag, step, y) -> None:
    """step: an int64 tensor of one element that is read when the kernel runs, or None."""
    _chk(_native().dropout(x, r, p, seed, stream_tag, step, y, _stream()), "ff_dropout")


KERNEL_CLASSES = ("gemm_fwd", "gemm_dw", "quant_act", "quant_grad", "quant_w", "update", "absmax", "small", "im2col",
                  "residual", "dwconv", "chain", "fused", "norm", "ckpt", "ckpt_dw",
                  "gated", "group_norm", "dropout")


def ff_timing_enable(on, classes: Optional[Sequence[str]] = None) -> None:
    """on: False = off, True = every kernel class, or restrict to the named `classes` (see KERNEL_CLASSES)."""
    mask = 0
    if on:
        mask = -1 if classes is None else sum(1 << KERNEL_CLASSES.index(c) for c in classes)
    _chk(lib().ff_timing_enable(mask), "ff_timing_enable")


def ff_timing_clock_probe(counters: Optional[torch.Tensor]) -> None:
    """counters: a zeroed int64 CUDA tensor of 16 elements (kept alive by the caller), or None to switch off."""
    _chk(lib().ff_timing_clock_probe(_ptr(counters)), "ff_timing_clock_probe")


def ff_probe_mfma_ceiling(operand_kind: int, iterations: int, sink: torch.Tensor, counters: Optional[torch.Tensor]) -> float:
    """Launches the register-resident MFMA loop on the current stream; returns the int8 operations of the launch."""
    ops = C.c_double(0.0)
    _chk(lib().ff_probe_mfma_ceiling(operand_kind, iterations, _ptr(sink), sink.numel() * sink.element_size(),
                                     _ptr(counters), C.byref(ops), _stream()), "ff_probe_mfma_ceiling")
    return ops.value


def ff_timing_fused_stamps(stamps: Optional[torch.Tensor]) -> None:
    """stamps: an int64 CUDA tensor of 32 elements (kept alive by the caller), or None to switch off."""
    _chk(lib().ff_timing_fused_stamps(_ptr(stamps)), "ff_timing_fused_stamps")


def ff_timing_reset() -> None:
    _chk(lib().ff_timing_reset(), "ff_timing_reset")


def ff_timing_read(kernel_class: int):
    """(total device milliseconds, launches) of one kernel class since the last reset."""
    ms, n = C.c_double(0.0), C.c_int64(0)
    _chk(lib().ff_timing_read(kernel_class, C.byref(ms), C.byref(n)), "ff_timing_read")
    return ms.value, n.value
