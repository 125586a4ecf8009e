"""ctypes binding of libdn: same names as include/dn.h, argument marshalling only.

PyTorch-ROCm is used for device memory (the arena and the data tensors) and for
the HIP stream handle; no torch operator takes part in a training step.  The
library must be built (``python -m paper_2001_04206_amd.build``); a missing
library is an error, there is no fallback path.
"""
from __future__ import annotations

import ctypes as C
import os
from typing import List, Optional, Sequence, Tuple

import numpy as np

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libdn.so")

DN_OK, DN_ERR_INVALID_ARG, DN_ERR_SHAPE, DN_ERR_UNSUPPORTED, DN_ERR_OOM, DN_ERR_DEVICE = range(6)
DN_ACT_LINEAR, DN_ACT_SIGMOID, DN_ACT_TANH, DN_ACT_RELU, DN_ACT_SOFTMAX = range(5)
DN_ACT_SILU, DN_ACT_GELU = 5, 6
DN_LOSS_MSE, DN_LOSS_CROSS_ENTROPY = 0, 1
DN_F32, DN_F16, DN_BF16 = range(3)
DN_NORM_NONE, DN_NORM_RMS, DN_NORM_LAYER = range(3)
DN_SCORE_SOFTMAX, DN_SCORE_SIGMOID = range(2)
DN_K_FORWARD, DN_K_DELTA, DN_K_GRAD_UPDATE, DN_K_OUTPUT, DN_K_ONLINE = range(5)
KERNEL_CLASS_NAMES = ["forward", "delta", "grad_update", "output", "online"]
(DN_SCHED_NONE, DN_SCHED_LAUNCHES, DN_SCHED_PER_SAMPLE, DN_SCHED_TWO_COPY, DN_SCHED_MINIBATCH,
 DN_SCHED_MINIBATCH_DEEP, DN_SCHED_ONE_WAVE, DN_SCHED_WIDE_HIDDEN, DN_SCHED_ONE_WAVE_REGISTERS,
 DN_SCHED_ONE_WORKGROUP, DN_SCHED_SAMPLE_BLOCKS, DN_SCHED_WIDE_BLOCKS, DN_SCHED_SLICES) = range(13)
# the kernel behind each persistent schedule (minibatches: or tile_epoch_kernel, dn_last_kernel says)
SCHEDULE_KERNELS = {DN_SCHED_PER_SAMPLE: "online_epoch_kernel", DN_SCHED_TWO_COPY: "twin_epoch_kernel",
                    DN_SCHED_MINIBATCH: "batch_epoch_kernel", DN_SCHED_MINIBATCH_DEEP: "deep_batch_epoch_kernel",
                    DN_SCHED_ONE_WAVE: "tiny_epoch_kernel", DN_SCHED_WIDE_HIDDEN: "wide_epoch_kernel",
                    DN_SCHED_ONE_WAVE_REGISTERS: "tiny_regs_epoch_kernel", DN_SCHED_ONE_WORKGROUP: "solo_epoch_kernel",
                    DN_SCHED_SAMPLE_BLOCKS: "block_epoch_kernel", DN_SCHED_WIDE_BLOCKS: "wide_block_epoch_kernel",
                    DN_SCHED_SLICES: "slice_epoch_kernel"}

EXPORTS = [
    "dn_status_string", "dn_net_arena_bytes", "dn_net_create", "dn_net_destroy", "dn_set_params",
    "dn_get_params", "dn_get_grads", "dn_forward", "dn_backward", "dn_update", "dn_train_epoch",
    "dn_train", "dn_evaluate", "dn_layer_backward_workspace_bytes", "dn_layer_backward_host",
    "dn_last_epoch_ms", "dn_last_schedule", "dn_last_kernel", "dn_kernel_time", "dn_kernel_flops", "dn_set_option",
    "dn_conv_forward", "dn_conv_backward_workspace_bytes", "dn_conv_backward", "dn_maxpool_forward",
    "dn_maxpool_backward", "dn_input_gradient", "dn_sgd_step",
    "dn_conv_backward_static", "dn_conv_backward_static_limit",
    "dn_cnn_arena_bytes", "dn_cnn_create", "dn_cnn_destroy", "dn_cnn_dense", "dn_cnn_flat_size",
    "dn_cnn_set_filters", "dn_cnn_get_filters", "dn_cnn_get_filter_grads", "dn_cnn_forward", "dn_cnn_train_epoch",
    "dn_linear_forward_workspace_bytes", "dn_linear_backward_workspace_bytes", "dn_linear_forward", "dn_linear_backward",
    "dn_ffn_forward_workspace_bytes", "dn_ffn_backward_workspace_bytes", "dn_ffn_forward", "dn_ffn_backward",
    "dn_norm_backward_workspace_bytes", "dn_norm_forward", "dn_norm_backward", "dn_dropout",
    "dn_route_workspace_bytes", "dn_route_forward", "dn_route_lists", "dn_route_backward",
    "dn_experts_forward_workspace_bytes", "dn_experts_backward_workspace_bytes", "dn_experts_forward", "dn_experts_backward",
    "dn_clip_workspace_bytes", "dn_clip",
]


class LinearDesc(C.Structure):
    """dn_linear_desc"""
    _fields_ = [("type", C.c_int32), ("grad_type", C.c_int32), ("act", C.c_int32), ("rows", C.c_int32),
                ("n_in", C.c_int32), ("n_out", C.c_int32), ("ldx", C.c_int64), ("ldw", C.c_int64), ("ldr", C.c_int64),
                ("ldy", C.c_int64), ("drop", C.c_float), ("grad_scale", C.c_float), ("seed", C.c_uint64),
                ("offset", C.c_uint64)]


class FfnDesc(C.Structure):
    """dn_ffn_desc"""
    _fields_ = [("type", C.c_int32), ("grad_type", C.c_int32), ("act", C.c_int32), ("rows", C.c_int32),
                ("d", C.c_int32), ("f", C.c_int32), ("ldx", C.c_int64), ("ldr", C.c_int64), ("ldy", C.c_int64),
                ("drop", C.c_float), ("grad_scale", C.c_float), ("seed", C.c_uint64), ("offset", C.c_uint64)]


class NormDesc(C.Structure):
    """dn_norm_desc"""
    _fields_ = [("type", C.c_int32), ("grad_type", C.c_int32), ("rows", C.c_int32), ("d", C.c_int32),
                ("post", C.c_int32), ("pre", C.c_int32), ("rows_per_gate", C.c_int32), ("scale", C.c_float),
                ("eps", C.c_float)]


class RouteDesc(C.Structure):
    """dn_route_desc"""
    _fields_ = [("type", C.c_int32), ("score", C.c_int32), ("rows", C.c_int32), ("experts", C.c_int32), ("k", C.c_int32),
                ("groups", C.c_int32), ("top_groups", C.c_int32), ("group_best", C.c_int32), ("renorm", C.c_int32),
                ("scale", C.c_float), ("ldl", C.c_int64)]


class ExpertsDesc(C.Structure):
    """dn_experts_desc"""
    _fields_ = [("type", C.c_int32), ("grad_type", C.c_int32), ("act", C.c_int32), ("rows", C.c_int32), ("d", C.c_int32),
                ("f", C.c_int32), ("experts", C.c_int32), ("k", C.c_int32), ("ldx", C.c_int64), ("ldr", C.c_int64),
                ("ldy", C.c_int64), ("grad_scale", C.c_float)]


class Span(C.Structure):
    """dn_span"""
    _fields_ = [("grad_dev", C.c_void_p), ("out_dev", C.c_void_p), ("count", C.c_int64), ("type", C.c_int32),
                ("out_type", C.c_int32)]


_lib = None


class DnError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        super().__init__("%s failed: %s (status %d)" % (where, status_string(status), status))


def lib():
    """Load libdn.so (raises if it has not been built)."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError("libdn.so is missing: build it with `python -m paper_2001_04206_amd.build`")
        # PyTorch ships its own HIP runtime (same soname as the system one).  Import it
        # first so that libdn binds to that copy: device pointers and streams handed
        # over from torch are only meaningful inside the runtime that created them.
        import torch  # noqa: F401
        l = C.CDLL(LIB_PATH)
        vp, i32, i64, f32 = C.c_void_p, C.c_int32, C.c_int64, C.c_float
        l.dn_status_string.restype = C.c_char_p
        l.dn_status_string.argtypes = [C.c_int]
        l.dn_net_arena_bytes.restype = C.c_size_t
        l.dn_net_arena_bytes.argtypes = [vp, i32, i32]
        l.dn_net_create.argtypes = [vp, i32, vp, C.c_int, i32, vp, C.c_size_t, vp, C.POINTER(vp)]
        l.dn_net_destroy.argtypes = [vp]
        for f in (l.dn_set_params, l.dn_get_params, l.dn_get_grads):
            f.argtypes = [vp, i32, vp, vp]
        l.dn_forward.argtypes = [vp, vp, i32, vp]
        l.dn_backward.argtypes = [vp, vp, i32, vp]
        l.dn_update.argtypes = [vp, f32, f32]
        l.dn_input_gradient.argtypes = [vp, i32, vp]
        l.dn_sgd_step.argtypes = [vp, vp, vp, i64, f32, f32, vp]
        l.dn_train_epoch.argtypes = [vp, vp, vp, i64, i32, f32, f32, C.POINTER(f32)]
        l.dn_train.argtypes = [vp, vp, vp, i64, i32, f32, f32, f32, i32, C.POINTER(i32), C.POINTER(f32)]
        l.dn_evaluate.argtypes = [vp, vp, vp, i64, i32, C.POINTER(f32), C.POINTER(i64)]
        l.dn_layer_backward_workspace_bytes.restype = C.c_size_t
        l.dn_layer_backward_workspace_bytes.argtypes = [i32, i32]
        l.dn_layer_backward_host.argtypes = [vp, vp, f32, i32, i32, vp, vp, vp, vp, C.c_size_t, vp,
                                             C.POINTER(f32), C.POINTER(f32), C.POINTER(f32)]
        l.dn_last_epoch_ms.argtypes = [vp, C.POINTER(f32)]
        l.dn_last_schedule.argtypes = [vp, C.POINTER(i32)]
        l.dn_last_kernel.argtypes = [vp, C.POINTER(C.c_char_p)]
        l.dn_kernel_time.argtypes = [vp, i32, C.POINTER(f32), C.POINTER(i64)]
        l.dn_kernel_flops.argtypes = [vp, i32, C.POINTER(C.c_double)]
        l.dn_set_option.argtypes = [vp, C.c_char_p, i64]
        l.dn_cnn_arena_bytes.argtypes = [i32, i32, i32, vp, i32, vp, i32, i32]
        l.dn_cnn_create.argtypes = [i32, i32, i32, vp, i32, vp, i32, vp, C.c_int, i32, vp, C.c_size_t, vp, C.POINTER(vp)]
        l.dn_cnn_destroy.argtypes = [vp]
        l.dn_cnn_dense.argtypes = [vp]
        l.dn_cnn_flat_size.argtypes = [vp]
        for f in (l.dn_cnn_set_filters, l.dn_cnn_get_filters, l.dn_cnn_get_filter_grads):
            f.argtypes = [vp, i32, vp, vp]
        l.dn_cnn_forward.argtypes = [vp, vp, i32, vp]
        l.dn_cnn_train_epoch.argtypes = [vp, vp, vp, i64, i32, f32, f32, C.POINTER(f32)]
        sz, u64 = C.c_size_t, C.c_uint64
        for f in (l.dn_linear_forward_workspace_bytes, l.dn_linear_backward_workspace_bytes, l.dn_ffn_forward_workspace_bytes,
                  l.dn_ffn_backward_workspace_bytes, l.dn_norm_backward_workspace_bytes):
            f.argtypes = [vp]
        l.dn_linear_forward.argtypes = [vp] * 8 + [sz, vp]
        l.dn_linear_backward.argtypes = [vp] * 9 + [sz, vp]
        l.dn_ffn_forward.argtypes = [vp] * 12 + [sz, vp]
        l.dn_ffn_backward.argtypes = [vp] * 15 + [sz, vp]
        l.dn_norm_forward.argtypes = [vp] * 11
        l.dn_norm_backward.argtypes = [vp] * 17 + [sz, vp]
        l.dn_dropout.argtypes = [i32, vp, vp, i32, i32, i64, i64, f32, u64, u64, vp]
        l.dn_route_workspace_bytes.argtypes = [i32, i32, i32]
        l.dn_route_forward.argtypes = [vp] * 9 + [sz, vp]
        l.dn_route_lists.argtypes = [vp, i32, i32, i32] + [vp] * 4 + [sz, vp]
        l.dn_route_backward.argtypes = [vp] * 6
        for f in (l.dn_experts_forward_workspace_bytes, l.dn_experts_backward_workspace_bytes):
            f.argtypes = [vp]
        l.dn_experts_forward.argtypes = [vp] * 13 + [sz, vp]
        l.dn_experts_backward.argtypes = [vp] * 17 + [sz, vp]
        l.dn_clip_workspace_bytes.argtypes = [vp, i32]
        l.dn_clip.argtypes = [vp, i32, f32, vp, vp, sz, vp]
        for name in EXPORTS[2:]:
            if name.endswith("_workspace_bytes") or name.endswith("_static_limit") or name.endswith("_arena_bytes"):
                getattr(l, name).restype = C.c_size_t
            elif name == "dn_cnn_dense":
                getattr(l, name).restype = vp
            elif name == "dn_cnn_flat_size":
                getattr(l, name).restype = i32
            else:
                getattr(l, name).restype = C.c_int
        _lib = l
    return _lib


def status_string(status: int) -> str:
    return lib().dn_status_string(int(status)).decode()


def _check(status: int, where: str):
    if status != DN_OK:
        raise DnError(status, where)


def _i32(a: Sequence[int]):
    arr = np.ascontiguousarray(a, dtype=np.int32)
    return arr, arr.ctypes.data_as(C.c_void_p)


def dn_net_arena_bytes(widths: Sequence[int], max_batch: int) -> int:
    arr, p = _i32(widths)
    return int(lib().dn_net_arena_bytes(p, len(arr), int(max_batch)))


def _dev_ptr(t, dtype, what: str):
    import torch
    if not isinstance(t, torch.Tensor) or not t.is_cuda or t.dtype != dtype or not t.is_contiguous():
        raise TypeError("%s must be a contiguous device tensor of dtype %s" % (what, dtype))
    return C.c_void_p(t.data_ptr())


def dn_layer_backward_host(deltas, inputs, learning_rate: float, gradients, delta_weights, delta_biases,
                           workspace=None):
    """One layer's backward step for one sample with host buffers copied in and out around the
    kernel.  All arrays are host tensors (torch CPU float32, pinned or not) or numpy float32
    arrays; `workspace` is a device uint8 tensor (allocated here if None).  Returns the device
    milliseconds of (copy in, kernel, copy out)."""
    import torch

    def host_ptr(a, n, what):
        if isinstance(a, torch.Tensor):
            if a.is_cuda or a.dtype != torch.float32 or not a.is_contiguous() or a.numel() != n:
                raise TypeError("%s must be a contiguous host float32 tensor of %d elements" % (what, n))
            return C.c_void_p(a.data_ptr())
        if not isinstance(a, np.ndarray) or a.dtype != np.float32 or not a.flags["C_CONTIGUOUS"] or a.size != n:
            raise TypeError("%s must be a contiguous float32 array of %d elements" % (what, n))
        return a.ctypes.data_as(C.c_void_p)

    cols_out = int(deltas.shape[0])
    cols_in = int(inputs.shape[0])
    need = int(lib().dn_layer_backward_workspace_bytes(cols_out, cols_in))
    if need == 0:
        raise DnError(DN_ERR_SHAPE, "dn_layer_backward_workspace_bytes")
    if workspace is None:
        workspace = torch.empty(need, dtype=torch.uint8, device="cuda:0")
    stream = torch.cuda.current_stream(workspace.device)
    t = [C.c_float(0.0), C.c_float(0.0), C.c_float(0.0)]
    with torch.cuda.device(workspace.device):
        st = lib().dn_layer_backward_host(
            host_ptr(deltas, cols_out, "deltas"), host_ptr(inputs, cols_in, "inputs"), float(learning_rate),
            cols_out, cols_in, host_ptr(gradients, cols_out * cols_in, "gradients"),
            host_ptr(delta_weights, cols_out * cols_in, "delta_weights"),
            host_ptr(delta_biases, cols_out, "delta_biases"), C.c_void_p(workspace.data_ptr()),
            int(workspace.numel()), C.c_void_p(stream.cuda_stream), C.byref(t[0]), C.byref(t[1]), C.byref(t[2]))
    _check(st, "dn_layer_backward_host")
    return t[0].value, t[1].value, t[2].value


def _shape_check(t, shape, what):
    if tuple(t.shape) != tuple(shape):
        raise TypeError("%s must have shape %s, not %s" % (what, tuple(shape), tuple(t.shape)))


def conv_out_size(n: int, k: int, stride: int, pad: int) -> int:
    return (n + 2 * pad - k) // stride + 1


def dn_conv_forward(X, W, bias, Y, stride: int, pad: int, act: int):
    """Y = f(conv(X, W) + bias).  X [B][Cin][H][W], W [Cout][Cin][KH][KW], bias [Cout],
    Y [B][Cout][Ho][Wo]: contiguous float32 device tensors.  Enqueued on torch's current stream."""
    import torch
    B, Cin, H, Wd = (int(v) for v in X.shape)
    Cout, Cin2, KH, KW = (int(v) for v in W.shape)
    if Cin2 != Cin:
        raise TypeError("filter channels do not match the input")
    _shape_check(bias, (Cout,), "bias")
    _shape_check(Y, (B, Cout, conv_out_size(H, KH, stride, pad), conv_out_size(Wd, KW, stride, pad)), "Y")
    f32 = torch.float32
    with torch.cuda.device(X.device):
        stream = torch.cuda.current_stream(X.device)
        _check(lib().dn_conv_forward(_dev_ptr(X, f32, "X"), _dev_ptr(W, f32, "W"), _dev_ptr(bias, f32, "bias"),
                                     _dev_ptr(Y, f32, "Y"), B, Cin, H, Wd, Cout, KH, KW, int(stride), int(pad),
                                     int(act), C.c_void_p(stream.cuda_stream)), "dn_conv_forward")


def dn_conv_backward(X, W, Y, dA, delta, dX, dW, dbias, stride: int, pad: int, act: int, workspace=None):
    """delta = dA * f'(Y); dW, dbias = batch means of the parameter gradients; dX (or None) = dE/dX.
    `workspace`: a device uint8 tensor of dn_conv_backward_workspace_bytes(...) bytes (allocated here if None)."""
    import torch
    B, Cin, H, Wd = (int(v) for v in X.shape)
    Cout, Cin2, KH, KW = (int(v) for v in W.shape)
    if Cin2 != Cin:
        raise TypeError("filter channels do not match the input")
    yshape = (B, Cout, conv_out_size(H, KH, stride, pad), conv_out_size(Wd, KW, stride, pad))
    for t, name in ((Y, "Y"), (dA, "dA"), (delta, "delta")):
        _shape_check(t, yshape, name)
    _shape_check(dW, W.shape, "dW")
    _shape_check(dbias, (Cout,), "dbias")
    if dX is not None:
        _shape_check(dX, X.shape, "dX")
    f32 = torch.float32
    need = int(lib().dn_conv_backward_workspace_bytes(B, Cin, H, Wd, Cout, KH, KW, int(stride), int(pad)))
    if need == 0:
        raise DnError(DN_ERR_INVALID_ARG, "dn_conv_backward_workspace_bytes")
    if workspace is None:
        workspace = torch.empty(need, dtype=torch.uint8, device=X.device)
    with torch.cuda.device(X.device):
        stream = torch.cuda.current_stream(X.device)
        _check(lib().dn_conv_backward(_dev_ptr(X, f32, "X"), _dev_ptr(W, f32, "W"), _dev_ptr(Y, f32, "Y"),
                                      _dev_ptr(dA, f32, "dA"), _dev_ptr(delta, f32, "delta"),
                                      None if dX is None else _dev_ptr(dX, f32, "dX"), _dev_ptr(dW, f32, "dW"),
                                      _dev_ptr(dbias, f32, "dbias"), _dev_ptr(workspace, torch.uint8, "workspace"),
                                      C.c_size_t(int(workspace.numel())), B, Cin, H, Wd, Cout, KH, KW, int(stride),
                                      int(pad), int(act), C.c_void_p(stream.cuda_stream)), "dn_conv_backward")


def dn_conv_backward_static_limit() -> int:
    return int(lib().dn_conv_backward_static_limit())


def dn_conv_backward_static(X, W, Y, dA, delta, dX, dW, dbias, stride: int, pad: int, act: int):
    """dn_conv_backward with the library's fixed scratch array in place of a workspace: nothing is
    allocated, here or in the library."""
    import torch
    B, Cin, H, Wd = (int(v) for v in X.shape)
    Cout, Cin2, KH, KW = (int(v) for v in W.shape)
    if Cin2 != Cin:
        raise TypeError("filter channels do not match the input")
    yshape = (B, Cout, conv_out_size(H, KH, stride, pad), conv_out_size(Wd, KW, stride, pad))
    for t, name in ((Y, "Y"), (dA, "dA"), (delta, "delta")):
        _shape_check(t, yshape, name)
    _shape_check(dW, W.shape, "dW")
    _shape_check(dbias, (Cout,), "dbias")
    if dX is not None:
        _shape_check(dX, X.shape, "dX")
    f32 = torch.float32
    with torch.cuda.device(X.device):
        stream = torch.cuda.current_stream(X.device)
        _check(lib().dn_conv_backward_static(_dev_ptr(X, f32, "X"), _dev_ptr(W, f32, "W"), _dev_ptr(Y, f32, "Y"),
                                             _dev_ptr(dA, f32, "dA"), _dev_ptr(delta, f32, "delta"),
                                             None if dX is None else _dev_ptr(dX, f32, "dX"),
                                             _dev_ptr(dW, f32, "dW"), _dev_ptr(dbias, f32, "dbias"), B, Cin, H, Wd,
                                             Cout, KH, KW, int(stride), int(pad), int(act),
                                             C.c_void_p(stream.cuda_stream)), "dn_conv_backward_static")


def dn_maxpool_forward(X, Y, k: int, stride: int):
    import torch
    B, Cn, H, Wd = (int(v) for v in X.shape)
    _shape_check(Y, (B, Cn, (H - k) // stride + 1, (Wd - k) // stride + 1), "Y")
    f32 = torch.float32
    with torch.cuda.device(X.device):
        stream = torch.cuda.current_stream(X.device)
        _check(lib().dn_maxpool_forward(_dev_ptr(X, f32, "X"), _dev_ptr(Y, f32, "Y"), B, Cn, H, Wd, int(k),
                                        int(stride), C.c_void_p(stream.cuda_stream)), "dn_maxpool_forward")


def dn_maxpool_backward(X, dY, dX, k: int, stride: int):
    import torch
    B, Cn, H, Wd = (int(v) for v in X.shape)
    _shape_check(dY, (B, Cn, (H - k) // stride + 1, (Wd - k) // stride + 1), "dY")
    _shape_check(dX, X.shape, "dX")
    f32 = torch.float32
    with torch.cuda.device(X.device):
        stream = torch.cuda.current_stream(X.device)
        _check(lib().dn_maxpool_backward(_dev_ptr(X, f32, "X"), _dev_ptr(dY, f32, "dY"), _dev_ptr(dX, f32, "dX"),
                                         B, Cn, H, Wd, int(k), int(stride), C.c_void_p(stream.cuda_stream)),
               "dn_maxpool_backward")


def dn_sgd_step(param, grad, velocity, lr: float, momentum: float):
    """The update rule of Net.dn_update for a parameter tensor the caller owns."""
    import torch
    f32 = torch.float32
    _shape_check(grad, param.shape, "grad")
    if velocity is not None:
        _shape_check(velocity, param.shape, "velocity")
    with torch.cuda.device(param.device):
        stream = torch.cuda.current_stream(param.device)
        _check(lib().dn_sgd_step(_dev_ptr(param, f32, "param"), _dev_ptr(grad, f32, "grad"),
                                 None if velocity is None else _dev_ptr(velocity, f32, "velocity"),
                                 int(param.numel()), float(lr), float(momentum), C.c_void_p(stream.cuda_stream)),
               "dn_sgd_step")


# ---- the residual feed-forward block -----------------------------------------------------------------------------

_TYPES = {}     # torch.dtype -> dn_type
_torch = _raw_stream = None


def _setup():
    global _torch, _raw_stream
    if _torch is None:
        import torch
        _torch, _raw_stream = torch, getattr(torch._C, "_cuda_getCurrentRawStream", None)
        _TYPES.update({torch.float32: DN_F32, torch.float16: DN_F16, torch.bfloat16: DN_BF16})


def _type_of(t, what: str) -> int:
    if _torch is None:
        _setup()
    kind = _TYPES.get(getattr(t, "dtype", None))
    if kind is None or not t.is_cuda:
        raise TypeError("%s must be a device tensor of float32, float16 or bfloat16" % what)
    return kind


def _matrix(t, dtype, dev: int, shape, what: str):
    """(pointer, elements between rows) of a matrix of that type on that device; rows may lie apart."""
    if t is None:
        return None, 0
    if t.dtype is not dtype or t.get_device() != dev:
        raise TypeError("%s must be a tensor of dtype %s on device %d" % (what, dtype, dev))
    if t.shape != shape:
        raise TypeError("%s must have shape %s, not %s" % (what, tuple(shape), tuple(t.shape)))
    step, one = t.stride()
    rows, cols = shape
    if (one != 1 and cols > 1) or (step < cols and rows > 1):
        raise TypeError("%s must have contiguous rows that do not overlap" % what)
    return t.data_ptr(), step if rows > 1 else cols


def _dense(t, dtype, dev: int, shape, what: str):
    """The pointer of a contiguous tensor of that type and shape on that device, None for None."""
    if t is None:
        return None
    if t.dtype is not dtype or t.get_device() != dev or not t.is_contiguous():
        raise TypeError("%s must be a contiguous tensor of dtype %s on device %d" % (what, dtype, dev))
    if t.shape != shape:
        raise TypeError("%s must have shape %s, not %s" % (what, tuple(shape), tuple(t.shape)))
    return t.data_ptr()


def _grad_type(grad, like):
    """Parameter gradients are of the tensors' own type or fp32."""
    kind = _type_of(like, "X")
    if grad is not None and _TYPES.get(grad.dtype) == DN_F32:
        return DN_F32, grad.dtype
    return kind, like.dtype


_REFUSED = C.c_size_t(-1).value


def _workspace(need: int, workspace, like):
    """(the tensor, its pointer, its bytes); allocated here if the caller brings none."""
    if workspace is None:
        if need == 0 or need == _REFUSED:      # refused: the call itself says why
            return None, None, 0
        workspace = _torch.empty(need, dtype=_torch.uint8, device=like.device)
    elif workspace.dtype != _torch.uint8 or workspace.device != like.device or not workspace.is_contiguous():
        raise TypeError("workspace must be a contiguous uint8 tensor on %s" % (like.device,))
    return workspace, workspace.data_ptr(), workspace.numel()


class _Here:
    """In place of torch.cuda.device where the tensors' device is the current one."""

    def __enter__(self):
        return self

    def __exit__(self, *a):
        return False


_here = _Here()


def _on(dev: int):
    return _here if _torch.cuda.current_device() == dev else _torch.cuda.device(dev)


def _stream(dev: int) -> int:
    # torch's own short way to current_stream(dev).cuda_stream, a microsecond less, where it has it
    return _raw_stream(dev) if _raw_stream else _torch.cuda.current_stream(dev).cuda_stream


def _two(t, what: str):
    if t.dim() != 2:
        raise TypeError("%s must be a matrix" % what)
    rows, cols = t.shape
    if (rows | cols) >> 31:     # the descriptors hold 32 bits
        raise DnError(DN_ERR_SHAPE, "%s of shape %s" % (what, tuple(t.shape)))
    return rows, cols


def _linear_desc(X, W, R, Y, Yname, act, drop, seed, offset, grad_type, grad_scale):
    kind = _type_of(X, "X")
    rows, n_in = _two(X, "X")
    n_out = _two(W, "W")[0]
    dtype, dev = X.dtype, X.get_device()
    x, ldx = _matrix(X, dtype, dev, (rows, n_in), "X")
    w, ldw = _matrix(W, dtype, dev, (n_out, n_in), "W")
    r, ldr = _matrix(R, dtype, dev, (rows, n_out), "R")
    y, ldy = _matrix(Y, dtype, dev, (rows, n_out), Yname)
    d = LinearDesc(kind, kind if grad_type is None else grad_type, act, rows, n_in, n_out, ldx, ldw, ldr, ldy, drop, grad_scale,
                   seed, offset)
    return d, x, w, r, y, rows, n_in, n_out, dtype, dev


def dn_linear_forward(X, W, bias, R, Y, Z=None, act: int = DN_ACT_LINEAR, drop: float = 0.0, seed: int = 0, offset: int = 0,
                      workspace=None):
    """Y = R + D(f(X W^T + bias)); Z receives X W^T + bias.  bias, R and Z may be None.  Enqueued on torch's current stream, as
    everything below; `workspace`: a uint8 tensor of dn_linear_forward_workspace_bytes bytes (allocated here if None)."""
    l = lib()
    d, x, w, r, y, rows, _, n_out, dtype, dev = _linear_desc(X, W, R, Y, "Y", act, drop, seed, offset, None, 1.0)
    b, z = _dense(bias, dtype, dev, (n_out,), "bias"), _dense(Z, dtype, dev, (rows, n_out), "Z")
    with _on(dev):
        at = C.addressof(d)
        _keep, ws, n = _workspace(l.dn_linear_forward_workspace_bytes(at), workspace, X)
        _check(l.dn_linear_forward(at, x, w, b, r, y, z, ws, n, _stream(dev)), "dn_linear_forward")


def dn_linear_backward(X, W, Z, dY, dX, dW, dbias, act: int = DN_ACT_LINEAR, drop: float = 0.0, seed: int = 0, offset: int = 0,
                       grad_scale: float = 1.0, workspace=None):
    """delta = D(dY) f'(Z); dX = delta W, dW = grad_scale delta^T X, dbias = grad_scale times delta's column sums.  Z may be
    None without an activation; dX, dW, dbias may be None; dW and dbias are of X's type or float32."""
    l = lib()
    gt, gdtype = _grad_type(dW, X)
    d, x, w, _, y, rows, n_in, n_out, dtype, dev = _linear_desc(X, W, None, dY, "dY", act, drop, seed, offset, gt, grad_scale)
    z, dx = _dense(Z, dtype, dev, (rows, n_out), "Z"), _dense(dX, dtype, dev, (rows, n_in), "dX")
    dw, db = _dense(dW, gdtype, dev, (n_out, n_in), "dW"), _dense(dbias, gdtype, dev, (n_out,), "dbias")
    with _on(dev):
        at = C.addressof(d)
        _keep, ws, n = _workspace(l.dn_linear_backward_workspace_bytes(at), workspace, X)
        _check(l.dn_linear_backward(at, x, w, z, y, dx, dw, db, ws, n, _stream(dev)), "dn_linear_backward")


def _ffn_desc(X, Wg, Wu, Wd, R, Y, Yname, act, drop, seed, offset, grad_type, grad_scale):
    kind = _type_of(X, "X")
    rows, d = _two(X, "X")
    f = _two(Wg, "Wg")[0]
    dtype, dev = X.dtype, X.get_device()
    x, ldx = _matrix(X, dtype, dev, (rows, d), "X")
    r, ldr = _matrix(R, dtype, dev, (rows, d), "R")
    y, ldy = _matrix(Y, dtype, dev, (rows, d), Yname)
    desc = FfnDesc(kind, kind if grad_type is None else grad_type, act, rows, d, f, ldx, ldr, ldy, drop, grad_scale, seed, offset)
    w = _dense(Wg, dtype, dev, (f, d), "Wg"), _dense(Wu, dtype, dev, (f, d), "Wu"), _dense(Wd, dtype, dev, (d, f), "Wd")
    return desc, x, r, y, w, rows, d, f, dtype, dev


def dn_ffn_forward(X, Wg, bg, Wu, bu, Wd, bd, R, Y, GU=None, act: int = DN_ACT_SILU, drop: float = 0.0, seed: int = 0,
                   offset: int = 0, workspace=None):
    """Y = R + D((f(X Wg^T + bg) * (X Wu^T + bu)) Wd^T + bd); GU [rows][2 f] receives both net inputs.  The biases, R and GU
    may be None."""
    l = lib()
    desc, x, r, y, (wg, wu, wd), rows, d, f, dtype, dev = _ffn_desc(X, Wg, Wu, Wd, R, Y, "Y", act, drop, seed, offset, None, 1.0)
    g, u = _dense(bg, dtype, dev, (f,), "bg"), _dense(bu, dtype, dev, (f,), "bu")
    b, gu = _dense(bd, dtype, dev, (d,), "bd"), _dense(GU, dtype, dev, (rows, 2 * f), "GU")
    with _on(dev):
        at = C.addressof(desc)
        _keep, ws, n = _workspace(l.dn_ffn_forward_workspace_bytes(at), workspace, X)
        _check(l.dn_ffn_forward(at, x, wg, g, wu, u, wd, b, r, y, gu, ws, n, _stream(dev)), "dn_ffn_forward")


def dn_ffn_backward(X, Wg, Wu, Wd, GU, dY, dX, dWg, dbg, dWu, dbu, dWd, dbd, act: int = DN_ACT_SILU, drop: float = 0.0,
                    seed: int = 0, offset: int = 0, grad_scale: float = 1.0, workspace=None):
    """The block's gradients; dX and the biases' may be None, the parameters' are all of X's type or all float32."""
    l = lib()
    gt, gdtype = _grad_type(dWg, X)
    desc, x, _, y, (wg, wu, wd), rows, d, f, dtype, dev = _ffn_desc(X, Wg, Wu, Wd, None, dY, "dY", act, drop, seed, offset, gt,
                                                                    grad_scale)
    gu, dx = _dense(GU, dtype, dev, (rows, 2 * f), "GU"), _dense(dX, dtype, dev, (rows, d), "dX")
    dwg, dwu = _dense(dWg, gdtype, dev, (f, d), "dWg"), _dense(dWu, gdtype, dev, (f, d), "dWu")
    dwd, b = _dense(dWd, gdtype, dev, (d, f), "dWd"), _dense(dbd, gdtype, dev, (d,), "dbd")
    g, u = _dense(dbg, gdtype, dev, (f,), "dbg"), _dense(dbu, gdtype, dev, (f,), "dbu")
    with _on(dev):
        at = C.addressof(desc)
        _keep, ws, n = _workspace(l.dn_ffn_backward_workspace_bytes(at), workspace, X)
        _check(l.dn_ffn_backward(at, x, wg, wu, wd, gu, y, dx, dwg, g, dwu, u, dwd, b, ws, n, _stream(dev)), "dn_ffn_backward")


def _norm_desc(like, post, pre, scale, eps, rows_per_gate, grad_type=None):
    kind = _type_of(like, "x")
    rows, d = _two(like, "x")
    per = rows if rows_per_gate is None else rows_per_gate
    # (more rows a gate than there are is one gate, and need not fit 32 bits)
    desc = NormDesc(kind, kind if grad_type is None else grad_type, rows, d, post, pre, max(min(per, rows), 0), scale, eps)
    return desc, (rows, d), (d,), (-(-rows // per) if per > 0 else 0, d), like.dtype, like.get_device()


def dn_norm_forward(x, b, gate, post_w, post_b, pre_w, pre_b, x_out, n_out, post: int = DN_NORM_RMS, pre: int = DN_NORM_RMS,
                    scale: float = 1.0, eps: float = 1e-5, rows_per_gate: Optional[int] = None):
    """x_out = x + scale gate post(b), n_out = pre(x_out).  b, gate, the norms' weights and shifts may be None (no block,
    ones, zeros); gate [ceil(rows / rows_per_gate)][d] (default: one row)."""
    l = lib()
    desc, big, one, gates, t, dev = _norm_desc(x, post, pre, scale, eps, rows_per_gate)
    with _on(dev):
        _check(l.dn_norm_forward(C.addressof(desc), _dense(x, t, dev, big, "x"), _dense(b, t, dev, big, "b"),
                                 _dense(gate, t, dev, gates, "gate"), _dense(post_w, t, dev, one, "post_w"),
                                 _dense(post_b, t, dev, one, "post_b"), _dense(pre_w, t, dev, one, "pre_w"),
                                 _dense(pre_b, t, dev, one, "pre_b"), _dense(x_out, t, dev, big, "x_out"),
                                 _dense(n_out, t, dev, big, "n_out"), _stream(dev)), "dn_norm_forward")


def dn_norm_backward(x, b, gate, post_w, post_b, pre_w, dx_out, dn, dx, db, dgate, dpost_w, dpost_b, dpre_w, dpre_b,
                     post: int = DN_NORM_RMS, pre: int = DN_NORM_RMS, scale: float = 1.0, eps: float = 1e-5,
                     rows_per_gate: Optional[int] = None, workspace=None):
    """The gradients of dn_norm_forward; x is its x_out.  dx_out may be None (zero), so may the gradients of gate, weights and
    shifts (not computed), which are all of x's type or all float32."""
    l = lib()
    like = x if x is not None else dx
    grads = [t for t in (dgate, dpost_w, dpost_b, dpre_w, dpre_b) if t is not None]
    gt, gdtype = _grad_type(grads[0] if grads else None, like)
    desc, big, one, gates, t, dev = _norm_desc(like, post, pre, scale, eps, rows_per_gate, gt)
    p = [_dense(v, t, dev, s, n) for v, s, n in ((x, big, "x"), (b, big, "b"), (gate, gates, "gate"), (post_w, one, "post_w"),
                                                 (post_b, one, "post_b"), (pre_w, one, "pre_w"), (dx_out, big, "dx_out"),
                                                 (dn, big, "dn"), (dx, big, "dx"), (db, big, "db"))]
    p += [_dense(v, gdtype, dev, s, n) for v, s, n in ((dgate, gates, "dgate"), (dpost_w, one, "dpost_w"), (dpost_b, one, "dpost_b"),
                                                       (dpre_w, one, "dpre_w"), (dpre_b, one, "dpre_b"))]
    with _on(dev):
        at = C.addressof(desc)
        _keep, ws, n = _workspace(l.dn_norm_backward_workspace_bytes(at), workspace, like)
        _check(l.dn_norm_backward(at, *p, ws, n, _stream(dev)), "dn_norm_backward")


def dn_dropout(X, Y, drop: float, seed: int, offset: int = 0):
    """Y = D(X), forward and backward alike; Y may be X, rows of either may lie apart."""
    kind = _type_of(X, "X")
    shape, dev = _two(X, "X"), X.get_device()
    x, ldx = _matrix(X, X.dtype, dev, shape, "X")
    y, ldy = _matrix(Y, X.dtype, dev, shape, "Y")
    with _on(dev):
        _check(lib().dn_dropout(kind, x, y, shape[0], shape[1], ldx, ldy, drop, seed, offset, _stream(dev)), "dn_dropout")


# ---- a block of experts ------------------------------------------------------------------------------------------

def _route_desc(L, k, score, groups, top_groups, group_best, renorm, scale):
    kind = _type_of(L, "L")
    rows, experts = _two(L, "L")
    l, ldl = _matrix(L, L.dtype, L.get_device(), (rows, experts), "L")
    return RouteDesc(kind, score, rows, experts, k, groups, top_groups, group_best, bool(renorm), scale, ldl), l, rows, experts


def _choices(t, what: str):
    """[rows][k] of a table of choices."""
    if t.dim() != 2:
        raise TypeError("%s must be a matrix" % what)
    return _two(t, what)


def dn_route_forward(L, bias, expert, weight, starts=None, order=None, place=None, score: int = DN_SCORE_SOFTMAX, groups: int = 1,
                     top_groups: int = 1, group_best: int = 1, renorm: bool = True, scale: float = 1.0, workspace=None):
    """Each row's k experts by the scores of its logits L, expert [rows][k] int32 (highest first, -1 for none), and their weights
    [rows][k] float32; with starts [experts + 1], order and place [rows * k] (int32) the lists of pairs by expert too.  bias: float32
    [experts] or None."""
    l = lib()
    rows, k = _choices(expert, "expert")
    d, at_l, _, experts = _route_desc(L, k, score, groups, top_groups, group_best, renorm, scale)
    i32, f32, dev = _torch.int32, _torch.float32, L.get_device()
    b, e, w = _dense(bias, f32, dev, (experts,), "bias"), _dense(expert, i32, dev, (d.rows, k), "expert"), _dense(weight, f32, dev, (d.rows, k), "weight")
    lists = (_dense(starts, i32, dev, (experts + 1,), "starts"), _dense(order, i32, dev, (rows * k,), "order"), _dense(place, i32, dev, (rows * k,), "place"))
    with _on(dev):
        need = l.dn_route_workspace_bytes(rows, experts, k) if starts is not None else 0
        _keep, ws, n = _workspace(need, workspace, L)
        _check(l.dn_route_forward(C.addressof(d), at_l, b, e, w, *lists, ws, n, _stream(dev)), "dn_route_forward")


def dn_route_lists(expert, starts, order, place, workspace=None):
    """The lists of a table of choices, expert [rows][k] int32 (numbers that are no expert's: none): starts [experts + 1], order and
    place [rows * k]."""
    l = lib()
    _setup()
    if not expert.is_cuda:
        raise TypeError("expert must be a device tensor")
    rows, k = _choices(expert, "expert")
    i32, dev, experts = _torch.int32, expert.get_device(), starts.numel() - 1
    p = (_dense(expert, i32, dev, (rows, k), "expert"), _dense(starts, i32, dev, (experts + 1,), "starts"),
         _dense(order, i32, dev, (rows * k,), "order"), _dense(place, i32, dev, (rows * k,), "place"))
    with _on(dev):
        _keep, ws, n = _workspace(l.dn_route_workspace_bytes(rows, experts, k), workspace, expert)
        _check(l.dn_route_lists(p[0], rows, experts, k, *p[1:], ws, n, _stream(dev)), "dn_route_lists")


def dn_route_backward(L, expert, dweight, dL, score: int = DN_SCORE_SOFTMAX, renorm: bool = True, scale: float = 1.0):
    """dL from the weights' gradient, for the choices in expert."""
    l = lib()
    rows, k = _choices(expert, "expert")
    d, at_l, _, experts = _route_desc(L, k, score, 1, 1, 1, renorm, scale)
    dev = L.get_device()
    e, w = _dense(expert, _torch.int32, dev, (d.rows, k), "expert"), _dense(dweight, _torch.float32, dev, (d.rows, k), "dweight")
    dl = _dense(dL, L.dtype, dev, (d.rows, experts), "dL")
    with _on(dev):
        _check(l.dn_route_backward(C.addressof(d), at_l, e, w, dl, _stream(dev)), "dn_route_backward")


def _experts_desc(X, Wg, Wu, Wd, weight, starts, order, place, R, Y, Yname, act, grad_type, grad_scale):
    kind = _type_of(X, "X")
    rows, d = _two(X, "X")
    if Wg.dim() != 3 or max(Wg.shape) >> 31:
        raise TypeError("Wg must be [experts][f][d]")
    experts, f, _ = Wg.shape
    k = _choices(weight, "weight")[1]
    dtype, dev, i32 = X.dtype, X.get_device(), _torch.int32
    x, ldx = _matrix(X, dtype, dev, (rows, d), "X")
    r, ldr = _matrix(R, dtype, dev, (rows, d), "R")
    y, ldy = _matrix(Y, dtype, dev, (rows, d), Yname)
    desc = ExpertsDesc(kind, kind if grad_type is None else grad_type, act, rows, d, f, experts, k, ldx, ldr, ldy, grad_scale)
    w = (_dense(Wg, dtype, dev, (experts, f, d), "Wg"), _dense(Wu, dtype, dev, (experts, f, d), "Wu"), _dense(Wd, dtype, dev, (experts, d, f), "Wd"))
    lists = (_dense(weight, _torch.float32, dev, (rows, k), "weight"), _dense(starts, i32, dev, (experts + 1,), "starts"),
             _dense(order, i32, dev, (rows * k,), "order"), _dense(place, i32, dev, (rows * k,), "place"))
    return desc, x, r, y, w, lists, (rows, d, f, experts, k), dtype, dev


def dn_experts_forward(X, Wg, Wu, Wd, weight, starts, order, place, R, Y, GU=None, act: int = DN_ACT_SILU, workspace=None):
    """Y_t = R_t + the sum over row t's choices of weight ((f(X Wg[e]^T) * (X Wu[e]^T)) Wd[e]^T), the choices by dn_route_forward's
    weight and lists.  GU [rows * k][2 f] receives both net inputs by place.  R and GU may be None."""
    l = lib()
    desc, x, r, y, w, lists, (rows, d, f, experts, k), dtype, dev = _experts_desc(X, Wg, Wu, Wd, weight, starts, order, place, R, Y, "Y", act,
                                                                                 None, 1.0)
    gu = _dense(GU, dtype, dev, (rows * k, 2 * f), "GU")
    with _on(dev):
        at = C.addressof(desc)
        _keep, ws, n = _workspace(l.dn_experts_forward_workspace_bytes(at), workspace, X)
        _check(l.dn_experts_forward(at, x, *w, *lists, r, y, gu, ws, n, _stream(dev)), "dn_experts_forward")


def dn_experts_backward(X, Wg, Wu, Wd, weight, starts, order, place, GU, dY, dX, dWg, dWu, dWd, dweight, act: int = DN_ACT_SILU,
                        grad_scale: float = 1.0, workspace=None):
    """The block's gradients; dX and dweight may be None, the matrices' are all of X's type or all float32."""
    l = lib()
    gt, gdtype = _grad_type(dWg, X)
    desc, x, _, y, w, lists, (rows, d, f, experts, k), dtype, dev = _experts_desc(X, Wg, Wu, Wd, weight, starts, order, place, None, dY, "dY",
                                                                                 act, gt, grad_scale)
    gu, dx = _dense(GU, dtype, dev, (rows * k, 2 * f), "GU"), _dense(dX, dtype, dev, (rows, d), "dX")
    dw = (_dense(dWg, gdtype, dev, (experts, f, d), "dWg"), _dense(dWu, gdtype, dev, (experts, f, d), "dWu"),
          _dense(dWd, gdtype, dev, (experts, d, f), "dWd"))
    dwt = _dense(dweight, _torch.float32, dev, (rows, k), "dweight")
    with _on(dev):
        at = C.addressof(desc)
        _keep, ws, n = _workspace(l.dn_experts_backward_workspace_bytes(at), workspace, X)
        _check(l.dn_experts_backward(at, x, *w, *lists, gu, y, dx, *dw, dwt, ws, n, _stream(dev)), "dn_experts_backward")


def dn_clip(grads, max_norm: float, norm, outs=None, workspace=None):
    """grads (tensors of any of the three types, each contiguous) times min(1, max_norm / n), n the norm of all of them together, which
    norm [1] float32 receives.  outs: where the results go, tensor by tensor: the gradient itself, another tensor of its type or of
    float32, or None (takes part in the norm only); outs None: into the gradients themselves."""
    l = lib()
    _type_of(norm, "norm")
    dev = norm.get_device()
    at_norm = _dense(norm, _torch.float32, dev, (1,), "norm")
    outs = grads if outs is None else outs
    if len(outs) != len(grads):
        raise TypeError("outs must be as many as grads")
    # the spans' 32 bytes as four words, the two types in the last: a tensor costs what asking it costs
    words, kinds = [], _TYPES
    for g, o in zip(grads, outs):
        kind = kinds.get(g.dtype)
        if kind is None or g.get_device() != dev or not g.is_contiguous():
            raise TypeError("gradients must be contiguous tensors of float32, float16 or bfloat16 on device %d" % dev)
        at, to, out_kind = g.data_ptr(), None, kind
        if o is g:
            to = at
        elif o is not None:
            out_kind = kinds.get(o.dtype)
            if out_kind is None or o.get_device() != dev or not o.is_contiguous() or o.shape != g.shape:
                raise TypeError("results must be contiguous tensors of their gradients' shapes on device %d" % dev)
            to = o.data_ptr()
        words += (at, to or 0, g.numel(), kind | out_kind << 32)
    n_spans = len(grads)
    spans = (C.c_int64 * max(len(words), 1))(*words)
    with _on(dev):
        at = C.addressof(spans)
        _keep, ws, n = _workspace(l.dn_clip_workspace_bytes(at, n_spans), workspace, norm)
        _check(l.dn_clip(at, n_spans, max_norm, at_norm, ws, n, _stream(dev)), "dn_clip")


class Net:
    """One network on the current device.  Owns the arena tensor (torch
    allocation) and the library handle; method names follow include/dn.h."""

    def __init__(self, widths: Sequence[int], acts: Sequence[int], loss: int, max_batch: int,
                 device: str = "cuda:0", _borrowed=None):
        import torch
        self._torch = torch
        self.widths = [int(w) for w in widths]
        self.L = len(self.widths) - 1
        self.max_batch = int(max_batch)
        self.device = torch.device(device)
        self._owned = _borrowed is None
        if _borrowed is not None:      # a handle that another object (Cnn) owns and destroys
            self._h = _borrowed
            return
        nbytes = dn_net_arena_bytes(self.widths, self.max_batch)
        if nbytes == 0:
            raise DnError(DN_ERR_SHAPE, "dn_net_arena_bytes")
        self.arena = torch.empty(nbytes, dtype=torch.uint8, device=self.device)
        self.stream = torch.cuda.current_stream(self.device)
        w_arr, w_p = _i32(self.widths)
        a_arr, a_p = _i32(acts)
        handle = C.c_void_p()
        with torch.cuda.device(self.device):
            st = lib().dn_net_create(w_p, len(w_arr), a_p, int(loss), self.max_batch,
                                     C.c_void_p(self.arena.data_ptr()), nbytes,
                                     C.c_void_p(self.stream.cuda_stream), C.byref(handle))
        _check(st, "dn_net_create")
        self._h = handle

    def close(self):
        if getattr(self, "_h", None):
            if self._owned:
                lib().dn_net_destroy(self._h)
            self._h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    # -- parameters ------------------------------------------------------------
    def dn_set_params(self, layer: int, W: Optional[np.ndarray], b: Optional[np.ndarray]):
        if not 1 <= layer <= self.L:
            raise DnError(DN_ERR_INVALID_ARG, "dn_set_params")
        Wc = None if W is None else np.ascontiguousarray(W, dtype=np.float32)
        bc = None if b is None else np.ascontiguousarray(b, dtype=np.float32)
        if Wc is not None and Wc.shape != (self.widths[layer], self.widths[layer - 1]):
            raise DnError(DN_ERR_SHAPE, "dn_set_params")
        if bc is not None and bc.shape != (self.widths[layer],):
            raise DnError(DN_ERR_SHAPE, "dn_set_params")
        _check(lib().dn_set_params(self._h, layer,
                                   None if Wc is None else Wc.ctypes.data_as(C.c_void_p),
                                   None if bc is None else bc.ctypes.data_as(C.c_void_p)), "dn_set_params")

    def _get(self, fn, name, layer) -> Tuple[np.ndarray, np.ndarray]:
        if not 1 <= layer <= self.L:          # the host buffers below are sized from the layer's widths
            raise DnError(DN_ERR_INVALID_ARG, name)
        W = np.empty((self.widths[layer], self.widths[layer - 1]), dtype=np.float32)
        b = np.empty(self.widths[layer], dtype=np.float32)
        _check(fn(self._h, layer, W.ctypes.data_as(C.c_void_p), b.ctypes.data_as(C.c_void_p)), name)
        return W, b

    def dn_get_params(self, layer: int):
        return self._get(lib().dn_get_params, "dn_get_params", layer)

    def dn_get_grads(self, layer: int):
        return self._get(lib().dn_get_grads, "dn_get_grads", layer)

    def set_all(self, W: Sequence[np.ndarray], b: Sequence[np.ndarray]):
        for l in range(1, self.L + 1):
            self.dn_set_params(l, W[l - 1], b[l - 1])

    def get_all(self) -> Tuple[List[np.ndarray], List[np.ndarray]]:
        pairs = [self.dn_get_params(l) for l in range(1, self.L + 1)]
        return [p[0] for p in pairs], [p[1] for p in pairs]

    def get_all_grads(self):
        pairs = [self.dn_get_grads(l) for l in range(1, self.L + 1)]
        return [p[0] for p in pairs], [p[1] for p in pairs]

    # -- the steps ---------------------------------------------------------------
    def dn_forward(self, X, out=None):
        t = self._torch
        batch = int(X.shape[0])
        _check(lib().dn_forward(self._h, _dev_ptr(X, t.float32, "X"), batch,
                                None if out is None else _dev_ptr(out, t.float32, "out")), "dn_forward")

    def dn_backward(self, labels, loss_out=None):
        t = self._torch
        _check(lib().dn_backward(self._h, _dev_ptr(labels, t.int32, "labels"), int(labels.shape[0]),
                                 None if loss_out is None else _dev_ptr(loss_out, t.float32, "loss")),
               "dn_backward")

    def dn_input_gradient(self, dX):
        t = self._torch
        _shape_check(dX, (int(dX.shape[0]), self.widths[0]), "dX")
        _check(lib().dn_input_gradient(self._h, int(dX.shape[0]), _dev_ptr(dX, t.float32, "dX")),
               "dn_input_gradient")

    def dn_update(self, lr: float, momentum: float):
        _check(lib().dn_update(self._h, float(lr), float(momentum)), "dn_update")

    def dn_train_epoch(self, X, labels, batch: int, lr: float, momentum: float,
                       n_samples: Optional[int] = None) -> float:
        t = self._torch
        n = int(X.shape[0]) if n_samples is None else int(n_samples)
        loss = C.c_float(0.0)
        _check(lib().dn_train_epoch(self._h, _dev_ptr(X, t.float32, "X"), _dev_ptr(labels, t.int32, "labels"),
                                    n, int(batch), float(lr), float(momentum), C.byref(loss)),
               "dn_train_epoch")
        return float(loss.value)

    def dn_train(self, X, labels, batch: int, lr: float, momentum: float, max_error: float,
                 max_epochs: int, n_samples: Optional[int] = None) -> Tuple[int, float]:
        """(epochs run, last epoch loss)."""
        t = self._torch
        n = int(X.shape[0]) if n_samples is None else int(n_samples)
        epochs, loss = C.c_int32(0), C.c_float(0.0)
        _check(lib().dn_train(self._h, _dev_ptr(X, t.float32, "X"), _dev_ptr(labels, t.int32, "labels"), n,
                              int(batch), float(lr), float(momentum), float(max_error), int(max_epochs),
                              C.byref(epochs), C.byref(loss)), "dn_train")
        return int(epochs.value), float(loss.value)

    def dn_evaluate(self, X, labels, batch: int, n_samples: Optional[int] = None) -> Tuple[float, int]:
        """(mean loss, number of samples whose largest output is at the label)."""
        t = self._torch
        n = int(X.shape[0]) if n_samples is None else int(n_samples)
        loss, correct = C.c_float(0.0), C.c_int64(0)
        _check(lib().dn_evaluate(self._h, _dev_ptr(X, t.float32, "X"), _dev_ptr(labels, t.int32, "labels"), n,
                                 int(batch), C.byref(loss), C.byref(correct)), "dn_evaluate")
        return float(loss.value), int(correct.value)

    # -- measurement ---------------------------------------------------------------
    def dn_last_epoch_ms(self) -> float:
        ms = C.c_float(0.0)
        _check(lib().dn_last_epoch_ms(self._h, C.byref(ms)), "dn_last_epoch_ms")
        return float(ms.value)

    def dn_last_schedule(self) -> int:
        v = C.c_int32(0)
        _check(lib().dn_last_schedule(self._h, C.byref(v)), "dn_last_schedule")
        return int(v.value)

    def dn_last_kernel(self) -> str:
        v = C.c_char_p()
        _check(lib().dn_last_kernel(self._h, C.byref(v)), "dn_last_kernel")
        return v.value.decode()

    def dn_kernel_time(self, kernel_class: int) -> Tuple[float, int]:
        ms, n = C.c_float(0.0), C.c_int64(0)
        _check(lib().dn_kernel_time(self._h, kernel_class, C.byref(ms), C.byref(n)), "dn_kernel_time")
        return float(ms.value), int(n.value)

    def dn_kernel_flops(self, kernel_class: int) -> float:
        f = C.c_double(0.0)
        _check(lib().dn_kernel_flops(self._h, kernel_class, C.byref(f)), "dn_kernel_flops")
        return float(f.value)

    def dn_set_option(self, name: str, value: int):
        _check(lib().dn_set_option(self._h, name.encode(), int(value)), "dn_set_option")


class Cnn:
    """A convolutional classifier on the current device (dn_cnn_* of include/dn.h): blocks of
    (c_out, k, stride, pad, act, pool_k, pool_stride) in front of a fully connected net.  Owns
    the arena tensor and the library handle; `dense` is the fully connected part as a Net."""

    def __init__(self, c: int, h: int, w: int, blocks: Sequence[Sequence[int]], dense_widths: Sequence[int],
                 dense_acts: Sequence[int], loss: int, max_batch: int, device: str = "cuda:0"):
        import torch
        self._torch = torch
        self.shape = (int(c), int(h), int(w))
        self.blocks = [tuple(int(v) for v in b) for b in blocks]
        if any(len(b) != 7 for b in self.blocks):
            raise DnError(DN_ERR_INVALID_ARG, "dn_cnn_create")
        self.max_batch = int(max_batch)
        self.device = torch.device(device)
        b_arr, b_p = _i32([v for b in self.blocks for v in b])
        w_arr, w_p = _i32(dense_widths)
        a_arr, a_p = _i32(dense_acts)
        nbytes = int(lib().dn_cnn_arena_bytes(c, h, w, b_p, len(self.blocks), w_p, len(w_arr), self.max_batch))
        if nbytes == 0:
            raise DnError(DN_ERR_SHAPE, "dn_cnn_arena_bytes")
        self.arena = torch.empty(nbytes, dtype=torch.uint8, device=self.device)
        self.stream = torch.cuda.current_stream(self.device)
        handle = C.c_void_p()
        with torch.cuda.device(self.device):
            st = lib().dn_cnn_create(c, h, w, b_p, len(self.blocks), w_p, len(w_arr), a_p, int(loss), self.max_batch,
                                     C.c_void_p(self.arena.data_ptr()), nbytes, C.c_void_p(self.stream.cuda_stream),
                                     C.byref(handle))
        _check(st, "dn_cnn_create")
        self._h = handle
        self.flat = int(lib().dn_cnn_flat_size(self._h))
        self.dense = Net([self.flat] + [int(v) for v in dense_widths], dense_acts, loss, self.max_batch, device,
                         _borrowed=C.c_void_p(lib().dn_cnn_dense(self._h)))
        # filter shapes, block by block
        self.filter_shapes, cin = [], int(c)
        for b in self.blocks:
            self.filter_shapes.append((b[0], cin, b[1], b[1]))
            cin = b[0]

    def close(self):
        if getattr(self, "_h", None):
            self.dense.close()
            lib().dn_cnn_destroy(self._h)
            self._h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def dn_cnn_set_filters(self, block: int, W: Optional[np.ndarray], bias: Optional[np.ndarray]):
        if not 0 <= block < len(self.blocks):
            raise DnError(DN_ERR_INVALID_ARG, "dn_cnn_set_filters")
        Wc = None if W is None else np.ascontiguousarray(W, dtype=np.float32)
        bc = None if bias is None else np.ascontiguousarray(bias, dtype=np.float32)
        if Wc is not None and Wc.shape != self.filter_shapes[block]:
            raise DnError(DN_ERR_SHAPE, "dn_cnn_set_filters")
        if bc is not None and bc.shape != (self.filter_shapes[block][0],):
            raise DnError(DN_ERR_SHAPE, "dn_cnn_set_filters")
        _check(lib().dn_cnn_set_filters(self._h, block, None if Wc is None else Wc.ctypes.data_as(C.c_void_p),
                                        None if bc is None else bc.ctypes.data_as(C.c_void_p)), "dn_cnn_set_filters")

    def _get(self, fn, name, block):
        if not 0 <= block < len(self.blocks):      # the host buffers below are sized from the block's shape
            raise DnError(DN_ERR_INVALID_ARG, name)
        W = np.empty(self.filter_shapes[block], dtype=np.float32)
        b = np.empty(self.filter_shapes[block][0], dtype=np.float32)
        _check(fn(self._h, block, W.ctypes.data_as(C.c_void_p), b.ctypes.data_as(C.c_void_p)), name)
        return W, b

    def dn_cnn_get_filters(self, block: int):
        return self._get(lib().dn_cnn_get_filters, "dn_cnn_get_filters", block)

    def dn_cnn_get_filter_grads(self, block: int):
        return self._get(lib().dn_cnn_get_filter_grads, "dn_cnn_get_filter_grads", block)

    def dn_cnn_forward(self, X, out=None):
        t = self._torch
        _shape_check(X, (int(X.shape[0]),) + self.shape, "X")
        _check(lib().dn_cnn_forward(self._h, _dev_ptr(X, t.float32, "X"), int(X.shape[0]),
                                    None if out is None else _dev_ptr(out, t.float32, "out")), "dn_cnn_forward")

    def dn_cnn_train_epoch(self, X, labels, batch: int, lr: float, momentum: float,
                           n_samples: Optional[int] = None) -> float:
        t = self._torch
        _shape_check(X, (int(X.shape[0]),) + self.shape, "X")
        n = int(X.shape[0]) if n_samples is None else int(n_samples)
        if n > int(X.shape[0]) or n > int(labels.shape[0]):
            raise DnError(DN_ERR_SHAPE, "dn_cnn_train_epoch")
        loss = C.c_float(0.0)
        _check(lib().dn_cnn_train_epoch(self._h, _dev_ptr(X, t.float32, "X"), _dev_ptr(labels, t.int32, "labels"), n,
                                        int(batch), float(lr), float(momentum), C.byref(loss)), "dn_cnn_train_epoch")
        return float(loss.value)
