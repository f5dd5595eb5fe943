"""Python binding of libpyramid_lstm.so (the MI355X PyraMiD-LSTM library).

Argument marshalling only: every function here has the name of a C entry point
declared in include/pyramid_lstm.h, converts torch tensors to device pointers
and the current HIP stream, calls the entry point and raises on a negative
status.  All computation runs in the library's HIP kernels; torch provides
device memory and streams.  There is no fallback: if the library is not built
the binding raises.
"""
from __future__ import annotations

import ctypes
import functools
import os

import torch

__all__ = [
    "PyramidLSTMError", "plstm_shape", "shape_for", "PLSTM_F32", "PLSTM_BF16",
    "pyramid_lstm_status_string", "pyramid_lstm_workspace_size", "pyramid_lstm_saved_size",
    "pyramid_lstm_forward", "pyramid_lstm_backward", "pyramid_fc_tanh_forward",
    "pyramid_fc_workspace_size", "pyramid_fc_tanh_backward", "pyramid_softmax_ce",
    "pyramid_head_workspace_size", "pyramid_head_train", "plstm_param_segment",
    "pyramid_head_forward", "pyramid_head_forward_supported",
    "pyramid_rmsprop_step", "pyramid_rmsprop_learning_rate", "RMSprop", "pyramid_softmax_sq",
    "pyramid_crop", "pyramid_stitch_clear", "pyramid_stitch_add", "pyramid_stitch_finish",
    "pyramid_lstm_timing_enable", "pyramid_lstm_timing_read", "pyramid_lstm_set_forward_path",
    "pyramid_lstm_set_backward_path", "pyramid_lstm_set_step_split", "pyramid_lstm_set_bf16_mfma",
    "pyramid_lstm_set_wgrad_staged",
    "library_path", "load", "plstm2d_shape", "shape2d_for", "pyramid_lstm2d_workspace_size",
    "pyramid_lstm2d_saved_size", "pyramid_lstm2d_forward", "pyramid_lstm2d_backward",
    "plstm_cube", "PLSTM_FLIP_Z", "PLSTM_FLIP_Y", "PLSTM_FLIP_X", "PLSTM_MAX_CUBES",
    "pyramid_sample_cubes", "draw_cubes", "pyramid_lstm_device_status",
    "pyramid_lstm_set_wait_test", "PLSTM_DEVICE_WAIT_GAVE_UP", "pyramid_lstm_forward_noalloc",
    "PLSTM_NOALLOC_SCRATCH_BYTES", "PLSTM_ESCRATCH",
    "pyramid_layer_norm_workspace_size", "pyramid_layer_norm_forward",
    "pyramid_layer_norm_backward", "pyramid_scan_workspace_size", "pyramid_scan_saved_size",
    "pyramid_scan_forward", "pyramid_scan_backward", "pyramid_checkpoint8_scales",
    "pyramid_checkpoint8_pack", "pyramid_checkpoint8_unpack", "checkpoint8_empty",
    "pyramid_causal_conv_workspace_size", "pyramid_causal_conv_forward",
    "pyramid_causal_conv_backward", "pyramid_selective_scan_workspace_size",
    "pyramid_selective_scan_saved_size", "pyramid_selective_scan_forward",
    "pyramid_selective_scan_backward", "pyramid_group_norm_workspace_size",
    "pyramid_group_norm_forward", "pyramid_group_norm_backward", "plstm_adamw_segment",
    "pyramid_adamw_scales", "pyramid_adamw_step", "pyramid_adamw_moments", "AdamW",
    "PLSTM_ADAMW_CLOCK_BYTES",
]

PLSTM_F32 = 0
PLSTM_BF16 = 1
PLSTM_FLIP_Z, PLSTM_FLIP_Y, PLSTM_FLIP_X = 1, 2, 4
PLSTM_MAX_CUBES = 64
PLSTM_DEVICE_WAIT_GAVE_UP = 1
PLSTM_NOALLOC_SCRATCH_BYTES = 256 << 20
PLSTM_ESCRATCH = -6
PLSTM_ADAMW_CLOCK_BYTES = 24

_PKG = os.path.dirname(os.path.abspath(__file__))
_LIB_PATH = os.path.join(_PKG, "libpyramid_lstm.so")
_lib = None


class PyramidLSTMError(RuntimeError):
    def __init__(self, fn, status):
        self.status = status
        super().__init__("%s failed: %s (%d)" % (fn, pyramid_lstm_status_string(status), status))


class plstm_shape(ctypes.Structure):
    _fields_ = [("N", ctypes.c_int32), ("D", ctypes.c_int32), ("H", ctypes.c_int32),
                ("W", ctypes.c_int32), ("C", ctypes.c_int32), ("O", ctypes.c_int32),
                ("dtype", ctypes.c_int32), ("K", ctypes.c_int32)]


class plstm2d_shape(ctypes.Structure):
    _fields_ = [("N", ctypes.c_int32), ("H", ctypes.c_int32), ("W", ctypes.c_int32),
                ("C", ctypes.c_int32), ("O", ctypes.c_int32), ("dtype", ctypes.c_int32),
                ("K", ctypes.c_int32)]


class plstm_cube(ctypes.Structure):
    _fields_ = [("n", ctypes.c_int32), ("z0", ctypes.c_int32), ("y0", ctypes.c_int32),
                ("x0", ctypes.c_int32), ("cos_t", ctypes.c_float), ("sin_t", ctypes.c_float),
                ("flips", ctypes.c_int32)]


class plstm_param_segment(ctypes.Structure):
    _fields_ = [("theta", ctypes.c_void_p), ("grad", ctypes.c_void_p), ("ms", ctypes.c_void_p),
                ("mom", ctypes.c_void_p), ("n", ctypes.c_int64)]


class plstm_adamw_segment(ctypes.Structure):
    _fields_ = [("theta", ctypes.c_void_p), ("copy", ctypes.c_void_p), ("grad", ctypes.c_void_p),
                ("m", ctypes.c_void_p), ("v", ctypes.c_void_p), ("mscale", ctypes.c_void_p),
                ("vscale", ctypes.c_void_p), ("n", ctypes.c_int64),
                ("weight_decay", ctypes.c_float), ("reserved", ctypes.c_int32)]


def library_path() -> str:
    return _LIB_PATH


def load():
    """Load the HIP library (raises if it has not been built)."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(_LIB_PATH):
        raise RuntimeError("libpyramid_lstm.so is not built; run "
                           "`python -m paper_1506_07452_amd.build` first")
    lib = ctypes.CDLL(_LIB_PATH)
    vp, sz, i32, i64 = ctypes.c_void_p, ctypes.c_size_t, ctypes.c_int32, ctypes.c_int64
    sp = ctypes.POINTER(plstm_shape)
    lib.pyramid_lstm_status_string.argtypes = [ctypes.c_int]
    lib.pyramid_lstm_status_string.restype = ctypes.c_char_p
    lib.pyramid_lstm_workspace_size.argtypes = [sp, ctypes.c_int]
    lib.pyramid_lstm_workspace_size.restype = sz
    lib.pyramid_lstm_saved_size.argtypes = [sp]
    lib.pyramid_lstm_saved_size.restype = sz
    lib.pyramid_lstm_forward.argtypes = [sp] + [vp] * 7 + [sz, vp]
    lib.pyramid_lstm_forward.restype = ctypes.c_int
    lib.pyramid_lstm_forward_noalloc.argtypes = [sp] + [vp] * 6
    lib.pyramid_lstm_forward_noalloc.restype = ctypes.c_int
    lib.pyramid_lstm_backward.argtypes = [sp] + [vp] * 11 + [sz, vp]
    lib.pyramid_lstm_backward.restype = ctypes.c_int
    sp2 = ctypes.POINTER(plstm2d_shape)
    lib.pyramid_lstm2d_workspace_size.argtypes = [sp2, ctypes.c_int]
    lib.pyramid_lstm2d_workspace_size.restype = sz
    lib.pyramid_lstm2d_saved_size.argtypes = [sp2]
    lib.pyramid_lstm2d_saved_size.restype = sz
    lib.pyramid_lstm2d_forward.argtypes = [sp2] + [vp] * 7 + [sz, vp]
    lib.pyramid_lstm2d_forward.restype = ctypes.c_int
    lib.pyramid_lstm2d_backward.argtypes = [sp2] + [vp] * 11 + [sz, vp]
    lib.pyramid_lstm2d_backward.restype = ctypes.c_int
    lib.pyramid_fc_tanh_forward.argtypes = [i64, i32, i32, i32] + [vp] * 4 + [vp]
    lib.pyramid_fc_tanh_forward.restype = ctypes.c_int
    lib.pyramid_fc_workspace_size.argtypes = [i64, i32, i32]
    lib.pyramid_fc_workspace_size.restype = sz
    lib.pyramid_fc_tanh_backward.argtypes = [i64, i32, i32] + [vp] * 8 + [sz, vp]
    lib.pyramid_fc_tanh_backward.restype = ctypes.c_int
    lib.pyramid_softmax_ce.argtypes = [i64, i32, i32, i32] + [vp] * 10 + [sz, vp]
    lib.pyramid_softmax_ce.restype = ctypes.c_int
    lib.pyramid_softmax_sq.argtypes = [i64, i32, i32, i32] + [vp] * 10 + [sz, vp]
    lib.pyramid_softmax_sq.restype = ctypes.c_int
    lib.pyramid_head_workspace_size.argtypes = [i64, i32, i32, i32]
    lib.pyramid_head_workspace_size.restype = sz
    lib.pyramid_head_train.argtypes = [i64, i32, i32, i32] + [vp] * 14 + [sz, vp]
    lib.pyramid_head_train.restype = ctypes.c_int
    lib.pyramid_head_forward_supported.argtypes = [i32, i32, i32, i32]
    lib.pyramid_head_forward_supported.restype = ctypes.c_int
    lib.pyramid_head_forward.argtypes = [i64, i32, i32, i32, i32] + [vp] * 7
    lib.pyramid_head_forward.restype = ctypes.c_int
    f32 = ctypes.c_float
    lib.pyramid_rmsprop_step.argtypes = [i32, ctypes.POINTER(plstm_param_segment), f32, f32, f32,
                                         f32, vp]
    lib.pyramid_rmsprop_step.restype = ctypes.c_int
    lib.pyramid_rmsprop_learning_rate.argtypes = [i32]
    lib.pyramid_rmsprop_learning_rate.restype = ctypes.c_double
    lib.pyramid_crop.argtypes = [i32] * 13 + [vp, vp, vp]
    lib.pyramid_crop.restype = ctypes.c_int
    lib.pyramid_sample_cubes.argtypes = [i32] * 7 + [ctypes.POINTER(plstm_cube)] + [i32] * 3 + \
        [vp] * 5
    lib.pyramid_sample_cubes.restype = ctypes.c_int
    lib.pyramid_stitch_clear.argtypes = [i32] * 4 + [vp, vp, vp]
    lib.pyramid_stitch_clear.restype = ctypes.c_int
    lib.pyramid_stitch_add.argtypes = [i32] * 10 + [f32, vp, vp, vp, vp]
    lib.pyramid_stitch_add.restype = ctypes.c_int
    lib.pyramid_stitch_finish.argtypes = [i32] * 4 + [vp, vp, vp, vp]
    lib.pyramid_stitch_finish.restype = ctypes.c_int
    lib.pyramid_layer_norm_workspace_size.argtypes = [i64, i32]
    lib.pyramid_layer_norm_workspace_size.restype = sz
    lib.pyramid_layer_norm_forward.argtypes = [i64, i32, i32, f32] + [vp] * 8
    lib.pyramid_layer_norm_forward.restype = ctypes.c_int
    lib.pyramid_layer_norm_backward.argtypes = [i64, i32, i32] + [vp] * 9 + [sz, vp]
    lib.pyramid_layer_norm_backward.restype = ctypes.c_int
    lib.pyramid_scan_workspace_size.argtypes = [i64] * 3
    lib.pyramid_scan_workspace_size.restype = sz
    lib.pyramid_scan_saved_size.argtypes = [i64] * 3
    lib.pyramid_scan_saved_size.restype = sz
    lib.pyramid_scan_forward.argtypes = [i64] * 3 + [i32] * 2 + [vp] * 8 + [sz, vp]
    lib.pyramid_scan_forward.restype = ctypes.c_int
    lib.pyramid_scan_backward.argtypes = [i64] * 3 + [i32] * 2 + [vp] * 12 + [sz, vp]
    lib.pyramid_scan_backward.restype = ctypes.c_int
    lib.pyramid_checkpoint8_scales.argtypes = [i64]
    lib.pyramid_checkpoint8_scales.restype = i64
    lib.pyramid_checkpoint8_pack.argtypes = [i64, i32] + [vp] * 4
    lib.pyramid_checkpoint8_pack.restype = ctypes.c_int
    lib.pyramid_checkpoint8_unpack.argtypes = [i64, i32] + [vp] * 4
    lib.pyramid_checkpoint8_unpack.restype = ctypes.c_int
    lib.pyramid_causal_conv_workspace_size.argtypes = [i64] * 3 + [i32]
    lib.pyramid_causal_conv_workspace_size.restype = sz
    lib.pyramid_causal_conv_forward.argtypes = [i64] * 3 + [i32] * 4 + [vp, i64] + [vp] * 7
    lib.pyramid_causal_conv_forward.restype = ctypes.c_int
    lib.pyramid_causal_conv_backward.argtypes = [i64] * 3 + [i32] * 4 + [vp, i64] + [vp] * 11 + \
        [sz, vp]
    lib.pyramid_causal_conv_backward.restype = ctypes.c_int
    lib.pyramid_selective_scan_workspace_size.argtypes = [i64] * 3 + [i32] * 2
    lib.pyramid_selective_scan_workspace_size.restype = sz
    lib.pyramid_selective_scan_saved_size.argtypes = [i64] * 3 + [i32]
    lib.pyramid_selective_scan_saved_size.restype = sz
    select = [i64] * 3 + [i32] * 4 + [vp, i64, vp, i64, vp, vp, i64, vp, i64, vp, vp, i64, vp, vp]
    lib.pyramid_selective_scan_forward.argtypes = select + [vp] * 5 + [sz, vp]
    lib.pyramid_selective_scan_forward.restype = ctypes.c_int
    lib.pyramid_selective_scan_backward.argtypes = select + [vp] * 13 + [sz, vp]
    lib.pyramid_selective_scan_backward.restype = ctypes.c_int
    lib.pyramid_group_norm_workspace_size.argtypes = [i64] * 2 + [i32] * 2
    lib.pyramid_group_norm_workspace_size.restype = sz
    lib.pyramid_group_norm_forward.argtypes = [i64] * 2 + [i32] * 4 + [f32] + [vp] * 6 + [sz, vp]
    lib.pyramid_group_norm_forward.restype = ctypes.c_int
    lib.pyramid_group_norm_backward.argtypes = [i64] * 2 + [i32] * 4 + [vp] * 9 + [sz, vp]
    lib.pyramid_group_norm_backward.restype = ctypes.c_int
    f64, segp = ctypes.c_double, ctypes.POINTER(plstm_adamw_segment)
    lib.pyramid_adamw_scales.argtypes = [i64]
    lib.pyramid_adamw_scales.restype = i64
    lib.pyramid_adamw_step.argtypes = [i32, segp, i32, i32, f64, f64, f64, f64, i64,
                                       ctypes.c_uint32, vp, vp, vp, vp]
    lib.pyramid_adamw_step.restype = ctypes.c_int
    lib.pyramid_adamw_moments.argtypes = [i32, segp, ctypes.POINTER(vp), ctypes.POINTER(vp), vp]
    lib.pyramid_adamw_moments.restype = ctypes.c_int
    lib.pyramid_lstm_timing_enable.argtypes = [ctypes.c_int]
    lib.pyramid_lstm_timing_enable.restype = ctypes.c_int
    lib.pyramid_lstm_timing_read.argtypes = [ctypes.c_int, ctypes.c_char_p,
                                             ctypes.POINTER(ctypes.c_double),
                                             ctypes.POINTER(ctypes.c_int),
                                             ctypes.POINTER(ctypes.c_int)]
    lib.pyramid_lstm_timing_read.restype = ctypes.c_int
    lib.pyramid_lstm_device_status.argtypes = [ctypes.POINTER(ctypes.c_int32), i32, vp]
    lib.pyramid_lstm_device_status.restype = ctypes.c_int
    lib.pyramid_lstm_set_wait_test.argtypes = [ctypes.c_int]
    lib.pyramid_lstm_set_wait_test.restype = ctypes.c_int
    lib.pyramid_lstm_set_bf16_mfma.argtypes = [ctypes.c_int]
    lib.pyramid_lstm_set_bf16_mfma.restype = ctypes.c_int
    lib.pyramid_lstm_set_step_split.argtypes = [ctypes.c_int]
    lib.pyramid_lstm_set_step_split.restype = ctypes.c_int
    lib.pyramid_lstm_set_wgrad_staged.argtypes = [ctypes.c_int]
    lib.pyramid_lstm_set_wgrad_staged.restype = ctypes.c_int
    lib.pyramid_lstm_set_forward_path.argtypes = [ctypes.c_int]
    lib.pyramid_lstm_set_forward_path.restype = ctypes.c_int
    lib.pyramid_lstm_set_backward_path.argtypes = [ctypes.c_int]
    lib.pyramid_lstm_set_backward_path.restype = ctypes.c_int
    _lib = lib
    return lib


# ----------------------------------------------------------------- marshalling
_DT = {torch.float32: PLSTM_F32, torch.bfloat16: PLSTM_BF16}


def _ptr(t):
    if t is None:
        return None
    if not isinstance(t, torch.Tensor):
        raise TypeError("expected a torch.Tensor, got %r" % type(t))
    if not t.is_cuda:
        raise ValueError("tensor must live on the GPU")
    if not t.is_contiguous():
        raise ValueError("tensor must be contiguous")
    return ctypes.c_void_p(t.data_ptr())


def _stream(stream):
    if stream is None:
        stream = torch.cuda.current_stream()
    return ctypes.c_void_p(stream.cuda_stream if hasattr(stream, "cuda_stream") else int(stream))


def _torch_stream(stream, device):
    """A stream argument (torch's or a handle) as a torch stream."""
    if isinstance(stream, torch.cuda.Stream):
        return stream
    return torch.cuda.ExternalStream(int(getattr(stream, "cuda_stream", stream)), device)


def _check(fn, rc):
    if rc != 0:
        raise PyramidLSTMError(fn, rc)


def shape_for(x: torch.Tensor, O: int, K: int = 3) -> plstm_shape:
    """plstm_shape of a [N][D][H][W][C] volume, hidden size O and K x K filters."""
    if x.dim() != 5:
        raise ValueError("x must be [N][D][H][W][C]")
    if x.dtype not in _DT:
        raise ValueError("x must be float32 or bfloat16")
    N, D, H, W, C = x.shape
    return plstm_shape(N, D, H, W, C, O, _DT[x.dtype], K)


def shape2d_for(x: torch.Tensor, O: int, K: int = 3) -> plstm2d_shape:
    """plstm2d_shape of a [N][H][W][C] image batch, hidden size O, filters of K taps."""
    if x.dim() != 4:
        raise ValueError("x must be [N][H][W][C]")
    if x.dtype not in _DT:
        raise ValueError("x must be float32 or bfloat16")
    N, H, W, C = x.shape
    return plstm2d_shape(N, H, W, C, O, _DT[x.dtype], K)


def _workspace(nbytes, device):
    return torch.empty(max(int(nbytes), 256), dtype=torch.uint8, device=device)


def _temporary(nbytes, device, stream):
    """A workspace of the call's stream: memory that torch may give away again
    once what the stream has by then been told is done."""
    if stream is None or device.type != "cuda" or \
            (_stream(stream).value or 0) == torch._C._cuda_getCurrentRawStream(device.index):
        return _workspace(nbytes, device)
    with torch.cuda.stream(_torch_stream(stream, device)):
        return _workspace(nbytes, device)


# --------------------------------------------------------------- entry points
def pyramid_lstm_status_string(status: int) -> str:
    return load().pyramid_lstm_status_string(int(status)).decode()


def pyramid_lstm_workspace_size(shape: plstm_shape, training: int) -> int:
    return int(load().pyramid_lstm_workspace_size(ctypes.byref(shape), int(training)))


def pyramid_lstm_saved_size(shape: plstm_shape) -> int:
    return int(load().pyramid_lstm_saved_size(ctypes.byref(shape)))


def pyramid_lstm_forward(shape, x, wx, wh, b, h, saved=None, ws=None, stream=None):
    """Layer forward.  ws=None allocates the workspace with torch."""
    lib = load()
    if ws is None:
        ws = _temporary(pyramid_lstm_workspace_size(shape, saved is not None), x.device, stream)
    _check("pyramid_lstm_forward", lib.pyramid_lstm_forward(
        ctypes.byref(shape), _ptr(x), _ptr(wx), _ptr(wh), _ptr(b), _ptr(h), _ptr(saved),
        _ptr(ws), ws.numel() * ws.element_size(), _stream(stream)))


def pyramid_lstm_forward_noalloc(shape, x, wx, wh, b, h, stream=None):
    """Inference forward on the library's own per-GPU scratch (no workspace,
    nothing allocated); raises PyramidLSTMError (PLSTM_ESCRATCH) for shapes
    whose workspace exceeds PLSTM_NOALLOC_SCRATCH_BYTES."""
    _check("pyramid_lstm_forward_noalloc", load().pyramid_lstm_forward_noalloc(
        ctypes.byref(shape), _ptr(x), _ptr(wx), _ptr(wh), _ptr(b), _ptr(h), _stream(stream)))


def pyramid_lstm_backward(shape, x, wx, wh, b, saved, dh, dx, dwx, dwh, db, ws=None,
                          stream=None):
    lib = load()
    if ws is None:
        ws = _temporary(pyramid_lstm_workspace_size(shape, 1), x.device, stream)
    _check("pyramid_lstm_backward", lib.pyramid_lstm_backward(
        ctypes.byref(shape), _ptr(x), _ptr(wx), _ptr(wh), _ptr(b), _ptr(saved), _ptr(dh),
        _ptr(dx), _ptr(dwx), _ptr(dwh), _ptr(db), _ptr(ws), ws.numel() * ws.element_size(),
        _stream(stream)))


def pyramid_lstm2d_workspace_size(shape: plstm2d_shape, training: int) -> int:
    return int(load().pyramid_lstm2d_workspace_size(ctypes.byref(shape), int(training)))


def pyramid_lstm2d_saved_size(shape: plstm2d_shape) -> int:
    return int(load().pyramid_lstm2d_saved_size(ctypes.byref(shape)))


def pyramid_lstm2d_forward(shape, x, wx, wh, b, h, saved=None, ws=None, stream=None):
    """2D layer forward over x [N][H][W][C].  ws=None allocates the workspace with torch."""
    lib = load()
    if ws is None:
        ws = _temporary(pyramid_lstm2d_workspace_size(shape, saved is not None), x.device, stream)
    _check("pyramid_lstm2d_forward", lib.pyramid_lstm2d_forward(
        ctypes.byref(shape), _ptr(x), _ptr(wx), _ptr(wh), _ptr(b), _ptr(h), _ptr(saved),
        _ptr(ws), ws.numel() * ws.element_size(), _stream(stream)))


def pyramid_lstm2d_backward(shape, x, wx, wh, b, saved, dh, dx, dwx, dwh, db, ws=None,
                            stream=None):
    lib = load()
    if ws is None:
        ws = _temporary(pyramid_lstm2d_workspace_size(shape, 1), x.device, stream)
    _check("pyramid_lstm2d_backward", lib.pyramid_lstm2d_backward(
        ctypes.byref(shape), _ptr(x), _ptr(wx), _ptr(wh), _ptr(b), _ptr(saved), _ptr(dh),
        _ptr(dx), _ptr(dwx), _ptr(dwh), _ptr(db), _ptr(ws), ws.numel() * ws.element_size(),
        _stream(stream)))


def pyramid_fc_tanh_forward(x, w, b, y, stream=None):
    """x [M][Cin], w [Cout][Cin], b [Cout], y [M][Cout] (same dtype)."""
    M, Cin = x.shape
    Cout = w.shape[0]
    _check("pyramid_fc_tanh_forward", load().pyramid_fc_tanh_forward(
        M, Cin, Cout, _DT[x.dtype], _ptr(x), _ptr(w), _ptr(b), _ptr(y), _stream(stream)))


def pyramid_fc_workspace_size(M: int, Cin: int, Cout: int) -> int:
    return int(load().pyramid_fc_workspace_size(M, Cin, Cout))


def pyramid_fc_tanh_backward(x, w, y, dy, dx, dw, db, ws=None, stream=None):
    M, Cin = x.shape
    Cout = w.shape[0]
    if ws is None:
        ws = _temporary(pyramid_fc_workspace_size(M, Cin, Cout), x.device, stream)
    _check("pyramid_fc_tanh_backward", load().pyramid_fc_tanh_backward(
        M, Cin, Cout, _ptr(x), _ptr(w), _ptr(y), _ptr(dy), _ptr(dx), _ptr(dw), _ptr(db),
        _ptr(ws), ws.numel() * ws.element_size(), _stream(stream)))


def pyramid_softmax_ce(x, w, b, p, labels=None, loss=None, dx=None, dw=None, db=None, ws=None,
                       stream=None, squared=False):
    """Final linear + softmax (+ mean cross-entropy, or with `squared` the
    squared error of Eq. (14), and its gradient)."""
    M, Cin = x.shape
    K = w.shape[0]
    if labels is not None and ws is None:
        ws = _temporary(pyramid_fc_workspace_size(M, Cin, K), x.device, stream)
    name = "pyramid_softmax_sq" if squared else "pyramid_softmax_ce"
    _check(name, getattr(load(), name)(
        M, Cin, K, _DT[x.dtype], _ptr(x), _ptr(w), _ptr(b), _ptr(labels), _ptr(p), _ptr(loss),
        _ptr(dx), _ptr(dw), _ptr(db), _ptr(ws),
        0 if ws is None else ws.numel() * ws.element_size(), _stream(stream)))


def pyramid_softmax_sq(x, w, b, p, labels=None, loss=None, dx=None, dw=None, db=None, ws=None,
                       stream=None):
    """Final linear + softmax (+ the squared loss of Eq. (14) and its gradient)."""
    pyramid_softmax_ce(x, w, b, p, labels, loss, dx, dw, db, ws, stream, squared=True)


def pyramid_head_workspace_size(M: int, Cin: int, F: int, K: int) -> int:
    return int(load().pyramid_head_workspace_size(M, Cin, F, K))


def pyramid_head_train(x, w1, b1, w2, b2, labels, p, loss, dx, dw1, db1, dw2, db2, ws=None,
                       stream=None):
    """Fused FC tanh + linear + softmax + mean cross-entropy and their backward."""
    M, Cin = x.shape
    F, K = w1.shape[0], w2.shape[0]
    if ws is None:
        ws = _temporary(max(pyramid_head_workspace_size(M, Cin, F, K), 256), x.device, stream)
    _check("pyramid_head_train", load().pyramid_head_train(
        M, Cin, F, K, _ptr(x), _ptr(w1), _ptr(b1), _ptr(w2), _ptr(b2), _ptr(labels), _ptr(p),
        _ptr(loss), _ptr(dx), _ptr(dw1), _ptr(db1), _ptr(dw2), _ptr(db2), _ptr(ws),
        ws.numel() * ws.element_size(), _stream(stream)))


def pyramid_head_forward_supported(dtype, Cin: int, F: int, K: int) -> bool:
    return bool(load().pyramid_head_forward_supported(_DT[dtype], Cin, F, K))


def pyramid_head_forward(x, w1, b1, w2, b2, p, stream=None):
    """Fused FC tanh + linear + softmax for inference: x [M][Cin], w1 [F][Cin],
    b1 [F], w2 [K][F], b2 [K] (same dtype), p [M][K] fp32."""
    M, Cin = x.shape
    F, K = w1.shape[0], w2.shape[0]
    _check("pyramid_head_forward", load().pyramid_head_forward(
        M, Cin, F, K, _DT[x.dtype], _ptr(x), _ptr(w1), _ptr(b1), _ptr(w2), _ptr(b2), _ptr(p),
        _stream(stream)))


def pyramid_rmsprop_step(params, grads, ms, mom, lr, rho_ms=0.9, rho_m=0.9, eps=1e-5,
                         stream=None):
    """RMS-prop with momentum (Section 3, Eq. (15)-(18)) over lists of fp32
    device tensors, in place, in one launch."""
    n = len(params)
    if not (len(grads) == len(ms) == len(mom) == n):
        raise ValueError("params, grads, ms and mom must have the same length")
    segs = (plstm_param_segment * max(n, 1))()
    for k, (t, g, a, m) in enumerate(zip(params, grads, ms, mom)):
        for u in (t, g, a, m):
            if u.dtype != torch.float32 or u.numel() != t.numel():
                raise ValueError("fp32 tensors of one size per parameter expected")
        segs[k] = plstm_param_segment(_ptr(t), _ptr(g), _ptr(a), _ptr(m), t.numel())
    _check("pyramid_rmsprop_step", load().pyramid_rmsprop_step(
        n, segs, float(lr), float(rho_ms), float(rho_m), float(eps), _stream(stream)))


def pyramid_rmsprop_learning_rate(epoch: int) -> float:
    """1e-6 + 1e-2 (2^(-1/100))^epoch (Section 3, "Training")."""
    return load().pyramid_rmsprop_learning_rate(int(epoch))


class RMSprop:
    """Optimiser state (zero-initialised) for a fixed list of parameter
    tensors; `step(grads, epoch)` applies one update with the paper's
    hyper-parameters and learning-rate schedule."""

    def __init__(self, params):
        self.params = list(params)
        self.ms = [torch.zeros_like(p) for p in self.params]
        self.mom = [torch.zeros_like(p) for p in self.params]

    def step(self, grads, epoch: int, stream=None):
        pyramid_rmsprop_step(self.params, list(grads), self.ms, self.mom,
                             pyramid_rmsprop_learning_rate(epoch), stream=stream)


def pyramid_crop(x, n, box, tile, stream=None):
    """tile [d][h][w][C] = x[n, z0:z0+d, y0:y0+h, x0:x0+w, :]; box = (z0, y0,
    x0, d, h, w)."""
    N, D, H, W, C = x.shape
    if tile.dtype != x.dtype or tuple(tile.shape[-4:]) != (box[3], box[4], box[5], C):
        raise ValueError("tile must be [d][h][w][C] of x's dtype")
    _check("pyramid_crop", load().pyramid_crop(N, D, H, W, C, _DT[x.dtype], n, *box, _ptr(x),
                                               _ptr(tile), _stream(stream)))


def pyramid_sample_cubes(x, cubes, size, out, labels=None, out_labels=None, stream=None):
    """Training cubes out [count][d][h][w][C] (and out_labels [count][d][h][w])
    from x [N][D][H][W][C] (labels [N][D][H][W] int32); `cubes` is a sequence
    of plstm_cube (at most PLSTM_MAX_CUBES), `size` = (d, h, w)."""
    N, D, H, W, C = x.shape
    d, h, w = size
    count = len(cubes)
    if count < 1 or count > PLSTM_MAX_CUBES:
        raise ValueError("between 1 and %d cubes per call" % PLSTM_MAX_CUBES)
    if out.dtype != x.dtype or tuple(out.shape) != (count, d, h, w, C):
        raise ValueError("out must be [count][d][h][w][C] of x's dtype")
    if labels is not None:
        if labels.dtype != torch.int32 or out_labels is None or out_labels.dtype != torch.int32:
            raise ValueError("labels and out_labels must be int32")
        if tuple(out_labels.shape) != (count, d, h, w) or tuple(labels.shape) != (N, D, H, W):
            raise ValueError("labels [N][D][H][W], out_labels [count][d][h][w]")
    arr = (plstm_cube * count)(*cubes)
    _check("pyramid_sample_cubes", load().pyramid_sample_cubes(
        N, D, H, W, C, _DT[x.dtype], count, arr, d, h, w, _ptr(x), _ptr(labels), _ptr(out),
        _ptr(out_labels), _stream(stream)))


def draw_cubes(rng, N, volume, size, count, rotate=True, flip_axes="zyx"):
    """Random training cubes (host side): a uniform batch element and corner
    among the boxes of `size` = (d, h, w) inside `volume` = (D, H, W); with
    `rotate` an angle uniform in [0, 2 pi) about z; each axis named in
    `flip_axes` flipped with probability 1/2.  The EM recipe is the default;
    the MR recipe is rotate=False, flip_axes="x".  `rng` is a
    numpy.random.Generator."""
    import math
    D, H, W = volume
    d, h, w = size
    bits = {"z": PLSTM_FLIP_Z, "y": PLSTM_FLIP_Y, "x": PLSTM_FLIP_X}
    out = []
    for _ in range(count):
        n = int(rng.integers(0, N))
        z0, y0, x0 = (int(rng.integers(0, E - e + 1)) for E, e in ((D, d), (H, h), (W, w)))
        theta = float(rng.uniform(0.0, 2.0 * math.pi)) if rotate else 0.0
        flips = 0
        for a in flip_axes:
            if rng.random() < 0.5:
                flips |= bits[a]
        out.append(plstm_cube(n, z0, y0, x0, math.cos(theta), math.sin(theta), flips))
    return out


def pyramid_stitch_clear(acc, wsum, stream=None):
    D, H, W, K = acc.shape
    _check("pyramid_stitch_clear", load().pyramid_stitch_clear(D, H, W, K, _ptr(acc),
                                                               _ptr(wsum), _stream(stream)))


def pyramid_stitch_add(p, box, acc, wsum, sigma_scale=0.25, stream=None):
    """acc += g p, wsum += g for the tile p [d][h][w][K] at box (z0, y0, x0, d,
    h, w) with Gaussian weights g."""
    D, H, W, K = acc.shape
    _check("pyramid_stitch_add", load().pyramid_stitch_add(
        D, H, W, K, *box, float(sigma_scale), _ptr(p), _ptr(acc), _ptr(wsum), _stream(stream)))


def pyramid_stitch_finish(acc, wsum, out, stream=None):
    D, H, W, K = acc.shape
    _check("pyramid_stitch_finish", load().pyramid_stitch_finish(
        D, H, W, K, _ptr(acc), _ptr(wsum), _ptr(out), _stream(stream)))


# The operators below run down to a few microseconds, so their marshalling keeps
# to plain integers: data_ptr(), device numbers and the raw stream instead of ctypes
# and torch objects, and no device switch where the tensors' device is current.
def _main(name, t, dims):
    """Storage type code, pointer and device number of an operator's main tensor of
    `dims` dimensions (None: any)."""
    if not isinstance(t, torch.Tensor):
        raise TypeError("expected a torch.Tensor, got %r" % type(t))
    code = _DT.get(t.dtype)
    if code is None or dims not in (None, t.dim()):
        raise ValueError("%s must be float32 or bfloat16%s" % (
            name, "" if dims is None else " with %d dimensions" % dims))
    if not t.is_cuda:
        raise ValueError("%s must live on the GPU" % name)
    if not t.is_contiguous():
        raise ValueError("%s must be contiguous" % name)
    return code, t.data_ptr(), t.get_device()


def _torch_tensor(t):
    if not isinstance(t, torch.Tensor):
        raise TypeError("expected a torch.Tensor, got %r" % type(t))
    return t


def _tensor(name, t, shape, dtype, dev):
    """Pointer of a tensor that has to have this shape, type and device (None: NULL)."""
    if t is None:
        return None
    try:
        # a host tensor's device number is -1
        if t.shape == shape and t.dtype == dtype and t.get_device() == dev and t.is_contiguous():
            return t.data_ptr()
    except (AttributeError, TypeError):     # an array of another library: its type is not comparable
        pass
    _torch_tensor(t)
    raise ValueError("%s must be %s %s on cuda:%d and contiguous, got %s %s on %s%s" % (
        name, dtype, list(shape), dev, t.dtype, list(t.shape), t.device,
        "" if t.is_contiguous() else ", not contiguous"))


def _bytes(ws, dev):
    if not ws.is_cuda or ws.get_device() != dev or not ws.is_contiguous():
        raise ValueError("ws must be contiguous and on cuda:%d" % dev)
    return ws.data_ptr(), ws.numel() * ws.element_size()


def _codes(name, q, scale, x, dev):
    """Pointers of an 8-bit checkpoint of a tensor of x's shape."""
    return (_tensor(name, q, x.shape, torch.int8, dev),
            _tensor(name + "'s scale", scale, (-(-x.numel() // 64),), torch.bfloat16, dev))


def _run(name, dev, stream, *args):
    """Calls entry point `name` with device `dev` current, on `stream` or that
    device's current stream."""
    fn = getattr(_lib or load(), name)
    if stream is None:
        stream = torch._C._cuda_getCurrentRawStream(dev)
    else:
        stream = _stream(stream)
    if dev == torch._C._cuda_getDevice():
        rc = fn(*args, stream)
    else:
        with torch.cuda.device(dev):
            rc = fn(*args, stream)
    if rc:
        raise PyramidLSTMError(name, rc)


def pyramid_layer_norm_workspace_size(M: int, C: int) -> int:
    return int(load().pyramid_layer_norm_workspace_size(M, C))


def pyramid_layer_norm_forward(x, gamma, beta, y, stats=None, xq=None, xscale=None, eps=1e-5,
                               stream=None):
    """Layer norm of the rows of x [M][C] (gamma, beta [C], y [M][C], one
    dtype).  stats [M][2] fp32 takes each row's (mean, rstd) for the backward;
    xq, xscale (see checkpoint8_empty) take x's 8-bit checkpoint."""
    dt, px, dev = _main("x", x, 2)
    M, C = x.shape
    if (xq is None) != (xscale is None):
        raise ValueError("xq and xscale go together")
    q, qs = _codes("xq", xq, xscale, x, dev) if xq is not None else (None, None)
    _run("pyramid_layer_norm_forward", dev, stream, M, C, dt, eps, px,
         _tensor("gamma", gamma, (C,), x.dtype, dev), _tensor("beta", beta, (C,), x.dtype, dev),
         _tensor("y", y, x.shape, x.dtype, dev), _tensor("stats", stats, (M, 2), torch.float32, dev),
         q, qs)


def pyramid_layer_norm_backward(x, gamma, stats, dy, dx, dgamma, dbeta, xscale=None, ws=None,
                                stream=None):
    """Gradients of pyramid_layer_norm_forward: dx [M][C] (or None), dgamma and
    dbeta [C] fp32, from dy [M][C] and the forward's input x, or its codes x
    with their scales xscale."""
    dt, pdy, dev = _main("dy", dy, 2)
    M, C = dy.shape
    if xscale is None:
        px, ps = _tensor("x", x, dy.shape, dy.dtype, dev), None
    else:
        px, ps = _codes("x", x, xscale, dy, dev)
    if ws is None:
        ws = _temporary(pyramid_layer_norm_workspace_size(M, C), dy.device, stream)
    _run("pyramid_layer_norm_backward", dev, stream, M, C, dt, px, ps,
         _tensor("gamma", gamma, (C,), dy.dtype, dev),
         _tensor("stats", stats, (M, 2), torch.float32, dev), pdy,
         _tensor("dx", dx, dy.shape, dy.dtype, dev),
         _tensor("dgamma", dgamma, (C,), torch.float32, dev),
         _tensor("dbeta", dbeta, (C,), torch.float32, dev), *_bytes(ws, dev))


@functools.lru_cache(maxsize=256)
def pyramid_scan_workspace_size(B: int, T: int, I: int) -> int:
    return int(load().pyramid_scan_workspace_size(B, T, I))


@functools.lru_cache(maxsize=256)
def pyramid_scan_saved_size(B: int, T: int, I: int) -> int:
    return int(load().pyramid_scan_saved_size(B, T, I))


def _saved(saved, B, T, I, dev):
    if saved is None:
        return None
    if not saved.is_cuda or saved.get_device() != dev or not saved.is_contiguous() or \
            saved.numel() * saved.element_size() < pyramid_scan_saved_size(B, T, I):
        raise ValueError("saved must hold pyramid_scan_saved_size bytes on cuda:%d" % dev)
    return saved.data_ptr()


_scan_ws = {}


def _shared_ws(x, dev):
    """256 bytes that calls which need no workspace share, as _scan_workspace gives one: they do
    not touch them."""
    shared = _scan_ws.get(dev)
    if shared is None:
        ws = _workspace(256, x.device)
        shared = _scan_ws[dev] = (ws,) + _bytes(ws, dev)
    return shared


def _scan_workspace(ws, x, dev, stream):
    """`ws`, or one made with torch, its pointer and its bytes.  A call that
    needs none takes 256 bytes as every call does, and shares them: it does not
    touch them."""
    if ws is None:
        need = pyramid_scan_workspace_size(*x.shape)
        if need <= 256:
            return _shared_ws(x, dev)
        ws = _temporary(need, x.device, stream)
    return (ws,) + _bytes(ws, dev)


def pyramid_scan_forward(g, u, h, reverse=False, lengths=None, h0=None, hT=None, saved=None,
                         ws=None, stream=None):
    """Gated linear recurrence along axis 1 of g, u [B][T][I] into h (same
    shape and dtype): f = sigmoid(g_t), h_t = f h_{t-1} + (1 - f) u_t, from the
    last step with `reverse`.  lengths [B] int32 gives each sequence its own
    number of steps; h0, hT [B][I] fp32 are the state before and after (hT may
    be h0); saved (pyramid_scan_saved_size bytes) keeps what the backward
    needs.  ws=None allocates the workspace with torch."""
    dt, pg, dev = _main("g", g, 3)
    B, T, I = g.shape
    ws, pws, nws = _scan_workspace(ws, g, dev, stream)
    _run("pyramid_scan_forward", dev, stream, B, T, I, dt, int(bool(reverse)), pg,
         _tensor("u", u, g.shape, g.dtype, dev), _tensor("lengths", lengths, (B,), torch.int32, dev),
         _tensor("h0", h0, (B, I), torch.float32, dev), _tensor("h", h, g.shape, g.dtype, dev),
         _tensor("hT", hT, (B, I), torch.float32, dev), _saved(saved, B, T, I, dev), pws, nws)


def pyramid_scan_backward(g, u, saved, dh, dg, du, reverse=False, lengths=None, dhT=None, dh0=None,
                          gscale=None, uscale=None, ws=None, stream=None):
    """Gradients of pyramid_scan_forward: dg, du [B][T][I] and dh0 [B][I] fp32
    (or None) from dh, dhT (or None) and the forward's inputs and saved
    buffer; g and u may be codes with their scales gscale and uscale."""
    dt, pdh, dev = _main("dh", dh, 3)
    B, T, I = dh.shape
    if (gscale is None) != (uscale is None):
        raise ValueError("g and u are both coded or neither")
    if gscale is None:
        pg, pgs = _tensor("g", g, dh.shape, dh.dtype, dev), None
        pu, pus = _tensor("u", u, dh.shape, dh.dtype, dev), None
    else:
        pg, pgs = _codes("g", g, gscale, dh, dev)
        pu, pus = _codes("u", u, uscale, dh, dev)
    ws, pws, nws = _scan_workspace(ws, dh, dev, stream)
    _run("pyramid_scan_backward", dev, stream, B, T, I, dt, int(bool(reverse)), pg, pgs, pu, pus,
         _tensor("lengths", lengths, (B,), torch.int32, dev), _saved(saved, B, T, I, dev),
         pdh, _tensor("dhT", dhT, (B, I), torch.float32, dev),
         _tensor("dg", dg, dh.shape, dh.dtype, dev), _tensor("du", du, dh.shape, dh.dtype, dev),
         _tensor("dh0", dh0, (B, I), torch.float32, dev), pws, nws)


def pyramid_checkpoint8_scales(n: int) -> int:
    return int(load().pyramid_checkpoint8_scales(n))


def checkpoint8_empty(x):
    """Uninitialised 8-bit checkpoint of a tensor like x: (codes of x's shape
    int8, scales bf16, one per 64 elements)."""
    return (torch.empty_like(x, dtype=torch.int8, memory_format=torch.contiguous_format),
            torch.empty(-(-x.numel() // 64), dtype=torch.bfloat16, device=x.device))


def pyramid_checkpoint8_pack(x, q, scale, stream=None):
    """Codes q (x's shape, int8) and scales of x (float32 or bfloat16, any shape)."""
    dt, px, dev = _main("x", x, None)
    pq, ps = _codes("q", q, scale, x, dev)
    _run("pyramid_checkpoint8_pack", dev, stream, x.numel(), dt, px, pq, ps)


def pyramid_checkpoint8_unpack(q, scale, x, stream=None):
    """x (float32 or bfloat16, q's shape) = the values of a checkpoint."""
    dt, px, dev = _main("x", x, None)
    pq, ps = _codes("q", q, scale, x, dev)
    _run("pyramid_checkpoint8_unpack", dev, stream, x.numel(), dt, pq, ps, px)


_ACT = {"none": 0, "silu": 1}


def _act(act):
    if act not in _ACT:
        raise ValueError("act must be one of %s" % ", ".join(_ACT))
    return _ACT[act]


def _pitched(name, t, shape, dtype, dev):
    """Pointer and pitch of an input [B][T][n] that may be a slice of wider rows: the
    elements of a row next to each other, rows (b, t) at (b T + t) pitch (0: dense)."""
    if t is None:
        return None, 0
    _torch_tensor(t)
    if t.shape != shape or t.dtype != dtype or t.get_device() != dev:
        raise ValueError("%s must be %s %s on cuda:%d, got %s %s on %s" % (
            name, dtype, list(shape), dev, t.dtype, list(t.shape), t.device))
    if t.is_contiguous():
        return t.data_ptr(), 0
    sb, st, sn = t.stride()
    B, T, n = shape
    pitch = st if T > 1 else sb if B > 1 else n
    if (n > 1 and sn != 1) or pitch < n or (B > 1 and sb != T * pitch):
        raise ValueError("%s must be contiguous or a slice of contiguous rows, got strides %s" % (
            name, (sb, st, sn)))
    return t.data_ptr(), pitch


def _main_pitched(name, t):
    """Storage type code, device number, pointer and pitch of a main input [B][T][n] that may
    be a slice of wider rows."""
    if not isinstance(t, torch.Tensor):
        raise TypeError("expected a torch.Tensor, got %r" % type(t))
    code = _DT.get(t.dtype)
    if code is None or t.dim() != 3:
        raise ValueError("%s must be float32 or bfloat16 with 3 dimensions" % name)
    dev = t.get_device()
    if dev < 0:
        raise ValueError("%s must live on the GPU" % name)
    if t.is_contiguous():
        return code, dev, t.data_ptr(), 0
    return (code, dev) + _pitched(name, t, t.shape, t.dtype, dev)


@functools.lru_cache(maxsize=256)
def pyramid_causal_conv_workspace_size(B: int, T: int, I: int, K: int) -> int:
    return int(load().pyramid_causal_conv_workspace_size(B, T, I, K))


def pyramid_causal_conv_forward(x, w, bias, y, act="none", reverse=False, lengths=None, state=None,
                                state_out=None, stream=None):
    """Short causal convolution along axis 1 of x [B][T][I] (contiguous, or a slice of
    wider rows) into y [B][T][I]: w [I][K], bias [I] or None, one dtype; act "none" or
    "silu".  state, state_out [B][K-1][I] of that dtype are the last inputs
    before and after (state_out may be state); lengths, reverse as in
    pyramid_scan_forward."""
    dt, dev, px, pitch = _main_pitched("x", x)
    B, T, I = x.shape
    K = w.shape[-1] if _torch_tensor(w).dim() == 2 else 0
    _run("pyramid_causal_conv_forward", dev, stream, B, T, I, K, dt, _act(act), int(bool(reverse)),
         px, pitch, _tensor("w", w, (I, K), x.dtype, dev), _tensor("bias", bias, (I,), x.dtype, dev),
         _tensor("lengths", lengths, (B,), torch.int32, dev),
         _tensor("state", state, (B, K - 1, I), x.dtype, dev) or None,
         _tensor("y", y, x.shape, x.dtype, dev),
         _tensor("state_out", state_out, (B, K - 1, I), x.dtype, dev) or None)


def pyramid_causal_conv_backward(x, w, bias, dy, dx, dw, db, act="none", reverse=False, lengths=None,
                                 state=None, dstate_out=None, dstate=None, ws=None, stream=None):
    """Gradients of pyramid_causal_conv_forward: dx [B][T][I], dw [I][K] and db [I] (or None) fp32,
    dstate [B][K-1][I] fp32 (or None), from dy, dstate_out fp32 (or None) and the
    forward's inputs."""
    dt, dev, px, pitch = _main_pitched("x", x)
    B, T, I = x.shape
    K = w.shape[-1] if _torch_tensor(w).dim() == 2 else 0
    if ws is None:
        ws = _temporary(pyramid_causal_conv_workspace_size(B, T, I, K), x.device, stream)
    _run("pyramid_causal_conv_backward", dev, stream, B, T, I, K, dt, _act(act), int(bool(reverse)),
         px, pitch, _tensor("w", w, (I, K), x.dtype, dev), _tensor("bias", bias, (I,), x.dtype, dev),
         _tensor("lengths", lengths, (B,), torch.int32, dev),
         _tensor("state", state, (B, K - 1, I), x.dtype, dev) or None,
         _tensor("dy", dy, x.shape, x.dtype, dev),
         _tensor("dstate_out", dstate_out, (B, K - 1, I), torch.float32, dev) or None,
         _tensor("dx", dx, x.shape, x.dtype, dev), _tensor("dw", dw, (I, K), torch.float32, dev),
         _tensor("db", db, (I,), torch.float32, dev),
         _tensor("dstate", dstate, (B, K - 1, I), torch.float32, dev) or None, *_bytes(ws, dev))


@functools.lru_cache(maxsize=256)
def pyramid_selective_scan_workspace_size(B: int, T: int, I: int, S: int, backward: int = 0) -> int:
    return int(load().pyramid_selective_scan_workspace_size(B, T, I, S, int(backward)))


@functools.lru_cache(maxsize=256)
def pyramid_selective_scan_saved_size(B: int, T: int, I: int, S: int) -> int:
    return int(load().pyramid_selective_scan_saved_size(B, T, I, S))


def _select_saved(saved, B, T, I, S, dev):
    if saved is None:
        return None
    if not saved.is_cuda or saved.get_device() != dev or not saved.is_contiguous() or \
            saved.numel() * saved.element_size() < pyramid_selective_scan_saved_size(B, T, I, S):
        raise ValueError("saved must hold pyramid_selective_scan_saved_size bytes on cuda:%d" % dev)
    return saved.data_ptr()


def _select_inputs(u, delta, A, Bm, Cm, D, z, delta_bias, softplus, reverse, lengths):
    """The device and the arguments of a selective scan call up to its lengths."""
    dt, dev, pu, lu = _main_pitched("u", u)
    shape, dtype, f32 = u.shape, u.dtype, torch.float32
    B, T, I = shape
    S = A.shape[-1] if _torch_tensor(A).dim() == 2 else 0
    pd, ld = _pitched("delta", delta, shape, dtype, dev)
    pB, lB = _pitched("Bm", Bm, (B, T, S), dtype, dev)
    pC, lC = _pitched("Cm", Cm, (B, T, S), dtype, dev)
    pz, lz = _pitched("z", z, shape, dtype, dev)
    return dev, (B, T, I, S, dt, 1 if reverse else 0, 1 if softplus else 0, pu, lu, pd, ld,
                 _tensor("A", A, (I, S), f32, dev), pB, lB, pC, lC, _tensor("D", D, (I,), f32, dev),
                 pz, lz, _tensor("delta_bias", delta_bias, (I,), f32, dev),
                 _tensor("lengths", lengths, (B,), torch.int32, dev))


def pyramid_selective_scan_forward(u, delta, A, Bm, Cm, y, D=None, z=None, delta_bias=None,
                                   softplus=False, reverse=False, lengths=None, h0=None, hT=None,
                                   saved=None, ws=None, stream=None):
    """Selective state space scan along axis 1 of u [B][T][I] into y (its shape and
    dtype): with d = delta + delta_bias (softplus of it, if asked), per channel i and
    state k: h = exp(d A[i][k]) h + d u Bm[t][k], y = sum_k Cm[t][k] h + D[i] u, times
    z sigmoid(z) with z.  delta, z [B][T][I], Bm, Cm [B][T][S] have u's dtype; u, delta, z, Bm and
    Cm may be slices of wider rows; A [I][S], D, delta_bias [I] are fp32.  lengths and
    reverse as in pyramid_scan_forward; h0, hT [B][I][S] fp32 are the state before and
    after (hT may be h0); saved (pyramid_selective_scan_saved_size bytes) keeps what
    the backward needs."""
    dev, args = _select_inputs(u, delta, A, Bm, Cm, D, z, delta_bias, softplus, reverse, lengths)
    B, T, I, S = args[:4]
    if ws is None:
        need = pyramid_selective_scan_workspace_size(B, T, I, S)
        ws = None if need <= 256 else _temporary(need, u.device, stream)
    _run("pyramid_selective_scan_forward", dev, stream, *args,
         _tensor("h0", h0, (B, I, S), torch.float32, dev), _tensor("y", y, u.shape, u.dtype, dev),
         _tensor("hT", hT, (B, I, S), torch.float32, dev), _select_saved(saved, B, T, I, S, dev),
         *(_shared_ws(u, dev)[1:] if ws is None else _bytes(ws, dev)))


def pyramid_selective_scan_backward(u, delta, A, Bm, Cm, saved, dy, du, ddelta, dA, dB, dC, D=None,
                                    z=None, delta_bias=None, softplus=False, dD=None, dz=None,
                                    ddelta_bias=None, reverse=False, lengths=None, dhT=None, dh0=None,
                                    ws=None, stream=None):
    """Gradients of pyramid_selective_scan_forward: du, ddelta (dz, with z) [B][T][I] and
    dB, dC [B][T][S] in u's dtype; dA [I][S], dD and ddelta_bias [I] (or None), dh0 [B][I][S]
    (or None) in fp32, from dy, dhT (or None) and the forward's inputs and saved buffer."""
    dev, args = _select_inputs(u, delta, A, Bm, Cm, D, z, delta_bias, softplus, reverse, lengths)
    B, T, I, S = args[:4]
    if ws is None:
        ws = _temporary(pyramid_selective_scan_workspace_size(B, T, I, S, 1), u.device, stream)
    f32 = torch.float32
    _run("pyramid_selective_scan_backward", dev, stream, *args, _select_saved(saved, B, T, I, S, dev),
         _tensor("dy", dy, u.shape, u.dtype, dev), _tensor("dhT", dhT, (B, I, S), f32, dev),
         _tensor("du", du, u.shape, u.dtype, dev), _tensor("ddelta", ddelta, u.shape, u.dtype, dev),
         _tensor("dA", dA, (I, S), f32, dev), _tensor("dB", dB, (B, T, S), u.dtype, dev),
         _tensor("dC", dC, (B, T, S), u.dtype, dev), _tensor("dD", dD, (I,), f32, dev),
         _tensor("dz", dz, u.shape, u.dtype, dev), _tensor("ddelta_bias", ddelta_bias, (I,), f32, dev),
         _tensor("dh0", dh0, (B, I, S), f32, dev), *_bytes(ws, dev))


@functools.lru_cache(maxsize=256)
def pyramid_group_norm_workspace_size(N: int, V: int, C: int, G: int) -> int:
    return int(load().pyramid_group_norm_workspace_size(N, V, C, G))


def _volumes(name, x):
    """Type code, pointer, device, N, V and C of x [N][...][C]."""
    dt, px, dev = _main(name, x, None)
    if x.dim() < 2:
        raise ValueError("%s must be [N][...][C]" % name)
    N, C = x.shape[0], x.shape[-1]
    return dt, px, dev, N, x.numel() // max(N * C, 1), C


def _group_norm_ws(ws, N, V, C, G, x, dev, stream):
    """`ws`, or one made with torch (the caller holds it until its call is under way), its pointer and its bytes."""
    if ws is None:
        need = pyramid_group_norm_workspace_size(N, V, C, G)
        if need <= 256:
            return _shared_ws(x, dev)
        ws = _temporary(need, x.device, stream)
        return ws, ws.data_ptr(), need
    return (ws,) + _bytes(ws, dev)


def pyramid_group_norm_forward(x, gamma, beta, y, groups, act="none", stats=None, eps=1e-5, ws=None,
                               stream=None):
    """Group norm over the voxels and C / groups consecutive channels of each volume of x
    [N][...][C], times gamma plus beta [C], act ("none" or "silu") of it into y; one dtype.
    stats [N][groups][2] fp32 takes (mean, rstd) for the backward."""
    dt, px, dev, N, V, C = _volumes("x", x)
    ws, pw, bw = _group_norm_ws(ws, N, V, C, groups, x, dev, stream)
    _run("pyramid_group_norm_forward", dev, stream, N, V, C, groups, dt, _act(act), eps, px,
         _tensor("gamma", gamma, (C,), x.dtype, dev), _tensor("beta", beta, (C,), x.dtype, dev),
         _tensor("y", y, x.shape, x.dtype, dev),
         _tensor("stats", stats, (N, groups, 2), torch.float32, dev),
         pw, bw)


def pyramid_group_norm_backward(x, gamma, beta, stats, dy, dx, dgamma, dbeta, groups, act="none",
                                ws=None, stream=None):
    """Gradients of pyramid_group_norm_forward: dx (or None) of x's shape, dgamma and dbeta [C]
    fp32, from dy, the forward's inputs and its stats."""
    dt, px, dev, N, V, C = _volumes("x", x)
    ws, pw, bw = _group_norm_ws(ws, N, V, C, groups, x, dev, stream)
    _run("pyramid_group_norm_backward", dev, stream, N, V, C, groups, dt, _act(act), px,
         _tensor("gamma", gamma, (C,), x.dtype, dev), _tensor("beta", beta, (C,), x.dtype, dev),
         _tensor("stats", stats, (N, groups, 2), torch.float32, dev),
         _tensor("dy", dy, x.shape, x.dtype, dev), _tensor("dx", dx, x.shape, x.dtype, dev),
         _tensor("dgamma", dgamma, (C,), torch.float32, dev),
         _tensor("dbeta", dbeta, (C,), torch.float32, dev),
         pw, bw)


def pyramid_adamw_scales(n: int) -> int:
    return int(load().pyramid_adamw_scales(n))


_data_ptr = torch.Tensor.data_ptr


def _adamw_segments(params, m, v, mscale, vscale, copies, weight_decay):
    """Segments of an AdamW call without its gradients, the bits of its moments and its device."""
    count = len(params)
    if count < 1 or not len(m) == len(v) == count or (copies is not None and len(copies) != count):
        raise ValueError("params, m, v (and copies) must have the same length, at least 1")
    if _torch_tensor(m[0]).dtype not in (torch.float32, torch.uint8):
        raise ValueError("moments must be float32 or (8-bit codes) uint8")
    bits = 32 if m[0].dtype == torch.float32 else 8
    if bits == 8 and (mscale is None or vscale is None or not len(mscale) == len(vscale) == count):
        raise ValueError("8-bit moments need mscale and vscale, one tensor per parameter")
    decay = weight_decay if isinstance(weight_decay, (list, tuple)) else [weight_decay] * count
    if len(decay) != count:
        raise ValueError("one weight decay, or one per parameter")
    segs = (plstm_adamw_segment * count)()
    f32 = torch.float32
    for k, p in enumerate(params):
        dt, pp, dev = _main("params", p, None)
        if dt != PLSTM_F32 or (k and dev != dev0):
            raise ValueError("parameters must be float32 on one device")
        dev0 = dev
        n = p.numel()
        segs[k].theta, segs[k].n, segs[k].weight_decay = pp, n, float(decay[k])
        segs[k].m = _tensor("m", m[k], p.shape, m[0].dtype, dev)
        segs[k].v = _tensor("v", v[k], p.shape, m[0].dtype, dev)
        if bits == 8:
            segs[k].mscale = _tensor("mscale", mscale[k], (-(-n // 256),), f32, dev)
            segs[k].vscale = _tensor("vscale", vscale[k], (-(-n // 256),), f32, dev)
        if copies is not None:
            segs[k].copy = _tensor("copies", copies[k], p.shape, torch.bfloat16, dev)
    _apart([(at, n * e) for s in segs for at, n, e in (
        (s.theta, s.n, 4), (s.m, s.n, bits // 8), (s.v, s.n, bits // 8), (s.copy, s.n, 2),
        (s.mscale, -(-s.n // 256), 4), (s.vscale, -(-s.n // 256), 4))])
    return segs, bits, dev0


def _apart(places):
    """Refuses memory (address and bytes) that is written under two names: lanes would race for it."""
    places = sorted((at, at + n) for at, n in places if at and n)
    if any(a[1] > b[0] for a, b in zip(places, places[1:])):
        raise ValueError("parameters, moments, scales and copies must not overlap (is one given twice?)")


def _adamw_grads(segs, shapes, grads, dev):
    """Puts the gradients into the segments (None: the tensor is left alone); their type."""
    if len(grads) != len(shapes):
        raise ValueError("one gradient (or None) per parameter")
    dtype = None
    try:
        for seg, shape, g in zip(segs, shapes, grads):
            if g is None:
                seg.n = 0
                continue
            if dtype is None:
                dtype = g.dtype
                if dtype not in _DT:
                    raise ValueError("gradients must be float32 or bfloat16")
            # _tensor's questions without its call (12 tensors 1 us of 13)
            if g.shape == shape and g.dtype == dtype and g.get_device() == dev and g.is_contiguous():
                seg.grad = g.data_ptr()
            else:
                seg.grad = _tensor("grads", g, shape, dtype, dev)
            if not seg.n:               # left alone before
                seg.n = shape.numel()
    except (AttributeError, TypeError, ValueError):
        _torch_tensor(g)
        raise
    return PLSTM_F32 if dtype is None else _DT[dtype]


def _adamw_run(segs, bits, grad_dtype, dev, stream, lr, betas, eps, step, seed, clock, grad_scale):
    lr_dev = None
    if isinstance(lr, torch.Tensor):
        lr, lr_dev = 0.0, _tensor("lr", lr, (1,), torch.float32, dev)
    _run("pyramid_adamw_step", dev, stream, len(segs), segs, bits, grad_dtype, lr, betas[0], betas[1],
         eps, step, seed & 0xffffffff, None if clock is None else _tensor("clock", clock, (3,), torch.int64, dev), lr_dev,
         None if grad_scale is None else _tensor("grad_scale", grad_scale, (1,), torch.float32, dev))


def pyramid_adamw_step(params, grads, m, v, lr, step, betas=(0.9, 0.999), eps=1e-8, weight_decay=0.01,
                       mscale=None, vscale=None, copies=None, seed=0, clock=None, grad_scale=None,
                       stream=None):
    """AdamW update number `step` (from 1, the same for all tensors) over lists of device tensors, in
    place: params fp32, grads fp32 or bf16 (None: that tensor is left alone), m and v fp32, or uint8 codes with their
    scales mscale and vscale (fp32, one per 256 elements, pyramid_adamw_scales).  copies: bf16
    tensors that take the updated parameters.  weight_decay: a number, or one per tensor.  lr: a
    number, or fp32 [1] on the device; grad_scale: None, or such a factor of the gradients.  clock:
    None, or int64 [3] on the device whose first element counts the updates (`step` is then
    ignored), for steps in captured graphs.  seed: of the rounding of 8-bit moments."""
    segs, bits, dev = _adamw_segments(params, m, v, mscale, vscale, copies, weight_decay)
    dtype = _adamw_grads(segs, [p.shape for p in params], grads, dev)
    _adamw_run(segs, bits, dtype, dev, stream, lr, betas, eps, step, seed, clock, grad_scale)


def pyramid_adamw_moments(m, v, mscale, vscale, mout, vout, stream=None):
    """fp32 values mout, vout of lists of 8-bit moments m, v with their scales."""
    segs, bits, dev = _adamw_segments(mout, m, v, mscale, vscale, None, 0.0)
    if bits != 8:
        raise ValueError("m and v must be 8-bit codes")
    count = len(mout)
    if len(vout) != count:
        raise ValueError("mout and vout must have the same length")
    pm, pv = (ctypes.c_void_p * count)(), (ctypes.c_void_p * count)()
    for k in range(count):
        pm[k] = segs[k].theta
        pv[k] = _tensor("vout", vout[k], mout[k].shape, torch.float32, dev)
    _apart([(at, 4 * s.n) for k, s in enumerate(segs) for at in (pm[k], pv[k])])
    _run("pyramid_adamw_moments", dev, stream, count, segs, pm, pv)


class AdamW:
    """AdamW for a fixed list of fp32 parameter tensors, beside RMSprop; moments in 32
    bits or in 8 (`bits`), zero at first or taken from `state` (what state() gives).
    copies: bf16 tensors (or None each) that take the updated parameters.
    weight_decay: a number or one per tensor.  capturable=True keeps the number of updates on
    the device, so that a step captured in a graph goes on counting when it is replayed.
    The count is one for all parameters: a first gradient after many updates without one moves its
    parameter by (1 - beta1) / sqrt(1 - beta2) times lr, as its moments are corrected for that many.
    An update works on the memory that params and copies have when it is called (a captured one on
    that of its capture).  The moments' memory, m and v (with 8 bits their codes, and the scales mscale and
    vscale), is the optimiser's from first to last: to go on from others, give them as `state`."""

    def __init__(self, params, lr=1e-3, betas=(0.9, 0.999), eps=1e-8, weight_decay=0.01, bits=32,
                 copies=None, seed=0, state=None, capturable=False):
        if bits not in (8, 32):
            raise ValueError("bits must be 8 or 32")
        self.params = list(params)
        self.lr, self.betas, self.eps, self.seed, self.bits = lr, betas, eps, seed, bits
        self.copies = None if copies is None else list(copies)
        ms = vs = None
        if state is None:
            dt = torch.float32 if bits == 32 else torch.uint8
            m, v = ([torch.zeros_like(p, dtype=dt, memory_format=torch.contiguous_format)
                     for p in self.params] for _ in range(2))
            if bits == 8:
                ms, vs = ([torch.zeros(-(-p.numel() // 256), device=p.device)
                           for p in self.params] for _ in range(2))
            t = 0
        else:
            m, v, t = state["m"], state["v"], int(state["t"])
            if bits == 8:
                ms, vs = state["mscale"], state["vscale"]
        # tensors of its own over their memory: a caller's may be given other memory
        self._m, self._v, self._ms, self._vs = (None if ts is None else [t.detach() for t in ts] for ts in (m, v, ms, vs))
        self._shown = {}
        self._decay = list(weight_decay) if isinstance(weight_decay, (list, tuple)) else weight_decay
        self._renew()
        self._t, self._clock = t, None
        if capturable:
            self._clock = torch.tensor([t, 0, 0], dtype=torch.int64, device=self.params[0].device)

    def _addresses(self):
        """Where the caller's tensors are that an update writes (0: a copy that is None)."""
        at = list(map(_data_ptr, self.params))
        if self.copies is not None:
            at += [0 if c is None else c.data_ptr() for c in self.copies]
        return at

    def _renew(self):
        """Segments of the tensors that are there now."""
        segs, bits, dev = _adamw_segments(self.params, self._m, self._v, self._ms, self._vs, self.copies, self._decay)
        if bits != self.bits:
            raise ValueError("state has moments in %d bits" % bits)
        self._segs, self._rows, self._dev = segs, list(segs), dev
        self._shapes, self._at = [p.shape for p in self.params], self._addresses()

    def _show(self, name):
        """Tensors for others over the moments or scales: new ones where one of them was given other memory."""
        shown = self._shown.get(name)
        if shown is None or list(map(_data_ptr, shown[0])) != shown[1]:
            held = getattr(self, name)
            if held is None:
                return None
            shown = self._shown[name] = tuple(t.detach() for t in held), list(map(_data_ptr, held))
        return shown[0]

    m = property(lambda self: self._show("_m"))
    v = property(lambda self: self._show("_v"))
    mscale = property(lambda self: self._show("_ms"))
    vscale = property(lambda self: self._show("_vs"))

    @property
    def t(self):
        """Updates so far (capturable: read from the device)."""
        return self._t if self._clock is None else int(self._clock[0])

    def state(self):
        """The moments, their scales and the number of updates: tensors of the memory itself."""
        out = {"m": list(self.m), "v": list(self.v), "t": self.t}
        if self.bits == 8:
            out.update(mscale=list(self.mscale), vscale=list(self.vscale))
        return out

    def step(self, grads, lr=None, grad_scale=None, stream=None):
        """One update from `grads` (one per parameter, None to leave it alone); lr and
        grad_scale as in pyramid_adamw_step."""
        if self._addresses() != self._at:       # a tensor was given other memory, or replaced
            self._renew()
        dtype = _adamw_grads(self._rows, self._shapes, list(grads), self._dev)
        _adamw_run(self._segs, self.bits, dtype, self._dev, stream, self.lr if lr is None else lr,
                   self.betas, self.eps, self._t + 1, self.seed, self._clock, grad_scale)
        self._t += 1

    def moments(self, stream=None):
        """fp32 (m, v) of each parameter: the moments themselves, or what their codes stand for."""
        if self.bits == 32:
            return list(zip(self._show("_m"), self._show("_v")))
        caller = torch.cuda.current_stream(self._dev)
        side = caller if stream is None else _torch_stream(stream, self.params[0].device)
        with torch.cuda.stream(side):
            mout, vout = ([torch.empty(p.shape, device=p.device) for p in self.params] for _ in range(2))
            pyramid_adamw_moments(self._m, self._v, self._ms, self._vs, mout, vout, side)
        for out in mout + vout:         # results are the caller's stream's as well
            out.record_stream(caller)
        return list(zip(mout, vout))


def pyramid_lstm_timing_enable(on: bool) -> None:
    """Start (clearing earlier records) or stop per-phase HIP-event timing."""
    _check("pyramid_lstm_timing_enable", load().pyramid_lstm_timing_enable(int(bool(on))))


def pyramid_lstm_timing_read(max_phases: int = 32):
    """{phase: (total_ms, launches)} accumulated since timing was enabled."""
    names = ctypes.create_string_buffer(32 * max_phases)
    ms = (ctypes.c_double * max_phases)()
    launches = (ctypes.c_int * max_phases)()
    count = ctypes.c_int(0)
    _check("pyramid_lstm_timing_read", load().pyramid_lstm_timing_read(
        max_phases, names, ms, launches, ctypes.byref(count)))
    out = {}
    for k in range(count.value):
        nm = names.raw[32 * k:32 * k + 32].split(b"\0", 1)[0].decode()
        out[nm] = (ms[k], launches[k])
    return out


def pyramid_lstm_set_forward_path(path: int) -> None:
    """0 = automatic, 1 = generic path only, 2 = MFMA sweep where supported,
    3 = MFMA sweep with every strip staged chunk by chunk, 4 = plane-step
    MFMA path where supported."""
    _check("pyramid_lstm_set_forward_path", load().pyramid_lstm_set_forward_path(int(path)))


def pyramid_lstm_set_backward_path(path: int) -> None:
    """0 = automatic, 1 = generic path only, 2 = MFMA sweep where supported,
    3 = plane-step MFMA path where supported."""
    _check("pyramid_lstm_set_backward_path", load().pyramid_lstm_set_backward_path(int(path)))


def pyramid_lstm_set_step_split(mode: int) -> None:
    """Plane steps, for testing: 0 = the default (fp32: split products);
    otherwise the fp32 steps on the fp32 instruction, 1 = each tile's K split
    over a workgroup's waves, 2 = not, 3 = not and the forward's operands read
    from L1 instead of LDS-staged pixel blocks."""
    _check("pyramid_lstm_set_step_split", load().pyramid_lstm_set_step_split(int(mode)))


def pyramid_lstm_set_bf16_mfma(on: int) -> None:
    """bf16-storage layers with 32 or 64 hidden units: 1 = bf16 MFMA (fp32
    accumulation) on pixel blocks staged in LDS, 2 = bf16 MFMA reading its
    operands from L1, 0 = fp32 MFMA."""
    _check("pyramid_lstm_set_bf16_mfma", load().pyramid_lstm_set_bf16_mfma(int(on)))


def pyramid_lstm_set_wgrad_staged(on: int) -> None:
    """Plane-step weight gradients: 1 = the LDS-staged GEMM where it applies
    (at most 32 hidden units, C a multiple of 4), 0 = the register-streamed
    kernel."""
    _check("pyramid_lstm_set_wgrad_staged", load().pyramid_lstm_set_wgrad_staged(int(on)))


def pyramid_lstm_device_status(clear: bool = False, stream=None) -> int:
    """This device's sticky status bits (synchronises `stream`):
    PLSTM_DEVICE_WAIT_GAVE_UP when a persistent sweep's bounded wait gave up
    since the last clear (that call's outputs were overwritten with NaN)."""
    out = ctypes.c_int32(0)
    _check("pyramid_lstm_device_status",
           load().pyramid_lstm_device_status(ctypes.byref(out), int(bool(clear)), _stream(stream)))
    return int(out.value)


def pyramid_lstm_set_wait_test(on: bool) -> None:
    """Failure-path test mode: every persistent-sweep wait expects a step that
    is never published and gives up after 16 polls (launches still finish)."""
    _check("pyramid_lstm_set_wait_test", load().pyramid_lstm_set_wait_test(int(bool(on))))
