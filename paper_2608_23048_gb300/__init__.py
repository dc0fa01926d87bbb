"""RoI mask-learning hot path on GB300: Python binding of libroi.so.

The binding only marshals arguments: every step of the op runs in the CUDA
library declared by include/roi.h.  Function names are the C names.  Tensors
are torch CUDA tensors (bfloat16 tensors are passed by their bit patterns);
calls are asynchronous on the current torch stream unless `stream` is given.
There is no fallback: if libroi.so is missing the import of the binding's
functions fails loudly.
"""
from __future__ import annotations

import ctypes
import os

__all__ = [
    "RoiError", "NoiseState", "lib", "roi_mask_fwd", "roi_mask_fwd_ex", "roi_mask_bwd",
    "roi_hard_mask_export", "roi_device_status", "roi_status_string", "roi_launch_count",
    "library_path", "hard_words", "roi_noise_words", "roi_gumbel_noise",
    "roi_mask_fwd_st", "roi_mask_bwd_st", "roi_export_compressed_2of4", "AdamW", "roi_mask_bwd_adamw",
    "roi_anneal", "roi_set_ring_wait_limit_ns",
    "roi_checkpoint_pitch", "roi_checkpoint_scale_pitch", "roi_checkpoint_save", "roi_checkpoint_load",
    "new_checkpoint", "roi_norm_fwd", "roi_norm_bwd", "roi_norm_bwd_workspace_size",
    "roi_masked_linear_wgrad", "roi_masked_linear_wgrad_workspace_size",
    "roi_fp8_pitch", "roi_fp8_scale_pitch", "new_fp8", "new_fp8_weight", "roi_fp8_save", "roi_fp8_save_weight",
    "roi_fp8_linear_fwd", "roi_fp8_linear_dgrad",
    "make_adamw_step_items", "make_adamw_step8_items", "make_adamw_state8_items", "new_adamw_state8",
    "roi_adamw_step", "roi_adamw_step8", "roi_adamw_state8_load",
]

_PKG = os.path.dirname(os.path.abspath(__file__))
library_path = os.path.join(_PKG, "libroi.so")

ROI_OK = 0
STATUS_NAMES = {0: "ROI_OK", 1: "ROI_ERR_NULL", 2: "ROI_ERR_SHAPE", 3: "ROI_ERR_NM", 4: "ROI_ERR_TAU",
                5: "ROI_ERR_ALIGN", 6: "ROI_ERR_ALIAS", 7: "ROI_ERR_CUDA", 8: "ROI_ERR_TIMEOUT", 9: "ROI_ERR_OPT",
                10: "ROI_ERR_TYPE"}


class RoiError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        super().__init__(f"{where}: {STATUS_NAMES.get(status, status)} ({roi_status_string(status)})")


class NoiseState(ctypes.Structure):
    """roi_noise_state: seed, step, tensor_id, lambda (sampling temperature), row_offset."""
    _fields_ = [("seed", ctypes.c_uint64), ("step", ctypes.c_uint32), ("tensor_id", ctypes.c_uint32),
                ("lam", ctypes.c_float), ("row_offset", ctypes.c_int64)]


class AdamW(ctypes.Structure):
    """roi_adamw: lr, beta1, beta2, eps, weight_decay, t (1-based step count)."""
    _fields_ = [("lr", ctypes.c_float), ("beta1", ctypes.c_float), ("beta2", ctypes.c_float),
                ("eps", ctypes.c_float), ("weight_decay", ctypes.c_float), ("t", ctypes.c_uint32)]


class FwdItem(ctypes.Structure):
    """roi_fwd_item: one tensor of roi_mask_fwd_batch."""
    _fields_ = [("logits", ctypes.c_void_p), ("W", ctypes.c_void_p), ("out_Wm", ctypes.c_void_p),
                ("out_soft", ctypes.c_void_p), ("out_hard", ctypes.c_void_p), ("rows", ctypes.c_int64),
                ("cols", ctypes.c_int64), ("st", NoiseState)]


class BwdItem(ctypes.Structure):
    """roi_bwd_item: one tensor of roi_mask_bwd_batch."""
    _fields_ = [("logits", ctypes.c_void_p), ("W", ctypes.c_void_p), ("dWm", ctypes.c_void_p),
                ("out_dlogits", ctypes.c_void_p), ("out_dW", ctypes.c_void_p), ("rows", ctypes.c_int64),
                ("cols", ctypes.c_int64), ("st", NoiseState)]


class AdamWItem(ctypes.Structure):
    """roi_adamw_item: one tensor of roi_mask_bwd_adamw_batch."""
    _fields_ = [("logits", ctypes.c_void_p), ("W", ctypes.c_void_p), ("dWm", ctypes.c_void_p),
                ("m", ctypes.c_void_p), ("v", ctypes.c_void_p), ("out_dlogits", ctypes.c_void_p),
                ("out_dW", ctypes.c_void_p), ("rows", ctypes.c_int64), ("cols", ctypes.c_int64),
                ("st", NoiseState)]


class BwdStItem(ctypes.Structure):
    """roi_bwd_st_item: one tensor of roi_mask_bwd_st_batch."""
    _fields_ = [("logits", ctypes.c_void_p), ("W", ctypes.c_void_p), ("dWm", ctypes.c_void_p),
                ("hard", ctypes.c_void_p), ("out_dlogits", ctypes.c_void_p), ("out_dW", ctypes.c_void_p),
                ("rows", ctypes.c_int64), ("cols", ctypes.c_int64), ("st", NoiseState)]


class AdamWStepItem(ctypes.Structure):
    """roi_adamw_step_item: one tensor of roi_adamw_step."""
    _fields_ = [("param", ctypes.c_void_p), ("grad", ctypes.c_void_p), ("m", ctypes.c_void_p), ("v", ctypes.c_void_p),
                ("out_copy", ctypes.c_void_p), ("n", ctypes.c_int64), ("grad_dtype", ctypes.c_int),
                ("copy_dtype", ctypes.c_int)]


class AdamWStep8Item(ctypes.Structure):
    """roi_adamw_step8_item: one tensor of roi_adamw_step8."""
    _fields_ = [("param", ctypes.c_void_p), ("grad", ctypes.c_void_p), ("m_codes", ctypes.c_void_p),
                ("u_codes", ctypes.c_void_p), ("scales", ctypes.c_void_p), ("out_copy", ctypes.c_void_p),
                ("n", ctypes.c_int64), ("grad_dtype", ctypes.c_int), ("copy_dtype", ctypes.c_int),
                ("tensor_id", ctypes.c_uint32)]


class AdamWState8Item(ctypes.Structure):
    """roi_adamw_state8_item: one tensor of roi_adamw_state8_load."""
    _fields_ = [("m_codes", ctypes.c_void_p), ("u_codes", ctypes.c_void_p), ("scales", ctypes.c_void_p),
                ("out_m", ctypes.c_void_p), ("out_u", ctypes.c_void_p), ("n", ctypes.c_int64), ("dtype", ctypes.c_int)]


_LIB = None
_P = ctypes.c_void_p


def lib() -> ctypes.CDLL:
    """The loaded libroi.so with argument types declared (loaded once)."""
    global _LIB
    if _LIB is not None:
        return _LIB
    if not os.path.exists(library_path):
        raise ImportError(f"{library_path} is not built; run `python -m paper_2608_23048_gb300._build` "
                          "(or __graft_entry__.build()) first")
    L = ctypes.CDLL(library_path)
    i32, u32, u64, i64, f32 = ctypes.c_int, ctypes.c_uint32, ctypes.c_uint64, ctypes.c_int64, ctypes.c_float
    L.roi_mask_fwd.argtypes = [_P, _P, i32, i32, f32, u64, u32, i64, i64, _P, _P, _P, _P]
    L.roi_mask_fwd_ex.argtypes = [_P, _P, i32, i32, f32, ctypes.POINTER(NoiseState), i64, i64, _P, _P, _P, _P]
    L.roi_mask_bwd.argtypes = [_P, _P, ctypes.POINTER(NoiseState), i32, i32, _P, f32, i64, i64, _P, _P, _P]
    L.roi_mask_fwd_st.argtypes = [_P, _P, i32, i32, f32, ctypes.POINTER(NoiseState), i64, i64, _P, _P, _P, _P]
    L.roi_mask_bwd_st.argtypes = [_P, _P, ctypes.POINTER(NoiseState), i32, i32, _P, _P, f32, i64, i64, _P, _P, _P]
    L.roi_export_compressed_2of4.argtypes = [_P, _P, i64, i64, _P, _P, _P]
    L.roi_mask_bwd_adamw.argtypes = [_P, _P, ctypes.POINTER(NoiseState), i32, i32, _P, f32, i64, i64, _P, _P,
                                     ctypes.POINTER(AdamW), _P, _P, _P]
    L.roi_masked_linear_fwd.argtypes = [_P, _P, _P, i32, i32, f32, ctypes.POINTER(NoiseState), i64, i64, i64, _P,
                                        _P, ctypes.c_size_t, _P]
    L.roi_masked_linear_fwd_noalloc.argtypes = [_P, _P, _P, i32, i32, f32, ctypes.POINTER(NoiseState), i64, i64,
                                                i64, _P, _P]
    L.roi_masked_linear_workspace_size.argtypes = [i64, i64, i64]
    L.roi_masked_linear_workspace_size.restype = ctypes.c_size_t
    L.roi_mask_fwd_batch.argtypes = [ctypes.POINTER(FwdItem), i32, i32, i32, f32, _P]
    L.roi_mask_bwd_batch.argtypes = [ctypes.POINTER(BwdItem), i32, i32, i32, f32, _P]
    L.roi_mask_fwd_st_batch.argtypes = [ctypes.POINTER(FwdItem), i32, i32, i32, f32, _P]
    L.roi_mask_bwd_st_batch.argtypes = [ctypes.POINTER(BwdStItem), i32, i32, i32, f32, _P]
    L.roi_mask_bwd_adamw_batch.argtypes = [ctypes.POINTER(AdamWItem), i32, i32, i32, f32, ctypes.POINTER(AdamW), _P]
    L.roi_anneal.argtypes = [f32, f32, u32, u32]
    L.roi_anneal.restype = f32
    L.roi_hard_mask_export.argtypes = [_P, i32, i32, i64, i64, _P, _P, _P, _P]
    L.roi_checkpoint_pitch.argtypes = [i64]
    L.roi_checkpoint_pitch.restype = i64
    L.roi_checkpoint_scale_pitch.argtypes = [i64]
    L.roi_checkpoint_scale_pitch.restype = i64
    L.roi_checkpoint_save.argtypes = [_P, i32, i64, i64, i64, _P, _P, _P]
    L.roi_checkpoint_load.argtypes = [_P, _P, i32, i64, i64, _P, i64, _P]
    L.roi_norm_fwd.argtypes = [_P, i32, i64, i64, i64, i32, _P, _P, i32, f32, _P, i64, _P, _P, _P, _P, _P, _P, _P]
    L.roi_norm_bwd.argtypes = [_P, i32, i64, i64, i64, _P, i64, _P, _P, i32, _P, i32, _P, _P, _P, i64, _P, _P, _P,
                               ctypes.c_size_t, _P]
    L.roi_norm_bwd_workspace_size.argtypes = [i64, i64]
    L.roi_norm_bwd_workspace_size.restype = ctypes.c_size_t
    L.roi_masked_linear_wgrad.argtypes = [_P, i64, _P, _P, i64, i64, i64, _P, _P, _P, ctypes.c_size_t, _P]
    L.roi_masked_linear_wgrad_workspace_size.argtypes = [i64, i64, i64, i64]
    L.roi_masked_linear_wgrad_workspace_size.restype = ctypes.c_size_t
    L.roi_fp8_pitch.argtypes = [i64]
    L.roi_fp8_pitch.restype = i64
    L.roi_fp8_scale_pitch.argtypes = [i64]
    L.roi_fp8_scale_pitch.restype = i64
    L.roi_fp8_save.argtypes = [_P, i32, i64, i64, i64, i32, _P, _P, _P]
    L.roi_fp8_save_weight.argtypes = [_P, i64, i64, _P, _P, _P]
    for name in ("roi_fp8_linear_fwd", "roi_fp8_linear_dgrad"):
        getattr(L, name).argtypes = [_P, _P, i32, _P, _P, i64, i64, i64, _P, i32, i64, _P]
    L.roi_adamw_step.argtypes = [ctypes.POINTER(AdamWStepItem), i32, ctypes.POINTER(AdamW), _P, _P]
    L.roi_adamw_step8.argtypes = [ctypes.POINTER(AdamWStep8Item), i32, ctypes.POINTER(AdamW), u64, _P, _P]
    L.roi_adamw_state8_load.argtypes = [ctypes.POINTER(AdamWState8Item), i32, _P]
    L.roi_device_status.argtypes = [_P]
    L.roi_set_ring_wait_limit_ns.argtypes = [u64]
    L.roi_noise_words.argtypes = [ctypes.POINTER(NoiseState), i64, i64, _P, _P]
    L.roi_gumbel_noise.argtypes = [ctypes.POINTER(NoiseState), i64, i64, _P, _P]
    L.roi_status_string.argtypes = [i32]
    L.roi_status_string.restype = ctypes.c_char_p
    L.roi_launch_count.argtypes = []
    L.roi_launch_count.restype = ctypes.c_uint64
    for name in ("roi_mask_fwd", "roi_mask_fwd_ex", "roi_mask_bwd", "roi_hard_mask_export", "roi_device_status",
                 "roi_noise_words", "roi_gumbel_noise", "roi_mask_fwd_st", "roi_mask_bwd_st",
                 "roi_export_compressed_2of4", "roi_mask_bwd_adamw", "roi_masked_linear_fwd",
                 "roi_masked_linear_fwd_noalloc", "roi_mask_fwd_batch", "roi_mask_bwd_batch",
                 "roi_mask_bwd_adamw_batch", "roi_mask_fwd_st_batch", "roi_mask_bwd_st_batch",
                 "roi_set_ring_wait_limit_ns", "roi_checkpoint_save", "roi_checkpoint_load", "roi_norm_fwd",
                 "roi_norm_bwd", "roi_masked_linear_wgrad", "roi_fp8_save", "roi_fp8_save_weight", "roi_fp8_linear_fwd",
                 "roi_fp8_linear_dgrad", "roi_adamw_step", "roi_adamw_step8", "roi_adamw_state8_load"):
        getattr(L, name).restype = i32
    _LIB = L
    return L


def roi_status_string(status: int) -> str:
    return lib().roi_status_string(int(status)).decode()


def roi_launch_count() -> int:
    return int(lib().roi_launch_count())


def _ptr(t):
    return None if t is None else t.data_ptr()


_RAW_STREAM = None  # torch's (raw current stream of a device, current device), once CUDA is initialised


def _stream(stream):
    global _RAW_STREAM
    if stream is None:
        if _RAW_STREAM is None:
            import torch
            if not torch.cuda.is_initialized():
                return torch.cuda.current_stream().cuda_stream
            # the same handle without a Stream object around it
            _RAW_STREAM = torch._C._cuda_getCurrentRawStream, torch._C._cuda_getDevice
        return _RAW_STREAM[0](_RAW_STREAM[1]())
    if isinstance(stream, int):
        return stream
    return stream.cuda_stream


def _check_tensor(t, name, dtype, shape=None):
    if t is None:
        return
    if t.dtype is dtype and t.is_cuda and t.is_contiguous() and (shape is None or t.shape == shape):
        return
    if t.dtype != dtype:
        raise TypeError(f"{name}: expected {dtype}, got {t.dtype}")
    if not t.is_cuda:
        raise ValueError(f"{name}: expected a CUDA tensor")
    if not t.is_contiguous():
        raise ValueError(f"{name}: must be contiguous")
    if shape is not None and tuple(t.shape) != tuple(shape):
        raise ValueError(f"{name}: expected shape {tuple(shape)}, got {tuple(t.shape)}")


def hard_words(rows: int, cols: int) -> int:
    """uint32 words of a hard mask over rows * cols elements."""
    return (rows * cols + 31) // 32


def _raise(status, where):
    if status != ROI_OK:
        raise RoiError(status, where)


def roi_mask_fwd_ex(logits, W, N, M, tau, state: NoiseState, out_Wm, out_soft=None, out_hard=None, stream=None):
    """Forward with full noise state; outputs are written in place.  Returns None."""
    import torch
    rows, cols = logits.shape
    _check_tensor(logits, "logits", torch.float32)
    _check_tensor(W, "W", torch.bfloat16, (rows, cols))
    _check_tensor(out_Wm, "out_Wm", torch.bfloat16, (rows, cols))
    _check_tensor(out_soft, "out_soft", torch.float32, (rows, cols))
    _check_tensor(out_hard, "out_hard", torch.int32, (hard_words(rows, cols),))
    st = state if isinstance(state, NoiseState) else NoiseState(*state)
    s = lib().roi_mask_fwd_ex(_ptr(logits), _ptr(W), int(N), int(M), float(tau), ctypes.byref(st), rows, cols,
                              _ptr(out_Wm), _ptr(out_soft), _ptr(out_hard), _stream(stream))
    _raise(s, "roi_mask_fwd_ex")


def _addr(t):
    return None if t is None else t.data_ptr()


def make_fwd_items(items):
    """ctypes array of FwdItem from (logits, W, state, out_Wm, out_soft, out_hard) tuples."""
    import torch
    arr = (FwdItem * len(items))()
    for k, (logits, W, state, out_Wm, out_soft, out_hard) in enumerate(items):
        rows, cols = logits.shape
        _check_tensor(logits, "logits", torch.float32)
        _check_tensor(W, "W", torch.bfloat16, (rows, cols))
        _check_tensor(out_Wm, "out_Wm", torch.bfloat16, (rows, cols))
        _check_tensor(out_soft, "out_soft", torch.float32, (rows, cols))
        _check_tensor(out_hard, "out_hard", torch.int32, (hard_words(rows, cols),))
        st = state if isinstance(state, NoiseState) else NoiseState(*state)
        arr[k] = FwdItem(_addr(logits), _addr(W), _addr(out_Wm), _addr(out_soft), _addr(out_hard), rows, cols, st)
    return arr


def make_bwd_items(items):
    """ctypes array of BwdItem from (logits, W, state, dWm, out_dlogits, out_dW) tuples."""
    import torch
    arr = (BwdItem * len(items))()
    for k, (logits, W, state, dWm, out_dlogits, out_dW) in enumerate(items):
        rows, cols = logits.shape
        _check_tensor(logits, "logits", torch.float32)
        _check_tensor(W, "W", torch.bfloat16, (rows, cols))
        _check_tensor(dWm, "dWm", torch.bfloat16, (rows, cols))
        _check_tensor(out_dlogits, "out_dlogits", torch.float32, (rows, cols))
        _check_tensor(out_dW, "out_dW", torch.bfloat16, (rows, cols))
        st = state if isinstance(state, NoiseState) else NoiseState(*state)
        arr[k] = BwdItem(_addr(logits), _addr(W), _addr(dWm), _addr(out_dlogits), _addr(out_dW), rows, cols, st)
    return arr


def make_adamw_items(items):
    """ctypes array of AdamWItem from (logits, W, state, dWm, m, v, out_dlogits, out_dW) tuples."""
    import torch
    arr = (AdamWItem * len(items))()
    for k, (logits, W, state, dWm, m, v, out_dlogits, out_dW) in enumerate(items):
        rows, cols = logits.shape
        _check_tensor(logits, "logits", torch.float32)
        for name, t, dt in (("W", W, torch.bfloat16), ("dWm", dWm, torch.bfloat16), ("m", m, torch.float32),
                            ("v", v, torch.float32), ("out_dlogits", out_dlogits, torch.float32),
                            ("out_dW", out_dW, torch.bfloat16)):
            _check_tensor(t, name, dt, (rows, cols))
        st = state if isinstance(state, NoiseState) else NoiseState(*state)
        arr[k] = AdamWItem(_addr(logits), _addr(W), _addr(dWm), _addr(m), _addr(v), _addr(out_dlogits),
                           _addr(out_dW), rows, cols, st)
    return arr


def roi_mask_bwd_adamw_batch(items, N, M, tau, opt: AdamW, stream=None):
    """Backward fused with the logits' AdamW step for many tensors (AdamWItem array from
    make_adamw_items, or a list of (logits, W, state, dWm, m, v, out_dlogits, out_dW) tuples)."""
    arr = items if isinstance(items, ctypes.Array) else make_adamw_items(items)
    s = lib().roi_mask_bwd_adamw_batch(arr, len(arr), int(N), int(M), float(tau), ctypes.byref(opt), _stream(stream))
    _raise(s, "roi_mask_bwd_adamw_batch")


def make_bwd_st_items(items):
    """ctypes array of BwdStItem from (logits, W, state, dWm, hard, out_dlogits, out_dW) tuples."""
    import torch
    arr = (BwdStItem * len(items))()
    for k, (logits, W, state, dWm, hard, out_dlogits, out_dW) in enumerate(items):
        rows, cols = logits.shape
        _check_tensor(logits, "logits", torch.float32)
        _check_tensor(W, "W", torch.bfloat16, (rows, cols))
        _check_tensor(dWm, "dWm", torch.bfloat16, (rows, cols))
        _check_tensor(hard, "hard", torch.int32, (hard_words(rows, cols),))
        _check_tensor(out_dlogits, "out_dlogits", torch.float32, (rows, cols))
        _check_tensor(out_dW, "out_dW", torch.bfloat16, (rows, cols))
        st = state if isinstance(state, NoiseState) else NoiseState(*state)
        arr[k] = BwdStItem(_addr(logits), _addr(W), _addr(dWm), _addr(hard), _addr(out_dlogits), _addr(out_dW),
                           rows, cols, st)
    return arr


def roi_mask_fwd_st_batch(items, N, M, tau, stream=None):
    """Straight-through forward of many tensors (items as for roi_mask_fwd_batch)."""
    arr = items if isinstance(items, ctypes.Array) else make_fwd_items(items)
    s = lib().roi_mask_fwd_st_batch(arr, len(arr), int(N), int(M), float(tau), _stream(stream))
    _raise(s, "roi_mask_fwd_st_batch")


def roi_mask_bwd_st_batch(items, N, M, tau, stream=None):
    """Straight-through backward of many tensors (BwdStItem array from make_bwd_st_items,
    or a list of (logits, W, state, dWm, hard, out_dlogits, out_dW) tuples)."""
    arr = items if isinstance(items, ctypes.Array) else make_bwd_st_items(items)
    s = lib().roi_mask_bwd_st_batch(arr, len(arr), int(N), int(M), float(tau), _stream(stream))
    _raise(s, "roi_mask_bwd_st_batch")


def roi_mask_fwd_batch(items, N, M, tau, stream=None):
    """Forward of many tensors in one call.  `items`: a FwdItem array from make_fwd_items
    (reusable across calls while its tensors live; update .st.step per step) or a list
    of (logits, W, state, out_Wm, out_soft, out_hard) tuples."""
    arr = items if isinstance(items, ctypes.Array) else make_fwd_items(items)
    s = lib().roi_mask_fwd_batch(arr, len(arr), int(N), int(M), float(tau), _stream(stream))
    _raise(s, "roi_mask_fwd_batch")


def roi_mask_bwd_batch(items, N, M, tau, stream=None):
    """Backward of many tensors in one call (BwdItem array from make_bwd_items, or a list
    of (logits, W, state, dWm, out_dlogits, out_dW) tuples)."""
    arr = items if isinstance(items, ctypes.Array) else make_bwd_items(items)
    s = lib().roi_mask_bwd_batch(arr, len(arr), int(N), int(M), float(tau), _stream(stream))
    _raise(s, "roi_mask_bwd_batch")


def roi_mask_fwd(logits, W, N, M, tau, seed, step, out_Wm, out_soft=None, out_hard=None, stream=None):
    """Forward, short form (lambda = 1, tensor_id = 0, row_offset = 0)."""
    import torch
    rows, cols = logits.shape
    _check_tensor(logits, "logits", torch.float32)
    _check_tensor(W, "W", torch.bfloat16, (rows, cols))
    _check_tensor(out_Wm, "out_Wm", torch.bfloat16, (rows, cols))
    _check_tensor(out_soft, "out_soft", torch.float32, (rows, cols))
    _check_tensor(out_hard, "out_hard", torch.int32, (hard_words(rows, cols),))
    s = lib().roi_mask_fwd(_ptr(logits), _ptr(W), int(N), int(M), float(tau), int(seed), int(step), rows, cols,
                           _ptr(out_Wm), _ptr(out_soft), _ptr(out_hard), _stream(stream))
    _raise(s, "roi_mask_fwd")


def roi_mask_bwd(logits, W, state: NoiseState, N, M, dWm, tau, out_dlogits, out_dW=None, stream=None):
    """Backward: logit gradients (overwritten) and optionally dW."""
    import torch
    rows, cols = logits.shape
    _check_tensor(logits, "logits", torch.float32)
    _check_tensor(W, "W", torch.bfloat16, (rows, cols))
    _check_tensor(dWm, "dWm", torch.bfloat16, (rows, cols))
    _check_tensor(out_dlogits, "out_dlogits", torch.float32, (rows, cols))
    _check_tensor(out_dW, "out_dW", torch.bfloat16, (rows, cols))
    st = state if isinstance(state, NoiseState) else NoiseState(*state)
    s = lib().roi_mask_bwd(_ptr(logits), _ptr(W), ctypes.byref(st), int(N), int(M), _ptr(dWm), float(tau),
                           rows, cols, _ptr(out_dlogits), _ptr(out_dW), _stream(stream))
    _raise(s, "roi_mask_bwd")


def roi_mask_fwd_st(logits, W, N, M, tau, state: NoiseState, out_Wm, out_soft=None, out_hard=None, stream=None):
    """Straight-through forward: Wm = W where the Gumbel-top-N hard mask is set, +0 elsewhere."""
    import torch
    rows, cols = logits.shape
    _check_tensor(logits, "logits", torch.float32)
    _check_tensor(W, "W", torch.bfloat16, (rows, cols))
    _check_tensor(out_Wm, "out_Wm", torch.bfloat16, (rows, cols))
    _check_tensor(out_soft, "out_soft", torch.float32, (rows, cols))
    _check_tensor(out_hard, "out_hard", torch.int32, (hard_words(rows, cols),))
    st = state if isinstance(state, NoiseState) else NoiseState(*state)
    s = lib().roi_mask_fwd_st(_ptr(logits), _ptr(W), int(N), int(M), float(tau), ctypes.byref(st), rows, cols,
                              _ptr(out_Wm), _ptr(out_soft), _ptr(out_hard), _stream(stream))
    _raise(s, "roi_mask_fwd_st")


def roi_mask_bwd_st(logits, W, state: NoiseState, N, M, dWm, hard, tau, out_dlogits, out_dW=None, stream=None):
    """Straight-through backward: logit gradients through the relaxation; dW = dWm where
    the forward's hard mask (`hard`, its out_hard words) is set."""
    import torch
    rows, cols = logits.shape
    _check_tensor(logits, "logits", torch.float32)
    _check_tensor(W, "W", torch.bfloat16, (rows, cols))
    _check_tensor(dWm, "dWm", torch.bfloat16, (rows, cols))
    _check_tensor(hard, "hard", torch.int32, (hard_words(rows, cols),))
    _check_tensor(out_dlogits, "out_dlogits", torch.float32, (rows, cols))
    _check_tensor(out_dW, "out_dW", torch.bfloat16, (rows, cols))
    st = state if isinstance(state, NoiseState) else NoiseState(*state)
    s = lib().roi_mask_bwd_st(_ptr(logits), _ptr(W), ctypes.byref(st), int(N), int(M), _ptr(dWm), _ptr(hard),
                              float(tau), rows, cols, _ptr(out_dlogits), _ptr(out_dW), _stream(stream))
    _raise(s, "roi_mask_bwd_st")


def roi_mask_bwd_adamw(logits, W, state: NoiseState, N, M, dWm, tau, m, v, opt: AdamW, out_dlogits=None,
                       out_dW=None, stream=None):
    """Backward fused with one AdamW step: `logits`, `m`, `v` are updated in place."""
    import torch
    rows, cols = logits.shape
    _check_tensor(logits, "logits", torch.float32)
    _check_tensor(W, "W", torch.bfloat16, (rows, cols))
    _check_tensor(dWm, "dWm", torch.bfloat16, (rows, cols))
    _check_tensor(m, "m", torch.float32, (rows, cols))
    _check_tensor(v, "v", torch.float32, (rows, cols))
    _check_tensor(out_dlogits, "out_dlogits", torch.float32, (rows, cols))
    _check_tensor(out_dW, "out_dW", torch.bfloat16, (rows, cols))
    st = state if isinstance(state, NoiseState) else NoiseState(*state)
    s = lib().roi_mask_bwd_adamw(_ptr(logits), _ptr(W), ctypes.byref(st), int(N), int(M), _ptr(dWm), float(tau),
                                 rows, cols, _ptr(m), _ptr(v), ctypes.byref(opt), _ptr(out_dlogits), _ptr(out_dW),
                                 _stream(stream))
    _raise(s, "roi_mask_bwd_adamw")


def roi_anneal(init, end, t, T_anneal):
    """Eq. 13: max(end, init * (end / init) ** (t / T_anneal)), evaluated by the library."""
    return float(lib().roi_anneal(float(init), float(end), int(t), int(T_anneal)))


def roi_export_compressed_2of4(logits, W, out_values, out_meta, stream=None):
    """Compressed 2:4 export: kept weights [rows, cols/2] and 4-bit index codes, 8 groups per word."""
    import torch
    rows, cols = logits.shape
    _check_tensor(logits, "logits", torch.float32)
    _check_tensor(W, "W", torch.bfloat16, (rows, cols))
    _check_tensor(out_values, "out_values", torch.bfloat16, (rows, cols // 2))
    _check_tensor(out_meta, "out_meta", torch.int32, ((rows * cols) // 32,))
    s = lib().roi_export_compressed_2of4(_ptr(logits), _ptr(W), rows, cols, _ptr(out_values), _ptr(out_meta),
                                         _stream(stream))
    _raise(s, "roi_export_compressed_2of4")


def roi_masked_linear_workspace_size(T, rows, cols) -> int:
    """Bytes of workspace that let roi_masked_linear_fwd split K fully on the current device."""
    return int(lib().roi_masked_linear_workspace_size(int(T), int(rows), int(cols)))


def roi_masked_linear_fwd(X, logits, W, N, M, tau, state: NoiseState, out_Y, workspace=None, stream=None):
    """Y[T, rows] = X[T, cols] @ bf16(W * S)^T with the mask formed inside the GEMM (float32 Y)."""
    import torch
    rows, cols = logits.shape
    T = X.shape[0]
    _check_tensor(logits, "logits", torch.float32)
    _check_tensor(X, "X", torch.bfloat16, (T, cols))
    _check_tensor(W, "W", torch.bfloat16, (rows, cols))
    _check_tensor(out_Y, "out_Y", torch.float32, (T, rows))
    ws_bytes = 0
    if workspace is not None:
        _check_tensor(workspace, "workspace", workspace.dtype)
        ws_bytes = workspace.numel() * workspace.element_size()
    st = state if isinstance(state, NoiseState) else NoiseState(*state)
    s = lib().roi_masked_linear_fwd(_ptr(X), _ptr(logits), _ptr(W), int(N), int(M), float(tau), ctypes.byref(st), T,
                                    rows, cols, _ptr(out_Y), _ptr(workspace), ws_bytes, _stream(stream))
    _raise(s, "roi_masked_linear_fwd")


def roi_masked_linear_fwd_noalloc(X, logits, W, N, M, tau, state: NoiseState, out_Y, stream=None):
    """roi_masked_linear_fwd with the library's static split-K scratch (no workspace argument)."""
    import torch
    rows, cols = logits.shape
    T = X.shape[0]
    _check_tensor(logits, "logits", torch.float32)
    _check_tensor(X, "X", torch.bfloat16, (T, cols))
    _check_tensor(W, "W", torch.bfloat16, (rows, cols))
    _check_tensor(out_Y, "out_Y", torch.float32, (T, rows))
    st = state if isinstance(state, NoiseState) else NoiseState(*state)
    s = lib().roi_masked_linear_fwd_noalloc(_ptr(X), _ptr(logits), _ptr(W), int(N), int(M), float(tau),
                                            ctypes.byref(st), T, rows, cols, _ptr(out_Y), _stream(stream))
    _raise(s, "roi_masked_linear_fwd_noalloc")


def roi_hard_mask_export(logits, N, M, out_bits, W=None, out_Wpruned=None, stream=None):
    """Deployment mask argtop_N(logits) (+ pruned weights)."""
    import torch
    rows, cols = logits.shape
    _check_tensor(logits, "logits", torch.float32)
    _check_tensor(out_bits, "out_bits", torch.int32, (hard_words(rows, cols),))
    _check_tensor(W, "W", torch.bfloat16, (rows, cols))
    _check_tensor(out_Wpruned, "out_Wpruned", torch.bfloat16, (rows, cols))
    s = lib().roi_hard_mask_export(_ptr(logits), int(N), int(M), rows, cols, _ptr(out_bits), _ptr(W),
                                   _ptr(out_Wpruned), _stream(stream))
    _raise(s, "roi_hard_mask_export")


# ---------------------------------------------------------------------------
# around the masked linear layers: 8-bit checkpoints, norms, weight gradients
# ---------------------------------------------------------------------------
NORM_KINDS = {"layer": 0, "rms": 1}


_TYPES = {}  # torch type -> roi_dtype, of the types that the calls take


def _type(t, name):
    code = _TYPES.get(t.dtype)
    if code is None:
        import torch
        _TYPES.update({torch.bfloat16: 0, torch.float16: 1, torch.float32: 2})
        code = _TYPES.get(t.dtype)
        if code is None:
            raise TypeError(f"{name}: expected bfloat16, float16 or float32, got {t.dtype}")
    return code


def _stride(t, name, shape=None):
    """Row stride, in elements, of a CUDA matrix whose rows may be apart."""
    if not t.is_cuda:
        raise ValueError(f"{name}: expected a CUDA tensor")
    have = t.shape
    if len(have) != 2 or (shape is not None and have != shape):
        raise ValueError(f"{name}: expected {'a matrix' if shape is None else f'shape {tuple(shape)}'}, got {tuple(have)}")
    if t.is_contiguous() or have[0] <= 1 and (have[1] <= 1 or t.stride(1) == 1):
        return have[1]  # (the stride of a single row says nothing)
    if have[1] > 1 and t.stride(1) != 1:
        raise ValueError(f"{name}: the elements of a row must be contiguous")
    return t.stride(0)


def roi_checkpoint_pitch(cols) -> int:
    """Codes in a row of a checkpoint of `cols` columns."""
    return int(lib().roi_checkpoint_pitch(int(cols)))


def roi_checkpoint_scale_pitch(cols) -> int:
    """Scale bytes in a row of a checkpoint of `cols` columns."""
    return int(lib().roi_checkpoint_scale_pitch(int(cols)))


def new_checkpoint(rows, cols, device="cuda"):
    """Uninitialised (codes, scales) for a matrix [rows, cols]."""
    import torch
    return (torch.empty(rows, roi_checkpoint_pitch(cols), dtype=torch.int8, device=device),
            torch.empty(rows, roi_checkpoint_scale_pitch(cols), dtype=torch.uint8, device=device))


def _checkpoint(pair, name, rows, cols):
    """Addresses of a checkpoint's codes and scales (of a matrix [rows, cols]; None: none)."""
    import torch
    if pair is None:
        return None, None
    codes, scales = pair
    if codes is None or scales is None:
        raise ValueError(f"{name}: codes and scales go together")
    _check_tensor(codes, f"{name} codes", torch.int8, (rows, (cols + 31) // 32 * 32))
    _check_tensor(scales, f"{name} scales", torch.uint8, (rows, (cols + 127) // 128 * 4))
    return codes.data_ptr(), scales.data_ptr()


def roi_checkpoint_save(x, out_codes, out_scales, stream=None):
    """Saves x [rows, cols] (bfloat16, float16 or float32; rows may be apart) in 8 bits."""
    ld = _stride(x, "x")
    rows, cols = x.shape
    codes, scales = _checkpoint((out_codes, out_scales), "out", rows, cols)
    s = lib().roi_checkpoint_save(x.data_ptr(), _type(x, "x"), rows, cols, ld, codes, scales, _stream(stream))
    _raise(s, "roi_checkpoint_save")


def roi_checkpoint_load(codes, scales, out_x, stream=None):
    """The values a checkpoint stands for, in the type of out_x [rows, cols]."""
    ld = _stride(out_x, "out_x")
    rows, cols = out_x.shape
    codes, scales = _checkpoint((codes, scales), "checkpoint", rows, cols)
    s = lib().roi_checkpoint_load(codes, scales, _type(out_x, "out_x"), rows, cols, out_x.data_ptr(), ld, _stream(stream))
    _raise(s, "roi_checkpoint_load")


def _norm_kind(kind):
    code = NORM_KINDS.get(kind)
    if code is None:
        raise ValueError(f"kind: expected one of {sorted(NORM_KINDS)}, got {kind!r}")
    return code


def _param(t, name, like, cols, other=None):
    """Type code of a norm's weight or bias: the type of `like`, or float32; that of `other`, if given."""
    code = _type(t, name)
    if (code != 2 and t.dtype != like.dtype) or (other is not None and t.dtype != other.dtype):
        raise TypeError(f"{name}: expected {like.dtype} or torch.float32, one type for all, got {t.dtype}")
    _check_tensor(t, name, t.dtype, (cols,))
    return code


def roi_norm_fwd(x, kind, gamma, beta, eps, out_y, out_mean=None, out_rstd=None, x_checkpoint=None, y_checkpoint=None,
                 stream=None):
    """Layer norm ("layer") or RMS norm ("rms") of the rows of x; the checkpoints of x and of
    out_y ((codes, scales) pairs) are written in the same pass where given."""
    import torch
    ldx = _stride(x, "x")
    dtype = param = _type(x, "x")
    shape = x.shape
    rows, cols = shape
    ldy = _stride(out_y, "out_y", shape)
    if out_y.dtype is not x.dtype:
        raise TypeError(f"out_y: expected {x.dtype}, got {out_y.dtype}")
    if gamma is not None:
        param = _param(gamma, "gamma", x, cols)
    if beta is not None:
        param = _param(beta, "beta", x, cols, gamma)
    if out_mean is not None:
        _check_tensor(out_mean, "out_mean", torch.float32, (rows,))
    if out_rstd is not None:
        _check_tensor(out_rstd, "out_rstd", torch.float32, (rows,))
    xq, xs = _checkpoint(x_checkpoint, "x_checkpoint", rows, cols)
    yq, ys = _checkpoint(y_checkpoint, "y_checkpoint", rows, cols)
    s = lib().roi_norm_fwd(x.data_ptr(), dtype, rows, cols, ldx, _norm_kind(kind), _ptr(gamma), _ptr(beta), param, eps,
                           out_y.data_ptr(), ldy, _ptr(out_mean), _ptr(out_rstd), xq, xs, yq, ys, _stream(stream))
    _raise(s, "roi_norm_fwd")


def roi_norm_bwd_workspace_size(rows, cols) -> int:
    """Bytes of workspace roi_norm_bwd needs for the gradients of weight and bias on the current device."""
    return int(lib().roi_norm_bwd_workspace_size(int(rows), int(cols)))


def _workspace(workspace):
    """(pointer, bytes) of a workspace tensor of any type."""
    if workspace is None:
        return None, 0
    _check_tensor(workspace, "workspace", workspace.dtype)
    return workspace.data_ptr(), workspace.nbytes


def roi_norm_bwd(dy, x, kind, gamma, mean, rstd, out_dx, out_dgamma=None, out_dbeta=None, workspace=None, stream=None):
    """Backward of roi_norm_fwd.  x: the forward's input, or its checkpoint, a (codes, scales) pair.
    out_dgamma, out_dbeta: float32 [cols], overwritten."""
    import torch
    lddy = _stride(dy, "dy")
    dtype = param = _type(dy, "dy")
    shape = dy.shape
    rows, cols = shape
    lddx = _stride(out_dx, "out_dx", shape)
    x_ptr = codes = scales = None
    ldx = cols
    if isinstance(x, (tuple, list)):
        codes, scales = _checkpoint(x, "x", rows, cols)
    else:
        ldx = _stride(x, "x", shape)
        if x.dtype is not dy.dtype:
            raise TypeError(f"x: expected {dy.dtype}, got {x.dtype}")
        x_ptr = x.data_ptr()
    if out_dx.dtype is not dy.dtype:
        raise TypeError(f"out_dx: expected {dy.dtype}, got {out_dx.dtype}")
    if gamma is not None:
        param = _param(gamma, "gamma", dy, cols)
    f32 = torch.float32
    if mean is not None:
        _check_tensor(mean, "mean", f32, (rows,))
    _check_tensor(rstd, "rstd", f32, (rows,))
    if out_dgamma is not None:
        _check_tensor(out_dgamma, "out_dgamma", f32, (cols,))
    if out_dbeta is not None:
        _check_tensor(out_dbeta, "out_dbeta", f32, (cols,))
    ws, ws_bytes = _workspace(workspace)
    s = lib().roi_norm_bwd(dy.data_ptr(), dtype, rows, cols, lddy, x_ptr, ldx, codes, scales, _norm_kind(kind),
                           _ptr(gamma), param, _ptr(mean), _ptr(rstd), out_dx.data_ptr(), lddx, _ptr(out_dgamma),
                           _ptr(out_dbeta), ws, ws_bytes, _stream(stream))
    _raise(s, "roi_norm_bwd")


def roi_masked_linear_wgrad_workspace_size(T, rows, cols, lddy=None) -> int:
    """Bytes of workspace roi_masked_linear_wgrad can use on the current device (lddy: row stride
    of dY in elements, `rows` unless given)."""
    return int(lib().roi_masked_linear_wgrad_workspace_size(int(T), int(rows), int(cols),
                                                            int(rows if lddy is None else lddy)))


def roi_masked_linear_wgrad(dY, x_checkpoint, out_dWm=None, acc=None, workspace=None, stream=None):
    """out_dWm[rows, cols] = bf16(dY[T, rows]^T x[T, cols] + acc), x the values of the (codes, scales)
    pair x_checkpoint; acc (float32), where given, is updated in place."""
    import torch
    lddy = _stride(dY, "dY")
    T, rows = dY.shape
    if dY.dtype is not torch.bfloat16:
        raise TypeError(f"dY: expected torch.bfloat16, got {dY.dtype}")
    out = out_dWm if out_dWm is not None else acc
    if out is None or out.dim() != 2:
        raise ValueError("out_dWm or acc: a matrix is required")
    cols = out.shape[1]
    codes, scales = _checkpoint(x_checkpoint, "x_checkpoint", T, cols)
    if out_dWm is not None:
        _check_tensor(out_dWm, "out_dWm", torch.bfloat16, (rows, cols))
    if acc is not None:
        _check_tensor(acc, "acc", torch.float32, (rows, cols))
    ws, ws_bytes = _workspace(workspace)
    s = lib().roi_masked_linear_wgrad(dY.data_ptr(), lddy, codes, scales, T, rows, cols, _ptr(out_dWm), _ptr(acc), ws,
                                      ws_bytes, _stream(stream))
    _raise(s, "roi_masked_linear_wgrad")


# ---------------------------------------------------------------------------
# the masked layers' products in 8-bit floating point
# ---------------------------------------------------------------------------
FP8_FORMATS = {"e4m3": 0, "e5m2": 1}


def _format(format):
    code = FP8_FORMATS.get(format)
    if code is None:
        raise ValueError(f"format: expected one of {sorted(FP8_FORMATS)}, got {format!r}")
    return code


def roi_fp8_pitch(cols) -> int:
    """Codes in a row of a copy of `cols` columns."""
    return int(lib().roi_fp8_pitch(int(cols)))


def roi_fp8_scale_pitch(cols) -> int:
    """Scale bytes in a row of a copy of `cols` columns."""
    return int(lib().roi_fp8_scale_pitch(int(cols)))


def new_fp8(rows, cols, device="cuda"):
    """Uninitialised (codes, scales) for the copy of an activation [rows, cols]."""
    import torch
    return (torch.empty(rows, roi_fp8_pitch(cols), dtype=torch.uint8, device=device),
            torch.empty(rows, roi_fp8_scale_pitch(cols), dtype=torch.uint8, device=device))


def new_fp8_weight(rows, cols, device="cuda"):
    """Uninitialised (codes, scales) for the copy of a weight [rows, cols]."""
    import torch
    return (torch.empty(rows, roi_fp8_pitch(cols), dtype=torch.uint8, device=device),
            torch.empty((rows + 127) // 128, roi_fp8_scale_pitch(cols), dtype=torch.uint8, device=device))


_UINT8 = None  # torch.uint8, once torch is there


def _fp8(pair, name, rows, pitch, scale_rows, scale_pitch, like):
    """Addresses of a copy's codes [rows, pitch] and scales, on the device of `like` (a CUDA tensor)."""
    global _UINT8
    codes, scales = pair
    if (codes.dtype is scales.dtype is _UINT8 and codes.get_device() == scales.get_device() == like.get_device()
            and codes.is_contiguous() and scales.is_contiguous() and codes.shape == (rows, pitch)
            and scales.shape == (scale_rows, scale_pitch)):
        return codes.data_ptr(), scales.data_ptr()
    import torch
    _UINT8 = torch.uint8
    _check_tensor(codes, f"{name} codes", torch.uint8, (rows, pitch))
    _check_tensor(scales, f"{name} scales", torch.uint8, (scale_rows, scale_pitch))
    _device((like, codes, scales), name)
    return codes.data_ptr(), scales.data_ptr()


def _pitches(cols):
    """Codes and scale bytes in a row of a copy of `cols` columns."""
    return (cols + 127) // 128 * 128, (cols + 2047) // 2048 * 16


def roi_fp8_save(x, format, out_codes, out_scales, stream=None):
    """Copies x [rows, cols] (bfloat16, float16 or float32; rows may be apart) in 8-bit floating point
    ("e4m3" or "e5m2") with a power of two for every 128 columns of a row."""
    ld = _stride(x, "x")
    rows, cols = x.shape
    pitch, scale_pitch = _pitches(cols)
    codes, scales = _fp8((out_codes, out_scales), "out", rows, pitch, rows, scale_pitch, x)
    s = lib().roi_fp8_save(x.data_ptr(), _type(x, "x"), rows, cols, ld, _format(format), codes, scales, _stream(stream))
    if s != ROI_OK:
        _raise(s, "roi_fp8_save")


def roi_fp8_save_weight(W, out_codes, out_scales, stream=None):
    """Copies a weight [rows, cols] (bfloat16) in e4m3 with a power of two for every block of 128 x 128."""
    import torch
    rows, cols = W.shape
    _check_tensor(W, "W", torch.bfloat16)
    pitch, scale_pitch = _pitches(cols)
    codes, scales = _fp8((out_codes, out_scales), "out", rows, pitch, (rows + 127) // 128, scale_pitch, W)
    s = lib().roi_fp8_save_weight(W.data_ptr(), rows, cols, codes, scales, _stream(stream))
    if s != ROI_OK:
        _raise(s, "roi_fp8_save_weight")


def roi_fp8_linear_fwd(x8, format, w8, out_y, stream=None):
    """out_y[T, rows] = x w^T from the (codes, scales) pairs of an activation (`format`) and of a weight, of the same number of
    columns (which a copy holds to the next 128 only)."""
    ld = _stride(out_y, "out_y")
    T, rows = out_y.shape
    # padding codes are zeros, so the whole blocks stand for the columns
    cols, scale_pitch = _pitches(w8[0].shape[1])
    xq, xs = _fp8(x8, "x8", T, cols, T, scale_pitch, out_y)
    wq, ws = _fp8(w8, "w8", rows, cols, (rows + 127) // 128, scale_pitch, out_y)
    s = lib().roi_fp8_linear_fwd(xq, xs, _format(format), wq, ws, T, rows, cols, out_y.data_ptr(), _type(out_y, "out_y"), ld,
                                 _stream(stream))
    if s != ROI_OK:
        _raise(s, "roi_fp8_linear_fwd")


def roi_fp8_linear_dgrad(dy8, format, w8, out_dx, stream=None):
    """out_dx[T, cols] = dy w, from the (codes, scales) pairs of dy [T, rows] (`format`; it holds its columns to the next 128
    only) and of the weight [rows, cols]."""
    ld = _stride(out_dx, "out_dx")
    T, cols = out_dx.shape
    rows = w8[0].shape[0]
    pitch, scale_pitch = _pitches(rows)
    dq, ds = _fp8(dy8, "dy8", T, pitch, T, scale_pitch, out_dx)
    pitch, scale_pitch = _pitches(cols)
    wq, ws = _fp8(w8, "w8", rows, pitch, (rows + 127) // 128, scale_pitch, out_dx)
    s = lib().roi_fp8_linear_dgrad(dq, ds, _format(format), wq, ws, T, rows, cols, out_dx.data_ptr(), _type(out_dx, "out_dx"), ld,
                                   _stream(stream))
    if s != ROI_OK:
        _raise(s, "roi_fp8_linear_dgrad")


# ---------------------------------------------------------------------------
# the AdamW step over many tensors
# ---------------------------------------------------------------------------
def _half(t, name, shape):
    """Type code of a copy in 16 bits (None: none)."""
    if t is None:
        return 0
    code = _type(t, name)
    if code == 2:
        raise TypeError(f"{name}: expected bfloat16 or float16, got {t.dtype}")
    _check_tensor(t, name, t.dtype, shape)
    return code


def _same_size(t, name, dtype, n):
    _check_tensor(t, name, dtype)
    if t.numel() != n:
        raise ValueError(f"{name}: expected {n} elements, got {t.numel()}")


def _device(tensors, name, first=None):
    """The one device of a call's tensors, of which those before lie on `first`."""
    for t in tensors:
        if t is not None:
            first = t.device if first is None else first
            if t.device != first:
                raise ValueError(f"{name}: tensors on {first} and on {t.device}")
    return first


def make_adamw_step_items(items):
    """ctypes array of AdamWStepItem from (param, grad, m, v, copy) tuples: tensors of any shape, copy (bfloat16 or
    float16) or None."""
    import torch
    arr, device = (AdamWStepItem * len(items))(), None
    for k, (param, grad, m, v, copy) in enumerate(items):
        shape = param.shape
        _check_tensor(param, "param", torch.float32)
        code = _type(grad, "grad")
        _check_tensor(grad, "grad", grad.dtype, shape)
        _check_tensor(m, "m", torch.float32, shape)
        _check_tensor(v, "v", torch.float32, shape)
        half = _half(copy, "copy", shape)
        device = _device((param, grad, m, v, copy), f"item {k}", device)
        arr[k] = AdamWStepItem(_addr(param), _addr(grad), _addr(m), _addr(v), _addr(copy), param.numel(), code, half)
    arr.device = device
    return arr


def new_adamw_state8(n, device="cuda"):
    """State in 8 bits before the first step of a tensor of n elements: (codes of m, codes of sqrt(v), scales)."""
    import torch
    blocks = (int(n) + 127) // 128
    return tuple(torch.zeros(s, dtype=torch.uint8, device=device) for s in ((blocks * 128,), (blocks * 128,), (blocks, 2)))


def _state8(state, n):
    import torch
    m, u, s = state
    blocks = (n + 127) // 128
    _check_tensor(m, "state's m", torch.uint8, (blocks * 128,))
    _check_tensor(u, "state's u", torch.uint8, (blocks * 128,))
    _check_tensor(s, "state's scales", torch.uint8, (blocks, 2))
    return m.data_ptr(), u.data_ptr(), s.data_ptr()


def make_adamw_step8_items(items):
    """ctypes array of AdamWStep8Item from (param, grad, state, copy, tensor_id) tuples, state as from new_adamw_state8."""
    import torch
    arr, device = (AdamWStep8Item * len(items))(), None
    for k, (param, grad, state, copy, tensor_id) in enumerate(items):
        shape = param.shape
        _check_tensor(param, "param", torch.float32)
        code = _type(grad, "grad")
        _check_tensor(grad, "grad", grad.dtype, shape)
        half = _half(copy, "copy", shape)
        n = param.numel()
        at = _state8(state, n)
        device = _device((param, grad, *state, copy), f"item {k}", device)
        arr[k] = AdamWStep8Item(_addr(param), _addr(grad), *at, _addr(copy), n, code, half, int(tensor_id))
    arr.device = device
    return arr


def make_adamw_state8_items(items):
    """ctypes array of AdamWState8Item from (state, out_m, out_u) tuples: tensors of one type, one of them or None."""
    arr, device = (AdamWState8Item * len(items))(), None
    for k, (state, out_m, out_u) in enumerate(items):
        like = out_m if out_m is not None else out_u
        if like is None:
            raise ValueError("out_m or out_u: a tensor is required")
        code, n = _type(like, "out_m"), like.numel()
        for t, name in ((out_m, "out_m"), (out_u, "out_u")):
            if t is not None:
                _same_size(t, name, like.dtype, n)
        at = _state8(state, n)
        device = _device((*state, out_m, out_u), f"item {k}", device)
        arr[k] = AdamWState8Item(*at, _addr(out_m), _addr(out_u), n, code)
    return arr


def _grad_scale(t, items):
    if t is None:
        return None
    import torch
    _same_size(t, "grad_scale", torch.float32, 1)
    _device((t,), "grad_scale", getattr(items, "device", None))
    return t.data_ptr()


def roi_adamw_step(items, opt: AdamW, grad_scale=None, stream=None):
    """One AdamW step of many tensors in place (an AdamWStepItem array from make_adamw_step_items, reusable while its
    tensors live, or a list of (param, grad, m, v, copy) tuples).  grad_scale: float32 [1] on the device, or None."""
    arr = items if isinstance(items, ctypes.Array) else make_adamw_step_items(items)
    s = lib().roi_adamw_step(arr, len(arr), ctypes.byref(opt), _grad_scale(grad_scale, arr), _stream(stream))
    _raise(s, "roi_adamw_step")


def roi_adamw_step8(items, opt: AdamW, seed, grad_scale=None, stream=None):
    """roi_adamw_step with states in 8 bits, rounded by the noise of (seed, opt.t, tensor_id) (an AdamWStep8Item array
    from make_adamw_step8_items, or a list of (param, grad, state, copy, tensor_id) tuples).  The seed is not one of the
    masks' NoiseState: the same words would round the moments and draw a mask."""
    arr = items if isinstance(items, ctypes.Array) else make_adamw_step8_items(items)
    s = lib().roi_adamw_step8(arr, len(arr), ctypes.byref(opt), int(seed), _grad_scale(grad_scale, arr), _stream(stream))
    _raise(s, "roi_adamw_step8")


def roi_adamw_state8_load(items, stream=None):
    """m and sqrt(v) of states in 8 bits (an AdamWState8Item array from make_adamw_state8_items, or a list of
    (state, out_m, out_u) tuples)."""
    arr = items if isinstance(items, ctypes.Array) else make_adamw_state8_items(items)
    _raise(lib().roi_adamw_state8_load(arr, len(arr), _stream(stream)), "roi_adamw_state8_load")


def roi_noise_words(state: NoiseState, rows, cols, out_words, stream=None):
    """Philox words of every element of a [rows, cols] call (int32 tensor of rows*cols)."""
    import torch
    _check_tensor(out_words, "out_words", torch.int32, (rows * cols,))
    st = state if isinstance(state, NoiseState) else NoiseState(*state)
    _raise(lib().roi_noise_words(ctypes.byref(st), rows, cols, _ptr(out_words), _stream(stream)), "roi_noise_words")


def roi_gumbel_noise(state: NoiseState, rows, cols, out_g, stream=None):
    """Gumbel noise of every element of a [rows, cols] call (float32 tensor of rows*cols)."""
    import torch
    _check_tensor(out_g, "out_g", torch.float32, (rows * cols,))
    st = state if isinstance(state, NoiseState) else NoiseState(*state)
    _raise(lib().roi_gumbel_noise(ctypes.byref(st), rows, cols, _ptr(out_g), _stream(stream)), "roi_gumbel_noise")


def roi_device_status(stream=None):
    """Synchronises the stream; raises RoiError if a kernel timed out or CUDA failed."""
    _raise(lib().roi_device_status(_stream(stream)), "roi_device_status")


ROI_DEFAULT_RING_WAIT_NS = 2_000_000_000


def roi_set_ring_wait_limit_ns(ns: int):
    """Wall-time limit (ns) of the kernels' waits for their staged copies on the
    current device; 0 gives up at once when a stage has not landed (tests)."""
    _raise(lib().roi_set_ring_wait_limit_ns(int(ns)), "roi_set_ring_wait_limit_ns")
