"""ctypes binding of libquan (include/quan.h).  Argument marshalling only: every
arithmetic step runs in the library's CUDA kernels.  Tensor arguments may be torch
tensors (their device pointer is passed), integer device addresses, or None.

The library must have been built (``paper_2509_05512_gb300.build.build_library()``);
there is no fallback implementation, and a missing library raises immediately.
"""
from __future__ import annotations

import ctypes
import os
import re
import struct
import threading
import typing

PKG_DIR = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(PKG_DIR, "libquan.so")
HEADER = os.path.join(os.path.dirname(PKG_DIR), "include", "quan.h")

QUAN_OK, QUAN_ERR_INVALID_ARG, QUAN_ERR_UNSUPPORTED, QUAN_ERR_CUDA, QUAN_ERR_DEVICE_TIMEOUT = range(5)
QUAN_ACT_NONE, QUAN_ACT_RELU, QUAN_ACT_SILU = 0, 1, 2
QUAN_PATH_AUTO, QUAN_PATH_TC, QUAN_PATH_SIMT = 0, 1, 2
QUAN_DTYPE_BF16, QUAN_DTYPE_F32 = 0, 1

_lock = threading.Lock()
_lib = None

_vp = ctypes.c_void_p
_i = ctypes.c_int
_conv_args = [_vp] * 8 + [_i] * 10


class QuanError(RuntimeError):
    def __init__(self, status: int, message: str):
        super().__init__("%s: %s" % (_status_name(status), message))
        self.status = status


def _status_name(st: int) -> str:
    names = ["QUAN_OK", "QUAN_ERR_INVALID_ARG", "QUAN_ERR_UNSUPPORTED", "QUAN_ERR_CUDA",
             "QUAN_ERR_DEVICE_TIMEOUT"]
    return names[st] if 0 <= st < len(names) else "QUAN_ERR_%d" % st


def header_functions() -> list:
    """Names of the functions include/quan.h declares."""
    with open(HEADER) as f:
        text = f.read()
    text = re.sub(r"/\*.*?\*/", "", text, flags=re.S)
    return sorted(set(re.findall(r"\b(quan_[a-z0-9_]+)\s*\(", text)))


def load():
    """Load libquan.so (raises if it has not been built)."""
    global _lib
    with _lock:
        if _lib is not None:
            return _lib
        if not os.path.exists(LIB_PATH):
            raise RuntimeError("libquan.so is not built; run "
                               "paper_2509_05512_gb300.build.build_library() first")
        lib = ctypes.CDLL(LIB_PATH)
        lib.quan_qconv2d_fwd.argtypes = _conv_args + [_vp, _vp]
        lib.quan_qconv2d_fwd_f32.argtypes = _conv_args + [_vp, _vp]
        lib.quan_qconv2d_fwd_res.argtypes = _conv_args + [_vp, _vp, _vp]
        lib.quan_qconv2d_fwd_ex.argtypes = _conv_args + [_vp, _vp, ctypes.c_size_t, _vp, _vp]
        lib.quan_qconv2d_fwd_shortcut.argtypes = (_conv_args + [_vp] * 7 + [_i, _i] +
                                                  [_vp, _vp, _vp])
        lib.quan_qconv2d_fwd_workspace_size.argtypes = []
        lib.quan_qconv2d_fwd_workspace_size.restype = ctypes.c_size_t
        lib.quan_qconv2d_sep_fwd.argtypes = _conv_args + [_vp, _vp]
        lib.quan_maxpool2d_fwd.argtypes = [_vp] + [_i] * 7 + [_vp, _vp]
        lib.quan_poincare_fwd.argtypes = [_vp, ctypes.c_longlong, _vp, _vp]
        _bwd_data_args = [_vp] * 5 + [_i] * 9 + [_vp, ctypes.c_size_t, _vp, _vp]
        lib.quan_qconv2d_bwd_data.argtypes = _bwd_data_args
        lib.quan_qconv2d_sep_bwd_data.argtypes = _bwd_data_args
        lib.quan_qconv2d_maxpool_fwd.argtypes = _conv_args + [_vp, ctypes.c_size_t, _vp, _vp]
        lib.quan_qconv2d_maxpool_rgb_fwd.argtypes = [_vp] * 8 + [_i] * 9 + [_vp, _vp]
        lib.quan_qconv2d_maxpool_workspace_size.argtypes = [_i] * 8
        lib.quan_qconv2d_maxpool_workspace_size.restype = ctypes.c_size_t
        lib.quan_iqbn_batch_stats.argtypes = [_vp, ctypes.c_longlong, _i, _vp, ctypes.c_size_t,
                                              _vp, _vp, _vp]
        lib.quan_iqbn_batch_stats_workspace_size.argtypes = [_i]
        lib.quan_iqbn_batch_stats_workspace_size.restype = ctypes.c_size_t
        lib.quan_iqbn_train_fwd.argtypes = ([_vp, ctypes.c_longlong, _i] + [_vp] * 4 +
                                            [ctypes.c_float, _i, _vp, _vp])
        lib.quan_qconv2d_bwd_data_static.argtypes = [_vp] * 5 + [_i] * 9 + [_vp, _vp]
        lib.quan_qconv2d_bwd_data_workspace_size.argtypes = [_i] * 4
        lib.quan_qconv2d_bwd_data_workspace_size.restype = ctypes.c_size_t
        lib.quan_qconv2d_bwd_data_workspace_size_ex.argtypes = [_i] * 9
        lib.quan_qconv2d_bwd_data_workspace_size_ex.restype = ctypes.c_size_t
        _bwd_weight_args = [_vp] * 2 + [_i] * 9 + [_vp] * 5
        lib.quan_qconv2d_bwd_weight.argtypes = _bwd_weight_args
        lib.quan_qconv2d_sep_bwd_weight.argtypes = _bwd_weight_args
        _ull, _ll, _f = ctypes.c_ulonglong, ctypes.c_longlong, ctypes.c_float
        lib.quan_dropout.argtypes = [_vp, _ll, _i, _f, _ull, _ull, _vp, _vp, _vp]
        _join_args = [_vp] * 3 + [_ll, _i, _i, _ll, _i, _f, _f, _f, _ull, _ull, _vp]
        lib.quan_residual_join_fwd.argtypes = [_vp] * 2 + _join_args + [_vp] * 3
        lib.quan_residual_join_bwd.argtypes = ([_vp] * 4 + _join_args + [_vp, ctypes.c_size_t] +
                                               [_vp] * 6)
        lib.quan_residual_join_bwd_workspace_size.argtypes = [_ll, _i, _i, _ll]
        lib.quan_residual_join_bwd_workspace_size.restype = ctypes.c_size_t
        lib.quan_f8_weights.argtypes = [_vp] * 4 + [_i, _i, _i, _vp, _vp, _vp]
        lib.quan_f8_weights_bytes.argtypes = [_i, _i, _i]
        lib.quan_f8_weights_bytes.restype = ctypes.c_size_t
        lib.quan_qpoint_f8_fwd.argtypes = ([_vp] * 6 + [_ll, _i, _i, _i, _vp, ctypes.c_size_t] +
                                           [_vp] * 2)
        lib.quan_qpoint_f8_bwd_data.argtypes = ([_vp] * 3 + [_ll, _i, _i, _vp, ctypes.c_size_t] +
                                                [_vp] * 2)
        lib.quan_qpoint_f8_workspace_size.argtypes = [_ll, _i, _i]
        lib.quan_qpoint_f8_workspace_size.restype = ctypes.c_size_t
        lib.quan_residual_join_f8_fwd.argtypes = [_vp] * 2 + _join_args + [_vp] * 5
        lib.quan_f8_rows_bytes.argtypes = [_ll, _i]
        lib.quan_f8_rows_bytes.restype = ctypes.c_size_t
        lib.quan_f8_rows_scales.argtypes = [_ll, _i]
        lib.quan_f8_rows_scales.restype = ctypes.c_size_t
        lib.quan_f8_rows_dequant.argtypes = [_vp] * 2 + [_ll, _i] + [_vp] * 2
        lib.quan_qpoint_f8_rows_fwd.argtypes = [_vp] * 7 + [_ll, _i, _i, _i] + [_vp] * 2
        lib.quan_w4_weights_bytes.argtypes = [_i] * 2
        lib.quan_w4_weights_bytes.restype = ctypes.c_size_t
        lib.quan_w4_weights_scales.argtypes = [_i] * 3
        lib.quan_w4_weights_scales.restype = ctypes.c_size_t
        lib.quan_w4_weights.argtypes = [_vp] * 4 + [_i] * 3 + [_vp] * 3
        lib.quan_qpoint_w4_fwd.argtypes = [_vp] * 6 + [_ll] + [_i] * 4 + [_vp] * 2
        _distill_sizes = [_ll] + [_i] * 6 + [_f]
        lib.quan_distill_fwd.argtypes = [_vp] * 3 + _distill_sizes + [_vp] * 3
        lib.quan_distill_bwd.argtypes = [_vp] * 5 + _distill_sizes + [_f] + [_vp] * 2
        lib.quan_distill_fwd_bwd.argtypes = [_vp] * 4 + _distill_sizes + [_f] + [_vp] * 3
        lib.quan_set_path.argtypes = [_i]
        lib.quan_last_path.argtypes = []
        lib.quan_last_kernel.argtypes = []
        lib.quan_last_kernel.restype = ctypes.c_char_p
        lib.quan_set_tc_tiles.argtypes = [_i, _i, _i, _i]
        lib.quan_set_wait_limit_ns.argtypes = [ctypes.c_ulonglong]
        lib.quan_set_tc_halo.argtypes = [_i]
        lib.quan_set_tc_issuers.argtypes = [_i]
        lib.quan_set_tc_band_rows.argtypes = [_i]
        lib.quan_device_status.argtypes = [_vp, ctypes.POINTER(ctypes.c_uint)]
        lib.quan_set_fault_injection.argtypes = [_i]
        lib.quan_status_string.argtypes = [_i]
        lib.quan_status_string.restype = ctypes.c_char_p
        lib.quan_last_error_message.argtypes = []
        lib.quan_last_error_message.restype = ctypes.c_char_p
        lib.quan_version.argtypes = []
        lib.quan_last_variant.argtypes = []
        lib.quan_last_variant.restype = ctypes.c_char_p
        lib.quan_packed_call.argtypes = [_i, ctypes.c_char_p]
        lib.quan_packed_call.restype = _i
        lib.quan_packed_bwd_workspace.argtypes = [ctypes.c_char_p]
        lib.quan_packed_bwd_workspace.restype = ctypes.c_size_t
        for name in ("quan_qconv2d_fwd", "quan_qconv2d_fwd_f32", "quan_qconv2d_fwd_res",
                     "quan_qconv2d_fwd_ex", "quan_qconv2d_fwd_shortcut",
                     "quan_qconv2d_sep_fwd", "quan_poincare_fwd", "quan_qconv2d_bwd_data",
                     "quan_qconv2d_sep_bwd_data", "quan_qconv2d_bwd_weight",
                     "quan_qconv2d_bwd_data_static", "quan_iqbn_batch_stats",
                     "quan_qconv2d_maxpool_fwd", "quan_qconv2d_maxpool_rgb_fwd",
                     "quan_iqbn_train_fwd", "quan_dropout", "quan_residual_join_fwd",
                     "quan_residual_join_bwd", "quan_f8_weights", "quan_qpoint_f8_fwd",
                     "quan_qpoint_f8_bwd_data", "quan_distill_fwd", "quan_distill_bwd",
                     "quan_distill_fwd_bwd", "quan_residual_join_f8_fwd", "quan_f8_rows_dequant",
                     "quan_qpoint_f8_rows_fwd", "quan_w4_weights", "quan_qpoint_w4_fwd",
                     "quan_qconv2d_sep_bwd_weight",
                     "quan_maxpool2d_fwd", "quan_set_path", "quan_set_tc_tiles",
                     "quan_set_wait_limit_ns", "quan_device_status", "quan_set_fault_injection",
                     "quan_set_tc_halo", "quan_set_tc_issuers", "quan_set_tc_band_rows"):
            getattr(lib, name).restype = _i
        lib.quan_last_path.restype = _i
        lib.quan_version.restype = _i
        _lib = lib
        return lib


def _ptr(t):
    if t is None:
        return None
    if isinstance(t, int):
        return t
    return t.data_ptr()


def _addr(t):
    """_ptr as an integer (None: 0)."""
    if t is None:
        return 0
    if t.__class__ is int:
        return t
    try:
        return t.data_ptr()
    except AttributeError:
        if isinstance(t, int):
            return t
        raise


_raw_stream = None


def _stream(stream, dev=None):
    """The handle of a stream; None: the current one of device `dev` (None: the current one)."""
    global _raw_stream
    if stream is None:
        # the handle of torch.cuda.current_stream() without building the Stream object
        # (0.4 us against 3)
        if dev is None or _raw_stream is None:
            import torch
            if _raw_stream is None:
                _raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (
                    lambda device: torch.cuda.current_stream(device).cuda_stream)
            if dev is None:
                dev = torch.cuda.current_device()
        return _raw_stream(dev)
    if isinstance(stream, int):
        return stream
    return stream.cuda_stream


# Packed calls (csrc/packed.cu): entry point number and the layout of its arguments, every
# integer and pointer a 64-bit word, in the order of the C function's.
_CONV = struct.Struct("20q").pack           # x, 4 letters, 3 vectors, 10 sizes, out, stream
_CONV_RES = struct.Struct("21q").pack
_CONV_EX = struct.Struct("23q").pack
_CONV_WS = struct.Struct("22q").pack
_CONV_RGB = struct.Struct("19q").pack
_BWD_DATA = struct.Struct("18q").pack
_BWD_WEIGHT = struct.Struct("16q").pack
_STATS = struct.Struct("8q").pack
_TRAIN = struct.Struct("7qd3q").pack
_SIZES = struct.Struct("9q").pack
_DROPOUT = struct.Struct("3qd2Q3q").pack
_JOIN_FWD = struct.Struct("10q3d2Q4q").pack
_QPOINT_F8 = struct.Struct("14q").pack
_QPOINT_F8_BWD = struct.Struct("10q").pack
_JOIN_BWD = struct.Struct("12q3d2Q9q").pack
_JOIN_F8 = struct.Struct("10q3d2Q6q").pack
_F8_ROWS = struct.Struct("6q").pack
_QPOINT_F8_ROWS = struct.Struct("13q").pack
_QPOINT_W4 = struct.Struct("13q").pack
_DISTILL_FWD = struct.Struct("10qd3q").pack
_DISTILL_BWD = struct.Struct("10q2d4q").pack


def _call(op: int, words: bytes) -> None:
    lib = _lib if _lib is not None else load()
    st = lib.quan_packed_call(op, words)
    if st != QUAN_OK:
        _check(st)


def _check(st: int):
    if st != QUAN_OK:
        msg = load().quan_last_error_message().decode(errors="replace")
        raise QuanError(st, msg)


def quan_qconv2d_fwd(x, wr, wi, wj, wk, bias, iqbn_scale, iqbn_shift, N, H, W, Cin, Cout, kh, kw,
                     stride, pad, act, out, stream=None) -> None:
    _call(0, _CONV(_addr(x), _addr(wr), _addr(wi), _addr(wj), _addr(wk), _addr(bias),
                   _addr(iqbn_scale), _addr(iqbn_shift), N, H, W, Cin, Cout, kh, kw, stride, pad,
                   act, _addr(out), _stream(stream)))


def quan_qconv2d_fwd_f32(x, wr, wi, wj, wk, bias, iqbn_scale, iqbn_shift, N, H, W, Cin, Cout, kh,
                         kw, stride, pad, act, out, stream=None) -> None:
    _call(1, _CONV(_addr(x), _addr(wr), _addr(wi), _addr(wj), _addr(wk), _addr(bias),
                   _addr(iqbn_scale), _addr(iqbn_shift), N, H, W, Cin, Cout, kh, kw, stride, pad,
                   act, _addr(out), _stream(stream)))


def quan_qconv2d_fwd_res(x, wr, wi, wj, wk, bias, iqbn_scale, iqbn_shift, N, H, W, Cin, Cout, kh,
                         kw, stride, pad, act, residual, out, stream=None) -> None:
    _call(2, _CONV_RES(_addr(x), _addr(wr), _addr(wi), _addr(wj), _addr(wk), _addr(bias),
                   _addr(iqbn_scale), _addr(iqbn_shift), N, H, W, Cin, Cout, kh, kw, stride, pad,
                   act, _addr(residual), _addr(out), _stream(stream)))


def quan_qconv2d_fwd_ex(x, wr, wi, wj, wk, bias, iqbn_scale, iqbn_shift, N, H, W, Cin, Cout, kh,
                        kw, stride, pad, act, residual, workspace, workspace_bytes, out,
                        stream=None) -> None:
    _call(3, _CONV_EX(_addr(x), _addr(wr), _addr(wi), _addr(wj), _addr(wk), _addr(bias),
                   _addr(iqbn_scale), _addr(iqbn_shift), N, H, W, Cin, Cout, kh, kw, stride, pad,
                   act, _addr(residual), _addr(workspace), workspace_bytes,
                   _addr(out), _stream(stream)))


def quan_qconv2d_fwd_shortcut(x, wr, wi, wj, wk, bias, iqbn_scale, iqbn_shift, N, H, W, Cin,
                              Cout, kh, kw, stride, pad, act, sc_wr, sc_wi, sc_wj, sc_wk,
                              sc_bias, sc_iqbn_scale, sc_iqbn_shift, Cout_sc, sc_act, out,
                              out_sc, stream=None) -> None:
    _check(load().quan_qconv2d_fwd_shortcut(
        _ptr(x), _ptr(wr), _ptr(wi), _ptr(wj), _ptr(wk), _ptr(bias), _ptr(iqbn_scale),
        _ptr(iqbn_shift), N, H, W, Cin, Cout, kh, kw, stride, pad, act, _ptr(sc_wr),
        _ptr(sc_wi), _ptr(sc_wj), _ptr(sc_wk), _ptr(sc_bias), _ptr(sc_iqbn_scale),
        _ptr(sc_iqbn_shift), Cout_sc, sc_act, _ptr(out), _ptr(out_sc), _stream(stream)))


def qconv2d_shortcut(x, w, sc_w, *, stride=2, pad=1, bias=None, scale=None, shift=None,
                     act=QUAN_ACT_NONE, sc_bias=None, sc_scale=None, sc_shift=None,
                     sc_act=QUAN_ACT_NONE, out=None, out_sc=None, stream=None):
    """A convolution (letters w = (wr, wi, wj, wk)) and the 1x1 shortcut of the same input
    (letters sc_w, same stride, no padding) in one call: returns (out, out_sc), allocated
    like qconv2d's when not given (bf16 CUDA tensors)."""
    import torch
    N, H, W, Cin = x.shape
    Qout, kh, kw, _ = w[0].shape
    Cout, Cout_sc = 4 * Qout, 4 * sc_w[0].shape[0]
    Ho, Wo = out_size(H, kh, stride, pad), out_size(W, kw, stride, pad)
    if out is None:
        out = torch.empty((N, Ho, Wo, Cout), dtype=x.dtype, device=x.device)
    if out_sc is None:
        out_sc = torch.empty((N, Ho, Wo, Cout_sc), dtype=x.dtype, device=x.device)
    quan_qconv2d_fwd_shortcut(x, *w, bias, scale, shift, N, H, W, Cin, Cout, kh, kw, stride, pad,
                              act, *sc_w, sc_bias, sc_scale, sc_shift, Cout_sc, sc_act, out,
                              out_sc, stream)
    return out, out_sc


def quan_qconv2d_fwd_workspace_size() -> int:
    return int(load().quan_qconv2d_fwd_workspace_size())


def fwd_workspace(device=None):
    """A zero-filled workspace (uint8 CUDA tensor) for quan_qconv2d_fwd_ex."""
    import torch
    return torch.zeros(quan_qconv2d_fwd_workspace_size(), dtype=torch.uint8,
                       device=device or "cuda")


def quan_maxpool2d_fwd(x, N, H, W, C, k, stride, pad, out, stream=None) -> None:
    _check(load().quan_maxpool2d_fwd(_ptr(x), N, H, W, C, k, stride, pad, _ptr(out),
                                     _stream(stream)))


def quan_set_path(path: int) -> None:
    _check(load().quan_set_path(path))


def quan_last_path() -> int:
    return load().quan_last_path()


def quan_last_kernel() -> str:
    return load().quan_last_kernel().decode()


def quan_set_tc_tiles(kappa: int = 0, bnq: int = 0, max_ctas: int = 0, mode: int = 0) -> None:
    _check(load().quan_set_tc_tiles(kappa, bnq, max_ctas, mode))


def quan_set_tc_halo(enable: bool) -> None:
    _check(load().quan_set_tc_halo(1 if enable else 0))


def quan_set_tc_issuers(issuers: int = 0) -> None:
    _check(load().quan_set_tc_issuers(issuers))


def quan_set_tc_band_rows(rows: int = 0) -> None:
    _check(load().quan_set_tc_band_rows(rows))


def quan_set_wait_limit_ns(ns: int) -> None:
    _check(load().quan_set_wait_limit_ns(ns))


def quan_set_fault_injection(enable: bool) -> None:
    _check(load().quan_set_fault_injection(1 if enable else 0))


def quan_device_status(stream=None) -> tuple:
    """Returns (status, bits); does not raise on QUAN_ERR_DEVICE_TIMEOUT."""
    bits = ctypes.c_uint(0)
    st = load().quan_device_status(_stream(stream), ctypes.byref(bits))
    if st not in (QUAN_OK, QUAN_ERR_DEVICE_TIMEOUT):
        _check(st)
    return st, bits.value


def quan_status_string(status: int) -> str:
    return load().quan_status_string(status).decode()


def quan_version() -> int:
    return load().quan_version()


def quan_qconv2d_sep_fwd(x, wr, wi, wj, wk, bias, iqbn_scale, iqbn_shift, N, H, W, Cin, Cout, kh,
                         kw, stride, pad, act, out, stream=None) -> None:
    _call(4, _CONV(_addr(x), _addr(wr), _addr(wi), _addr(wj), _addr(wk), _addr(bias),
                   _addr(iqbn_scale), _addr(iqbn_shift), N, H, W, Cin, Cout, kh, kw, stride, pad,
                   act, _addr(out), _stream(stream)))


# ------------------------------------------------------------------ tensor helpers

def out_size(n: int, k: int, stride: int, pad: int) -> int:
    return (n + 2 * pad - k) // stride + 1


def qconv2d(x, wr, wi, wj, wk, *, stride=1, pad=0, bias=None, scale=None, shift=None,
            act=QUAN_ACT_NONE, residual=None, out=None, stream=None, separable=False,
            workspace=None):
    """Allocate the output (torch, same dtype/device as x) and run the convolution.
    x: [N, H, W, Cin] (bf16 or fp32, CUDA); w*: [Cout/4, kh, kw, Cin/4].  separable=True
    runs the separable form of Eq. 7 (bf16 only, no residual).  workspace (a zero-filled
    uint8 CUDA tensor, see fwd_workspace) runs the bf16 full form through
    quan_qconv2d_fwd_ex."""
    import torch
    N, H, W, Cin = x.shape
    Qout, kh, kw, _ = wr.shape
    Cout = 4 * Qout
    Ho, Wo = out_size(H, kh, stride, pad), out_size(W, kw, stride, pad)
    if out is None:
        out = torch.empty((N, Ho, Wo, Cout), dtype=x.dtype, device=x.device)
    if separable:
        if x.dtype != torch.bfloat16 or residual is not None:
            raise ValueError("the separable form takes bf16 tensors and no residual")
        quan_qconv2d_sep_fwd(x, wr, wi, wj, wk, bias, scale, shift, N, H, W, Cin, Cout, kh, kw,
                             stride, pad, act, out, stream)
    elif x.dtype == torch.float32:
        if residual is not None:
            raise ValueError("the fp32 entry point has no residual input")
        quan_qconv2d_fwd_f32(x, wr, wi, wj, wk, bias, scale, shift, N, H, W, Cin, Cout, kh, kw,
                             stride, pad, act, out, stream)
    elif workspace is not None:
        quan_qconv2d_fwd_ex(x, wr, wi, wj, wk, bias, scale, shift, N, H, W, Cin, Cout, kh, kw,
                            stride, pad, act, residual, workspace,
                            workspace.numel() * workspace.element_size(), out, stream)
    elif residual is not None:
        quan_qconv2d_fwd_res(x, wr, wi, wj, wk, bias, scale, shift, N, H, W, Cin, Cout, kh, kw,
                             stride, pad, act, residual, out, stream)
    else:
        quan_qconv2d_fwd(x, wr, wi, wj, wk, bias, scale, shift, N, H, W, Cin, Cout, kh, kw,
                         stride, pad, act, out, stream)
    return out


def quan_poincare_fwd(rgb, npix, out, stream=None) -> None:
    _check(load().quan_poincare_fwd(_ptr(rgb), npix, _ptr(out), _stream(stream)))


def poincare(rgb, *, out=None, stream=None):
    """Eq. 4 on the GPU: fp32 rgb [..., 3] (CUDA) -> bf16 quaternion pixels [..., 4]."""
    import torch
    if rgb.dtype != torch.float32 or rgb.shape[-1] != 3:
        raise ValueError("rgb must be float32 with a last dimension of 3")
    if out is None:
        out = torch.empty(rgb.shape[:-1] + (4,), dtype=torch.bfloat16, device=rgb.device)
    quan_poincare_fwd(rgb, rgb.numel() // 3, out, stream)
    return out


def quan_qconv2d_bwd_data_workspace_size(Cin, Cout, kh, kw) -> int:
    return load().quan_qconv2d_bwd_data_workspace_size(Cin, Cout, kh, kw)


def quan_qconv2d_bwd_data_workspace_size_ex(N, H, W, Cin, Cout, kh, kw, stride, pad) -> int:
    return load().quan_packed_bwd_workspace(_SIZES(N, H, W, Cin, Cout, kh, kw, stride, pad))


def quan_qconv2d_bwd_data(dy, wr, wi, wj, wk, N, H, W, Cin, Cout, kh, kw, stride, pad, workspace,
                          workspace_bytes, dx, stream=None) -> None:
    _call(5, _BWD_DATA(_addr(dy), _addr(wr), _addr(wi), _addr(wj), _addr(wk), N, H, W, Cin, Cout, kh,
                       kw, stride, pad, _addr(workspace), workspace_bytes, _addr(dx),
                       _stream(stream)))


def quan_qconv2d_bwd_data_static(dy, wr, wi, wj, wk, N, H, W, Cin, Cout, kh, kw, stride, pad,
                                 dx, stream=None) -> None:
    _check(load().quan_qconv2d_bwd_data_static(_ptr(dy), _ptr(wr), _ptr(wi), _ptr(wj),
                                               _ptr(wk), N, H, W, Cin, Cout, kh, kw, stride,
                                               pad, _ptr(dx), _stream(stream)))


def quan_qconv2d_sep_bwd_data(dy, wr, wi, wj, wk, N, H, W, Cin, Cout, kh, kw, stride, pad,
                              workspace, workspace_bytes, dx, stream=None) -> None:
    _call(6, _BWD_DATA(_addr(dy), _addr(wr), _addr(wi), _addr(wj), _addr(wk), N, H, W, Cin, Cout, kh,
                       kw, stride, pad, _addr(workspace), workspace_bytes, _addr(dx),
                       _stream(stream)))


def quan_qconv2d_bwd_weight(x, dy, N, H, W, Cin, Cout, kh, kw, stride, pad, dwr, dwi, dwj, dwk,
                            stream=None) -> None:
    _call(7, _BWD_WEIGHT(_addr(x), _addr(dy), N, H, W, Cin, Cout, kh, kw, stride, pad, _addr(dwr),
                         _addr(dwi), _addr(dwj), _addr(dwk), _stream(stream)))


def quan_qconv2d_sep_bwd_weight(x, dy, N, H, W, Cin, Cout, kh, kw, stride, pad, dwr, dwi, dwj,
                                dwk, stream=None) -> None:
    _call(8, _BWD_WEIGHT(_addr(x), _addr(dy), N, H, W, Cin, Cout, kh, kw, stride, pad, _addr(dwr),
                         _addr(dwi), _addr(dwj), _addr(dwk), _stream(stream)))


def qconv2d_backward_data(dy, wr, wi, wj, wk, *, H, W, stride=1, pad=0, separable=False,
                          workspace=None, out=None, stream=None):
    """Input gradient of the pre-epilogue convolution: dy [N, Ho, Wo, Cout] (bf16, CUDA) ->
    dx [N, H, W, Cin] bf16.  `workspace` (a uint8 CUDA tensor) is allocated when not given,
    with quan_qconv2d_bwd_data_workspace_size_ex bytes (the tensor-core path of strided
    layers included)."""
    import torch
    N, Ho, Wo, Cout = dy.shape
    Qout, kh, kw, Qin = wr.shape
    Cin = 4 * Qin
    need = quan_qconv2d_bwd_data_workspace_size_ex(N, H, W, Cin, Cout, kh, kw, stride, pad)
    if workspace is None:
        workspace = torch.empty(need, dtype=torch.uint8, device=dy.device)
    if out is None:
        out = torch.empty((N, H, W, Cin), dtype=torch.bfloat16, device=dy.device)
    fn = quan_qconv2d_sep_bwd_data if separable else quan_qconv2d_bwd_data
    fn(dy, wr, wi, wj, wk, N, H, W, Cin, Cout, kh, kw, stride, pad, workspace,
       workspace.numel() * workspace.element_size(), out, stream)
    return out


def qconv2d_backward_weight(x, dy, *, kh, kw, stride=1, pad=0, separable=False, out=None,
                            stream=None):
    """Weight gradients of the pre-epilogue convolution: x [N, H, W, Cin], dy
    [N, Ho, Wo, Cout] (bf16, CUDA) -> (dW_r, dW_i, dW_j, dW_k), fp32 [Cout/4, kh, kw, Cin/4]."""
    import torch
    N, H, W, Cin = x.shape
    Cout = dy.shape[-1]
    if out is None:
        out = tuple(torch.empty((Cout // 4, kh, kw, Cin // 4), dtype=torch.float32,
                                device=x.device) for _ in range(4))
    fn = quan_qconv2d_sep_bwd_weight if separable else quan_qconv2d_bwd_weight
    fn(x, dy, N, H, W, Cin, Cout, kh, kw, stride, pad, *out, stream)
    return out


def quan_qconv2d_maxpool_workspace_size(N, H, W, Cout, kh, kw, stride, pad) -> int:
    return load().quan_qconv2d_maxpool_workspace_size(N, H, W, Cout, kh, kw, stride, pad)


def quan_qconv2d_maxpool_rgb_fwd(rgb, wr, wi, wj, wk, bias, iqbn_scale, iqbn_shift, N, H, W,
                                 Cout, kh, kw, stride, pad, act, out, stream=None) -> None:
    _call(11, _CONV_RGB(_addr(rgb), _addr(wr), _addr(wi), _addr(wj), _addr(wk), _addr(bias),
                        _addr(iqbn_scale), _addr(iqbn_shift), N, H, W, Cout, kh, kw, stride,
                        pad, act, _addr(out), _stream(stream)))


def quan_qconv2d_maxpool_fwd(x, wr, wi, wj, wk, bias, iqbn_scale, iqbn_shift, N, H, W, Cin,
                             Cout, kh, kw, stride, pad, act, workspace, workspace_bytes, out,
                             stream=None) -> None:
    _call(12, _CONV_WS(_addr(x), _addr(wr), _addr(wi), _addr(wj), _addr(wk), _addr(bias),
                   _addr(iqbn_scale), _addr(iqbn_shift), N, H, W, Cin, Cout, kh, kw, stride, pad,
                   act, _addr(workspace), workspace_bytes, _addr(out),
                   _stream(stream)))


def quan_iqbn_batch_stats_workspace_size(C) -> int:
    return load().quan_iqbn_batch_stats_workspace_size(C)


def quan_iqbn_batch_stats(x, npix, C, workspace, workspace_bytes, mean, var,
                          stream=None) -> None:
    _call(9, _STATS(_addr(x), npix, C, _addr(workspace), workspace_bytes, _addr(mean),
                    _addr(var), _stream(stream)))


def quan_iqbn_train_fwd(x, npix, C, mean, var, gamma, beta, eps, act, out, stream=None) -> None:
    _call(10, _TRAIN(_addr(x), npix, C, _addr(mean), _addr(var), _addr(gamma), _addr(beta), eps,
                     act, _addr(out), _stream(stream)))


def iqbn_batch_stats(x, *, workspace=None, stream=None):
    """Eq. 11 on the GPU: bf16 x [..., C] (CUDA) -> (mean, biased var), fp32 [C] each.
    `workspace` (a CUDA tensor of at least quan_iqbn_batch_stats_workspace_size(C) bytes)
    is allocated when not given."""
    import torch
    C = x.shape[-1]
    if workspace is None:
        workspace = torch.empty(quan_iqbn_batch_stats_workspace_size(C), dtype=torch.uint8,
                                device=x.device)
    mean = torch.empty(C, dtype=torch.float32, device=x.device)
    var = torch.empty(C, dtype=torch.float32, device=x.device)
    quan_iqbn_batch_stats(x, x.numel() // C, C, workspace,
                          workspace.numel() * workspace.element_size(), mean, var, stream)
    return mean, var


def iqbn_train(x, gamma=None, beta=None, *, eps=1e-5, act=QUAN_ACT_NONE, out=None,
               stream=None):
    """Training-mode IQBN (Eq. 11-12) with the batch's statistics, then the activation:
    bf16 x [..., C] -> bf16, same shape; returns (out, mean, var)."""
    import torch
    mean, var = iqbn_batch_stats(x, stream=stream)
    if out is None:
        out = torch.empty_like(x)
    C = x.shape[-1]
    quan_iqbn_train_fwd(x, x.numel() // C, C, mean, var, gamma, beta, eps, act, out, stream)
    return out, mean, var


def maxpool2d(x, *, k=3, stride=2, pad=1, out=None, stream=None):
    import torch
    N, H, W, C = x.shape
    Ho, Wo = out_size(H, k, stride, pad), out_size(W, k, stride, pad)
    if out is None:
        out = torch.empty((N, Ho, Wo, C), dtype=x.dtype, device=x.device)
    quan_maxpool2d_fwd(x, N, H, W, C, k, stride, pad, out, stream)
    return out


# ------------------------------------------------------------------ residual blocks

def quan_dropout(x, n, dtype, p, seed, offset, counter, out, stream=None) -> None:
    _call(13, _DROPOUT(_addr(x), n, dtype, p, seed, offset, _addr(counter), _addr(out),
                       _stream(stream)))


def quan_residual_join_fwd(x, h, post, gate, pre, rows, C, groups, images, dtype, alpha, eps, p,
                           seed, offset, counter, y, n, stream=None) -> None:
    _call(14, _JOIN_FWD(_addr(x), _addr(h), _addr(post), _addr(gate), _addr(pre), rows, images, C,
                        groups, dtype, alpha, eps, p, seed, offset, _addr(counter), _addr(y),
                        _addr(n), _stream(stream)))


def quan_residual_join_bwd_workspace_size(rows, C, groups, images) -> int:
    return load().quan_residual_join_bwd_workspace_size(rows, C, groups, images)


def quan_residual_join_bwd(dy, dn, y, h, post, gate, pre, rows, C, groups, images, dtype, alpha,
                           eps, p, seed, offset, counter, workspace, workspace_bytes, dx, dh,
                           dpost, dgate, dpre, stream=None) -> None:
    _call(15, _JOIN_BWD(_addr(dy), _addr(dn), _addr(y), _addr(h), _addr(post), _addr(gate),
                        _addr(pre), rows, images, C, groups, dtype, alpha, eps, p, seed, offset,
                        _addr(counter), _addr(workspace), workspace_bytes, _addr(dx), _addr(dh),
                        _addr(dpost), _addr(dgate), _addr(dpre), _stream(stream)))


def _empty(stream, shape, dtype, device):
    """An empty tensor whose memory belongs to `stream` (None: the current one), so that the
    allocator hands it on only after that stream's work."""
    torch = _torch or _get_torch()
    if stream is None:
        return torch.empty(shape, dtype=dtype, device=device)
    if not isinstance(stream, int):
        s = stream
    elif stream == 0:  # (an ExternalStream of 0 is a new stream, not the default one)
        s = torch.cuda.default_stream(device)
    else:
        s = torch.cuda.ExternalStream(stream)
    with torch.cuda.stream(s):
        return torch.empty(shape, dtype=dtype, device=device)


def _device(name, t):
    """The device that a call's tensors have to be on: its first tensor's, which has to be the
    current one, for that is where the kernels are launched."""
    dev = t.get_device()
    if dev < 0:
        raise ValueError("%s must be a contiguous CUDA tensor (got one on %s)" % (name, t.device))
    current = (_torch or _get_torch()).cuda.current_device()
    if dev != current:
        raise ValueError("%s is on cuda:%d, but the current device is cuda:%d" % (name, dev,
                                                                                 current))
    return dev


def _check_tensor(name, t, shape, dtype, dev):
    if t.dtype is not dtype or t.shape != shape or t.get_device() != dev or \
            not t.is_contiguous():
        raise ValueError("%s must be a contiguous CUDA tensor %s of %s on cuda:%d (got %s of %s "
                         "on %s)" % (name, list(shape), dtype, dev, list(t.shape), t.dtype,
                                     t.device))


def _workspace_bytes(workspace, dev):
    """The bytes of a workspace that a caller gives."""
    if workspace.get_device() != dev or not workspace.is_contiguous():
        raise ValueError("workspace must be a contiguous CUDA tensor on cuda:%d" % dev)
    return workspace.numel() * workspace.element_size()


_torch = None


def _get_torch():
    global _torch
    if _torch is None:
        import torch
        _torch = torch
    return _torch


def _dtype_of(name, t):
    torch = _torch or _get_torch()
    if t.dtype is torch.bfloat16:
        return QUAN_DTYPE_BF16
    if t.dtype is torch.float32:
        return QUAN_DTYPE_F32
    raise ValueError("%s must be bfloat16 or float32 (got %s)" % (name, t.dtype))


def _check_counter(counter, dev):
    _check_tensor("counter", counter.reshape(-1), (1,), _get_torch().int64, dev)


def dropout(x, p, seed, offset=0, *, counter=None, out=None, stream=None):
    """Dropout of a bf16 or fp32 CUDA tensor with probability p in steps of 2^-16: kept elements
    are multiplied by 1 / (1 - p), the others become 0.  The mask is a function of seed, offset
    and the element's index and is never stored: the same call on the gradient is the backward
    pass.  A call uses ceil(n / 8) counters from `offset` on (plus the int64 CUDA scalar
    `counter`, read when the kernel runs), so calls of one seed take offsets that far apart.
    out may be x."""
    torch = _torch or _get_torch()
    t, shape = x.dtype, x.shape
    dtype = QUAN_DTYPE_BF16 if t is torch.bfloat16 else _dtype_of("x", x)
    dev = _device("x", x)
    if not x.is_contiguous():
        _check_tensor("x", x, shape, t, dev)
    if counter is not None:
        _check_counter(counter, dev)
    if out is not None:
        _check_tensor("out", out, shape, t, dev)
    else:
        out = _empty(stream, shape, t, x.device)
    _call(13, _DROPOUT(x.data_ptr(), x.numel(), dtype, p, seed, offset,
                       0 if counter is None else counter.data_ptr(), out.data_ptr(),
                       _stream(stream, dev)))
    return out


def quan_f8_weights(wr, wi, wj, wk, Cin, Cout, transpose, q, scale, stream=None) -> None:
    _check(load().quan_f8_weights(_ptr(wr), _ptr(wi), _ptr(wj), _ptr(wk), Cin, Cout,
                                  1 if transpose else 0, _ptr(q), _ptr(scale), _stream(stream)))


def quan_f8_weights_bytes(Cin, Cout, transpose) -> int:
    return load().quan_f8_weights_bytes(Cin, Cout, 1 if transpose else 0)


def quan_qpoint_f8_workspace_size(rows, Cin, Cout) -> int:
    return load().quan_qpoint_f8_workspace_size(rows, Cin, Cout)


def quan_qpoint_f8_fwd(x, wq, wscale, bias, iqbn_scale, iqbn_shift, rows, Cin, Cout, act,
                       workspace, workspace_bytes, out, stream=None) -> None:
    _call(16, _QPOINT_F8(_addr(x), _addr(wq), _addr(wscale), _addr(bias), _addr(iqbn_scale),
                         _addr(iqbn_shift), rows, Cin, Cout, act, _addr(workspace),
                         workspace_bytes, _addr(out), _stream(stream)))


def quan_qpoint_f8_bwd_data(dy, wq, wscale, rows, Cin, Cout, workspace, workspace_bytes, dx,
                            stream=None) -> None:
    _call(17, _QPOINT_F8_BWD(_addr(dy), _addr(wq), _addr(wscale), rows, Cin, Cout,
                             _addr(workspace), workspace_bytes, _addr(dx), _stream(stream)))


def quan_f8_rows_bytes(rows, C) -> int:
    return load().quan_f8_rows_bytes(rows, C)


def quan_f8_rows_scales(rows, C) -> int:
    return load().quan_f8_rows_scales(rows, C)


def quan_residual_join_f8_fwd(x, h, post, gate, pre, rows, C, groups, images, dtype, alpha, eps, p,
                              seed, offset, counter, y, n, q, scale, stream=None) -> None:
    _call(21, _JOIN_F8(_addr(x), _addr(h), _addr(post), _addr(gate), _addr(pre), rows, images, C,
                       groups, dtype, alpha, eps, p, seed, offset, _addr(counter), _addr(y),
                       _addr(n), _addr(q), _addr(scale), _stream(stream)))


def quan_f8_rows_dequant(q, scale, rows, C, out, stream=None) -> None:
    _call(22, _F8_ROWS(_addr(q), _addr(scale), rows, C, _addr(out), _stream(stream)))


def quan_qpoint_f8_rows_fwd(xq, xscale, wq, wscale, bias, iqbn_scale, iqbn_shift, rows, Cin, Cout,
                            act, out, stream=None) -> None:
    _call(23, _QPOINT_F8_ROWS(_addr(xq), _addr(xscale), _addr(wq), _addr(wscale), _addr(bias),
                              _addr(iqbn_scale), _addr(iqbn_shift), rows, Cin, Cout, act,
                              _addr(out), _stream(stream)))


class F8Rows(typing.NamedTuple):
    """Rows (pixels) in 8-bit floating point, as residual_join_f8 writes them: q e4m3
    [..., 4, pitch], scale fp32 [4, ceil(channels / 512), rows rounded up to 128]; component by
    component, pitch = channels / 4 rounded up to 16."""
    q: object
    scale: object
    channels: int


def _f8_rows(name, x, dev):
    """The leading shape and the number of 8-bit rows, which are looked at."""
    torch = _torch or _get_torch()
    q, scale, C = x
    if C % 4 or C < 4:
        raise ValueError("%s has %s channels, not a multiple of 4" % (name, C))
    lead, pitch = tuple(q.shape[:-2]), (C + 63) // 64 * 16
    if q.dtype is not torch.float8_e4m3fn or q.shape[-2:] != (4, pitch) or \
            not q.is_contiguous():
        _check_tensor(name + ".q", q, lead + (4, pitch), torch.float8_e4m3fn, dev)
    rows = q.numel() // (4 * pitch)
    want = (4, (C + 511) // 512, (rows + 127) // 128 * 128)
    if scale.dtype is not torch.float32 or scale.shape != want or scale.get_device() != dev or \
            not scale.is_contiguous():
        _check_tensor(name + ".scale", scale, want, torch.float32, dev)
    return lead, rows


def dequantize_f8_rows(x, *, out=None, stream=None):
    """F8Rows read back: bf16 [..., channels]."""
    bf16 = (_torch or _get_torch()).bfloat16
    dev = _device("x.q", x.q)
    lead, rows = _f8_rows("x", x, dev)
    shape = lead + (x.channels,)
    if out is None:
        out = _empty(stream, shape, bf16, x.q.device)
    else:
        _check_tensor("out", out, shape, bf16, dev)
    _call(22, _F8_ROWS(x.q.data_ptr(), x.scale.data_ptr(), rows, x.channels, out.data_ptr(),
                       _stream(stream, dev)))
    return out


class F8Weights(typing.NamedTuple):
    """Letters of a pointwise layer in 8-bit floating point, as quantize_f8_weights lays them
    out: q e4m3 [4, n, pitch], scale fp32 [4, ceil(n / 128), ceil(k / 128)]; n, k = Cout / 4,
    Cin / 4, or the other way round when transposed (for the input gradient)."""
    q: object
    scale: object
    Cin: int
    Cout: int
    transposed: bool


def quantize_f8_weights(wr, wi, wj, wk, *, transpose=False, stream=None):
    """The four letters [Cout/4, 1, 1, Cin/4] (bf16, CUDA) of a pointwise layer as F8Weights for
    qpointwise_f8, or with transpose=True for qpointwise_f8_backward_data: e4m3 with a
    power-of-two scale for each 128 x 128 block."""
    import torch
    Qout, kh, kw, Qin = wr.shape
    if kh != 1 or kw != 1:
        raise ValueError("the letters of a pointwise layer are [Cout/4, 1, 1, Cin/4]")
    dev = _device("wr", wr)
    for name, w in (("wr", wr), ("wi", wi), ("wj", wj), ("wk", wk)):
        _check_tensor(name, w, wr.shape, torch.bfloat16, dev)
    n, k = (Qin, Qout) if transpose else (Qout, Qin)
    if 4 * max(n, k) >= 1 << 31:  # (past the arguments' int; the library's own limit is lower)
        raise ValueError("a layer of %d -> %d channels is too large" % (4 * Qin, 4 * Qout))
    need = quan_f8_weights_bytes(4 * Qin, 4 * Qout, transpose)
    if need == 0:
        raise ValueError("a layer has at least four input and output channels")
    q = _empty(stream, (4, n, need // (4 * n)), torch.float8_e4m3fn, wr.device)
    scale = _empty(stream, (4, -(-n // 128), -(-k // 128)), torch.float32, wr.device)
    quan_f8_weights(wr, wi, wj, wk, 4 * Qin, 4 * Qout, transpose, q, scale, stream)
    return F8Weights(q, scale, 4 * Qin, 4 * Qout, bool(transpose))


def _qpoint_f8(x, q, scale, K, N, workspace, out, stream, dev):
    """rows, workspace, its bytes and the output of one 8-bit product of K input and N output
    channels with the letters q, scale, which are looked at too."""
    torch = _torch or _get_torch()
    shape, bf16 = tuple(x.shape), torch.bfloat16  # (torch.empty takes a tuple 1 us faster)
    if x.dtype is not bf16 or shape[-1] != K or not x.is_contiguous():
        _check_tensor("x", x, shape[:-1] + (K,), bf16, dev)
    _f8_letters(q, scale, K, N, dev)
    rows = x.numel() // K
    shape = shape[:-1] + (N,)
    if out is None:
        out = _empty(stream, shape, bf16, x.device)
    else:
        _check_tensor("out", out, shape, bf16, dev)
    if workspace is not None:
        return rows, workspace, _workspace_bytes(workspace, dev), out
    nbytes = (_lib or load()).quan_qpoint_f8_workspace_size(rows, K, N)
    if nbytes:
        workspace = _empty(stream, nbytes, torch.uint8, x.device)
    return rows, workspace, nbytes, out


def _f8_letters(q, scale, K, N, dev):
    """Looks at the letters of an 8-bit product of K input and N output channels."""
    torch = _torch or _get_torch()
    # (pitch K / 4 rounded up to 16, a scale for each 128 x 128)
    blocks = ((N + 511) // 512, (K + 511) // 512)
    if q.numel() != N * 16 * ((K + 63) // 64) or q.dtype is not torch.float8_e4m3fn or \
            q.get_device() != dev or not q.is_contiguous():
        _check_tensor("w.q", q, (4, N // 4, 16 * ((K + 63) // 64)), torch.float8_e4m3fn, dev)
    if scale.numel() != 4 * blocks[0] * blocks[1] or scale.dtype is not torch.float32 or \
            scale.get_device() != dev or not scale.is_contiguous():
        _check_tensor("w.scale", scale, (4,) + blocks, torch.float32, dev)


def qpointwise_f8(x, w, *, bias=None, scale=None, shift=None, act=QUAN_ACT_NONE, workspace=None,
                  out=None, stream=None):
    """Pointwise quaternion convolution in 8-bit floating point: bf16 x [..., Cin] (CUDA), which
    is quantised in the call, and w = quantize_f8_weights(...) -> bf16 [..., Cout],
    act(scale * (x W + bias) + shift) with fp32 vectors [Cout] as in qconv2d.  x may be F8Rows
    (residual_join_f8): no workspace, the same bits.  Half the bytes of
    bf16 letters; faster than qconv2d in wide layers only (25,600 rows: 4096 -> 4096 420 us
    against 485, 2048 -> 1024 86 against 78; 102,400 rows of 512 -> 1024 109 against 84)."""
    if w.transposed:
        raise ValueError("w holds transposed letters: quantize_f8_weights(..., transpose=False)")
    q, wscale, Cin, Cout, _ = w
    in8 = x.__class__ is F8Rows
    dev = _device("x", x.q if in8 else x)
    vectors = (0, 0, 0)
    if bias is not None or scale is not None or shift is not None:
        f32 = (_torch or _get_torch()).float32
        for name, v in (("bias", bias), ("scale", scale), ("shift", shift)):
            if v is not None:
                _check_tensor(name, v, (Cout,), f32, dev)
        vectors = (_addr(bias), _addr(scale), _addr(shift))
    if in8:
        if x.channels != Cin or workspace is not None:
            raise ValueError("x has %d channels, w %d, and 8-bit rows need no workspace" %
                             (x.channels, Cin))
        lead, rows = _f8_rows("x", x, dev)
        _f8_letters(q, wscale, Cin, Cout, dev)
        shape, bf16 = lead + (Cout,), (_torch or _get_torch()).bfloat16
        if out is None:
            out = _empty(stream, shape, bf16, x.q.device)
        else:
            _check_tensor("out", out, shape, bf16, dev)
        _call(23, _QPOINT_F8_ROWS(x.q.data_ptr(), x.scale.data_ptr(), q.data_ptr(),
                                  wscale.data_ptr(), *vectors, rows, Cin, Cout, act,
                                  out.data_ptr(), _stream(stream, dev)))
        return out
    rows, workspace, nbytes, out = _qpoint_f8(x, q, wscale, Cin, Cout, workspace, out,
                                              stream, dev)
    _call(16, _QPOINT_F8(x.data_ptr(), q.data_ptr(), wscale.data_ptr(), *vectors, rows, Cin, Cout,
                         act, _addr(workspace), nbytes, out.data_ptr(), _stream(stream, dev)))
    return out


def qpointwise_f8_backward_data(dy, w, *, workspace=None, out=None, stream=None):
    """Input gradient of that convolution before its epilogue: bf16 dy [..., Cout] (CUDA),
    quantised in the call, and w = quantize_f8_weights(..., transpose=True) -> bf16 [..., Cin]."""
    if not w.transposed:
        raise ValueError("w holds the forward letters: quantize_f8_weights(..., transpose=True)")
    q, wscale, Cin, Cout, _ = w
    dev = _device("dy", dy)
    rows, workspace, nbytes, out = _qpoint_f8(dy, q, wscale, Cout, Cin, workspace, out,
                                              stream, dev)
    _call(17, _QPOINT_F8_BWD(dy.data_ptr(), q.data_ptr(), wscale.data_ptr(), rows, Cin, Cout,
                             _addr(workspace), nbytes, out.data_ptr(), _stream(stream, dev)))
    return out


# ------------------------------------------------------------------ letters in 4 bits

def quan_w4_weights(wr, wi, wj, wk, Cin, Cout, group, q, scale, stream=None) -> None:
    _check(load().quan_w4_weights(_ptr(wr), _ptr(wi), _ptr(wj), _ptr(wk), Cin, Cout, group, _ptr(q),
                                  _ptr(scale), _stream(stream)))


def quan_w4_weights_bytes(Cin, Cout) -> int:
    return load().quan_w4_weights_bytes(Cin, Cout)


def quan_w4_weights_scales(Cin, Cout, group) -> int:
    return load().quan_w4_weights_scales(Cin, Cout, group)


def quan_qpoint_w4_fwd(x, wq, wscale, bias, iqbn_scale, iqbn_shift, rows, Cin, Cout, group, act,
                       out, stream=None) -> None:
    _call(24, _QPOINT_W4(_addr(x), _addr(wq), _addr(wscale), _addr(bias), _addr(iqbn_scale),
                         _addr(iqbn_shift), rows, Cin, Cout, group, act, _addr(out),
                         _stream(stream)))


class W4Weights(typing.NamedTuple):
    """Letters of a pointwise layer in 4 bits, as quantize_w4_weights lays them out: q uint8
    [4, ceil(Cout / 64), ceil(Cin / 256), 512], scale bf16 [4, ceil(Cout / 64), groups, 16] (the
    order inside is include/quan.h's)."""
    q: object
    scale: object
    Cin: int
    Cout: int
    group: int


def quantize_w4_weights(wr, wi, wj, wk, *, group=64, stream=None):
    """The four letters [Cout/4, 1, 1, Cin/4] (bf16, CUDA) of a pointwise layer as W4Weights for
    qpointwise_w4: whole numbers -7 .. 7 with a bf16 scale for each `group` (32, 64 or 128) input
    channels of an output channel."""
    import torch
    Qout, kh, kw, Qin = wr.shape
    if kh != 1 or kw != 1:
        raise ValueError("the letters of a pointwise layer are [Cout/4, 1, 1, Cin/4]")
    if group not in (32, 64, 128):
        raise ValueError("group must be 32, 64 or 128 (got %s)" % (group,))
    dev = _device("wr", wr)
    for name, w in (("wr", wr), ("wi", wi), ("wj", wj), ("wk", wk)):
        _check_tensor(name, w, wr.shape, torch.bfloat16, dev)
    if min(Qin, Qout) < 1 or 4 * max(Qin, Qout) >= 1 << 31:
        raise ValueError("a layer of %d -> %d channels is empty or too large" % (4 * Qin, 4 * Qout))
    tiles = -(-Qout // 16)
    q = _empty(stream, (4, tiles, -(-Qin // 64), 512), torch.uint8, wr.device)
    scale = _empty(stream, (4, tiles, -(-Qin // group), 16), torch.bfloat16, wr.device)
    quan_w4_weights(wr, wi, wj, wk, 4 * Qin, 4 * Qout, group, q, scale, stream)
    return W4Weights(q, scale, 4 * Qin, 4 * Qout, group)


def qpointwise_w4(x, w, *, bias=None, scale=None, shift=None, act=QUAN_ACT_NONE, out=None,
                  stream=None):
    """Pointwise quaternion convolution of a few pixels with 4-bit letters: bf16 x [..., Cin] (CUDA)
    and w = quantize_w4_weights(...) -> bf16 [..., Cout], act(scale * (x W + bias) + shift) with
    fp32 vectors [Cout] as in qconv2d.  About a quarter of the bytes of bf16 letters (0.27 with
    groups of 64), for serving.  qpointwise_f8 is faster from some number of pixels on: between 16 and 32
    for 8192 -> 8192, 32 and 49 for 4096 -> 4096, 64 and 96 for 2048 -> 2048, 256 and 512 for 512 -> 1024."""
    torch = _torch or _get_torch()
    q, wscale, Cin, Cout, group = w
    dev, shape, bf16 = _device("x", x), tuple(x.shape), torch.bfloat16
    if x.dtype is not bf16 or shape[-1] != Cin or not x.is_contiguous():
        _check_tensor("x", x, shape[:-1] + (Cin,), bf16, dev)
    tiles = (Cout + 63) // 64
    want = (4, tiles, (Cin + 255) // 256, 512)
    if q.dtype is not torch.uint8 or q.shape != want or q.get_device() != dev or \
            not q.is_contiguous():
        _check_tensor("w.q", q, want, torch.uint8, dev)
    want = (4, tiles, (Cin + 4 * group - 1) // (4 * group), 16)
    if wscale.dtype is not bf16 or wscale.shape != want or wscale.get_device() != dev or \
            not wscale.is_contiguous():
        _check_tensor("w.scale", wscale, want, bf16, dev)
    vectors = (0, 0, 0)
    if bias is not None or scale is not None or shift is not None:
        for name, v in (("bias", bias), ("scale", scale), ("shift", shift)):
            if v is not None:
                _check_tensor(name, v, (Cout,), torch.float32, dev)
        vectors = (_addr(bias), _addr(scale), _addr(shift))
    shape = shape[:-1] + (Cout,)
    if out is None:
        out = _empty(stream, shape, bf16, x.device)
    else:
        _check_tensor("out", out, shape, bf16, dev)
    _call(24, _QPOINT_W4(x.data_ptr(), q.data_ptr(), wscale.data_ptr(), *vectors, x.numel() // Cin,
                         Cin, Cout, group, act, out.data_ptr(), _stream(stream, dev)))
    return out


def _join_shape(like, shape, post, gate, pre, dev):
    """(rows, C, images) of a join's tensors, its vectors checked."""
    f32 = (_torch or _get_torch()).float32
    C = shape[-1]
    vec, images = (C,), 1
    if gate is not None:
        want = vec
        if gate.dim() != 1:
            images = shape[0]
            want = (images, C)
        if gate.dtype is not f32 or gate.shape != want or gate.get_device() != dev or \
                not gate.is_contiguous():
            _check_tensor("gate", gate, want, f32, dev)
    if post is not None and (post.dtype is not f32 or post.shape != vec or
                             post.get_device() != dev or not post.is_contiguous()):
        _check_tensor("post", post, vec, f32, dev)
    if pre is not None and (pre.dtype is not f32 or pre.shape != vec or
                            pre.get_device() != dev or not pre.is_contiguous()):
        _check_tensor("pre", pre, vec, f32, dev)
    return like.numel() // C if C else 0, C, max(images, 1)


def residual_join(x, h=None, *, post=None, gate=None, pre=None, alpha=1.0, groups=1, eps=1e-5,
                  p=0.0, seed=0, offset=0, counter=None, y=None, n=None, stream=None):
    """The end of a residual branch and the norm in front of the next one, in one pass:
        u = h / rms(h) * post,  y = x + alpha * gate * dropout(u),  n = y / rms(y) * pre
    x, h: bf16 or fp32 [N, ..., C] (CUDA).  post, pre: fp32 [C]; without one, no such norm (u = h;
    no n).  gate: fp32 [C], or [N, C] for a gate of each image.  groups=4 normalises each
    quaternion component by itself.  p, seed, offset, counter: see `dropout`.  Without h only the
    norm of x is taken.  Returns (y, n); y may be given as x and n as h (in place)."""
    torch = _torch or _get_torch()
    t, shape = x.dtype, x.shape
    dtype = QUAN_DTYPE_BF16 if t is torch.bfloat16 else _dtype_of("x", x)
    dev = _device("x", x)
    if not x.is_contiguous():
        _check_tensor("x", x, shape, t, dev)
    rows, C, images = _join_shape(x, shape, post, gate, pre, dev)
    if counter is not None:
        _check_counter(counter, dev)
    if h is not None:
        if h.dtype is not t or h.shape != shape or h.get_device() != dev or not h.is_contiguous():
            _check_tensor("h", h, shape, t, dev)
        if y is None:
            y = _empty(stream, shape, t, x.device)
        else:
            _check_tensor("y", y, shape, t, dev)
    elif y is not None:
        raise ValueError("y is given without h")
    if n is not None:
        _check_tensor("n", n, shape, t, dev)
    elif pre is not None:
        n = _empty(stream, shape, t, x.device)
    _call(14, _JOIN_FWD(x.data_ptr(), _addr(h), _addr(post), _addr(gate), _addr(pre), rows, images,
                        C, groups, dtype, alpha, eps, p, seed, offset, _addr(counter), _addr(y),
                        _addr(n), _stream(stream, dev)))
    return y, n


def residual_join_f8(x, h=None, *, post=None, gate=None, pre, alpha=1.0, groups=1, eps=1e-5,
                     p=0.0, seed=0, offset=0, counter=None, keep=False, y=None, n=None, n8=None,
                     stream=None):
    """`residual_join` whose n comes out as F8Rows for qpointwise_f8, rounded to bf16 and then
    quantised: the bits (groups=4) of residual_join and the product's own quantisation, without
    that pass.  keep=True, or n given: n in bf16 too, for the weight gradient.  Returns (y, n, n8),
    None for what is absent; y may be given as x, n as a bf16 h (in place), n8 as F8Rows to write
    to.  The gradients are residual_join_backward's: the quantisation has none of its own."""
    torch = _torch or _get_torch()
    t, shape = x.dtype, x.shape
    dtype = QUAN_DTYPE_BF16 if t is torch.bfloat16 else _dtype_of("x", x)
    dev = _device("x", x)
    if not x.is_contiguous():
        _check_tensor("x", x, shape, t, dev)
    if pre is None:
        raise ValueError("pre is needed: the 8-bit rows are the norm")
    rows, C, images = _join_shape(x, shape, post, gate, pre, dev)
    if C % 4 or C < 4:
        raise ValueError("x has %d channels, not a multiple of 4" % C)
    if counter is not None:
        _check_counter(counter, dev)
    if h is not None:
        if h.dtype is not t or h.shape != shape or h.get_device() != dev or not h.is_contiguous():
            _check_tensor("h", h, shape, t, dev)
        if y is None:
            y = _empty(stream, shape, t, x.device)
        else:
            _check_tensor("y", y, shape, t, dev)
    elif y is not None:
        raise ValueError("y is given without h")
    if n is not None:
        _check_tensor("n", n, shape, torch.bfloat16, dev)
    elif keep:
        n = _empty(stream, shape, torch.bfloat16, x.device)
    if n8 is None:
        n8 = F8Rows(_empty(stream, tuple(shape[:-1]) + (4, (C + 63) // 64 * 16),
                           torch.float8_e4m3fn, x.device),
                    _empty(stream, (4, (C + 511) // 512, (rows + 127) // 128 * 128),
                           torch.float32, x.device), C)
    elif n8.channels != C or _f8_rows("n8", n8, dev)[0] != tuple(shape[:-1]) or \
            n8.q.get_device() != dev:
        raise ValueError("n8 does not have the rows and channels of x")
    _call(21, _JOIN_F8(x.data_ptr(), _addr(h), _addr(post), _addr(gate), _addr(pre), rows, images,
                       C, groups, dtype, alpha, eps, p, seed, offset, _addr(counter), _addr(y),
                       _addr(n), n8.q.data_ptr(), n8.scale.data_ptr(), _stream(stream, dev)))
    return y, n, n8


def residual_join_backward(dy, dn, y, h=None, *, post=None, gate=None, pre=None, alpha=1.0,
                           groups=1, eps=1e-5, p=0.0, seed=0, offset=0, counter=None,
                           workspace=None, dx=None, dh=None, stream=None):
    """Gradients of `residual_join`, from dy (None: 0) and dn (None without pre) and the forward
    call's y (needed with pre) and h.  Returns (dx, dh, dpost, dgate, dpre), fp32 sums shaped as
    their vectors, None for what is absent; without pre, dx is dy itself, or its copy in a dx that
    is given.  dx may be given as dy or dn, dh as dn or h (in place)."""
    torch = _torch or _get_torch()
    like = dy if dy is not None else dn
    if like is None:
        raise ValueError("dy or dn must be given")
    t, shape, device = like.dtype, like.shape, like.device
    dtype = QUAN_DTYPE_BF16 if t is torch.bfloat16 else \
        _dtype_of("dy" if dy is not None else "dn", like)
    dev = _device("dy" if dy is not None else "dn", like)
    rows, C, images = _join_shape(like, shape, post, gate, pre, dev)
    if counter is not None:
        _check_counter(counter, dev)
    for name, v in (("dy", dy), ("dn", dn), ("y", y), ("h", h), ("dx", dx), ("dh", dh)):
        if v is not None and (v.dtype is not t or v.shape != shape or v.get_device() != dev or
                              not v.is_contiguous()):
            _check_tensor(name, v, shape, t, dev)
    if pre is None:
        y = None
        if h is None and post is None and gate is None and dn is None and dx is None and \
                dh is None:
            return dy, None, None, None, None
    elif dx is None:
        dx = _empty(stream, shape, t, device)
    if h is not None and dh is None:
        dh = _empty(stream, shape, t, device)
    f32 = torch.float32
    dpost = None if post is None else _empty(stream, C, f32, device)
    dgate = None if gate is None else _empty(stream, gate.shape, f32, device)
    dpre = None if pre is None else _empty(stream, C, f32, device)
    if workspace is None:
        nbytes = (_lib or load()).quan_residual_join_bwd_workspace_size(rows, C, groups, images)
        if nbytes:
            workspace = _empty(stream, nbytes, torch.uint8, device)
    else:
        nbytes = _workspace_bytes(workspace, dev)
    _call(15, _JOIN_BWD(_addr(dy), _addr(dn), _addr(y), _addr(h), _addr(post), _addr(gate),
                        _addr(pre), rows, images, C, groups, dtype, alpha, eps, p, seed, offset,
                        _addr(counter), _addr(workspace), nbytes, _addr(dx), _addr(dh),
                        _addr(dpost), _addr(dgate), _addr(dpre), _stream(stream, dev)))
    return (dy if dx is None else dx, dh, dpost, dgate, dpre)


# ------------------------------------------------------------------ distillation

def quan_distill_fwd(z, index, teacher, rows, classes, pitch, top, dtype, teacher_dtype, index_bits,
                     temperature, loss, lse, stream=None) -> None:
    _call(18, _DISTILL_FWD(_addr(z), _addr(index), _addr(teacher), rows, classes, pitch, top, dtype,
                           teacher_dtype, index_bits, temperature, _addr(loss), _addr(lse),
                           _stream(stream)))


def quan_distill_bwd(dloss, z, lse, index, teacher, rows, classes, pitch, top, dtype, teacher_dtype,
                     index_bits, temperature, scale, dz, stream=None) -> None:
    _call(19, _DISTILL_BWD(_addr(z), _addr(index), _addr(teacher), rows, classes, pitch, top, dtype,
                           teacher_dtype, index_bits, temperature, scale, _addr(dloss), _addr(lse),
                           _addr(dz), _stream(stream)))


def quan_distill_fwd_bwd(z, index, teacher, dloss, rows, classes, pitch, top, dtype, teacher_dtype,
                         index_bits, temperature, scale, loss, dz, stream=None) -> None:
    _call(20, _DISTILL_BWD(_addr(z), _addr(index), _addr(teacher), rows, classes, pitch, top, dtype,
                           teacher_dtype, index_bits, temperature, scale, _addr(dloss), _addr(loss),
                           _addr(dz), _stream(stream)))


def _distill(logits, index, teacher, classes):
    """The device, the leading shape and the packed sizes of a distillation's tensors, checked."""
    torch = _torch or _get_torch()
    t, shape = logits.dtype, logits.shape
    dtype = QUAN_DTYPE_BF16 if t is torch.bfloat16 else _dtype_of("logits", logits)
    dev = _device("logits", logits)
    if not logits.is_contiguous():
        _check_tensor("logits", logits, shape, t, dev)
    lead, pitch = shape[:-1], shape[-1]
    slots = index.shape
    if slots[:-1] != lead or index.get_device() != dev or not index.is_contiguous() or \
            (index.dtype is not torch.int64 and index.dtype is not torch.int32):
        _check_tensor("index", index, lead + slots[-1:], torch.int64, dev)
    teacher_dtype = QUAN_DTYPE_BF16 if teacher.dtype is torch.bfloat16 else \
        _dtype_of("teacher", teacher)
    if teacher.shape != slots or teacher.get_device() != dev or not teacher.is_contiguous():
        _check_tensor("teacher", teacher, slots, teacher.dtype, dev)
    if classes is None:
        classes = pitch
    rows = logits.numel() // pitch if pitch else 0
    return dev, lead, (rows, classes, pitch, slots[-1], dtype, teacher_dtype,
                       64 if index.dtype is torch.int64 else 32)


def distill_loss(logits, index, teacher, *, classes=None, temperature=1.0, loss=None, lse=None,
                 stream=None):
    """The loss of each row of bf16 or fp32 logits [..., C] (CUDA) against a teacher's top logits:
    teacher [..., K] (bf16 or fp32) and their classes, index [..., K] (int64 or int32), as
    torch.topk gives them (K up to 256):
        p = softmax(teacher / T),  q = softmax(logits / T),  T^2 sum_k p_k (ln p_k - ln q_index_k)
    classes: the first so many channels are the classes (all by default), the others padding.
    Slots with a class outside [0, classes) are empty; a row of empty slots (an ignored pixel) has
    loss 0.  Returns (loss, lse), fp32 [...]; lse is for distill_loss_backward."""
    f32 = (_torch or _get_torch()).float32
    dev, lead, sizes = _distill(logits, index, teacher, classes)
    if loss is None:
        loss = _empty(stream, lead, f32, logits.device)
    else:
        _check_tensor("loss", loss, lead, f32, dev)
    if lse is None:
        lse = _empty(stream, lead, f32, logits.device)
    else:
        _check_tensor("lse", lse, lead, f32, dev)
    _call(18, _DISTILL_FWD(logits.data_ptr(), index.data_ptr(), teacher.data_ptr(), *sizes,
                           temperature, loss.data_ptr(), lse.data_ptr(), _stream(stream, dev)))
    return loss, lse


def distill_loss_backward(dloss, logits, lse, index, teacher, *, classes=None, temperature=1.0,
                          scale=1.0, out=None, stream=None):
    """Gradient of distill_loss with respect to its logits, times scale: from dloss, fp32 [...]
    (None: 1), and the forward call's lse and arguments.  Channels behind the classes get 0.  out
    may be logits (in place).  q is e^(logits / T - lse) with lse as fp32 holds it: off by about
    2^-23 (|logits| / T + |lse|) of itself, 1e-3 where those are 5000.  distill_loss_and_gradient has no
    such error."""
    f32 = (_torch or _get_torch()).float32
    dev, lead, sizes = _distill(logits, index, teacher, classes)
    if dloss is not None:
        _check_tensor("dloss", dloss, lead, f32, dev)
    _check_tensor("lse", lse, lead, f32, dev)
    if out is None:
        out = _empty(stream, logits.shape, logits.dtype, logits.device)
    else:
        _check_tensor("out", out, logits.shape, logits.dtype, dev)
    _call(19, _DISTILL_BWD(logits.data_ptr(), index.data_ptr(), teacher.data_ptr(), *sizes,
                           temperature, scale, _addr(dloss), lse.data_ptr(), out.data_ptr(),
                           _stream(stream, dev)))
    return out


def distill_loss_and_gradient(logits, index, teacher, dloss=None, *, classes=None,
                              temperature=1.0, scale=1.0, loss=None, out=None, stream=None):
    """distill_loss and distill_loss_backward in one pass over the logits: (loss, dlogits), for a
    dloss (a row's weight in the sum that is minimised; None: 1) that is known beforehand.  out may
    be logits (in place)."""
    f32 = (_torch or _get_torch()).float32
    dev, lead, sizes = _distill(logits, index, teacher, classes)
    if dloss is not None:
        _check_tensor("dloss", dloss, lead, f32, dev)
    if loss is None:
        loss = _empty(stream, lead, f32, logits.device)
    else:
        _check_tensor("loss", loss, lead, f32, dev)
    if out is None:
        out = _empty(stream, logits.shape, logits.dtype, logits.device)
    else:
        _check_tensor("out", out, logits.shape, logits.dtype, dev)
    _call(20, _DISTILL_BWD(logits.data_ptr(), index.data_ptr(), teacher.data_ptr(), *sizes,
                           temperature, scale, _addr(dloss), loss.data_ptr(), out.data_ptr(),
                           _stream(stream, dev)))
    return loss, out
