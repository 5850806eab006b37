"""ctypes binding of libpcl_dnn.so: same names as the C ABI, argument
marshalling only (of the calls whose kernels last no longer than that, compiled: csrc/fast_calls.cpp).  Tensors are torch CUDA tensors (device memory and streams
are all torch is used for); every step of the path runs in the library's
kernels.  There is no CPU or library fallback: if the shared library is missing
or a call fails, an exception is raised.
"""
from __future__ import annotations

import ctypes
import os
import warnings

import torch

from . import build

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libpcl_dnn.so")

ACT_NONE, ACT_RELU, ACT_SIGMOID = 0, 1, 2
PASS_FWD, PASS_BWD_DATA, PASS_BWD_WEIGHTS = 0, 1, 2
PATH_AUTO, PATH_TENSOR, PATH_GENERIC = 0, 1, 2
OK = 0
ERR_BAD_ARG, ERR_UNSUPPORTED_SHAPE, ERR_MISALIGNED, ERR_WORKSPACE, ERR_CUDA, ERR_DEVICE_TIMEOUT = 1, 2, 3, 4, 5, 6
ERR_SCRATCH_LIMIT = 7
ERR_BAD_LABEL = 8
F32, BF16, F16 = 0, 1, 2
NO_ID = -2 ** 31

EXPORTS = [
    "pcl_set_path", "pcl_conv_out_dims", "pcl_conv_workspace_bytes", "pcl_fc_workspace_bytes",
    "pcl_conv_fwd", "pcl_conv_bwd_data", "pcl_conv_bwd_weights", "pcl_fc_fwd", "pcl_fc_bwd",
    "pcl_sgd_update", "pcl_maxpool2x2_fwd", "pcl_maxpool2x2_bwd", "pcl_softmax_xent",
    "pcl_last_device_status", "pcl_launch_count", "pcl_status_string", "pcl_profile_begin", "pcl_profile_end", "pcl_conv_bwd_data_noalloc", "pcl_noalloc_scratch_bytes",
    "pcl_conv_bwd_data_colsum_workspace_bytes", "pcl_conv_bwd_data_colsum",
    "pcl_maxpool2x2_bwd_colsum_workspace_bytes", "pcl_maxpool2x2_bwd_colsum", "pcl_conv_fwd_pool", "pcl_conv_fwd_pool_is_fused",
    "pcl_conv_bwd_weights_pooled", "pcl_conv_bwd_weights_pooled_is_fused", "pcl_conv_bwd_weights_pooled_workspace_bytes",
    "pcl_maxpool2x2_fwd_codes", "pcl_maxpool2x2_bwd_codes", "pcl_last_wait_code", "pcl_set_tuning", "pcl_reset_tuning", "pcl_fc_bwd_fused", "pcl_conv_plan_describe", "pcl_conv_staged_input_bytes",
    "pcl_embedding_fwd", "pcl_embedding_workspace_bytes", "pcl_embedding_bwd", "pcl_embedding_bwd_sgd",
    "pcl_fc_softmax_xent_workspace_bytes", "pcl_fc_softmax_xent_fwd", "pcl_fc_softmax_xent_bwd",
    "pcl_orthogonalize_workspace_bytes", "pcl_orthogonalize", "pcl_orthogonal_update",
    "pcl_conv_bwd_weights_pooled_staged", "pcl_conv_bwd_weights_sgd", "pcl_conv_bwd_weights_sgd_workspace_bytes",
    "pcl_fc_bwd_fused_sgd", "pcl_fc_bwd_fused_sgd_workspace_bytes", "pcl_plan_cache_stats",
    "pcl_rms_norm_fwd", "pcl_rms_norm_fwd_q8", "pcl_rms_norm_workspace_bytes", "pcl_rms_norm_bwd", "pcl_quantize_rows",
    "pcl_fc_q8_workspace_bytes", "pcl_fc_q8_fwd",
    "pcl_grad_norm_workspace_bytes", "pcl_grad_norm", "pcl_grad_clip", "pcl_sgd_update_clipped",
    "pcl_sample_tokens_workspace_bytes", "pcl_sample_tokens",
]


class PclError(RuntimeError):
    def __init__(self, code: int, where: str):
        self.code = code
        super().__init__(f"{where}: {status_string(code)} (status {code})")


class KernelStat(ctypes.Structure):
    _fields_ = [("name", ctypes.c_char * 64), ("launches", ctypes.c_ulonglong), ("total_ms", ctypes.c_double),
                ("work", ctypes.c_double)]


class ConvDesc(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int) for n in
                ("N", "C", "K", "H", "W", "R", "S", "stride_h", "stride_w", "pad_h", "pad_w")]


_lib = None
_calls = None           # compiled checks and marshalling (csrc/fast_calls.cpp) of the calls that have them, once the library is loaded


def lib() -> ctypes.CDLL:
    """Loads the CUDA library; fails loudly if it has not been built."""
    global _lib, _calls
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(f"{LIB_PATH} is missing: run `python -m paper_1602_06709_b200.build` "
                               "(there is no fallback path)")
        L = ctypes.CDLL(LIB_PATH)
        vp, sz, ci, cf = ctypes.c_void_p, ctypes.c_size_t, ctypes.c_int, ctypes.c_float
        dp = ctypes.POINTER(ConvDesc)
        L.pcl_set_path.argtypes = [ci]
        L.pcl_set_tuning.argtypes = [ctypes.c_char_p, ci]
        L.pcl_conv_plan_describe.argtypes = [dp, ci, ctypes.c_char_p, sz]
        L.pcl_conv_out_dims.argtypes = [dp, ctypes.POINTER(ci), ctypes.POINTER(ci)]
        L.pcl_conv_workspace_bytes.argtypes = [dp, ci]
        L.pcl_conv_workspace_bytes.restype = sz
        L.pcl_fc_workspace_bytes.argtypes = [ci, ci, ci, ci]
        L.pcl_fc_workspace_bytes.restype = sz
        L.pcl_conv_fwd.argtypes = [dp, vp, vp, vp, vp, ci, vp, sz, vp]
        L.pcl_conv_bwd_data.argtypes = [dp, vp, vp, vp, vp, vp, sz, vp]
        L.pcl_conv_fwd_pool.argtypes = [dp, vp, vp, vp, vp, vp, vp, ci, vp, sz, vp]
        L.pcl_conv_fwd_pool_is_fused.argtypes = [dp]
        L.pcl_conv_bwd_weights_pooled_is_fused.argtypes = [dp]
        L.pcl_conv_bwd_weights_pooled_workspace_bytes.argtypes = [dp]
        L.pcl_conv_bwd_weights_pooled_workspace_bytes.restype = sz
        L.pcl_conv_bwd_weights_pooled.argtypes = [dp, vp, vp, vp, ci, vp, vp, vp, sz, vp]
        L.pcl_conv_bwd_weights_pooled_staged.argtypes = [dp, vp, vp, vp, ci, vp, vp, vp, sz, vp]
        L.pcl_conv_staged_input_bytes.argtypes = [dp]
        L.pcl_conv_staged_input_bytes.restype = sz
        L.pcl_maxpool2x2_fwd_codes.argtypes = [ci, ci, ci, ci, vp, vp, vp, vp]
        L.pcl_maxpool2x2_bwd_codes.argtypes = [ci, ci, ci, ci, vp, vp, ci, vp, vp, vp, sz, vp]
        L.pcl_conv_bwd_weights.argtypes = [dp, vp, vp, vp, vp, ci, vp, sz, vp]
        L.pcl_fc_fwd.argtypes = [ci, ci, ci, vp, vp, vp, vp, ci, vp, sz, vp]
        L.pcl_fc_bwd.argtypes = [ci, ci, ci, vp, vp, vp, ci, vp, vp, vp, vp, vp, sz, vp]
        L.pcl_fc_bwd_fused.argtypes = [ci, ci, ci, vp, vp, vp, ci, vp, vp, ci, vp, vp, vp, vp, sz, vp]
        L.pcl_sgd_update.argtypes = [vp, vp, sz, cf, vp]
        L.pcl_conv_bwd_weights_sgd_workspace_bytes.argtypes = [dp]
        L.pcl_conv_bwd_weights_sgd_workspace_bytes.restype = sz
        L.pcl_conv_bwd_weights_sgd.argtypes = [dp, vp, vp, vp, cf, vp, vp, sz, vp]
        L.pcl_fc_bwd_fused_sgd_workspace_bytes.argtypes = [ci, ci, ci]
        L.pcl_fc_bwd_fused_sgd_workspace_bytes.restype = sz
        L.pcl_fc_bwd_fused_sgd.argtypes = [ci, ci, ci, vp, vp, vp, ci, vp, vp, ci, vp, cf, vp, vp, sz, vp]
        L.pcl_maxpool2x2_fwd.argtypes = [ci, ci, ci, ci, vp, vp, vp]
        L.pcl_maxpool2x2_bwd.argtypes = [ci, ci, ci, ci, vp, vp, vp, vp, vp]
        L.pcl_softmax_xent.argtypes = [ci, ci, vp, vp, vp, vp, vp]
        L.pcl_embedding_fwd.argtypes = [ci, ci, ci, ci, vp, vp, cf, ci, vp, vp]
        L.pcl_embedding_workspace_bytes.argtypes = [ci, ci, ci]
        L.pcl_embedding_workspace_bytes.restype = sz
        L.pcl_embedding_bwd.argtypes = [ci, ci, ci, ci, vp, vp, cf, ci, vp, vp, sz, vp]
        L.pcl_embedding_bwd_sgd.argtypes = [ci, ci, ci, ci, vp, vp, cf, ci, vp, cf, vp, sz, vp]
        L.pcl_fc_softmax_xent_workspace_bytes.argtypes = [ci, ci, ci, ci, ci]
        L.pcl_fc_softmax_xent_workspace_bytes.restype = sz
        L.pcl_fc_softmax_xent_fwd.argtypes = [ci, ci, ci, ci, vp, vp, vp, vp, ci, vp, vp, vp, vp, sz, vp]
        L.pcl_fc_softmax_xent_bwd.argtypes = [ci, ci, ci, ci, vp, vp, vp, vp, ci, vp, vp, vp, vp, vp, vp, sz, vp]
        L.pcl_orthogonalize_workspace_bytes.argtypes = [ci, ci, ci]
        L.pcl_orthogonalize_workspace_bytes.restype = sz
        L.pcl_orthogonalize.argtypes = [ci, ci, ci, ci, vp, vp, ci, vp, sz, vp]
        L.pcl_orthogonal_update.argtypes = [ci, ci, ci, ci, vp, vp, vp, cf, ci, cf, cf, ci, vp, sz, vp]
        L.pcl_rms_norm_fwd.argtypes = [ci, ci, ci, vp, vp, vp, cf, vp, vp, vp, vp]
        L.pcl_rms_norm_fwd_q8.argtypes = [ci, ci, ci, vp, vp, vp, cf, vp, vp, vp, vp, vp]
        L.pcl_rms_norm_workspace_bytes.argtypes = [ci, ci]
        L.pcl_rms_norm_workspace_bytes.restype = sz
        L.pcl_rms_norm_bwd.argtypes = [ci, ci, ci, vp, vp, vp, vp, vp, vp, vp, vp, sz, vp]
        L.pcl_quantize_rows.argtypes = [ci, ci, ci, vp, vp, vp, vp]
        L.pcl_fc_q8_workspace_bytes.argtypes = [ci, ci, ci]
        L.pcl_fc_q8_workspace_bytes.restype = sz
        L.pcl_fc_q8_fwd.argtypes = [ci, ci, ci, ci, vp, vp, vp, vp, vp, vp, ci, vp, sz, vp]
        L.pcl_grad_norm_workspace_bytes.argtypes = [ci]
        L.pcl_grad_norm_workspace_bytes.restype = sz
        L.pcl_grad_norm.argtypes = [ci, vp, vp, vp, vp, vp, sz, vp]
        L.pcl_grad_clip.argtypes = [ci, vp, vp, vp, vp, cf, vp, vp, sz, vp]
        L.pcl_sgd_update_clipped.argtypes = [ci, vp, vp, vp, vp, cf, cf, vp, vp, sz, vp]
        L.pcl_sample_tokens_workspace_bytes.argtypes = [ci, ci]
        L.pcl_sample_tokens_workspace_bytes.restype = sz
        L.pcl_sample_tokens.argtypes = [ci, ci, ci, vp, vp, vp, vp, vp, vp, vp, vp, vp, sz, vp]
        L.pcl_last_device_status.argtypes = [vp]
        L.pcl_launch_count.restype = ctypes.c_ulonglong
        L.pcl_last_wait_code.restype = ctypes.c_uint
        L.pcl_profile_end.argtypes = [ctypes.POINTER(KernelStat), ci, ctypes.POINTER(ci)]
        L.pcl_conv_bwd_data_colsum_workspace_bytes.argtypes = [dp]
        L.pcl_conv_bwd_data_colsum_workspace_bytes.restype = sz
        L.pcl_conv_bwd_data_colsum.argtypes = [dp, vp, vp, vp, vp, vp, vp, sz, vp]
        L.pcl_maxpool2x2_bwd_colsum_workspace_bytes.argtypes = [ci, ci, ci, ci]
        L.pcl_maxpool2x2_bwd_colsum_workspace_bytes.restype = sz
        L.pcl_maxpool2x2_bwd_colsum.argtypes = [ci, ci, ci, ci, vp, vp, vp, vp, vp, vp, sz, vp]
        L.pcl_conv_bwd_data_noalloc.argtypes = [dp, vp, vp, vp, vp, vp]
        L.pcl_noalloc_scratch_bytes.restype = sz
        L.pcl_status_string.argtypes = [ci]
        L.pcl_status_string.restype = ctypes.c_char_p
        _lib, _calls = L, _compiled_calls(L)
    return _lib


_COMPILED = ["pcl_rms_norm_fwd", "pcl_rms_norm_fwd_q8", "pcl_rms_norm_bwd", "pcl_quantize_rows", "pcl_fc_q8_fwd", "pcl_grad_norm",
             "pcl_grad_clip", "pcl_sgd_update_clipped", "pcl_sample_tokens"]


def _compiled_calls(L):
    """The compiled marshalling, bound to the library; None where it was not built, or for another Python or torch: every call has its checks here
    too, which take a few microseconds longer."""
    try:
        from . import _pcl_calls
    except ImportError as e:
        why = str(e)
    else:
        want, have = build.calls_built_for(), getattr(_pcl_calls, "built_for", None)
        if have == want:
            _pcl_calls.bind({n: ctypes.cast(getattr(L, n), ctypes.c_void_p).value for n in _COMPILED})
            return _pcl_calls
        why = f"it was built for {have}, this is {want}"
    warnings.warn(f"{os.path.join(_HERE, '_pcl_calls.so')} is not used ({why}): run `python -m paper_1602_06709_b200.build`", RuntimeWarning, stacklevel=3)
    return None


def _done(code: int, where: str) -> bool:
    """Whether a compiled call has been made (-1: an argument is not what it takes; the checks here say which)."""
    if code > 0:
        raise PclError(code, where)
    return code == 0


def status_string(code: int) -> str:
    return lib().pcl_status_string(code).decode()


def _check(code: int, where: str):
    if code != OK:
        raise PclError(code, where)


def _ptr(t):
    if t is None:
        return None
    assert t.is_cuda and t.is_contiguous(), "tensors must be contiguous CUDA tensors"
    return ctypes.c_void_p(t.data_ptr())


def _stream(stream=None):
    s = stream if stream is not None else torch.cuda.current_stream()
    return ctypes.c_void_p(s.cuda_stream)


def conv_desc(N, C, K, H, W, R, S, stride=1, pad=0, stride_w=None, pad_w=None) -> ConvDesc:
    return ConvDesc(N, C, K, H, W, R, S, stride, stride if stride_w is None else stride_w,
                    pad, pad if pad_w is None else pad_w)


UNSET = -2 ** 31
TILINGS = {"plain": 0, "halo0": 1, "halo1": 2, "halo2": 3, "auto": UNSET}      # auto: the launcher's own rule


def set_tuning(name: str, value):
    """Pins one of the launchers' choices (see pcl_set_tuning in the header).  value None unsets the knob; the
    TILING knob also takes the names plain / halo0 / halo1 / halo2 / auto."""
    if value is None:
        value = UNSET
    elif name == "TILING" and isinstance(value, str):
        value = TILINGS[value]
    _check(lib().pcl_set_tuning(name.encode(), int(value)), f"pcl_set_tuning({name})")


def conv_plan_describe(d: ConvDesc, pass_: int) -> str:
    """The tiling the pass would launch with under the current knobs and the cost model's prediction for it."""
    buf = ctypes.create_string_buffer(512)
    _check(lib().pcl_conv_plan_describe(ctypes.byref(d), pass_, buf, 512), "pcl_conv_plan_describe")
    return buf.value.decode()


def reset_tuning():
    _check(lib().pcl_reset_tuning(), "pcl_reset_tuning")


def set_path(path: int):
    _check(lib().pcl_set_path(path), "pcl_set_path")


def conv_out_dims(d: ConvDesc):
    P, Q = ctypes.c_int(), ctypes.c_int()
    _check(lib().pcl_conv_out_dims(ctypes.byref(d), ctypes.byref(P), ctypes.byref(Q)), "pcl_conv_out_dims")
    return P.value, Q.value


def conv_workspace_bytes(d: ConvDesc, which: int) -> int:
    return int(lib().pcl_conv_workspace_bytes(ctypes.byref(d), which))


def fc_workspace_bytes(N, C, K, which: int) -> int:
    return int(lib().pcl_fc_workspace_bytes(N, C, K, which))


def _ws(ws):
    if ws is None:
        return None, 0
    return _ptr(ws), ws.numel() * ws.element_size()


def conv_fwd(d, x, w, bias, y, act=ACT_NONE, ws=None, stream=None):
    wp, wb = _ws(ws)
    _check(lib().pcl_conv_fwd(ctypes.byref(d), _ptr(x), _ptr(w), _ptr(bias), _ptr(y), act, wp, wb, _stream(stream)),
           "pcl_conv_fwd")


def conv_fwd_pool_is_fused(d) -> bool:
    return bool(lib().pcl_conv_fwd_pool_is_fused(ctypes.byref(d)))


def conv_fwd_pool(d, x, w, bias, y, y_pool, act=ACT_NONE, ws=None, stream=None, pool_codes=None):
    """y may be None where conv_fwd_pool_is_fused(d): the full-resolution output is then not stored."""
    wp, wb = _ws(ws)
    _check(lib().pcl_conv_fwd_pool(ctypes.byref(d), _ptr(x), _ptr(w), _ptr(bias), _ptr(y), _ptr(y_pool),
                                   _ptr(pool_codes), act, wp, wb, _stream(stream)), "pcl_conv_fwd_pool")


def conv_bwd_weights_pooled_is_fused(d) -> bool:
    return bool(lib().pcl_conv_bwd_weights_pooled_is_fused(ctypes.byref(d)))


def conv_bwd_weights_pooled_workspace_bytes(d) -> int:
    return int(lib().pcl_conv_bwd_weights_pooled_workspace_bytes(ctypes.byref(d)))


def conv_bwd_weights_pooled(d, x, dy_pool, pool_codes, relu_mask, dw, dbias=None, ws=None, stream=None):
    wp, wb = _ws(ws)
    _check(lib().pcl_conv_bwd_weights_pooled(ctypes.byref(d), _ptr(x), _ptr(dy_pool), _ptr(pool_codes),
                                             int(bool(relu_mask)), _ptr(dw), _ptr(dbias), wp, wb, _stream(stream)),
           "pcl_conv_bwd_weights_pooled")


def conv_staged_input_bytes(d) -> int:
    return int(lib().pcl_conv_staged_input_bytes(ctypes.byref(d)))


def conv_bwd_weights_pooled_staged(d, x_staged, dy_pool, pool_codes, relu_mask, dw, dbias=None, ws=None, stream=None):
    """conv_bwd_weights_pooled from the staged input that the layer's forward call left at the start of its workspace
    (x_staged: that workspace tensor, kept untouched since)."""
    wp, wb = _ws(ws)
    _check(lib().pcl_conv_bwd_weights_pooled_staged(ctypes.byref(d), _ptr(x_staged), _ptr(dy_pool), _ptr(pool_codes),
                                                    int(bool(relu_mask)), _ptr(dw), _ptr(dbias), wp, wb, _stream(stream)),
           "pcl_conv_bwd_weights_pooled_staged")


def maxpool2x2_fwd_codes(N, H, W, C, x, y, codes, stream=None):
    _check(lib().pcl_maxpool2x2_fwd_codes(N, H, W, C, _ptr(x), _ptr(y), _ptr(codes), _stream(stream)),
           "pcl_maxpool2x2_fwd_codes")


def maxpool2x2_bwd_codes(N, H, W, C, codes, dy, relu_mask, dx, dx_colsum=None, ws=None, stream=None):
    wp, wb = _ws(ws)
    _check(lib().pcl_maxpool2x2_bwd_codes(N, H, W, C, _ptr(codes), _ptr(dy), int(bool(relu_mask)), _ptr(dx),
                                          _ptr(dx_colsum), wp, wb, _stream(stream)), "pcl_maxpool2x2_bwd_codes")


def last_wait_code() -> int:
    return int(lib().pcl_last_wait_code())


def conv_bwd_data(d, dy, w, relu_mask_src, dx, ws=None, stream=None):
    wp, wb = _ws(ws)
    _check(lib().pcl_conv_bwd_data(ctypes.byref(d), _ptr(dy), _ptr(w), _ptr(relu_mask_src), _ptr(dx), wp, wb,
                                   _stream(stream)), "pcl_conv_bwd_data")


def conv_bwd_data_colsum_workspace_bytes(d: ConvDesc) -> int:
    return int(lib().pcl_conv_bwd_data_colsum_workspace_bytes(ctypes.byref(d)))


def conv_bwd_data_colsum(d, dy, w, relu_mask_src, dx, dx_colsum, ws=None, stream=None):
    wp, wb = _ws(ws)
    _check(lib().pcl_conv_bwd_data_colsum(ctypes.byref(d), _ptr(dy), _ptr(w), _ptr(relu_mask_src), _ptr(dx),
                                          _ptr(dx_colsum), wp, wb, _stream(stream)), "pcl_conv_bwd_data_colsum")


def maxpool2x2_bwd_colsum_workspace_bytes(N, H, W, C) -> int:
    return int(lib().pcl_maxpool2x2_bwd_colsum_workspace_bytes(N, H, W, C))


def maxpool2x2_bwd_colsum(N, H, W, C, x, dy, relu_mask_src, dx, dx_colsum, ws=None, stream=None):
    wp, wb = _ws(ws)
    _check(lib().pcl_maxpool2x2_bwd_colsum(N, H, W, C, _ptr(x), _ptr(dy), _ptr(relu_mask_src), _ptr(dx),
                                           _ptr(dx_colsum), wp, wb, _stream(stream)), "pcl_maxpool2x2_bwd_colsum")


def conv_bwd_data_noalloc(d, dy, w, relu_mask_src, dx, stream=None):
    """Backward-data without a caller workspace (for callers that cannot allocate device memory): the
    library's built-in 16 MiB scratch array is used instead.  Calls that may overlap on the GPU race on it."""
    _check(lib().pcl_conv_bwd_data_noalloc(ctypes.byref(d), _ptr(dy), _ptr(w), _ptr(relu_mask_src), _ptr(dx),
                                           _stream(stream)), "pcl_conv_bwd_data_noalloc")


def noalloc_scratch_bytes() -> int:
    return int(lib().pcl_noalloc_scratch_bytes())


def conv_bwd_weights(d, x, dy, dw, dbias=None, deterministic=True, ws=None, stream=None):
    wp, wb = _ws(ws)
    _check(lib().pcl_conv_bwd_weights(ctypes.byref(d), _ptr(x), _ptr(dy), _ptr(dw), _ptr(dbias),
                                      1 if deterministic else 0, wp, wb, _stream(stream)), "pcl_conv_bwd_weights")


def fc_fwd(N, C, K, x, w, bias, y, act=ACT_NONE, ws=None, stream=None):
    wp, wb = _ws(ws)
    _check(lib().pcl_fc_fwd(N, C, K, _ptr(x), _ptr(w), _ptr(bias), _ptr(y), act, wp, wb, _stream(stream)),
           "pcl_fc_fwd")


def fc_bwd(N, C, K, x, w, y, act, dy, dx, dw, dbias, ws=None, stream=None):
    wp, wb = _ws(ws)
    _check(lib().pcl_fc_bwd(N, C, K, _ptr(x), _ptr(w), _ptr(y), act, _ptr(dy), _ptr(dx), _ptr(dw), _ptr(dbias),
                            wp, wb, _stream(stream)), "pcl_fc_bwd")


def fc_bwd_fused(N, C, K, x, w, y, act, dy, dx, x_act, dx_colsum, dw, dbias, ws=None, stream=None):
    """fc_bwd with the gradient of the activation that produced x (x_act) and the column sums of dx (the bias
    gradient of the layer below) formed in the backpropagation kernel's epilogue."""
    wp, wb = _ws(ws)
    _check(lib().pcl_fc_bwd_fused(N, C, K, _ptr(x), _ptr(w), _ptr(y), act, _ptr(dy), _ptr(dx), x_act, _ptr(dx_colsum),
                                  _ptr(dw), _ptr(dbias), wp, wb, _stream(stream)), "pcl_fc_bwd_fused")


def conv_bwd_weights_sgd_workspace_bytes(d) -> int:
    return int(lib().pcl_conv_bwd_weights_sgd_workspace_bytes(ctypes.byref(d)))


def conv_bwd_weights_sgd(d, x, dy, w, lr, dbias=None, ws=None, stream=None):
    """w <- w - lr * dw(x, dy) in place, the update applied by the weight gradient's second pass (dw is not stored)."""
    wp, wb = _ws(ws)
    _check(lib().pcl_conv_bwd_weights_sgd(ctypes.byref(d), _ptr(x), _ptr(dy), _ptr(w), ctypes.c_float(lr), _ptr(dbias),
                                          wp, wb, _stream(stream)), "pcl_conv_bwd_weights_sgd")


def fc_bwd_fused_sgd_workspace_bytes(N, C, K) -> int:
    return int(lib().pcl_fc_bwd_fused_sgd_workspace_bytes(N, C, K))


def fc_bwd_fused_sgd(N, C, K, x, w, y, act, dy, dx, x_act, dx_colsum, lr, dbias, ws=None, stream=None):
    """fc_bwd_fused with the SGD step folded in: dx from the old weights first, then w <- w - lr * dw in place."""
    wp, wb = _ws(ws)
    _check(lib().pcl_fc_bwd_fused_sgd(N, C, K, _ptr(x), _ptr(w), _ptr(y), act, _ptr(dy), _ptr(dx), x_act, _ptr(dx_colsum),
                                      ctypes.c_float(lr), _ptr(dbias), wp, wb, _stream(stream)), "pcl_fc_bwd_fused_sgd")


def plan_cache_stats():
    """(hits, misses): tensor-core launches served from the launch-plan cache / launches that built their plan."""
    h, m = ctypes.c_ulonglong(0), ctypes.c_ulonglong(0)
    _check(lib().pcl_plan_cache_stats(ctypes.byref(h), ctypes.byref(m)), "pcl_plan_cache_stats")
    return int(h.value), int(m.value)


def sgd_update(w, dw, lr, stream=None):
    _check(lib().pcl_sgd_update(_ptr(w), _ptr(dw), w.numel(), ctypes.c_float(lr), _stream(stream)), "pcl_sgd_update")


def maxpool2x2_fwd(N, H, W, C, x, y, stream=None):
    _check(lib().pcl_maxpool2x2_fwd(N, H, W, C, _ptr(x), _ptr(y), _stream(stream)), "pcl_maxpool2x2_fwd")


def maxpool2x2_bwd(N, H, W, C, x, dy, relu_mask_src, dx, stream=None):
    _check(lib().pcl_maxpool2x2_bwd(N, H, W, C, _ptr(x), _ptr(dy), _ptr(relu_mask_src), _ptr(dx), _stream(stream)),
           "pcl_maxpool2x2_bwd")


def softmax_xent(N, K, logits, labels, loss, dlogits, stream=None):
    assert labels.dtype == torch.int32
    _check(lib().pcl_softmax_xent(N, K, _ptr(logits), _ptr(labels), _ptr(loss), _ptr(dlogits), _stream(stream)),
           "pcl_softmax_xent")


_DTYPES = {torch.float32: F32, torch.bfloat16: BF16, torch.float16: F16}


def dtype_code(t) -> int:
    """The library's type code of a tensor (PCL_F32 / PCL_BF16 / PCL_F16)."""
    if t.dtype not in _DTYPES:
        raise TypeError(f"fp32, bf16 or fp16 tensors are wanted, not {t.dtype}")
    return _DTYPES[t.dtype]


def _typed(where, sizes, typed, fp32=(), int32=(), stream=None, ws=None):
    """Checks the tensors of a call -- (tensor, element count) pairs, None allowed; all contiguous, on the current device,
    and so the workspace -- and returns the type code that those of `typed` share, and the stream handle.  (Written for few interpreter steps: the
    smallest of these calls launch a kernel of two microseconds.)"""
    for n in sizes:
        if type(n) is not int or n <= 0 or n > 2147483647:          # (ctypes would cut larger ones to 32 bits)
            raise PclError(ERR_BAD_ARG, where)
    first = typed[0][0]
    want, dev = first.dtype, first.get_device()
    code = _DTYPES.get(want, -1)
    ok = code >= 0 and dev >= 0
    for t, n in typed:
        if t is not None and not (t.dtype is want and t.numel() == n and t.get_device() == dev and t.is_contiguous()):
            ok = False
    for t, n in fp32:
        if t is not None and not (t.dtype is torch.float32 and t.numel() == n and t.get_device() == dev and t.is_contiguous()):
            ok = False
    for t, n in int32:
        if not (t.dtype is torch.int32 and t.numel() == n and t.get_device() == dev and t.is_contiguous()):
            ok = False
    if ws is not None and ws.get_device() != dev:
        ok = False
    if not ok:
        _explain(where, typed, fp32, int32)
    if dev != torch.cuda.current_device():
        raise ValueError(f"{where}: all tensors must be on the current CUDA device")
    return code, (stream.cuda_stream if stream is not None else _raw_stream(dev))


def _explain(where, typed, fp32, int32):
    """Raises what is wrong with the tensors of a call."""
    first = typed[0][0]
    dtype_code(first)
    for group, want in ((typed, first.dtype), (fp32, torch.float32), (int32, torch.int32)):
        for t, n in group:
            if t is None:
                continue
            if t.dtype != want:
                raise TypeError(f"{where}: a {want} tensor is wanted, not {t.dtype}")
            if t.numel() != n or not t.is_contiguous():
                raise ValueError(f"{where}: a contiguous tensor of {n} elements is wanted")
    raise ValueError(f"{where}: all tensors must be on the current CUDA device")


def _raw_stream(dev: int) -> int:
    return torch.cuda.current_stream(dev).cuda_stream


if hasattr(torch._C, "_cuda_getCurrentRawStream"):          # (the handle without a Stream object around it)
    _raw_stream = torch._C._cuda_getCurrentRawStream


def _addr(t):
    """Address of a tensor that _typed() has checked (0 for None)."""
    return 0 if t is None else t.data_ptr()


def _id(v):
    """pad_id / ignore_label as the library takes it."""
    if v is None:
        return NO_ID
    v = int(v)
    if not -2 ** 31 <= v < 2 ** 31:          # (ctypes would cut it to 32 bits, i.e. to another id)
        raise ValueError(f"an id or label is a 32-bit integer, not {v}")
    return v


def _size(n):
    """A size as the library takes it: what does not fit in 32 bits is refused there like the largest that does."""
    return min(n, 2147483647)


def embedding_workspace_bytes(N, V, C) -> int:
    return int(lib().pcl_embedding_workspace_bytes(*map(_size, (N, V, C))))


def embedding_fwd(N, V, C, ids, table, scale, out, pad_id=None, stream=None):
    """out[n] = scale * table[ids[n]]; rows of pad_id are zero."""
    d, s = _typed("pcl_embedding_fwd", (N, V, C), [(table, V * C), (out, N * C)], int32=[(ids, N)], stream=stream)
    _check(lib().pcl_embedding_fwd(N, V, C, d, _addr(ids), _addr(table), scale, _id(pad_id), _addr(out),
                                   s), "pcl_embedding_fwd")


def embedding_bwd(N, V, C, ids, dy, scale, dtable, pad_id=None, ws=None, stream=None):
    """dtable[v] = scale * sum of dy[n] over the tokens n with ids[n] == v; every row is written."""
    d, s = _typed("pcl_embedding_bwd", (N, V, C), [(dy, N * C), (dtable, V * C)], int32=[(ids, N)], stream=stream, ws=ws)
    wp, wb = _ws(ws)
    _check(lib().pcl_embedding_bwd(N, V, C, d, _addr(ids), _addr(dy), scale, _id(pad_id), _addr(dtable), wp, wb,
                                   s), "pcl_embedding_bwd")


def embedding_bwd_sgd(N, V, C, ids, dy, scale, table, lr, pad_id=None, ws=None, stream=None):
    """table[v] -= lr * dtable[v] in place for the rows that occur; dtable is not stored."""
    d, s = _typed("pcl_embedding_bwd_sgd", (N, V, C), [(dy, N * C), (table, V * C)], int32=[(ids, N)], stream=stream, ws=ws)
    wp, wb = _ws(ws)
    _check(lib().pcl_embedding_bwd_sgd(N, V, C, d, _addr(ids), _addr(dy), scale, _id(pad_id), _addr(table),
                                       lr, wp, wb, s), "pcl_embedding_bwd_sgd")


def fc_softmax_xent_workspace_bytes(N, C, K, dtype: int, which: int) -> int:
    """dtype: dtype_code() of the operands; which: PASS_FWD or PASS_BWD_DATA."""
    return int(lib().pcl_fc_softmax_xent_workspace_bytes(*map(_size, (N, C, K)), dtype, which))


def fc_softmax_xent_fwd(N, C, K, x, w, bias, labels, loss, row_loss, lse, ignore_label=None, ws=None, stream=None):
    """Mean loss, loss and log-sum-exp of each row of softmax(x w^T + bias), without storing the logits."""
    d, s = _typed("pcl_fc_softmax_xent_fwd", (N, C, K), [(x, N * C), (w, K * C), (bias, K)],
               [(loss, 1), (row_loss, N), (lse, N)], [(labels, N)], stream=stream, ws=ws)
    wp, wb = _ws(ws)
    _check(lib().pcl_fc_softmax_xent_fwd(N, C, K, d, _addr(x), _addr(w), _addr(bias), _addr(labels), _id(ignore_label),
                                         _addr(loss), _addr(row_loss), _addr(lse), wp, wb, s),
           "pcl_fc_softmax_xent_fwd")


def fc_softmax_xent_bwd(N, C, K, x, w, bias, labels, lse, row_grad, dx, dw, dbias, ignore_label=None, ws=None, stream=None):
    """dx (or None), dw and dbias (or None) from the forward call's lse; row_grad: gradient of each row's loss, or None for
    the gradient of the mean."""
    d, s = _typed("pcl_fc_softmax_xent_bwd", (N, C, K), [(x, N * C), (w, K * C), (bias, K), (dx, N * C), (dw, K * C), (dbias, K)],
               [(lse, N), (row_grad, N)], [(labels, N)], stream=stream, ws=ws)
    wp, wb = _ws(ws)
    _check(lib().pcl_fc_softmax_xent_bwd(N, C, K, d, _addr(x), _addr(w), _addr(bias), _addr(labels), _id(ignore_label), _addr(lse),
                                         _addr(row_grad), _addr(dx), _addr(dw), _addr(dbias), wp, wb, s),
           "pcl_fc_softmax_xent_bwd")


def orthogonalize_workspace_bytes(count, M, N) -> int:
    return int(lib().pcl_orthogonalize_workspace_bytes(*map(_size, (count, M, N))))


def orthogonalize(count, M, N, g, out, steps=5, ws=None, stream=None):
    """out = g / |g| after `steps` Newton-Schulz steps, for each of `count` M x N matrices."""
    d, s = _typed("pcl_orthogonalize", (count, M, N, steps), [(g, count * M * N), (out, count * M * N)], stream=stream, ws=ws)
    wp, wb = _ws(ws)
    _check(lib().pcl_orthogonalize(count, M, N, d, _addr(g), _addr(out), steps, wp, wb, s), "pcl_orthogonalize")


def orthogonal_update(count, M, N, w, dw, momentum, mu, nesterov, lr, weight_decay=0.0, steps=5, ws=None, stream=None):
    """momentum <- mu momentum + dw, then w <- (1 - lr weight_decay) w - lr sqrt(max(1, M/N)) * orthogonalize(direction)."""
    d, s = _typed("pcl_orthogonal_update", (count, M, N, steps), [(w, count * M * N), (dw, count * M * N)], [(momentum, count * M * N)], stream=stream, ws=ws)
    wp, wb = _ws(ws)
    _check(lib().pcl_orthogonal_update(count, M, N, d, _addr(w), _addr(dw), _addr(momentum), mu,
                                       1 if nesterov else 0, lr, weight_decay, steps, wp, wb,
                                       s), "pcl_orthogonal_update")


E4M3 = torch.float8_e4m3fn


def _bytes8(where, like, tensors, types=(E4M3, torch.uint8)):
    """Checks the 8-bit tensors of a call: (tensor, element count) pairs, contiguous, on the device of `like`."""
    dev = like.get_device()
    for t, n in tensors:
        if t.dtype not in types:
            raise TypeError(f"{where}: an 8-bit tensor (float8_e4m3fn or uint8) is wanted, not {t.dtype}")
        if t.numel() != n or not t.is_contiguous():
            raise ValueError(f"{where}: a contiguous tensor of {n} elements is wanted")
        if t.get_device() != dev:
            raise ValueError(f"{where}: all tensors must be on the current CUDA device")


def rms_norm_fwd(N, C, x, residual, w, eps, h, y, rstd=None, stream=None):
    """h = x + residual (residual and h may be None), y = h / sqrt(mean(h^2) + eps) * w, rstd = 1 / sqrt(mean(h^2) + eps)."""
    if _calls is not None and _done(_calls.rms_norm_fwd(N, C, x, residual, w, eps, h, y, rstd, stream), "pcl_rms_norm_fwd"):
        return
    d, s = _typed("pcl_rms_norm_fwd", (N, C), [(x, N * C), (residual, N * C), (w, C), (h, N * C), (y, N * C)], [(rstd, N)], stream=stream)
    _check(lib().pcl_rms_norm_fwd(N, C, d, _addr(x), _addr(residual), _addr(w), eps, _addr(h), _addr(y), _addr(rstd), s),
           "pcl_rms_norm_fwd")


def rms_norm_fwd_q8(N, C, x, residual, w, eps, h, y8, y_scale, rstd=None, stream=None):
    """rms_norm_fwd with y as e4m3 values (a float8_e4m3fn or uint8 tensor) and a scale for each row."""
    if _calls is not None and _done(_calls.rms_norm_fwd_q8(N, C, x, residual, w, eps, h, y8, y_scale, rstd, stream), "pcl_rms_norm_fwd_q8"):
        return
    d, s = _typed("pcl_rms_norm_fwd_q8", (N, C), [(x, N * C), (residual, N * C), (w, C), (h, N * C)], [(rstd, N), (y_scale, N)], stream=stream)
    _bytes8("pcl_rms_norm_fwd_q8", x, [(y8, N * C)])
    _check(lib().pcl_rms_norm_fwd_q8(N, C, d, _addr(x), _addr(residual), _addr(w), eps, _addr(h), _addr(y8), _addr(y_scale),
                                     _addr(rstd), s), "pcl_rms_norm_fwd_q8")


def rms_norm_workspace_bytes(N, C) -> int:
    return int(lib().pcl_rms_norm_workspace_bytes(*map(_size, (N, C))))


def rms_norm_bwd(N, C, h, w, rstd, dy, dh, dx, dw, ws=None, stream=None):
    """dx = dh (or 0) + the gradient through the norm; dw (or None): the gradient of its weights."""
    if _calls is not None and _done(_calls.rms_norm_bwd(N, C, h, w, rstd, dy, dh, dx, dw, ws, stream), "pcl_rms_norm_bwd"):
        return
    d, s = _typed("pcl_rms_norm_bwd", (N, C), [(h, N * C), (w, C), (dy, N * C), (dh, N * C), (dx, N * C), (dw, C)], [(rstd, N)],
                  stream=stream, ws=ws)
    wp, wb = _ws(ws)
    _check(lib().pcl_rms_norm_bwd(N, C, d, _addr(h), _addr(w), _addr(rstd), _addr(dy), _addr(dh), _addr(dx), _addr(dw), wp, wb, s),
           "pcl_rms_norm_bwd")


def quantize_rows(N, C, x, q, scale, stream=None):
    """q: the rows of x as e4m3 values, scale: max |row| / 448."""
    if _calls is not None and _done(_calls.quantize_rows(N, C, x, q, scale, stream), "pcl_quantize_rows"):
        return
    d, s = _typed("pcl_quantize_rows", (N, C), [(x, N * C)], [(scale, N)], stream=stream)
    _bytes8("pcl_quantize_rows", x, [(q, N * C)])
    _check(lib().pcl_quantize_rows(N, C, d, _addr(x), _addr(q), _addr(scale), s), "pcl_quantize_rows")


def fc_q8_workspace_bytes(N, C, K) -> int:
    return int(lib().pcl_fc_q8_workspace_bytes(*map(_size, (N, C, K))))


def fc_q8_fwd(N, C, K, x, x_scale, w, w_scale, bias, y, act=ACT_NONE, ws=None, stream=None):
    """y = act(x_scale[n] * w_scale[k] * (x w^T) + bias) of e4m3 operands (float8_e4m3fn or uint8 tensors)."""
    if _calls is not None and _done(_calls.fc_q8_fwd(N, C, K, y, bias, x, x_scale, w, w_scale, act, ws, stream), "pcl_fc_q8_fwd"):
        return
    d, s = _typed("pcl_fc_q8_fwd", (N, C, K), [(y, N * K), (bias, K)], [(x_scale, N), (w_scale, K)], stream=stream, ws=ws)
    _bytes8("pcl_fc_q8_fwd", y, [(x, N * C), (w, K * C)])
    wp, wb = _ws(ws)
    _check(lib().pcl_fc_q8_fwd(N, C, K, d, _addr(x), _addr(x_scale), _addr(w), _addr(w_scale), _addr(bias), _addr(y), act, wp, wb, s),
           "pcl_fc_q8_fwd")


class TensorList:
    """Several tensors (contiguous, of one device, each fp32, bf16 or fp16) as the calls over many tensors take them.  The list is of the
    tensors' memory as it is when the list is made, and keeps that memory alive."""

    def __init__(self, tensors):
        self.tensors = [t.detach() for t in tensors]
        n = len(self.tensors)
        if n == 0:
            raise ValueError("a list of one tensor or more is wanted")
        self.device = self.tensors[0].get_device()
        for t in self.tensors:
            if t.get_device() != self.device or self.device < 0 or not t.is_contiguous():
                raise ValueError("contiguous tensors on one CUDA device are wanted")
        self.dtypes = tuple(dtype_code(t) for t in self.tensors)
        self.sizes = tuple(t.numel() for t in self.tensors)
        self._pointers = (ctypes.c_void_p * n)(*[t.data_ptr() if t.numel() else None for t in self.tensors])
        self._sizes = (ctypes.c_size_t * n)(*self.sizes)
        self._dtypes = (ctypes.c_int * n)(*self.dtypes)
        self.layout = bytes((ctypes.c_int * 1)(self.device)) + bytes(self._sizes) + bytes(self._dtypes)       # (alike for lists that are alike)
        spans = sorted((t.data_ptr(), t.data_ptr() + t.numel() * t.element_size()) for t in self.tensors if t.numel())
        self.overlaps = any(a[1] > b[0] for a, b in zip(spans, spans[1:]))       # (then it can only be read)
        self.pointers, self.counts, self.types = (ctypes.addressof(a) for a in (self._pointers, self._sizes, self._dtypes))

    def __len__(self):
        return len(self.tensors)


def _lists(where, lists, norm, stream, ws):
    """Checks tensor lists (alike in sizes and types), the norm and the workspace; returns the stream handle."""
    first = lists[0]
    dev = first.device
    for other in lists[1:]:
        if other.layout != first.layout:
            raise ValueError(f"{where}: lists of the same sizes and types, on the same device, are wanted")
    if norm.dtype is not torch.float32:
        raise TypeError(f"{where}: a torch.float32 tensor is wanted, not {norm.dtype}")
    if norm.numel() != 1:
        raise ValueError(f"{where}: a tensor of 1 element is wanted")
    if norm.get_device() != dev or (ws is not None and ws.get_device() != dev) or dev != torch.cuda.current_device():
        raise ValueError(f"{where}: all tensors must be on the current CUDA device")
    return stream.cuda_stream if stream is not None else _raw_stream(dev)


def grad_norm_workspace_bytes(tensors) -> int:
    """tensors: a TensorList, or how many tensors."""
    return int(lib().pcl_grad_norm_workspace_bytes(_size(tensors if isinstance(tensors, int) else len(tensors))))


def grad_norm(grads, norm, ws=None, stream=None):
    """norm = the 2-norm of all tensors of the list `grads` together."""
    if _calls is not None and _done(_calls.grad_norm(grads.device, len(grads.tensors), grads.pointers, grads.counts, grads.types, norm, ws, stream), "pcl_grad_norm"):
        return
    s = _lists("pcl_grad_norm", (grads,), norm, stream, ws)
    wp, wb = _ws(ws)
    _check(lib().pcl_grad_norm(len(grads), grads.pointers, grads.counts, grads.types, _addr(norm), wp, wb, s), "pcl_grad_norm")


def grad_clip(grads, out, max_norm, norm, ws=None, stream=None):
    """out[i] = grads[i] * min(1, max_norm / (norm + 1e-6)); out may be grads."""
    if out.overlaps:
        raise ValueError("pcl_grad_clip: tensors that are written must not overlap")
    if _calls is not None and out.layout == grads.layout and _done(_calls.grad_clip(
            grads.device, len(grads.tensors), grads.pointers, out.pointers, grads.counts, grads.types, max_norm, norm, ws, stream), "pcl_grad_clip"):
        return
    s = _lists("pcl_grad_clip", (grads, out), norm, stream, ws)
    wp, wb = _ws(ws)
    _check(lib().pcl_grad_clip(len(grads), grads.pointers, out.pointers, grads.counts, grads.types, max_norm, _addr(norm), wp, wb, s),
           "pcl_grad_clip")


def sgd_update_clipped(params, grads, lr, max_norm, norm, ws=None, stream=None):
    """params[i] -= lr * min(1, max_norm / (norm + 1e-6)) * grads[i], in place."""
    if params.overlaps:
        raise ValueError("pcl_sgd_update_clipped: tensors that are written must not overlap")
    if _calls is not None and params.layout == grads.layout and _done(_calls.sgd_update_clipped(
            grads.device, len(grads.tensors), params.pointers, grads.pointers, grads.counts, grads.types, lr, max_norm, norm, ws, stream),
            "pcl_sgd_update_clipped"):
        return
    s = _lists("pcl_sgd_update_clipped", (grads, params), norm, stream, ws)
    wp, wb = _ws(ws)
    _check(lib().pcl_sgd_update_clipped(len(grads), params.pointers, grads.pointers, grads.counts, grads.types, lr, max_norm,
                                        _addr(norm), wp, wb, s), "pcl_sgd_update_clipped")


def sample_tokens_workspace_bytes(N, K) -> int:
    return int(lib().pcl_sample_tokens_workspace_bytes(*map(_size, (N, K))))


def sample_tokens(N, K, logits, uniform, token, temperature=None, top_k=None, top_p=None, min_p=None, logprob=None, ws=None, stream=None):
    """token[n] of each row of logits, chosen by uniform[n] after temperature, top-k, top-p and min-p ([N] tensors, top_k int32)."""
    if _calls is not None and _done(_calls.sample_tokens(N, K, logits, uniform, token, temperature, top_k, top_p, min_p, logprob, ws, stream), "pcl_sample_tokens"):
        return
    ints = [(token, N)] if top_k is None else [(token, N), (top_k, N)]
    d, s = _typed("pcl_sample_tokens", (N, K), [(logits, N * K)], [(uniform, N), (temperature, N), (top_p, N), (min_p, N), (logprob, N)], ints,
                  stream=stream, ws=ws)
    wp, wb = _ws(ws)
    _check(lib().pcl_sample_tokens(N, K, d, _addr(logits), _addr(uniform), _addr(temperature), _addr(top_k), _addr(top_p), _addr(min_p),
                                   _addr(token), _addr(logprob), wp, wb, s), "pcl_sample_tokens")


def last_device_status(stream=None) -> int:
    return int(lib().pcl_last_device_status(_stream(stream)))


def check_device_status(stream=None):
    _check(last_device_status(stream), "device status")


def launch_count() -> int:
    return int(lib().pcl_launch_count())


def profile_begin():
    _check(lib().pcl_profile_begin(), "pcl_profile_begin")


def profile_end():
    """Returns {"<pass>/<kernel>": dict(launches, total_ms, work)} for the launches since profile_begin()."""
    arr = (KernelStat * 128)()
    n = ctypes.c_int(0)
    _check(lib().pcl_profile_end(arr, 128, ctypes.byref(n)), "pcl_profile_end")
    return {arr[i].name.decode(): dict(launches=int(arr[i].launches), total_ms=float(arr[i].total_ms),
                                       work=float(arr[i].work)) for i in range(n.value)}
