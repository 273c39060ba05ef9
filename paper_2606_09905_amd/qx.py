"""Thin Python binding of libqx (the C ABI in include/qx.h).

Argument marshalling only: every step of every operation runs in the HIP
kernels of libqx.so.  torch supplies device memory and the current stream.
If the library is missing, every call raises; there is no fallback.
"""
from __future__ import annotations

import ctypes
import math
import os
import re

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libqx.so")
HEADER_PATH = os.path.join(os.path.dirname(_HERE), "include", "qx.h")

# qx_status
OK, ERR_INVALID_ARG, ERR_UNSUPPORTED, ERR_RANGE, ERR_OUT_OF_MEMORY, ERR_DEVICE = range(6)
STATUS_NAMES = ["OK", "INVALID_ARG", "UNSUPPORTED", "RANGE", "OUT_OF_MEMORY", "DEVICE"]

# qx_attn_dtype
DT_F32, DT_I32 = 0, 1
# qx_pool_kind
POOL_AVG_I32, POOL_MAX_F32 = 0, 1

# qx_float_type
FT_F32, FT_F16, FT_BF16 = 0, 1, 2

# qx_route
ROUTE = {
    "auto": 0, "i8_direct": 1, "f16_exact": 2, "i8_karatsuba": 3, "i8_offset4": 4,
    "valu_dot2": 5, "s24_valu": 6, "s24_i8limb": 7,
    "attn_f32_mfma": 8, "attn_i32_mfma": 9, "attn_i32_valu": 10, "attn_f32_valu": 11,
    "f32_mfma": 12, "f32_valu": 13, "lin_mfma": 14, "lin_step": 15,
}
ROUTE_NAME = {v: k for k, v in ROUTE.items()}


class QxError(RuntimeError):
    def __init__(self, status: int, message: str):
        self.status = status
        name = STATUS_NAMES[status] if 0 <= status < len(STATUS_NAMES) else str(status)
        super().__init__(f"qx {name}: {message}")


class PlanInfo(ctypes.Structure):
    _fields_ = [
        ("route", ctypes.c_int32), ("chunk", ctypes.c_int32), ("products", ctypes.c_int32),
        ("tile_m", ctypes.c_int32), ("tile_n", ctypes.c_int32), ("tile_k", ctypes.c_int32),
        ("kernels", ctypes.c_int32), ("exact_no_wrap", ctypes.c_int32),
        ("operand_format", ctypes.c_int32), ("k_splits", ctypes.c_int32),
        ("workspace_bytes", ctypes.c_int64),
    ]

    def as_dict(self) -> dict:
        d = {f: getattr(self, f) for f, _ in self._fields_}
        d["route_name"] = ROUTE_NAME.get(self.route, str(self.route))
        return d


_lib = None
_i64, _i32, _p, _f32 = ctypes.c_int64, ctypes.c_int32, ctypes.c_void_p, ctypes.c_float


def lib() -> ctypes.CDLL:
    """Load libqx.so (built in-tree); raises if it has not been built."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(f"{LIB_PATH} is missing: build it with "
                               "`python -m paper_2606_09905_amd.build`")
        L = ctypes.CDLL(LIB_PATH)
        sig = {
            "qgemm_i16i32": [_p, _p, _p, _i64, _i64, _i64, _i64, _i32, _i32, _p],
            "qgemm_i32_s24": [_p, _p, _p, _i64, _i64, _i64, _i64, _p],
            "qgemm_i16i32_noalloc": [_p, _p, _p, _i64, _i64, _i64, _i64, _i32, _i32, _p],
            "conv2d_gemm": [_p, _p, _p] + [_i64] * 9 + [_i32, _i32, _p],
            "conv2d_gemm_t": [_i32, _p, _p, _p] + [_i64] * 9 + [_p],
            "attn_core": [_i32, _p, _p, _p, _p, _i64, _i64, _i32, _p],
            "qx_exec_create_gemm_i16i32": [_p, _i64, _i64, _i64, _i64, _i32, _i32],
            "qx_exec_create_gemm_i32_s24": [_p, _i64, _i64, _i64, _i64],
            "qx_exec_create_conv2d": [_p] + [_i64] * 9 + [_i32, _i32],
            "qx_exec_create_attn": [_p, _i32, _i64, _i64, _i32],
            "qx_exec_create_gemm_i16i32_route": [_p, _i64, _i64, _i64, _i64, _i32, _i32, _i32],
            "qx_exec_create_gemm_i32_s24_route": [_p, _i64, _i64, _i64, _i64, _i32],
            "qx_exec_create_conv2d_route": [_p] + [_i64] * 9 + [_i32, _i32, _i32],
            "qx_exec_create_attn_route": [_p, _i32, _i64, _i64, _i32, _i32],
            "qx_exec_create_conv2d_t": [_p, _i32] + [_i64] * 9 + [_i32],
            "qx_testing_host_double": [_i32],
            "qx_exec_run": [_p, _p, _p, _p],
            "qx_exec_plan": [_p, _p],
            "qx_exec_profile": [_p, _p, _p, _p, _i32, _p, _p, _i32],
            "qx_exec_destroy": [_p],
            "qx_plan_gemm_i16i32": [_p, _i64, _i64, _i64, _i64, _i32, _i32, _i32],
            "qx_plan_gemm_i32_s24": [_p, _i64, _i64, _i64, _i64, _i32],
            "qx_plan_conv2d": [_p] + [_i64] * 9 + [_i32, _i32, _i32],
            "qx_plan_conv2d_t": [_p, _i32] + [_i64] * 9 + [_i32],
            "qx_plan_attn": [_p, _i32, _i64, _i64, _i32, _i32],
            "minmax": [_p, _i64, _i32, _p, _p],
            "pool2x2": [_i32, _p, _p, _i64, _i64, _i64, _i64, _p],
            "qx_exec_create_minmax": [_p, _i64, _i32],
            "qx_exec_create_pool2x2": [_p, _i32, _i64, _i64, _i64, _i64],
            "qx_plan_minmax": [_p, _i64, _i32],
            "qx_plan_lenet_i32": [_p, _i64],
            "qx_exec_create_lenet_i32": [_p, _i64],
            "qx_plan_pool2x2": [_p, _i32, _i64, _i64, _i64, _i64],
            "sdpa_f32": [_p, _p, _p, _p, _i64, _i64, _i64, _f32, _i32, _p],
            "qx_exec_create_sdpa_f32": [_p, _i64, _i64, _i64, _f32, _i32],
            "qx_plan_sdpa_f32": [_p, _i64, _i64, _i64, _f32, _i32],
            "quantize_rows_i8": [_i32, _p, _p, _p, _i64, _i64, _i64, _p],
            "qgemm_i8_scaled": [_i32] + [_p] * 6 + [_i64] * 3 + [_p],
            "linear_i8": [_i32] + [_p] * 5 + [_i64] * 4 + [_p, _i64, _p],
            "lin_attn": [_i32] + [_p] * 8 + [_i64] * 5 + [_p, _f32, _p, _i64, _p],
            "lin_attn_step": [_i32] + [_p] * 6 + [_i64] * 4 + [_p, _f32, _p],
            "lin_attn_backward": [_i32] + [_p] * 12 + [_i64] * 5 + [_p, _f32, _p, _i64, _p],
            "qx_exec_create_gemm_i8_scaled": [_p, _i32] + [_i64] * 3 + [_i32],
            "qx_exec_create_linear_i8": [_p, _i32] + [_i64] * 3 + [_i32],
            "qx_exec_create_lin_attn": [_p, _i32] + [_i64] * 5 + [_f32],
            "qx_exec_create_lin_attn_step": [_p, _i32] + [_i64] * 4 + [_f32],
            "qx_plan_quantize_rows_i8": [_p, _i32, _i64, _i64],
            "qx_plan_gemm_i8_scaled": [_p, _i32] + [_i64] * 3,
            "qx_plan_linear_i8": [_p, _i32] + [_i64] * 3,
            "qx_plan_lin_attn": [_p, _i32] + [_i64] * 5,
            "qx_plan_lin_attn_step": [_p, _i32] + [_i64] * 4,
            "qx_plan_lin_attn_backward": [_p, _i32] + [_i64] * 5,
        }
        for name, args in sig.items():
            fn = getattr(L, name)
            fn.argtypes = args
            fn.restype = ctypes.c_int
        L.qx_last_error.argtypes = []
        L.qx_last_error.restype = ctypes.c_char_p
        L.qx_release_cache.argtypes = []
        L.qx_release_cache.restype = None
        L.qx_testing_counters.argtypes = [_p, _i32]
        L.qx_testing_counters.restype = None
        _lib = L
    return _lib


def header_functions(path: str = HEADER_PATH) -> list[str]:
    """Names of every function a header (default include/qx.h) declares."""
    with open(path) as f:
        text = f.read()
    text = re.sub(r"/\*.*?\*/", "", text, flags=re.S)
    text = re.sub(r"^\s*#.*$", "", text, flags=re.M)     # preprocessor lines
    return sorted(set(re.findall(r"\b([A-Za-z_]\w*)\s*\(", text)) -
                  {"if", "defined", "sizeof"})


def check(status: int) -> None:
    if status != OK:
        msg = lib().qx_last_error()
        raise QxError(status, msg.decode() if msg else "")


# ---------------------------------------------------------------------------
# torch marshalling
# ---------------------------------------------------------------------------
_torch_module = None


def _torch():
    global _torch_module
    if _torch_module is None:
        import torch
        _torch_module = torch
    return _torch_module


_current = None   # (device getter, current raw stream of a device), once CUDA is initialised


def _stream(stream):
    """The HIP stream handle (an int) of a torch stream, a raw handle, or
    None for torch's current stream."""
    global _current
    if stream is None:
        # the handle straight from torch's native getters where it has them:
        # building a Stream object costs as much as the rest of a small call
        if _current is not None:
            return _current[1](_current[0]())
        torch = _torch()
        handle = torch.cuda.current_stream().cuda_stream
        get = [getattr(torch._C, n, None) for n in ("_cuda_getDevice", "_cuda_getCurrentRawStream")]
        if all(get):
            _current = tuple(get)
        return handle
    handle = getattr(stream, "cuda_stream", None)
    return handle if handle is not None else int(stream)


def _dev_tensor(t, dtype, name):
    torch = _torch()
    if not isinstance(t, torch.Tensor):
        raise TypeError(f"{name} must be a torch.Tensor")
    if t.dtype != dtype:
        raise TypeError(f"{name} must be {dtype}, got {t.dtype}")
    if t.device.type != "cuda":
        raise ValueError(f"{name} must be on a GPU device")
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    return ctypes.c_void_p(t.data_ptr())


def _gemm_shapes(A, B):
    if A.dim() == 2 and B.dim() == 2:
        (M, K), (K2, N) = A.shape, B.shape
        batch, out_shape = 1, (M, N)
    elif A.dim() == 3 and B.dim() == 3:
        (batch, M, K), (b2, K2, N) = A.shape, B.shape
        if b2 != batch:
            raise ValueError("batch mismatch")
        out_shape = (batch, M, N)
    else:
        raise ValueError("A and B must both be 2-D or both 3-D")
    if K2 != K:
        raise ValueError(f"inner dimensions differ: {K} vs {K2}")
    return batch, M, N, K, out_shape


def qgemm_i16i32(A, B, bound_a: int = 0, bound_b: int = 0, out=None, stream=None):
    """C = A @ B, int16 in, int32 out (exact mod 2^32); [M,K]@[K,N] or batched."""
    torch = _torch()
    batch, M, N, K, shape = _gemm_shapes(A, B)
    if out is None:
        out = torch.empty(shape, dtype=torch.int32, device=A.device)
    check(lib().qgemm_i16i32(_dev_tensor(A, torch.int16, "A"), _dev_tensor(B, torch.int16, "B"),
                             _dev_tensor(out, torch.int32, "C"), M, N, K, batch,
                             int(bound_a), int(bound_b), _stream(stream)))
    return out


def qgemm_i16i32_noalloc(A, B, out, bound_a: int = 0, bound_b: int = 0, stream=None):
    """qgemm_i16i32 into a caller-provided `out`, with no device allocation
    (the library's fixed per-device scratch serves as workspace)."""
    torch = _torch()
    batch, M, N, K, shape = _gemm_shapes(A, B)
    if tuple(out.shape) != tuple(shape):
        raise ValueError(f"out must have shape {shape}")
    check(lib().qgemm_i16i32_noalloc(_dev_tensor(A, torch.int16, "A"), _dev_tensor(B, torch.int16, "B"),
                                     _dev_tensor(out, torch.int32, "C"), M, N, K, batch,
                                     int(bound_a), int(bound_b), _stream(stream)))
    return out


def qgemm_i32_s24(A, B, out=None, stream=None):
    """C = sext24(A) @ sext24(B) mod 2^32, int32 in and out."""
    torch = _torch()
    batch, M, N, K, shape = _gemm_shapes(A, B)
    if out is None:
        out = torch.empty(shape, dtype=torch.int32, device=A.device)
    check(lib().qgemm_i32_s24(_dev_tensor(A, torch.int32, "A"), _dev_tensor(B, torch.int32, "B"),
                              _dev_tensor(out, torch.int32, "C"), M, N, K, batch, _stream(stream)))
    return out


def conv_out_hw(H, W, KH, KW, stride, pad):
    return (H + 2 * pad - KH) // stride + 1, (W + 2 * pad - KW) // stride + 1


def conv2d_gemm(x, w, stride: int = 1, pad: int = 0, bound_x: int = 0, bound_w: int = 0,
                out=None, stream=None):
    """NCHW int16 x, OIHW int16 w -> NCHW int32 y (cross-correlation, zero padding)."""
    torch = _torch()
    N, Ci, H, W = x.shape
    Co, Ci2, KH, KW = w.shape
    if Ci2 != Ci:
        raise ValueError("channel mismatch")
    Ho, Wo = conv_out_hw(H, W, KH, KW, stride, pad)
    if out is None:
        out = torch.empty((N, Co, max(Ho, 0), max(Wo, 0)), dtype=torch.int32, device=x.device)
    check(lib().conv2d_gemm(_dev_tensor(x, torch.int16, "x"), _dev_tensor(w, torch.int16, "w"),
                            _dev_tensor(out, torch.int32, "y"), N, Ci, H, W, Co, KH, KW,
                            stride, pad, int(bound_x), int(bound_w), _stream(stream)))
    return out


def conv2d_gemm_t(x, w, stride: int = 1, pad: int = 0, out=None, stream=None):
    """Conv2D on float32 (fp32 sum) or int32 (smul24 contract, exact mod 2^32)
    NCHW x and OIHW w -> NCHW y of the same dtype."""
    torch = _torch()
    if x.dtype == torch.float32:
        dt = DT_F32
    elif x.dtype == torch.int32:
        dt = DT_I32
    else:
        raise TypeError("x must be float32 or int32")
    N, Ci, H, W = x.shape
    Co, Ci2, KH, KW = w.shape
    if Ci2 != Ci:
        raise ValueError("channel mismatch")
    Ho, Wo = conv_out_hw(H, W, KH, KW, stride, pad)
    if out is None:
        out = torch.empty((N, Co, max(Ho, 0), max(Wo, 0)), dtype=x.dtype, device=x.device)
    check(lib().conv2d_gemm_t(dt, _dev_tensor(x, x.dtype, "x"), _dev_tensor(w, x.dtype, "w"),
                              _dev_tensor(out, x.dtype, "y"), N, Ci, H, W, Co, KH, KW, stride, pad,
                              _stream(stream)))
    return out


def attn_core(Q, K, V, bound: int = 0, out=None, stream=None):
    """O = (Q K^T) V for [L, d] float32 or int32 tensors."""
    torch = _torch()
    if Q.dtype == torch.float32:
        dt = DT_F32
    elif Q.dtype == torch.int32:
        dt = DT_I32
    else:
        raise TypeError("Q must be float32 or int32")
    L, d = Q.shape
    if out is None:
        out = torch.empty((L, d), dtype=Q.dtype, device=Q.device)
    check(lib().attn_core(dt, _dev_tensor(Q, Q.dtype, "Q"), _dev_tensor(K, Q.dtype, "K"),
                          _dev_tensor(V, Q.dtype, "V"), _dev_tensor(out, Q.dtype, "O"), L, d,
                          int(bound), _stream(stream)))
    return out


def sdpa_f32(Q, K, V, scale: float = 1.0, causal: bool = False, out=None, stream=None):
    """softmax(scale Q K^T [causal mask]) V per head for float32 [..., L, d]
    tensors; leading dimensions are flattened into heads."""
    torch = _torch()
    if Q.dtype != torch.float32:
        raise TypeError("Q must be float32")
    if Q.dim() < 2 or K.shape != Q.shape or V.shape != Q.shape:
        raise ValueError("Q, K, V must share one shape [..., L, d]")
    L, d = Q.shape[-2], Q.shape[-1]
    BH = math.prod(Q.shape[:-2])
    if out is None:
        out = torch.empty(Q.shape, dtype=Q.dtype, device=Q.device)
    check(lib().sdpa_f32(_dev_tensor(Q, Q.dtype, "Q"), _dev_tensor(K, Q.dtype, "K"),
                         _dev_tensor(V, Q.dtype, "V"), _dev_tensor(out, Q.dtype, "O"), BH, L, d,
                         float(scale), 1 if causal else 0, _stream(stream)))
    return out


def minmax(x, out=None, stream=None):
    """(min, max) of a non-empty int32 or int16 tensor, as a 2-element tensor."""
    torch = _torch()
    if x.dtype not in (torch.int32, torch.int16):
        raise TypeError("x must be int32 or int16")
    if out is None:
        out = torch.empty(2, dtype=x.dtype, device=x.device)
    check(lib().minmax(_dev_tensor(x, x.dtype, "x"), x.numel(), x.element_size(),
                       _dev_tensor(out, x.dtype, "out"), _stream(stream)))
    return out


def pool2x2(x, out=None, stream=None):
    """2x2 / stride 2 pooling of an NCHW tensor: int32 -> floor average, float32 -> maximum."""
    torch = _torch()
    if x.dtype == torch.int32:
        kind = POOL_AVG_I32
    elif x.dtype == torch.float32:
        kind = POOL_MAX_F32
    else:
        raise TypeError("x must be int32 (average) or float32 (maximum)")
    N, C, H, W = x.shape
    if out is None:
        out = torch.empty((N, C, H // 2, W // 2), dtype=x.dtype, device=x.device)
    check(lib().pool2x2(kind, _dev_tensor(x, x.dtype, "x"), _dev_tensor(out, x.dtype, "y"),
                        N, C, H, W, _stream(stream)))
    return out


# ---------------------------------------------------------------------------
# operators of a language model's layer
#
# A token's step is a few microseconds on the GPU, so these keep the host's
# part short: one condition over all operands, and the checks one by one only
# where it fails, to say what is wrong.  None of them records an autograd
# graph, whatever its operands require.
# ---------------------------------------------------------------------------
_ftype = {}    # torch dtype -> qx_float_type
_need = {}     # (query, type, sizes) -> workspace bytes
_t_f32 = _t_i8 = _t_i32 = _get_device = None


def _serve_init():
    global _t_f32, _t_i8, _t_i32, _get_device
    torch = _torch()
    _t_f32, _t_i8, _t_i32 = torch.float32, torch.int8, torch.int32
    # torch's native getter where it has one (a CPU build of torch has none)
    _get_device = getattr(torch._C, "_cuda_getDevice", torch.cuda.current_device)
    _ftype.update({torch.float32: FT_F32, torch.float16: FT_F16, torch.bfloat16: FT_BF16})
    return torch


def _float_type(dtype, name):
    if not _ftype:
        _serve_init()
    try:
        return _ftype[dtype]
    except KeyError:
        raise TypeError(f"{name} must be float32, float16 or bfloat16, got {dtype}") from None


def _refuse(first, *rest):
    """Raises for the operand that is wrong: (name, tensor, dtype, shape,
    whether it must be dense), `first` being the tensor that sets the device."""
    torch = _torch()
    dev = first.device
    if dev.type != "cuda":
        raise ValueError("tensors must be on a GPU device")
    for name, t, dtype, shape, dense in rest:
        if t is None:
            continue
        if t.device != dev:
            raise ValueError(f"{name} is on {t.device}, expected {dev}")
        if t.dtype != dtype:
            raise TypeError(f"{name} must be {dtype}, got {t.dtype}")
        if tuple(t.shape) != tuple(shape):
            raise ValueError(f"{name} must have shape {tuple(shape)}, got {tuple(t.shape)}")
        if dense and not t.is_contiguous():
            raise ValueError(f"{name} must be contiguous")
    # the launches go to the current device
    if dev.index != torch.cuda.current_device():
        raise ValueError(f"tensors are on {dev}, the current device is cuda:{torch.cuda.current_device()}")


def _ok(t, dev, dtype, shape):
    """An optional dense operand is absent or right."""
    return t is None or (t.dtype is dtype and t.get_device() == dev and t.shape == shape and t.is_contiguous())


def _new(like, shape, dtype, stream, zeros=False):
    """A new tensor on the stream that is going to use it: one of the current
    stream's could be taken up again while another stream still works on it."""
    make = like.new_zeros if zeros else like.new_empty
    if stream is None:
        return make(shape, dtype=dtype)
    cuda = _torch_module.cuda
    if not hasattr(stream, "cuda_stream"):
        stream = cuda.ExternalStream(int(stream)) if int(stream) else cuda.default_stream()
    with cuda.stream(stream):
        return make(shape, dtype=dtype)


def _workspace(query, dt, sizes, like, workspace, stream):
    """(pointer, bytes, tensor) of a workspace: the caller's, or a new one."""
    key = (query, dt, sizes)
    need = _need.get(key)
    if need is None:
        info = PlanInfo()
        check(getattr(lib(), query)(ctypes.byref(info), dt, *sizes))
        if len(_need) >= 4096:
            _need.clear()
        need = _need[key] = info.workspace_bytes
    if workspace is None:
        if need == 0:
            return None, 0, None
        workspace = _new(like, need, _torch_module.uint8, stream)
    elif workspace.device != like.device or not workspace.is_contiguous():
        raise ValueError(f"workspace must be contiguous and on {like.device}")
    return workspace.data_ptr(), workspace.numel() * workspace.element_size(), workspace


def _rows_of(x, name):
    """[..., K] as rows of one stride: (rows, K, stride)."""
    shape = x.shape
    if len(shape) and x.is_contiguous():
        return (shape[0] if len(shape) == 2 else math.prod(shape[:-1])), shape[-1], shape[-1]
    if len(shape) != 2 or x.stride(1) != 1 and shape[1] > 1 or x.stride(0) < shape[1]:
        raise ValueError(f"{name} must be contiguous, or 2-D with contiguous rows that do not overlap")
    return shape[0], shape[1], x.stride(0)


def quantize_rows_i8(x, out=None, scale=None, stream=None):
    """Rows of x [..., K] (float32, float16 or bfloat16) as (int8 values
    [..., K], float32 scales [...]): scale = max|row| / 127, values = round(row / scale)."""
    dt = _float_type(x.dtype, "x")
    rows, cols, ld = _rows_of(x, "x")
    shape = x.shape
    dev = x.get_device()
    if out is None:
        out = _new(x, shape, _t_i8, stream)
    if scale is None:
        scale = _new(x, shape[:-1], _t_f32, stream)
    if dev < 0 or dev != _get_device() or not _ok(out, dev, _t_i8, shape) or not _ok(scale, dev, _t_f32, shape[:-1]):
        _refuse(x, ("out", out, _t_i8, shape, True), ("scale", scale, _t_f32, shape[:-1], True))
    st = lib().quantize_rows_i8(dt, x.data_ptr(), out.data_ptr(), scale.data_ptr(), rows, cols, ld, _stream(stream))
    if st:
        check(st)
    return out, scale


def qgemm_i8_scaled(a, w, scale_a, scale_w, bias=None, dtype=None, out=None, stream=None):
    """scale_a[:, None] * scale_w * (a @ w.T) + bias for int8 a [..., K] and w
    [N, K]; exact int32 sums, result [..., N] of `dtype` (default: out's, else bfloat16)."""
    torch = _torch()
    T = dtype or (torch.bfloat16 if out is None else out.dtype)
    dt = _float_type(T, "out")
    M, K, ld = _rows_of(a, "a")
    if ld != K:
        raise ValueError("a must be contiguous")
    lead, dev = a.shape[:-1], a.get_device()
    N = w.shape[0]
    if out is None:
        out = _new(a, (*lead, N), T, stream)
    if dev < 0 or dev != _get_device() or a.dtype is not _t_i8 or not (
            _ok(w, dev, _t_i8, (N, K)) and _ok(scale_a, dev, _t_f32, lead) and _ok(scale_w, dev, _t_f32, (N,)) and
            _ok(bias, dev, _t_f32, (N,)) and _ok(out, dev, T, (*lead, N))):
        _refuse(a, ("a", a, _t_i8, a.shape, True), ("w", w, _t_i8, (N, K), True), ("scale_a", scale_a, _t_f32, lead, True),
                ("scale_w", scale_w, _t_f32, (N,), True), ("bias", bias, _t_f32, (N,), True),
                ("out", out, T, (*lead, N), True))
    st = lib().qgemm_i8_scaled(dt, a.data_ptr(), w.data_ptr(), scale_a.data_ptr(), scale_w.data_ptr(),
                               None if bias is None else bias.data_ptr(), out.data_ptr(), M, N, K, _stream(stream))
    if st:
        check(st)
    return out


def linear_i8(x, w, scale_w, bias=None, out=None, workspace=None, stream=None):
    """x [..., K] through a linear layer with int8 weights w [N, K] and one
    scale an output channel: rows are quantised to 8 bits as
    quantize_rows_i8 does; the result [..., N] has x's type."""
    T = x.dtype
    dt = _float_type(T, "x")
    M, K, ld = _rows_of(x, "x")
    dev = x.get_device()
    N = w.shape[0]
    shape = (*x.shape[:-1], N)
    if out is None:
        out = _new(x, shape, T, stream)
    if dev < 0 or dev != _get_device() or not (
            _ok(w, dev, _t_i8, (N, K)) and _ok(scale_w, dev, _t_f32, (N,)) and _ok(bias, dev, _t_f32, (N,)) and
            _ok(out, dev, T, shape)):
        _refuse(x, ("w", w, _t_i8, (N, K), True), ("scale_w", scale_w, _t_f32, (N,), True),
                ("bias", bias, _t_f32, (N,), True), ("out", out, T, shape, True))
    wp, wb, _keep = _workspace("qx_plan_linear_i8", dt, (M, N, K), x, workspace, stream)
    st = lib().linear_i8(dt, x.data_ptr(), w.data_ptr(), scale_w.data_ptr(), None if bias is None else bias.data_ptr(),
                         out.data_ptr(), M, N, K, ld, wp, wb, _stream(stream))
    if st:
        check(st)
    return out


def _lin_strides(named):
    """(batch, head[, row]) strides of tensors whose last dimension is
    contiguous, where not all are dense."""
    st = []
    for name, t in named:
        if t.shape[-1] > 1 and t.stride(-1) != 1:
            raise ValueError(f"{name}: the last dimension must be contiguous")
        st += [s if n > 1 else 0 for s, n in zip(t.stride()[:-1], t.shape[:-1])]
    return (_i64 * len(st))(*st)


def lin_attn(q, k, v, log_decay, scale: float = 1.0, state=None, lens=None, out=None, out_state=None, workspace=None,
             stream=None):
    """Causal linear attention with a decay for each head:
        S_i = exp(log_decay[h]) S_{i-1} + k_i^T v_i,   o_i = scale q_i S_i
    q, k [B, H, L, dk], v [B, H, L, dv] of one floating type, any strides with
    a contiguous last dimension; log_decay [H], state [B, H, dk, dv] float32
    (None: zeros); lens [B] int32 (None: L), rows of `out` behind a sequence's
    end are left as they were, zeros where the call makes it.  Returns (out,
    state after the last token); out_state may be `state` itself.  Records no
    autograd graph: lin_attn_backward gives the gradients."""
    T = q.dtype
    dt = _float_type(T, "q")
    shape = q.shape
    if len(shape) != 4:
        raise ValueError("q, k, v must be [B, H, L, d]")
    B, H, L, dk = shape
    dv = v.shape[-1]
    dev = q.get_device()
    vs, ss = (B, H, L, dv), (B, H, dk, dv)
    if out is None:
        out = _new(q, vs, T, stream, lens is not None)
    if out_state is None:
        out_state = _new(q, ss, _t_f32, stream)
    if (dev < 0 or dev != _get_device() or k.dtype is not T or v.dtype is not T or out.dtype is not T or
            k.shape != shape or v.shape != vs or out.shape != vs or k.get_device() != dev or v.get_device() != dev or
            out.get_device() != dev or not (_ok(log_decay, dev, _t_f32, (H,)) and _ok(state, dev, _t_f32, ss) and
                                            _ok(lens, dev, _t_i32, (B,)) and _ok(out_state, dev, _t_f32, ss))):
        _refuse(q, ("k", k, T, shape, False), ("v", v, T, vs, False), ("out", out, T, vs, False),
                ("log_decay", log_decay, _t_f32, (H,), True), ("state", state, _t_f32, ss, True),
                ("lens", lens, _t_i32, (B,), True), ("out_state", out_state, _t_f32, ss, True))
    dense = q.is_contiguous() and k.is_contiguous() and v.is_contiguous() and out.is_contiguous()
    st = None if dense else _lin_strides((("q", q), ("k", k), ("v", v), ("out", out)))
    wp, wb, _keep = _workspace("qx_plan_lin_attn", dt, (B, H, L, dk, dv), q, workspace, stream)
    st = lib().lin_attn(dt, q.data_ptr(), k.data_ptr(), v.data_ptr(), log_decay.data_ptr(),
                        None if state is None else state.data_ptr(), None if lens is None else lens.data_ptr(),
                        out.data_ptr(), out_state.data_ptr(), B, H, L, dk, dv, st, scale, wp, wb, _stream(stream))
    if st:
        check(st)
    return out, out_state


def lin_attn_step(q, k, v, log_decay, state, scale: float = 1.0, out=None, stream=None):
    """lin_attn for one token of every sequence: q, k [B, H, dk], v [B, H, dv];
    `state` [B, H, dk, dv] float32 is updated in place.  Returns out [B, H, dv]."""
    T = q.dtype
    dt = _float_type(T, "q")
    shape = q.shape
    if len(shape) != 3:
        raise ValueError("q, k, v must be [B, H, d]")
    B, H, dk = shape
    dv = v.shape[-1]
    dev = q.get_device()
    vs, ss = (B, H, dv), (B, H, dk, dv)
    if out is None:
        out = _new(q, vs, T, stream)
    if (dev < 0 or dev != _get_device() or k.dtype is not T or v.dtype is not T or out.dtype is not T or
            k.shape != shape or v.shape != vs or out.shape != vs or k.get_device() != dev or v.get_device() != dev or
            out.get_device() != dev or not (_ok(log_decay, dev, _t_f32, (H,)) and _ok(state, dev, _t_f32, ss))):
        _refuse(q, ("k", k, T, shape, False), ("v", v, T, vs, False), ("out", out, T, vs, False),
                ("log_decay", log_decay, _t_f32, (H,), True), ("state", state, _t_f32, ss, True))
    dense = q.is_contiguous() and k.is_contiguous() and v.is_contiguous() and out.is_contiguous()
    st = None if dense else _lin_strides((("q", q), ("k", k), ("v", v), ("out", out)))
    st = lib().lin_attn_step(dt, q.data_ptr(), k.data_ptr(), v.data_ptr(), log_decay.data_ptr(), state.data_ptr(),
                             out.data_ptr(), B, H, dk, dv, st, scale, _stream(stream))
    if st:
        check(st)
    return out


def lin_attn_backward(q, k, v, d_out, log_decay, scale: float = 1.0, state=None, d_state=None, lens=None, out=None,
                      out_state=None, workspace=None, stream=None):
    """Gradients (dq, dk, dv, dstate) of lin_attn from d_out [B, H, L, dv] and
    d_state [B, H, dk, dv] (None: zeros), the gradients of its two results.
    `out`: three tensors for dq, dk, dv, whose rows behind a sequence's end are
    left as they were; zeros where the call makes them."""
    T = q.dtype
    dt = _float_type(T, "q")
    shape = q.shape
    if len(shape) != 4:
        raise ValueError("q, k, v must be [B, H, L, d]")
    B, H, L, dk = shape
    dv = v.shape[-1]
    dev = q.get_device()
    vs, ss = (B, H, L, dv), (B, H, dk, dv)
    if out is None:
        out = [_new(q, t, T, stream, lens is not None) for t in (shape, shape, vs)]
    gq, gk, gv = out
    if out_state is None:
        out_state = _new(q, ss, _t_f32, stream)
    _refuse(q, ("k", k, T, shape, False), ("v", v, T, vs, False), ("d_out", d_out, T, vs, False),
            ("dq", gq, T, shape, False), ("dk", gk, T, shape, False), ("dv", gv, T, vs, False),
            ("log_decay", log_decay, _t_f32, (H,), True), ("state", state, _t_f32, ss, True),
            ("d_state", d_state, _t_f32, ss, True), ("lens", lens, _t_i32, (B,), True),
            ("out_state", out_state, _t_f32, ss, True))
    named = (("q", q), ("k", k), ("v", v), ("d_out", d_out), ("dq", gq), ("dk", gk), ("dv", gv))
    st = None if all(t.is_contiguous() for _, t in named) else _lin_strides(named)
    wp, wb, _keep = _workspace("qx_plan_lin_attn_backward", dt, (B, H, L, dk, dv), q, workspace, stream)
    check(lib().lin_attn_backward(dt, q.data_ptr(), k.data_ptr(), v.data_ptr(), d_out.data_ptr(), log_decay.data_ptr(),
                                  None if state is None else state.data_ptr(),
                                  None if d_state is None else d_state.data_ptr(),
                                  None if lens is None else lens.data_ptr(), gq.data_ptr(), gk.data_ptr(),
                                  gv.data_ptr(), out_state.data_ptr(), B, H, L, dk, dv, st, scale, wp, wb,
                                  _stream(stream)))
    return gq, gk, gv, out_state


# ---------------------------------------------------------------------------
# planner queries (host only)
# ---------------------------------------------------------------------------
def _route(route) -> int:
    return ROUTE[route] if isinstance(route, str) else int(route)


def plan_gemm_i16i32(M, N, K, batch=1, bound_a=0, bound_b=0, route="auto") -> dict:
    info = PlanInfo()
    check(lib().qx_plan_gemm_i16i32(ctypes.byref(info), M, N, K, batch, bound_a, bound_b, _route(route)))
    return info.as_dict()


def plan_gemm_i32_s24(M, N, K, batch=1, route="auto") -> dict:
    info = PlanInfo()
    check(lib().qx_plan_gemm_i32_s24(ctypes.byref(info), M, N, K, batch, _route(route)))
    return info.as_dict()


def plan_conv2d(N, Ci, H, W, Co, KH, KW, stride=1, pad=0, bound_x=0, bound_w=0, route="auto") -> dict:
    info = PlanInfo()
    check(lib().qx_plan_conv2d(ctypes.byref(info), N, Ci, H, W, Co, KH, KW, stride, pad,
                               bound_x, bound_w, _route(route)))
    return info.as_dict()


def plan_conv2d_t(dtype: str, N, Ci, H, W, Co, KH, KW, stride=1, pad=0, route="auto") -> dict:
    info = PlanInfo()
    check(lib().qx_plan_conv2d_t(ctypes.byref(info), DT_F32 if dtype == "f32" else DT_I32, N, Ci, H, W,
                                 Co, KH, KW, stride, pad, _route(route)))
    return info.as_dict()


def plan_minmax(n, elem_bytes) -> dict:
    info = PlanInfo()
    check(lib().qx_plan_minmax(ctypes.byref(info), n, elem_bytes))
    return info.as_dict()


def plan_pool2x2(kind: str, N, C, H, W) -> dict:
    info = PlanInfo()
    check(lib().qx_plan_pool2x2(ctypes.byref(info), POOL_AVG_I32 if kind == "avg_i32" else POOL_MAX_F32,
                                N, C, H, W))
    return info.as_dict()


def plan_lenet_i32(batch) -> dict:
    info = PlanInfo()
    check(lib().qx_plan_lenet_i32(ctypes.byref(info), batch))
    return info.as_dict()


def plan_sdpa_f32(BH, L, d, scale=1.0, causal=False) -> dict:
    info = PlanInfo()
    check(lib().qx_plan_sdpa_f32(ctypes.byref(info), BH, L, d, float(scale), 1 if causal else 0))
    return info.as_dict()


def _torch_type(dtype: str):
    torch = _torch()
    return {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}[dtype]


_FT = {"f32": FT_F32, "f16": FT_F16, "bf16": FT_BF16}


def plan_quantize_rows_i8(dtype: str, rows, cols) -> dict:
    info = PlanInfo()
    check(lib().qx_plan_quantize_rows_i8(ctypes.byref(info), _FT[dtype], rows, cols))
    return info.as_dict()


def plan_gemm_i8_scaled(dtype: str, M, N, K) -> dict:
    info = PlanInfo()
    check(lib().qx_plan_gemm_i8_scaled(ctypes.byref(info), _FT[dtype], M, N, K))
    return info.as_dict()


def plan_linear_i8(dtype: str, M, N, K) -> dict:
    info = PlanInfo()
    check(lib().qx_plan_linear_i8(ctypes.byref(info), _FT[dtype], M, N, K))
    return info.as_dict()


def plan_lin_attn(dtype: str, B, H, L, dk, dv) -> dict:
    info = PlanInfo()
    check(lib().qx_plan_lin_attn(ctypes.byref(info), _FT[dtype], B, H, L, dk, dv))
    return info.as_dict()


def plan_lin_attn_step(dtype: str, B, H, dk, dv) -> dict:
    info = PlanInfo()
    check(lib().qx_plan_lin_attn_step(ctypes.byref(info), _FT[dtype], B, H, dk, dv))
    return info.as_dict()


def plan_lin_attn_backward(dtype: str, B, H, L, dk, dv) -> dict:
    info = PlanInfo()
    check(lib().qx_plan_lin_attn_backward(ctypes.byref(info), _FT[dtype], B, H, L, dk, dv))
    return info.as_dict()


def plan_attn(dtype: str, L, d, bound=0, route="auto") -> dict:
    info = PlanInfo()
    check(lib().qx_plan_attn(ctypes.byref(info), DT_F32 if dtype == "f32" else DT_I32, L, d,
                             bound, _route(route)))
    return info.as_dict()


# ---------------------------------------------------------------------------
# persistent executor
# ---------------------------------------------------------------------------
class Executor:
    """Owns a qx_exec handle: planned and allocated once, re-dispatched by run()."""

    def __init__(self, handle: ctypes.c_void_p, out_shape, out_dtype, n_inputs: int):
        self._h = handle
        self.out_shape = tuple(out_shape)
        self.out_dtype = out_dtype
        self.n_inputs = n_inputs
        self._ptrs = ctypes.c_void_p * n_inputs
        self._run = lib().qx_exec_run

    @classmethod
    def gemm_i16i32(cls, M, N, K, batch=1, bound_a=0, bound_b=0, route="auto"):
        torch = _torch()
        h = ctypes.c_void_p()
        if _route(route) == 0:
            check(lib().qx_exec_create_gemm_i16i32(ctypes.byref(h), M, N, K, batch, bound_a, bound_b))
        else:
            check(lib().qx_exec_create_gemm_i16i32_route(ctypes.byref(h), M, N, K, batch, bound_a, bound_b,
                                                         _route(route)))
        return cls(h, (batch, M, N), torch.int32, 2)

    @classmethod
    def gemm_i32_s24(cls, M, N, K, batch=1, route="auto"):
        torch = _torch()
        h = ctypes.c_void_p()
        if _route(route) == 0:
            check(lib().qx_exec_create_gemm_i32_s24(ctypes.byref(h), M, N, K, batch))
        else:
            check(lib().qx_exec_create_gemm_i32_s24_route(ctypes.byref(h), M, N, K, batch, _route(route)))
        return cls(h, (batch, M, N), torch.int32, 2)

    @classmethod
    def conv2d(cls, N, Ci, H, W, Co, KH, KW, stride=1, pad=0, bound_x=0, bound_w=0, route="auto"):
        torch = _torch()
        h = ctypes.c_void_p()
        if _route(route) == 0:
            check(lib().qx_exec_create_conv2d(ctypes.byref(h), N, Ci, H, W, Co, KH, KW, stride, pad,
                                              bound_x, bound_w))
        else:
            check(lib().qx_exec_create_conv2d_route(ctypes.byref(h), N, Ci, H, W, Co, KH, KW, stride, pad,
                                                    bound_x, bound_w, _route(route)))
        Ho, Wo = conv_out_hw(H, W, KH, KW, stride, pad)
        return cls(h, (N, Co, Ho, Wo), torch.int32, 2)

    @classmethod
    def conv2d_t(cls, dtype: str, N, Ci, H, W, Co, KH, KW, stride=1, pad=0, route="auto"):
        torch = _torch()
        h = ctypes.c_void_p()
        dt = DT_F32 if dtype == "f32" else DT_I32
        check(lib().qx_exec_create_conv2d_t(ctypes.byref(h), dt, N, Ci, H, W, Co, KH, KW, stride, pad,
                                            _route(route)))
        Ho, Wo = conv_out_hw(H, W, KH, KW, stride, pad)
        return cls(h, (N, Co, Ho, Wo), torch.float32 if dtype == "f32" else torch.int32, 2)

    @classmethod
    def minmax(cls, n, dtype: str):
        """dtype "i32" or "i16"; the output is 2 elements (min, max)."""
        torch = _torch()
        h = ctypes.c_void_p()
        check(lib().qx_exec_create_minmax(ctypes.byref(h), n, 4 if dtype == "i32" else 2))
        return cls(h, (2,), torch.int32 if dtype == "i32" else torch.int16, 1)

    @classmethod
    def pool2x2(cls, kind: str, N, C, H, W):
        """kind "avg_i32" or "max_f32"."""
        torch = _torch()
        h = ctypes.c_void_p()
        k = POOL_AVG_I32 if kind == "avg_i32" else POOL_MAX_F32
        check(lib().qx_exec_create_pool2x2(ctypes.byref(h), k, N, C, H, W))
        return cls(h, (N, C, H // 2, W // 2), torch.int32 if k == POOL_AVG_I32 else torch.float32, 1)

    @classmethod
    def lenet_i32(cls, batch):
        """inputs (x, w1, w2, f1, f2, f3) int32; output [batch][10] int32."""
        torch = _torch()
        h = ctypes.c_void_p()
        check(lib().qx_exec_create_lenet_i32(ctypes.byref(h), batch))
        return cls(h, (batch, 10), torch.int32, 6)

    @classmethod
    def attn(cls, dtype: str, L, d, bound=0, route="auto"):
        torch = _torch()
        h = ctypes.c_void_p()
        dt = DT_F32 if dtype == "f32" else DT_I32
        if _route(route) == 0:
            check(lib().qx_exec_create_attn(ctypes.byref(h), dt, L, d, bound))
        else:
            check(lib().qx_exec_create_attn_route(ctypes.byref(h), dt, L, d, bound, _route(route)))
        return cls(h, (L, d), torch.float32 if dtype == "f32" else torch.int32, 3)

    @classmethod
    def sdpa_f32(cls, BH, L, d, scale=1.0, causal=False):
        """inputs (Q, K, V) float32 [BH][L][d]; output [BH][L][d]."""
        torch = _torch()
        h = ctypes.c_void_p()
        check(lib().qx_exec_create_sdpa_f32(ctypes.byref(h), BH, L, d, float(scale), 1 if causal else 0))
        return cls(h, (BH, L, d), torch.float32, 3)

    @classmethod
    def gemm_i8_scaled(cls, dtype: str, M, N, K, bias=False):
        """inputs (a, w, scale_a, scale_w[, bias]); output [M][N] of dtype "f32", "f16" or "bf16"."""
        h = ctypes.c_void_p()
        check(lib().qx_exec_create_gemm_i8_scaled(ctypes.byref(h), _FT[dtype], M, N, K, 1 if bias else 0))
        return cls(h, (M, N), _torch_type(dtype), 5 if bias else 4)

    @classmethod
    def linear_i8(cls, dtype: str, M, N, K, bias=False):
        """inputs (x, w, scale_w[, bias]); output [M][N]."""
        h = ctypes.c_void_p()
        check(lib().qx_exec_create_linear_i8(ctypes.byref(h), _FT[dtype], M, N, K, 1 if bias else 0))
        return cls(h, (M, N), _torch_type(dtype), 4 if bias else 3)

    @classmethod
    def lin_attn(cls, dtype: str, B, H, L, dk, dv, scale=1.0):
        """inputs (q, k, v, log_decay, state), dense; the state is updated in place; output [B][H][L][dv]."""
        h = ctypes.c_void_p()
        check(lib().qx_exec_create_lin_attn(ctypes.byref(h), _FT[dtype], B, H, L, dk, dv, float(scale)))
        return cls(h, (B, H, L, dv), _torch_type(dtype), 5)

    @classmethod
    def lin_attn_step(cls, dtype: str, B, H, dk, dv, scale=1.0):
        """inputs (q, k, v, log_decay, state), dense; the state is updated in place; output [B][H][dv]."""
        h = ctypes.c_void_p()
        check(lib().qx_exec_create_lin_attn_step(ctypes.byref(h), _FT[dtype], B, H, dk, dv, float(scale)))
        return cls(h, (B, H, dv), _torch_type(dtype), 5)

    def plan(self) -> dict:
        info = PlanInfo()
        check(lib().qx_exec_plan(self._h, ctypes.byref(info)))
        return info.as_dict()

    def run_ptrs(self, in_ptrs, out_ptr: int, stream=None) -> None:
        """Enqueue with raw device pointers (ints).  Kept lean: for small
        problems the host's cost per call is what bounds back-to-back runs."""
        n = len(in_ptrs)
        arr = self._ptrs(*in_ptrs) if n == self.n_inputs else (ctypes.c_void_p * n)(*in_ptrs)
        st = self._run(self._h, arr, out_ptr, _stream(stream))
        if st != OK:
            check(st)

    def run(self, inputs, out=None, stream=None):
        if len(inputs) != self.n_inputs:
            raise ValueError(f"expected {self.n_inputs} inputs")
        if out is None:
            out = _torch().empty(self.out_shape, dtype=self.out_dtype, device=inputs[0].device)
        ptrs = []
        for i, t in enumerate(inputs):
            if not t.is_cuda or not t.is_contiguous():
                raise ValueError(f"input {i} must be a contiguous GPU tensor")
            ptrs.append(t.data_ptr())
        if not out.is_contiguous() or out.dtype != self.out_dtype:
            raise ValueError("bad output tensor")
        self.run_ptrs(ptrs, out.data_ptr(), stream)
        return out

    def profile(self, inputs, out, reps: int = 10, stream=None) -> list:
        """Mean execute-only duration (ms) of every launch: [(kernel, ms), ...]."""
        nk = self.plan()["kernels"]
        ms = (ctypes.c_float * max(nk, 1))()
        names = (ctypes.c_char_p * max(nk, 1))()
        arr = (ctypes.c_void_p * len(inputs))(*[ctypes.c_void_p(t.data_ptr()) for t in inputs])
        check(lib().qx_exec_profile(self._h, arr, ctypes.c_void_p(out.data_ptr()), _stream(stream),
                                    int(reps), ms, names, nk))
        return [(names[i].decode(), float(ms[i])) for i in range(nk)]

    def close(self) -> None:
        if self._h:
            check(lib().qx_exec_destroy(self._h))
            self._h = None

    def __enter__(self):
        return self

    def __exit__(self, *exc):
        self.close()

    def __del__(self):
        try:
            if self._h:
                lib().qx_exec_destroy(self._h)
        except Exception:
            pass


# ---------------------------------------------------------------------------
# test seams (include/qx_testing.h): no result is computed under the double
# ---------------------------------------------------------------------------
COUNTERS = ("allocs", "frees", "events", "events_freed", "launches", "live_handles")


def testing_host_double(on: bool) -> None:
    """Switch executor creation to the host-only runtime double (or back)."""
    check(lib().qx_testing_host_double(1 if on else 0))


def testing_counters() -> dict:
    vals = (ctypes.c_int64 * len(COUNTERS))()
    lib().qx_testing_counters(vals, len(COUNTERS))
    return dict(zip(COUNTERS, list(vals)))


class HostTensor:
    """Stand-in for a device tensor under the host double: a pointer, a
    shape and a dtype (nothing is ever read or written through it)."""

    def __init__(self, ptr: int, shape, dtype=None):
        self.ptr, self.shape, self.dtype = ptr, tuple(shape), dtype

    def data_ptr(self) -> int:
        return self.ptr
