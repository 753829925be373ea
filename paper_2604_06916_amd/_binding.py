"""Thin binding of libsolfp4.so (declared in include/solfp4.h).

Argument marshalling only: torch supplies device memory and the current
stream; every step of the computation runs in the library's HIP kernels.
Loading fails loudly if the library has not been built.

Calls on the current stream go through _host.so, which makes the same checks
and allocations in native code; whatever it does not take (another stream,
an operand that is not exactly what the call needs) runs through the checks
here, which raise the errors, and ctypes.
"""
from __future__ import annotations

import ctypes
import os

import torch

LIB_PATH = os.path.join(os.path.dirname(os.path.abspath(__file__)), "libsolfp4.so")

if not os.path.exists(LIB_PATH):
    raise ImportError(f"{LIB_PATH} is missing: build it with `python -m paper_2604_06916_amd.build`")

lib = ctypes.CDLL(LIB_PATH)

if not os.path.exists(os.path.join(os.path.dirname(LIB_PATH), "_host.so")):
    raise ImportError("_host.so is missing: build it with `python -m paper_2604_06916_amd.build`")
from . import _host  # noqa: E402  (links against the library loaded above)

_p = ctypes.c_void_p
_i64 = ctypes.c_int64
_sz = ctypes.c_size_t

lib.solfp4_strerror.restype = ctypes.c_char_p
lib.solfp4_strerror.argtypes = [ctypes.c_int]
lib.solfp4_version.restype = ctypes.c_int
lib.solfp4_version.argtypes = []
lib.nvfp4_quantize_workspace_bytes.restype = _sz
lib.nvfp4_quantize_workspace_bytes.argtypes = [_i64, _i64]
lib.nvfp4_quantize.restype = ctypes.c_int
lib.nvfp4_quantize.argtypes = [_p, _i64, _i64, _p, _p, _p, _p, _sz, _p]
lib.nvfp4_quantize_amax.restype = ctypes.c_int
lib.nvfp4_quantize_amax.argtypes = [_p, _i64, _i64, _p, _sz, _p]
lib.nvfp4_gelu_amax.restype = ctypes.c_int
lib.nvfp4_gelu_amax.argtypes = [_p, _i64, _i64, _p, _sz, _p]
lib.nvfp4_quantize_encode.restype = ctypes.c_int
lib.nvfp4_quantize_encode.argtypes = [_p, _i64, _i64, _p, _p, _p, _p, _sz, _p]
lib.nvfp4_quantize_noalloc.restype = ctypes.c_int
lib.nvfp4_quantize_noalloc.argtypes = [_p, _i64, _i64, _p, _p, _p, _p]
lib.nvfp4_gemm.restype = ctypes.c_int
lib.nvfp4_gemm.argtypes = [_p, _p, _p, _p, _p, _p, _p, _p, _p, _sz, _i64, _i64, _i64, _p]
lib.nvfp4_gemm_workspace_bytes.restype = _sz
lib.nvfp4_gemm_workspace_bytes.argtypes = [_i64, _i64, _i64]
lib.nvfp4_linear_workspace_bytes.restype = _sz
lib.nvfp4_linear_workspace_bytes.argtypes = [_i64, _i64, _i64]
lib.nvfp4_linear.restype = ctypes.c_int
lib.nvfp4_linear.argtypes = [_p, _p, _p, _p, _p, _p, _p, _sz, _i64, _i64, _i64, _p]

lib.solfp4_gemm_plan.restype = ctypes.c_int
lib.solfp4_gemm_plan.argtypes = [ctypes.c_int, _i64, _i64, _i64, ctypes.c_int,
                                 ctypes.POINTER(ctypes.c_int), ctypes.POINTER(ctypes.c_int),
                                 ctypes.POINTER(ctypes.c_int64), ctypes.POINTER(ctypes.c_int)]

lib.mxfp4_quantize.restype = ctypes.c_int
lib.mxfp4_quantize.argtypes = [_p, _i64, _i64, _p, _p, _p]
lib.mxfp4_gemm.restype = ctypes.c_int
lib.mxfp4_gemm.argtypes = [_p, _p, _p, _p, _p, _p, _i64, _i64, _i64, _p]
lib.mxfp4_linear_workspace_bytes.restype = _sz
lib.mxfp4_linear_workspace_bytes.argtypes = [_i64, _i64]
lib.mxfp4_linear.restype = ctypes.c_int
lib.mxfp4_linear.argtypes = [_p, _p, _p, _p, _p, _p, _sz, _i64, _i64, _i64, _p]

_int, _f32, _f64 = ctypes.c_int, ctypes.c_float, ctypes.c_double
_norm_in = [_int, _p, _i64, _p, _i64, _p, _i64, _i64, _f32, _p, _i64]
lib.solfp4_add_rmsnorm.restype = _int
lib.solfp4_add_rmsnorm.argtypes = [*_norm_in, _p, _i64, _i64, _i64, _p]
lib.mxfp8_add_rmsnorm.restype = _int
lib.mxfp8_add_rmsnorm.argtypes = [*_norm_in, _p, _p, _i64, _i64, _p]
lib.mxfp4_add_rmsnorm.restype = _int
lib.mxfp4_add_rmsnorm.argtypes = [*_norm_in, _p, _p, _i64, _i64, _p]
lib.solfp4_rmsnorm_backward_workspace_bytes.restype = _sz
lib.solfp4_rmsnorm_backward_workspace_bytes.argtypes = [_i64, _i64, _i64]
lib.solfp4_rmsnorm_backward.restype = _int
lib.solfp4_rmsnorm_backward.argtypes = [_int, _p, _i64, _p, _i64, _p, _i64, _i64, _p, _i64, _f32, _p, _i64, _p, _p,
                                        _sz, _i64, _i64, _p]
lib.solfp4_rotary_table.restype = _int
lib.solfp4_rotary_table.argtypes = [_p, _i64, _p, _i64, _p, _int, _f64, _p, _p]
lib.solfp4_rotary.restype = _int
lib.solfp4_rotary.argtypes = [_int, _int, _int, *2 * [_p, _i64, _i64, _p, _i64, _i64, _i64], _p, _i64, _p, _int, _i64,
                              _i64, _i64, _p]
lib.nvfp4_weight_linear.restype = _int
lib.nvfp4_weight_linear.argtypes = [*6 * [_p], _i64, _i64, _i64, _p]
lib.mxfp4_weight_linear.restype = _int
lib.mxfp4_weight_linear.argtypes = [*5 * [_p], _i64, _i64, _i64, _p]
lib.mxfp8_linear.restype = _int
lib.mxfp8_linear.argtypes = [*6 * [_p], _i64, _i64, _i64, _p]

EXPORTED = ["solfp4_strerror", "solfp4_version", "solfp4_gemm_plan",
            "nvfp4_quantize_workspace_bytes", "nvfp4_quantize", "nvfp4_quantize_amax",
            "nvfp4_gelu_amax", "nvfp4_quantize_encode", "nvfp4_quantize_noalloc",
            "nvfp4_gemm",
            "nvfp4_gemm_workspace_bytes", "nvfp4_linear_workspace_bytes", "nvfp4_linear",
            "mxfp4_quantize", "mxfp4_gemm", "mxfp4_linear_workspace_bytes", "mxfp4_linear",
            "solfp4_add_rmsnorm", "mxfp8_add_rmsnorm", "mxfp4_add_rmsnorm",
            "solfp4_rmsnorm_backward_workspace_bytes", "solfp4_rmsnorm_backward",
            "solfp4_rotary_table", "solfp4_rotary",
            "nvfp4_weight_linear", "mxfp4_weight_linear", "mxfp8_linear"]

FORMAT_NVFP4, FORMAT_MXFP4 = 0, 1
KERNEL_NAMES = {0: None, 1: "nvfp4_gemm_lane_kernel", 2: "nvfp4_gemm_kernel",
                3: "mxfp4_gemm_kernel", 4: "nvfp4_gemm_small_kernel", 5: "nvfp4_gemm_wavek_kernel",
                6: "mxfp4_gemm_wavek_kernel"}


class Solfp4Error(RuntimeError):
    def __init__(self, status: int):
        self.status = status
        super().__init__(f"solfp4 status {status}: {lib.solfp4_strerror(status).decode()}")


def _check(status: int):
    if status != 0:
        raise Solfp4Error(status)


def _native(r):
    """A result of _host that took the call: the outputs, or a failed status."""
    if type(r) is int:
        raise Solfp4Error(r)
    return r


def _ptr(t):
    return None if t is None else ctypes.c_void_p(t.data_ptr())


def _stream(stream, device):
    if stream is None:
        stream = torch.cuda.current_stream(device)
    return stream


def _alloc(shape, dtype, device, stream):
    """A temporary or output on `device`, allocated under `stream` so the
    caching allocator does not hand its memory to other work before the
    library's kernels on that stream are done with it."""
    with torch.cuda.stream(stream):
        return torch.empty(shape, dtype=dtype, device=device)


def _is_gpu(t):
    return t.is_cuda


def _need(t, dtype, shape, name, device=None):
    """Every tensor crossing the boundary: contiguous, on the GPU (on the
    same device as the call's other tensors), of the dtype and shape the
    C-ABI expects for these sizes; else ValueError before any launch."""
    if not isinstance(t, torch.Tensor):
        raise ValueError(f"{name}: expected a torch.Tensor, got {type(t).__name__}")
    if (t.dtype != dtype or tuple(t.shape) != tuple(shape) or not t.is_contiguous() or not _is_gpu(t)
            or (device is not None and t.device != device)):
        want = f"contiguous CUDA {dtype} {tuple(shape)}" + (f" on {device}" if device is not None else "")
        raise ValueError(f"{name}: expected {want}, got {t.dtype} {tuple(t.shape)} on {t.device}"
                         f"{'' if t.is_contiguous() else ' (not contiguous)'}")


def _need_workspace(t, nbytes, name, device):
    if not isinstance(t, torch.Tensor) or t.dtype != torch.uint8 or t.dim() != 1 \
            or not t.is_contiguous() or not _is_gpu(t) or t.device != device:
        raise ValueError(f"{name}: expected a contiguous 1-D CUDA uint8 tensor on {device}")
    if t.numel() < nbytes:
        raise ValueError(f"{name}: {t.numel()} bytes, at least {nbytes} needed")


def _dims(x, name, block):
    if not isinstance(x, torch.Tensor) or x.dim() != 2:
        raise ValueError(f"{name}: expected a 2-D tensor")
    rows, K = x.shape
    if K % block:
        raise ValueError(f"{name}: K = {K} is not a multiple of {block}")
    return rows, K


def nvfp4_quantize_workspace_bytes(rows: int, K: int) -> int:
    return lib.nvfp4_quantize_workspace_bytes(rows, K)


def nvfp4_gemm_workspace_bytes(M: int, N: int, K: int) -> int:
    return lib.nvfp4_gemm_workspace_bytes(M, N, K)


def nvfp4_linear_workspace_bytes(M: int, N: int, K: int) -> int:
    return lib.nvfp4_linear_workspace_bytes(M, N, K)


def gemm_plan(M: int, N: int, K: int, fmt: int = FORMAT_NVFP4, with_workspace: bool = True) -> dict:
    """The library's own account of how a GEMM of this shape runs (host
    only): kernel name, output tile edge, workgroups, K ranges per tile of
    the last round."""
    kernel, tile, splits = ctypes.c_int(), ctypes.c_int(), ctypes.c_int()
    wgs = ctypes.c_int64()
    _check(lib.solfp4_gemm_plan(fmt, M, N, K, int(with_workspace), ctypes.byref(kernel),
                                ctypes.byref(tile), ctypes.byref(wgs), ctypes.byref(splits)))
    return {"kernel": KERNEL_NAMES.get(kernel.value, f"kernel {kernel.value}"), "tile": tile.value,
            "workgroups": wgs.value, "splits": splits.value}


def nvfp4_quantize(x, codes=None, scales=None, global_scale=None, workspace=None, stream=None):
    """x: BF16 [rows, K] -> (codes uint8 [rows, K/2], scales uint8 [rows, K/16],
    global_scale float32 [1]).  Outputs may be passed in to avoid allocation."""
    if stream is None:
        r = _host.nvfp4_quantize(x, codes, scales, global_scale, workspace)
        if r is not None:
            return _native(r)
    rows, K = _dims(x, "x", 16)
    dev = x.device
    _need(x, torch.bfloat16, (rows, K), "x")
    need = nvfp4_quantize_workspace_bytes(rows, K)
    if codes is not None:
        _need(codes, torch.uint8, (rows, K // 2), "codes", dev)
    if scales is not None:
        _need(scales, torch.uint8, (rows, K // 16), "scales", dev)
    if global_scale is not None:
        _need(global_scale, torch.float32, (1,), "global_scale", dev)
    if workspace is not None:
        _need_workspace(workspace, need, "workspace", dev)
    st = _stream(stream, dev)
    if codes is None:
        codes = _alloc((rows, K // 2), torch.uint8, dev, st)
    if scales is None:
        scales = _alloc((rows, K // 16), torch.uint8, dev, st)
    if global_scale is None:
        global_scale = _alloc((1,), torch.float32, dev, st)
    if workspace is None:
        workspace = _alloc((max(need, 256),), torch.uint8, dev, st)
    _check(lib.nvfp4_quantize(_ptr(x), rows, K, _ptr(codes), _ptr(scales), _ptr(global_scale),
                              _ptr(workspace), workspace.numel(), ctypes.c_void_p(st.cuda_stream)))
    return codes, scales, global_scale


def nvfp4_quantize_amax(x, workspace, stream=None):
    """The first pass of nvfp4_quantize: x's partial maxima into `workspace`
    (uint8, at least nvfp4_quantize_workspace_bytes(rows, K))."""
    rows, K = _dims(x, "x", 16)
    dev = x.device
    _need(x, torch.bfloat16, (rows, K), "x")
    _need_workspace(workspace, nvfp4_quantize_workspace_bytes(rows, K), "workspace", dev)
    st = _stream(stream, dev)
    _check(lib.nvfp4_quantize_amax(_ptr(x), rows, K, _ptr(workspace), workspace.numel(),
                                   ctypes.c_void_p(st.cuda_stream)))


def nvfp4_gelu_amax(x, workspace, stream=None):
    """x <- gelu(x) in place (tanh form) and nvfp4_quantize_amax of the
    result, in one pass."""
    rows, K = _dims(x, "x", 16)
    dev = x.device
    _need(x, torch.bfloat16, (rows, K), "x")
    _need_workspace(workspace, nvfp4_quantize_workspace_bytes(rows, K), "workspace", dev)
    st = _stream(stream, dev)
    _check(lib.nvfp4_gelu_amax(_ptr(x), rows, K, _ptr(workspace), workspace.numel(),
                               ctypes.c_void_p(st.cuda_stream)))
    return x


def nvfp4_quantize_encode(x, codes, scales, global_scale, workspace, stream=None):
    """The second pass of nvfp4_quantize (after nvfp4_quantize_amax on the
    same x and workspace): codes, scales and alpha."""
    rows, K = _dims(x, "x", 16)
    dev = x.device
    _need(x, torch.bfloat16, (rows, K), "x")
    _need(codes, torch.uint8, (rows, K // 2), "codes", dev)
    _need(scales, torch.uint8, (rows, K // 16), "scales", dev)
    _need(global_scale, torch.float32, (1,), "global_scale", dev)
    _need_workspace(workspace, nvfp4_quantize_workspace_bytes(rows, K), "workspace", dev)
    st = _stream(stream, dev)
    _check(lib.nvfp4_quantize_encode(_ptr(x), rows, K, _ptr(codes), _ptr(scales), _ptr(global_scale),
                                     _ptr(workspace), workspace.numel(), ctypes.c_void_p(st.cuda_stream)))
    return codes, scales, global_scale


def nvfp4_quantize_noalloc(x, codes, scales, global_scale, stream=None):
    """nvfp4_quantize into caller-provided outputs with no workspace: the
    library's fixed per-device scratch holds the partial maxima, so this
    call allocates nothing (usable where allocation is not allowed).  Calls
    that may overlap on one device race on that scratch."""
    rows, K = _dims(x, "x", 16)
    dev = x.device
    _need(x, torch.bfloat16, (rows, K), "x")
    _need(codes, torch.uint8, (rows, K // 2), "codes", dev)
    _need(scales, torch.uint8, (rows, K // 16), "scales", dev)
    _need(global_scale, torch.float32, (1,), "global_scale", dev)
    st = _stream(stream, dev)
    _check(lib.nvfp4_quantize_noalloc(_ptr(x), rows, K, _ptr(codes), _ptr(scales),
                                      _ptr(global_scale), ctypes.c_void_p(st.cuda_stream)))
    return codes, scales, global_scale


def nvfp4_gemm(a_codes, a_scales, a_global_scale, b_codes, b_scales, b_global_scale,
               bias=None, out=None, workspace=None, stream=None, split=True):
    """Block-scaled NVFP4 GEMM: A [M, K] (packed), B [N, K] (packed) -> BF16 [M, N].
    `workspace` (uint8, at least nvfp4_gemm_workspace_bytes(M, N, K)) is
    allocated when needed and not given; split=False passes none (no split
    of the last round's tiles)."""
    if stream is None and split:
        r = _host.nvfp4_gemm(a_codes, a_scales, a_global_scale, b_codes, b_scales, b_global_scale, bias, out,
                             workspace)
        if r is not None:
            return _native(r)
    M, Kh = _dims(a_codes, "a_codes", 1)
    N = _dims(b_codes, "b_codes", 1)[0]
    K = 2 * Kh
    if K % 16:
        raise ValueError(f"K = {K} is not a multiple of 16")
    dev = a_codes.device
    _need(a_codes, torch.uint8, (M, K // 2), "a_codes")
    _need(a_scales, torch.uint8, (M, K // 16), "a_scales", dev)
    _need(a_global_scale, torch.float32, (1,), "a_global_scale", dev)
    _need(b_codes, torch.uint8, (N, K // 2), "b_codes (A and B must agree on K)", dev)
    _need(b_scales, torch.uint8, (N, K // 16), "b_scales", dev)
    _need(b_global_scale, torch.float32, (1,), "b_global_scale", dev)
    if bias is not None:
        _need(bias, torch.bfloat16, (N,), "bias", dev)
    if out is not None:
        _need(out, torch.bfloat16, (M, N), "out", dev)
    if split and workspace is not None:
        _need_workspace(workspace, nvfp4_gemm_workspace_bytes(M, N, K), "workspace", dev)
    st = _stream(stream, dev)
    if out is None:
        out = _alloc((M, N), torch.bfloat16, dev, st)
    if not split:
        workspace = None
    elif workspace is None:
        need = nvfp4_gemm_workspace_bytes(M, N, K)
        if need:
            workspace = _alloc((need,), torch.uint8, dev, st)
    _check(lib.nvfp4_gemm(_ptr(a_codes), _ptr(a_scales), _ptr(a_global_scale), _ptr(b_codes),
                          _ptr(b_scales), _ptr(b_global_scale), _ptr(bias), _ptr(out),
                          _ptr(workspace), 0 if workspace is None else workspace.numel(),
                          M, N, K, ctypes.c_void_p(st.cuda_stream)))
    return out


def nvfp4_linear(x, w_codes, w_scales, w_global_scale, bias=None, out=None, workspace=None,
                 stream=None):
    """NVFP4 linear: quantize BF16 x [M, K] on the fly, GEMM with the packed
    weight [N, K], add bias -> BF16 [M, N]."""
    if stream is None:
        r = _host.nvfp4_linear(x, w_codes, w_scales, w_global_scale, bias, out, workspace)
        if r is not None:
            return _native(r)
    M, K = _dims(x, "x", 16)
    dev = x.device
    _need(x, torch.bfloat16, (M, K), "x")
    N = _dims(w_codes, "w_codes", 1)[0]
    _need(w_codes, torch.uint8, (N, K // 2), "w_codes (x and w must agree on K)", dev)
    _need(w_scales, torch.uint8, (N, K // 16), "w_scales", dev)
    _need(w_global_scale, torch.float32, (1,), "w_global_scale", dev)
    if bias is not None:
        _need(bias, torch.bfloat16, (N,), "bias", dev)
    if out is not None:
        _need(out, torch.bfloat16, (M, N), "out", dev)
    need = nvfp4_linear_workspace_bytes(M, N, K)
    if workspace is not None:
        _need_workspace(workspace, need, "workspace", dev)
    st = _stream(stream, dev)
    if out is None:
        out = _alloc((M, N), torch.bfloat16, dev, st)
    if workspace is None:
        workspace = _alloc((need,), torch.uint8, dev, st)
    _check(lib.nvfp4_linear(_ptr(x), _ptr(w_codes), _ptr(w_scales), _ptr(w_global_scale),
                            _ptr(bias), _ptr(out), _ptr(workspace), workspace.numel(),
                            M, N, K, ctypes.c_void_p(st.cuda_stream)))
    return out


def mxfp4_linear_workspace_bytes(M: int, K: int) -> int:
    return lib.mxfp4_linear_workspace_bytes(M, K)


def mxfp4_quantize(x, codes=None, scales=None, stream=None):
    """x: BF16 [rows, K] (K % 32 == 0) -> (codes uint8 [rows, K/2],
    scales uint8 [rows, K/32], E8M0)."""
    if stream is None:
        r = _host.mxfp4_quantize(x, codes, scales)
        if r is not None:
            return _native(r)
    rows, K = _dims(x, "x", 32)
    dev = x.device
    _need(x, torch.bfloat16, (rows, K), "x")
    if codes is not None:
        _need(codes, torch.uint8, (rows, K // 2), "codes", dev)
    if scales is not None:
        _need(scales, torch.uint8, (rows, K // 32), "scales", dev)
    st = _stream(stream, dev)
    if codes is None:
        codes = _alloc((rows, K // 2), torch.uint8, dev, st)
    if scales is None:
        scales = _alloc((rows, K // 32), torch.uint8, dev, st)
    _check(lib.mxfp4_quantize(_ptr(x), rows, K, _ptr(codes), _ptr(scales),
                              ctypes.c_void_p(st.cuda_stream)))
    return codes, scales


def mxfp4_gemm(a_codes, a_scales, b_codes, b_scales, bias=None, out=None, stream=None):
    """MXFP4 GEMM: A [M, K] (packed), B [N, K] (packed) -> BF16 [M, N]."""
    if stream is None:
        r = _host.mxfp4_gemm(a_codes, a_scales, b_codes, b_scales, bias, out)
        if r is not None:
            return _native(r)
    M, Kh = _dims(a_codes, "a_codes", 1)
    N = _dims(b_codes, "b_codes", 1)[0]
    K = 2 * Kh
    if K % 32:
        raise ValueError(f"K = {K} is not a multiple of 32")
    dev = a_codes.device
    _need(a_codes, torch.uint8, (M, K // 2), "a_codes")
    _need(a_scales, torch.uint8, (M, K // 32), "a_scales", dev)
    _need(b_codes, torch.uint8, (N, K // 2), "b_codes (A and B must agree on K)", dev)
    _need(b_scales, torch.uint8, (N, K // 32), "b_scales", dev)
    if bias is not None:
        _need(bias, torch.bfloat16, (N,), "bias", dev)
    if out is not None:
        _need(out, torch.bfloat16, (M, N), "out", dev)
    st = _stream(stream, dev)
    if out is None:
        out = _alloc((M, N), torch.bfloat16, dev, st)
    _check(lib.mxfp4_gemm(_ptr(a_codes), _ptr(a_scales), _ptr(b_codes), _ptr(b_scales),
                          _ptr(bias), _ptr(out), M, N, K, ctypes.c_void_p(st.cuda_stream)))
    return out


def mxfp4_linear(x, w_codes, w_scales, bias=None, out=None, workspace=None, stream=None):
    """MXFP4 linear: quantize BF16 x [M, K] on the fly, GEMM with the packed
    weight [N, K], add bias -> BF16 [M, N]."""
    if stream is None:
        r = _host.mxfp4_linear(x, w_codes, w_scales, bias, out, workspace)
        if r is not None:
            return _native(r)
    M, K = _dims(x, "x", 32)
    dev = x.device
    _need(x, torch.bfloat16, (M, K), "x")
    N = _dims(w_codes, "w_codes", 1)[0]
    _need(w_codes, torch.uint8, (N, K // 2), "w_codes (x and w must agree on K)", dev)
    _need(w_scales, torch.uint8, (N, K // 32), "w_scales", dev)
    if bias is not None:
        _need(bias, torch.bfloat16, (N,), "bias", dev)
    if out is not None:
        _need(out, torch.bfloat16, (M, N), "out", dev)
    need = mxfp4_linear_workspace_bytes(M, K)
    if workspace is not None:
        _need_workspace(workspace, need, "workspace", dev)
    st = _stream(stream, dev)
    if out is None:
        out = _alloc((M, N), torch.bfloat16, dev, st)
    if workspace is None:
        workspace = _alloc((need,), torch.uint8, dev, st)
    _check(lib.mxfp4_linear(_ptr(x), _ptr(w_codes), _ptr(w_scales), _ptr(bias), _ptr(out),
                            _ptr(workspace), workspace.numel(), M, N, K,
                            ctypes.c_void_p(st.cuda_stream)))
    return out


# ---- operators around the linears -----------------------------------------

TYPES = {torch.bfloat16: 0, torch.float16: 1, torch.float32: 2}
LAYOUTS = {"half": 0, "interleaved": 1}


def _type(t, name):
    if not isinstance(t, torch.Tensor):
        raise ValueError(f"{name}: expected a torch.Tensor, got {type(t).__name__}")
    if t.dtype not in TYPES:
        raise ValueError(f"{name}: expected bfloat16, float16 or float32, got {t.dtype}")
    return TYPES[t.dtype]


def _need_strided(t, dtype, shape, name, device):
    """A GPU tensor of this type and shape whose last dimension is contiguous;
    the others may have any stride."""
    if not isinstance(t, torch.Tensor):
        raise ValueError(f"{name}: expected a torch.Tensor, got {type(t).__name__}")
    if t.layout != torch.strided or t.dtype != dtype or tuple(t.shape) != tuple(shape) or not _is_gpu(t) \
            or t.device != device or (shape[-1] > 1 and t.stride(-1) != 1):
        raise ValueError(f"{name}: expected CUDA {dtype} {tuple(shape)} on {device} with a contiguous last dimension, "
                         f"got {t.dtype} {tuple(t.shape)} strides {t.stride()} on {t.device}")


def _norm_operands(x, residual, gain, eps, sum_out):
    """Checked: (type, rows, width, device, groups, gain stride)."""
    kind = _type(x, "x")
    if x.dim() != 2:
        raise ValueError("x: expected a 2-D tensor")
    rows, width = x.shape
    dev = x.device
    _need_strided(x, x.dtype, (rows, width), "x", dev)
    if residual is not None:
        _need_strided(residual, x.dtype, (rows, width), "residual", dev)
    if sum_out is not None:
        if residual is None:
            raise ValueError("sum_out: given without a residual")
        _need_strided(sum_out, x.dtype, (rows, width), "sum_out", dev)
    groups, gain_stride = _gain(gain, x, rows, width, dev)
    if not eps >= 0:
        raise ValueError(f"eps: expected a number of at least 0, got {eps}")
    return kind, rows, width, dev, groups, gain_stride


def _gain(gain, x, rows, width, dev):
    if gain is None:
        return 1, 0
    if not isinstance(gain, torch.Tensor) or gain.dim() not in (1, 2):
        raise ValueError("gain: expected a tensor [width] or [groups, width]")
    groups = 1 if gain.dim() == 1 else gain.shape[0]
    _need_strided(gain, x.dtype, (width,) if gain.dim() == 1 else (groups, width), "gain", dev)
    if groups < 1 or rows % groups:
        raise ValueError(f"gain: {rows} rows cannot be dealt to {groups} groups evenly")
    return groups, 0 if gain.dim() == 1 else gain.stride(0)


def _rows_of(t):
    """Pointer and row stride, as the C-ABI takes them."""
    return (None, 0) if t is None else (_ptr(t), t.stride(0))


def add_rmsnorm(x, residual=None, gain=None, eps=1e-6, out=None, sum_out=None, stream=None):
    """Root-mean-square norm of the rows of x + residual, times gain
    ([width], or [groups, width] with the rows dealt to the groups in order)
    -> (out, sum); sum, x + residual rounded to x's type, is None without a
    residual.  x [rows, width] BF16, FP16 or FP32, rows of any stride; sum_out
    may be x or residual.  Nothing is recorded for autograd here or in the other
    calls: gradients are rmsnorm_backward's and rotary's with inverse=True."""
    if stream is None:
        r = _host.add_rmsnorm(x, residual, gain, eps, out, sum_out)
        if r is not None:
            return _native(r)
    kind, rows, width, dev, groups, gain_stride = _norm_operands(x, residual, gain, eps, sum_out)
    if out is not None:
        _need_strided(out, x.dtype, (rows, width), "out", dev)
    st = _stream(stream, dev)
    if out is None:
        out = _alloc((rows, width), x.dtype, dev, st)
    if residual is not None and sum_out is None:
        sum_out = _alloc((rows, width), x.dtype, dev, st)
    _check(lib.solfp4_add_rmsnorm(kind, *_rows_of(x), *_rows_of(residual), _ptr(gain), gain_stride, groups, eps,
                                  *_rows_of(sum_out), *_rows_of(out), rows, width, ctypes.c_void_p(st.cuda_stream)))
    return out, sum_out


def _quantized_add_rmsnorm(fn, native, pack, x, residual, gain, eps, codes, scales, sum_out, stream):
    if stream is None:
        r = native(x, residual, gain, eps, codes, scales, sum_out)
        if r is not None:
            return _native(r)
    kind, rows, width, dev, groups, gain_stride = _norm_operands(x, residual, gain, eps, sum_out)
    if width % 32:
        raise ValueError(f"x: width {width} is not a multiple of 32")
    if codes is not None:
        _need(codes, torch.uint8, (rows, width // pack), "codes", dev)
    if scales is not None:
        _need(scales, torch.uint8, (rows, width // 32), "scales", dev)
    st = _stream(stream, dev)
    if codes is None:
        codes = _alloc((rows, width // pack), torch.uint8, dev, st)
    if scales is None:
        scales = _alloc((rows, width // 32), torch.uint8, dev, st)
    if residual is not None and sum_out is None:
        sum_out = _alloc((rows, width), x.dtype, dev, st)
    _check(fn(kind, *_rows_of(x), *_rows_of(residual), _ptr(gain), gain_stride, groups, eps, *_rows_of(sum_out),
              _ptr(codes), _ptr(scales), rows, width, ctypes.c_void_p(st.cuda_stream)))
    return codes, scales, sum_out


def mxfp8_add_rmsnorm(x, residual=None, gain=None, eps=1e-6, codes=None, scales=None, sum_out=None, stream=None):
    """add_rmsnorm with its output in MXFP8 -> (codes uint8 [rows, width],
    E4M3, scales uint8 [rows, width/32], E8M0, sum).  width % 32 == 0."""
    return _quantized_add_rmsnorm(lib.mxfp8_add_rmsnorm, _host.mxfp8_add_rmsnorm, 1, x, residual, gain, eps, codes,
                                  scales, sum_out, stream)


def mxfp4_add_rmsnorm(x, residual=None, gain=None, eps=1e-6, codes=None, scales=None, sum_out=None, stream=None):
    """add_rmsnorm with its output in MXFP4, as mxfp4_gemm takes it -> (codes
    uint8 [rows, width/2], scales uint8 [rows, width/32], sum).  width % 32 == 0."""
    return _quantized_add_rmsnorm(lib.mxfp4_add_rmsnorm, _host.mxfp4_add_rmsnorm, 2, x, residual, gain, eps, codes,
                                  scales, sum_out, stream)


def rmsnorm_backward_workspace_bytes(rows: int, width: int, groups: int = 1) -> int:
    return lib.solfp4_rmsnorm_backward_workspace_bytes(rows, width, groups)


def rmsnorm_backward(dy, x, gain=None, dsum=None, eps=1e-6, dx=None, dgain=None, workspace=None, stream=None):
    """Backward pass of add_rmsnorm: dy, the output's gradient; x, the sum
    (or the x of a call without a residual); dsum, what reaches the sum past
    the norm -> (dx, dgain).  dx is the gradient of x and of the residual alike;
    dgain is FP32 in gain's shape, None without a gain."""
    if stream is None:
        r = _host.rmsnorm_backward(dy, x, gain, dsum, eps, dx, dgain, workspace)
        if r is not None:
            return _native(r)
    kind = _type(x, "x")
    if x.dim() != 2:
        raise ValueError("x: expected a 2-D tensor")
    rows, width = x.shape
    dev = x.device
    _need_strided(x, x.dtype, (rows, width), "x", dev)
    _need_strided(dy, x.dtype, (rows, width), "dy", dev)
    if dsum is not None:
        _need_strided(dsum, x.dtype, (rows, width), "dsum", dev)
    if dx is not None:
        _need_strided(dx, x.dtype, (rows, width), "dx", dev)
    groups, gain_stride = _gain(gain, x, rows, width, dev)
    if not eps >= 0:
        raise ValueError(f"eps: expected a number of at least 0, got {eps}")
    need = 0
    if gain is None:
        if dgain is not None:
            raise ValueError("dgain: given without a gain")
    else:
        if dgain is not None:
            _need(dgain, torch.float32, tuple(gain.shape), "dgain", dev)
        need = rmsnorm_backward_workspace_bytes(rows, width, groups)
        if workspace is not None:
            _need_workspace(workspace, need, "workspace", dev)
    st = _stream(stream, dev)
    if dx is None:
        dx = _alloc((rows, width), x.dtype, dev, st)
    if gain is not None:
        if dgain is None:
            dgain = _alloc(tuple(gain.shape), torch.float32, dev, st)
        if workspace is None:
            workspace = _alloc((max(need, 256),), torch.uint8, dev, st)
    _check(lib.solfp4_rmsnorm_backward(kind, *_rows_of(dy), *_rows_of(x), _ptr(gain), gain_stride, groups,
                                       *_rows_of(dsum), eps, *_rows_of(dx), _ptr(dgain), _ptr(workspace),
                                       0 if workspace is None else workspace.numel(), rows, width,
                                       ctypes.c_void_p(st.cuda_stream)))
    return dx, dgain


def rotary_frequencies(rotated: int, base: float = 10000.0, scaling: str | None = None, factor: float = 1.0,
                       original_length: int = 0, low_turns: float = 1.0, high_turns: float = 32.0):
    """Angle per position of each of the rotated/2 pairs, float64 on the host:
    base ** (-2 i / rotated), and for contexts `factor` times longer than the
    one a model was trained on

        "linear"   every frequency divided by factor
        "base"     base * factor ** (rotated / (rotated - 2)) as the base: the
                   fastest pair keeps its frequency, the slowest is divided
                   by factor
        "by-parts" pairs that turn more than high_turns times over
                   original_length keep their frequency, those under low_turns
                   have it divided by factor, in between linearly mixed by
                   their number of turns
    """
    if rotated < 0 or rotated % 2:
        raise ValueError(f"rotated: expected an even number, got {rotated}")
    if scaling not in (None, "linear", "base", "by-parts"):
        raise ValueError(f"scaling: expected None, 'linear', 'base' or 'by-parts', got {scaling!r}")
    if not base > 0 or not factor > 0:
        raise ValueError("base and factor: expected positive numbers")
    i = torch.arange(rotated // 2, dtype=torch.float64)
    if scaling == "base":
        if rotated <= 2:
            raise ValueError("scaling 'base' needs more than one pair")
        base = base * factor ** (rotated / (rotated - 2))
    f = base ** (-2.0 * i / max(rotated, 1))
    if scaling == "linear":
        f = f / factor
    if scaling == "by-parts":
        if original_length <= 0 or not high_turns > low_turns:
            raise ValueError("scaling 'by-parts' needs original_length and high_turns above low_turns")
        turns = original_length * f / (2 * torch.pi)
        keep = ((turns - low_turns) / (high_turns - low_turns)).clamp(0, 1)
        f = f * keep + f / factor * (1 - keep)
    return f


def rotary_table(frequencies, positions, axis_pairs=None, magnitude=1.0, device=None, out=None, stream=None):
    """cos and sin of position x frequency, FP32 [rows, 2 pairs], for rotary.

    frequencies: float64 [pairs].  positions: a row count (row p is position
    p) or an int64 tensor [rows], or [rows, axes] with axis_pairs giving each
    axis's number of pairs (image positions: the first axis_pairs[0] pairs turn
    with axis 0, ...).  magnitude scales both.  The table is on the
    device of a positions tensor, else on `device` (default: the current one)."""
    if not isinstance(frequencies, torch.Tensor) or frequencies.dim() != 1 or frequencies.dtype != torch.float64:
        raise ValueError("frequencies: expected a 1-D float64 tensor")
    pairs = frequencies.numel()
    axes = 1
    if isinstance(positions, torch.Tensor):
        dev = positions.device
        if positions.dim() not in (1, 2):
            raise ValueError("positions: expected [rows] or [rows, axes]")
        _need(positions, torch.int64, positions.shape, "positions")
        rows = positions.shape[0]
        axes = 1 if positions.dim() == 1 else positions.shape[1]
        at = positions
    else:
        rows, at = int(positions), None
        if rows < 0:
            raise ValueError(f"positions: expected at least 0 rows, got {rows}")
        dev = torch.device("cuda" if device is None else device)
        if dev.type != "cuda":
            raise ValueError(f"device: expected a CUDA device, got {dev}")
    if axes > 1 or axis_pairs is not None:
        if axis_pairs is None or len(axis_pairs) != axes or sum(axis_pairs) != pairs or min(axis_pairs) < 0:
            raise ValueError(f"axis_pairs: expected {axes} counts that add up to {pairs}")
    if at is None and dev.index is None:
        dev = torch.device("cuda", torch.cuda.current_device())
    if out is not None:
        _need(out, torch.float32, (rows, 2 * pairs), "out", dev)
    st = _stream(stream, dev)
    with torch.cuda.stream(st):
        f = frequencies.to(dev).contiguous()   # the kernel reads them one after another
    if out is None:
        out = _alloc((rows, 2 * pairs), torch.float32, dev, st)
    counts = None if axis_pairs is None else (ctypes.c_int64 * axes)(*axis_pairs)
    _check(lib.solfp4_rotary_table(_ptr(at), rows, _ptr(f), pairs, counts, axes, float(magnitude), _ptr(out),
                                   ctypes.c_void_p(st.cuda_stream)))
    return out


def _heads_of(t):
    return (None, 0, 0) if t is None else (_ptr(t), t.stride(0), t.stride(1))


def rotary(q, k, table, positions=None, layout="half", inverse=False, q_out=None, k_out=None, stream=None):
    """Rotary positions on q [tokens, q_heads, dim] and k [tokens, k_heads,
    dim] or None -> (q, k) in new tensors, or in q_out and k_out, which may be q
    and k themselves.  Views of a packed QKV buffer are taken as they are.

    table: FP32 [table_rows, rotated] from rotary_table; the first `rotated`
    elements of a head turn.  positions: int32 or int64 [tokens], the table
    row of each token; None: token t takes row t % table_rows.  A position
    outside the table gives NaN.  layout: "half" (pairs i, i + rotated/2) or
    "interleaved" (pairs 2i, 2i + 1).  inverse: the transposed rotation, which
    takes the outputs' gradients to the inputs'."""
    if stream is None:
        r = _host.rotary(q, k, table, positions, LAYOUTS.get(layout, -1), inverse, q_out, k_out)
        if r is not None:
            return _native(r)
    kind = _type(q, "q")
    if q.dim() != 3:
        raise ValueError("q: expected a 3-D tensor [tokens, heads, dim]")
    tokens, heads, dim = q.shape
    dev = q.device
    _need_strided(q, q.dtype, (tokens, heads, dim), "q", dev)
    k_heads = 0
    if k is not None:
        if not isinstance(k, torch.Tensor) or k.dim() != 3:
            raise ValueError("k: expected a 3-D tensor [tokens, heads, dim] or None")
        k_heads = k.shape[1]
        _need_strided(k, q.dtype, (tokens, k_heads, dim), "k", dev)
    elif k_out is not None:
        raise ValueError("k_out: given without k")
    if layout not in LAYOUTS:
        raise ValueError(f"layout: expected 'half' or 'interleaved', got {layout!r}")
    if not isinstance(table, torch.Tensor) or table.dim() != 2:
        raise ValueError("table: expected a 2-D tensor [rows, rotated]")
    table_rows, rotated = table.shape
    _need(table, torch.float32, (table_rows, rotated), "table", dev)
    if rotated % 2 or rotated > dim:
        raise ValueError(f"table: {rotated} elements to rotate, expected an even number of at most {dim}")
    if table_rows == 0 and tokens > 0:
        raise ValueError("table: no rows")
    position_bytes = 0
    if positions is not None:
        if not isinstance(positions, torch.Tensor) or positions.dtype not in (torch.int32, torch.int64):
            raise ValueError("positions: expected an int32 or int64 tensor")
        _need(positions, positions.dtype, (tokens,), "positions", dev)
        position_bytes = positions.element_size()
    if q_out is not None:
        _need_strided(q_out, q.dtype, (tokens, heads, dim), "q_out", dev)
    if k_out is not None:
        _need_strided(k_out, q.dtype, (tokens, k_heads, dim), "k_out", dev)
    st = _stream(stream, dev)
    if q_out is None:
        q_out = _alloc((tokens, heads, dim), q.dtype, dev, st)
    if k is not None and k_out is None:
        k_out = _alloc((tokens, k_heads, dim), q.dtype, dev, st)
    _check(lib.solfp4_rotary(kind, LAYOUTS[layout], int(bool(inverse)), *_heads_of(q), *_heads_of(q_out), heads,
                             *_heads_of(k), *_heads_of(k_out), k_heads, _ptr(table), table_rows, _ptr(positions),
                             position_bytes, tokens, dim, rotated, ctypes.c_void_p(st.cuda_stream)))
    return q_out, k_out


def nvfp4_weight_linear(x, w_codes, w_scales, w_global_scale, bias=None, out=None, stream=None):
    """Linear of few tokens with BF16 activations x [M, K] (not quantized) and
    a packed NVFP4 weight [N, K], plus bias -> BF16 [M, N]."""
    if stream is None:
        r = _host.nvfp4_weight_linear(x, w_codes, w_scales, w_global_scale, bias, out)
        if r is not None:
            return _native(r)
    M, K = _dims(x, "x", 16)
    N = _dims(w_codes, "w_codes", 1)[0]
    dev = x.device
    _need(x, torch.bfloat16, (M, K), "x")
    _need(w_codes, torch.uint8, (N, K // 2), "w_codes (x and w must agree on K)", dev)
    _need(w_scales, torch.uint8, (N, K // 16), "w_scales", dev)
    _need(w_global_scale, torch.float32, (1,), "w_global_scale", dev)
    st, out = _weight_linear_out(bias, out, M, N, dev, stream)
    _check(lib.nvfp4_weight_linear(_ptr(x), _ptr(w_codes), _ptr(w_scales), _ptr(w_global_scale), _ptr(bias),
                                   _ptr(out), M, N, K, ctypes.c_void_p(st.cuda_stream)))
    return out


def _weight_linear_out(bias, out, M, N, dev, stream):
    if bias is not None:
        _need(bias, torch.bfloat16, (N,), "bias", dev)
    if out is not None:
        _need(out, torch.bfloat16, (M, N), "out", dev)
    st = _stream(stream, dev)
    return st, _alloc((M, N), torch.bfloat16, dev, st) if out is None else out


def mxfp4_weight_linear(x, w_codes, w_scales, bias=None, out=None, stream=None):
    """Linear of few tokens with BF16 activations x [M, K] (not quantized) and
    a packed MXFP4 weight [N, K], plus bias -> BF16 [M, N]."""
    if stream is None:
        r = _host.mxfp4_weight_linear(x, w_codes, w_scales, bias, out)
        if r is not None:
            return _native(r)
    M, K = _dims(x, "x", 32)
    N = _dims(w_codes, "w_codes", 1)[0]
    dev = x.device
    _need(x, torch.bfloat16, (M, K), "x")
    _need(w_codes, torch.uint8, (N, K // 2), "w_codes (x and w must agree on K)", dev)
    _need(w_scales, torch.uint8, (N, K // 32), "w_scales", dev)
    st, out = _weight_linear_out(bias, out, M, N, dev, stream)
    _check(lib.mxfp4_weight_linear(_ptr(x), _ptr(w_codes), _ptr(w_scales), _ptr(bias), _ptr(out), M, N, K,
                                   ctypes.c_void_p(st.cuda_stream)))
    return out


def mxfp8_linear(x_codes, x_scales, w_codes, w_scales, bias=None, out=None, stream=None):
    """Linear of few tokens with MXFP8 activations [M, K] (as mxfp8_add_rmsnorm
    writes them) and a packed MXFP4 weight [N, K], plus bias -> BF16 [M, N]."""
    if stream is None:
        r = _host.mxfp8_linear(x_codes, x_scales, w_codes, w_scales, bias, out)
        if r is not None:
            return _native(r)
    M, K = _dims(x_codes, "x_codes", 32)
    N = _dims(w_codes, "w_codes", 1)[0]
    dev = x_codes.device
    _need(x_codes, torch.uint8, (M, K), "x_codes")
    _need(x_scales, torch.uint8, (M, K // 32), "x_scales", dev)
    _need(w_codes, torch.uint8, (N, K // 2), "w_codes (x and w must agree on K)", dev)
    _need(w_scales, torch.uint8, (N, K // 32), "w_scales", dev)
    st, out = _weight_linear_out(bias, out, M, N, dev, stream)
    _check(lib.mxfp8_linear(_ptr(x_codes), _ptr(x_scales), _ptr(w_codes), _ptr(w_scales), _ptr(bias), _ptr(out),
                            M, N, K, ctypes.c_void_p(st.cuda_stream)))
    return out
