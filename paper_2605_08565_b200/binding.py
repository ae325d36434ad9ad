"""Thin binding of libmxq (argument marshalling only; every step runs in the CUDA kernels).

The calls of an inner loop go through the extension module ``_native`` (csrc/mxq_python.cpp), which unpacks the usual
arguments in C++; everything else, and whatever ``_native`` does not take, goes through ctypes (all of it where ``_native``
has not been built).

The functions carry the names of the C-ABI declared in ``include/mxq.h`` and take torch CUDA
tensors (torch supplies device memory and streams, nothing else).  There is no CPU fallback: if
``libmxq.so`` is missing or a call is made without a CUDA device, an exception is raised.
"""
from __future__ import annotations

import ctypes
import importlib.util
import os
import warnings

import torch

from .build import native_path

_HERE = os.path.dirname(os.path.abspath(__file__))
# MXQ_LIB: path of another build of the library; the default is the in-tree build
LIB_PATH = os.environ.get("MXQ_LIB") or os.path.join(_HERE, "libmxq.so")

MXQ_F32, MXQ_BF16 = 0, 1
MXQ_SF_UE8M0, MXQ_SF_UE4M3, MXQ_SF_UE5M3 = 0, 1, 2
MXQ_ABSMAX, MXQ_ABSMAX_PZ, MXQ_4O6, MXQ_4O6_PZ, MXQ_BRUTE, MXQ_BRUTE_PZ, MXQ_ABSMAX_OCP, MXQ_ABSMAX_CLIP7 = range(8)
MXQ_E4M3, MXQ_E5M2 = 0, 1
MXQ_OPT_BRUTE_PRUNE = 1

EXPORTS = (
    "mxq_quantize", "mxq_quantize_ex", "mxq_quantize_mse", "mxq_quantize_batch", "mxq_fake_quantize", "mxq_tensor_amax", "mxq_global_scale_from_amax",
    "mxq_tensor_mse_workspace_bytes", "mxq_tensor_mse", "mxq_tensor_mse_static", "mxq_dequantize", "mxq_dequantize_ex",
    "mxq_block_clip_sse", "mxq_histograms", "mxq_segment_mse", "mxq_mask_interval",
    "mxq_quantize8", "mxq_dequantize8", "mxq_add_rmsnorm8", "mxq_add_rmsnorm8_workspace_bytes", "mxq_add_rmsnorm8_backward", "mxq_swiglu8",
    "mxq_swiglu8_backward", "mxq_set_option", "mxq_get_option", "mxq_launch_count",
    "mxq_status_string", "mxq_last_cuda_error", "mxq_version",
)


class MxqError(RuntimeError):
    pass


class TensorDesc(ctypes.Structure):
    """mxq_tensor_desc of include/mxq.h (one tensor of a multi-tensor launch)."""
    _fields_ = [("x", ctypes.c_void_p), ("out_codes", ctypes.c_void_p), ("out_scales", ctypes.c_void_p),
                ("out_block_sse", ctypes.c_void_p), ("n", ctypes.c_size_t)]


class _CtypesOnly:
    """In the place of the extension module where it is missing: knows no arguments."""

    def __getattr__(self, name):
        return lambda *args: -1


def _import_native():
    path = native_path()
    spec = importlib.util.spec_from_file_location(__package__ + "._native", path)
    if not os.path.exists(path):
        raise ImportError(f"no {os.path.basename(path)}")
    native = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(native)
    return native


_lib = None
_native = None


def load_library() -> ctypes.CDLL:
    """dlopen libmxq.so (built by ``paper_2605_08565_b200.build``); raises if it is missing."""
    global _lib, _native
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise MxqError(f"{LIB_PATH} not found: build it with `python -m paper_2605_08565_b200.build` "
                       "(there is no CPU fallback)")
    L = ctypes.CDLL(LIB_PATH)
    c = ctypes
    vp, sz, i32, f32 = c.c_void_p, c.c_size_t, c.c_int, c.c_float
    L.mxq_quantize.restype = i32
    L.mxq_quantize.argtypes = [vp, sz, i32, i32, i32, f32, vp, vp, vp]
    L.mxq_quantize_ex.restype = i32
    L.mxq_quantize_ex.argtypes = [vp, i32, sz, i32, i32, i32, f32, vp, vp, vp, vp, vp]
    L.mxq_quantize_mse.restype = i32
    L.mxq_quantize_mse.argtypes = [vp, i32, sz, i32, i32, i32, f32, vp, vp, vp, vp, vp, vp, sz, vp]
    L.mxq_quantize_batch.restype = i32
    L.mxq_quantize_batch.argtypes = [vp, vp, sz, i32, i32, i32, i32, f32, vp, vp]
    L.mxq_fake_quantize.restype = i32
    L.mxq_fake_quantize.argtypes = [vp, i32, sz, i32, i32, i32, f32, vp, vp, i32, vp]
    L.mxq_tensor_amax.restype = i32
    L.mxq_tensor_amax.argtypes = [vp, i32, sz, vp, vp, vp]
    L.mxq_global_scale_from_amax.restype = f32
    L.mxq_global_scale_from_amax.argtypes = [f32]
    L.mxq_tensor_mse_workspace_bytes.restype = sz
    L.mxq_tensor_mse_workspace_bytes.argtypes = [sz]
    L.mxq_tensor_mse.restype = i32
    L.mxq_tensor_mse.argtypes = [vp, sz, sz, vp, vp, sz, vp]
    L.mxq_tensor_mse_static.restype = i32
    L.mxq_tensor_mse_static.argtypes = [vp, sz, sz, vp, vp]
    L.mxq_dequantize.restype = i32
    L.mxq_dequantize.argtypes = [vp, vp, sz, i32, i32, f32, vp, i32, vp]
    L.mxq_dequantize_ex.restype = i32
    L.mxq_dequantize_ex.argtypes = [vp, vp, sz, i32, i32, f32, vp, vp, i32, vp]
    L.mxq_block_clip_sse.restype = i32
    L.mxq_block_clip_sse.argtypes = [vp, i32, sz, i32, i32, f32, vp, vp, vp, vp]
    L.mxq_histograms.restype = i32
    L.mxq_histograms.argtypes = [vp, vp, sz, i32, vp, vp, vp]
    L.mxq_segment_mse.restype = i32
    L.mxq_segment_mse.argtypes = [vp, sz, sz, sz, vp, vp]
    L.mxq_mask_interval.restype = i32
    L.mxq_mask_interval.argtypes = [vp, i32, sz, f32, f32, vp, vp]
    L.mxq_quantize8.restype = i32
    L.mxq_quantize8.argtypes = [vp, i32, sz, sz, sz, i32, i32, vp, vp, vp]
    L.mxq_dequantize8.restype = i32
    L.mxq_dequantize8.argtypes = [vp, vp, sz, sz, i32, i32, vp, i32, sz, vp]
    L.mxq_add_rmsnorm8.restype = i32
    L.mxq_add_rmsnorm8.argtypes = [vp, vp, vp, i32, i32, sz, sz, sz, sz, f32, i32, i32, vp, sz, vp, vp, vp, vp, vp, vp]
    L.mxq_add_rmsnorm8_workspace_bytes.restype = sz
    L.mxq_add_rmsnorm8_workspace_bytes.argtypes = [sz, sz]
    L.mxq_add_rmsnorm8_backward.restype = i32
    L.mxq_add_rmsnorm8_backward.argtypes = [vp, vp, vp, i32, i32, sz, sz, sz, sz, vp, vp, vp, i32, i32, vp, sz, vp, vp, sz, vp]
    L.mxq_swiglu8.restype = i32
    L.mxq_swiglu8.argtypes = [vp, vp, i32, sz, sz, sz, sz, i32, i32, vp, vp, vp, vp, vp, vp, vp]
    L.mxq_swiglu8_backward.restype = i32
    L.mxq_swiglu8_backward.argtypes = [vp, i32, sz, sz, sz, vp, vp, vp, vp, i32, i32, vp, sz, vp, sz, vp]
    L.mxq_set_option.restype = i32
    L.mxq_set_option.argtypes = [i32, i32]
    L.mxq_get_option.restype = i32
    L.mxq_get_option.argtypes = [i32, c.POINTER(c.c_int)]
    L.mxq_launch_count.restype = c.c_ulonglong
    L.mxq_launch_count.argtypes = []
    L.mxq_status_string.restype = c.c_char_p
    L.mxq_status_string.argtypes = [i32]
    L.mxq_last_cuda_error.restype = i32
    L.mxq_last_cuda_error.argtypes = []
    L.mxq_version.restype = i32
    L.mxq_version.argtypes = []
    try:
        native = _import_native()
        native.bind({name: c.cast(getattr(L, name), vp).value for name in EXPORTS})
    except ImportError as e:
        warnings.warn(f"extension module _native not usable ({e}): every call goes through ctypes, 2 to 3 us slower; build it with "
                      "`python -m paper_2605_08565_b200.build`", RuntimeWarning, stacklevel=2)
        native = _CtypesOnly()
    _native = native
    _lib = L
    return L


def _check(status: int) -> None:
    if status != 0:
        L = load_library()
        msg = L.mxq_status_string(status).decode()
        if status == 7:
            msg += f" [cudaError {L.mxq_last_cuda_error()}]"
        raise MxqError(f"libmxq status {status}: {msg}")


def _load_native():
    load_library()
    return _native


def _ptr(t) -> int:
    if t is None:
        return 0
    if not t.is_cuda:
        raise MxqError("libmxq takes CUDA tensors only (no CPU fallback)")
    if not t.is_contiguous():
        raise MxqError("tensor must be contiguous")
    return t.data_ptr()


def _dtype_id(t: torch.Tensor) -> int:
    if t.dtype == torch.float32:
        return MXQ_F32
    if t.dtype == torch.bfloat16:
        return MXQ_BF16
    raise MxqError(f"unsupported dtype {t.dtype}")


_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)


def _stream(stream, like=None) -> int:
    """cudaStream_t of `stream`, or of torch's current stream on the device of tensor `like`."""
    if stream is not None:
        return stream.cuda_stream
    if _raw_stream is not None and like is not None and like.is_cuda:
        return _raw_stream(like.device.index if like.device.index is not None else torch.cuda.current_device())
    return torch.cuda.current_stream().cuda_stream


# ---- C-ABI names ---------------------------------------------------------------------------
def mxq_quantize(x, n, block_size, scale_fmt, recipe, global_scale, out_codes, out_scales, out_block_sse) -> None:
    """float32 input, default stream (synchronises with torch's current stream by stream order
    only if that is the default stream)."""
    _check(load_library().mxq_quantize(_ptr(x), n, block_size, scale_fmt, recipe, global_scale,
                                       _ptr(out_codes), _ptr(out_scales), _ptr(out_block_sse)))


def mxq_quantize_ex(x, n, block_size, scale_fmt, recipe, global_scale, d_global_scale, out_codes, out_scales,
                    out_block_sse, stream=None) -> None:
    st = (_native or _load_native()).quantize_ex(x, n, block_size, scale_fmt, recipe, global_scale, d_global_scale,
                                                 out_codes, out_scales, out_block_sse, stream)
    if st == 0:
        return
    if st > 0:
        _check(st)
    _check(load_library().mxq_quantize_ex(_ptr(x), _dtype_id(x), n, block_size, scale_fmt, recipe, global_scale,
                                          _ptr(d_global_scale), _ptr(out_codes), _ptr(out_scales),
                                          _ptr(out_block_sse), _stream(stream, x)))


def mxq_quantize_mse(x, n, block_size, scale_fmt, recipe, global_scale, d_global_scale, out_codes, out_scales,
                     out_block_sse, d_out_mse, d_workspace, stream=None) -> None:
    """Quantize and score in one call: the tensor MSE comes from partial sums formed inside the quantization kernel."""
    st = (_native or _load_native()).quantize_mse(x, n, block_size, scale_fmt, recipe, global_scale, d_global_scale,
                                                  out_codes, out_scales, out_block_sse, d_out_mse, d_workspace,
                                                  stream)
    if st == 0:
        return
    if st > 0:
        _check(st)
    ws_bytes = d_workspace.numel() * d_workspace.element_size() if d_workspace is not None else 0
    _check(load_library().mxq_quantize_mse(_ptr(x), _dtype_id(x), n, block_size, scale_fmt, recipe, global_scale,
                                           _ptr(d_global_scale), _ptr(out_codes), _ptr(out_scales), _ptr(out_block_sse),
                                           _ptr(d_out_mse), _ptr(d_workspace), ws_bytes, _stream(stream, x)))


def make_tensor_descs(items):
    """Descriptor arrays for ``mxq_quantize_batch``: items = [(x, out_codes, out_scales, out_block_sse or None), ...]
    (flat CUDA tensors of one dtype on one device).  Returns (host ctypes array, device uint8 tensor holding
    the same bytes); both must be kept alive until the launch that uses them has run."""
    if not items:
        raise MxqError("empty tensor list")
    arr = (TensorDesc * len(items))()
    for d, (x, codes, scales, sse) in zip(arr, items):
        d.x, d.out_codes, d.out_scales, d.out_block_sse, d.n = _ptr(x), _ptr(codes), _ptr(scales), _ptr(sse), x.numel()
    host = torch.frombuffer(bytearray(bytes(arr)), dtype=torch.uint8)
    return arr, host.to(items[0][0].device)


def mxq_quantize_batch(h_descs, d_descs, n_tensors, dtype_id, block_size, scale_fmt, recipe, global_scale=1.0,
                       d_global_scale=None, stream=None) -> None:
    """One launch over a list of tensors; h_descs / d_descs from ``make_tensor_descs``."""
    st = (_native or _load_native()).quantize_batch(ctypes.addressof(h_descs), d_descs, n_tensors, dtype_id,
                                                    block_size, scale_fmt, recipe, global_scale, d_global_scale,
                                                    stream)
    if st == 0:
        return
    if st > 0:
        _check(st)
    _check(load_library().mxq_quantize_batch(ctypes.addressof(h_descs), _ptr(d_descs), n_tensors, dtype_id, block_size,
                                             scale_fmt, recipe, global_scale, _ptr(d_global_scale),
                                             _stream(stream, d_descs)))


def mxq_fake_quantize(x, n, block_size, scale_fmt, recipe, global_scale, d_global_scale, d_out, stream=None) -> None:
    st = (_native or _load_native()).fake_quantize(x, n, block_size, scale_fmt, recipe, global_scale, d_global_scale,
                                                   d_out, stream)
    if st == 0:
        return
    if st > 0:
        _check(st)
    _check(load_library().mxq_fake_quantize(_ptr(x), _dtype_id(x), n, block_size, scale_fmt, recipe, global_scale,
                                            _ptr(d_global_scale), _ptr(d_out), _dtype_id(d_out), _stream(stream, x)))


def mxq_tensor_amax(x, n, d_out_amax, d_out_global_scale=None, stream=None) -> None:
    st = (_native or _load_native()).tensor_amax(x, n, d_out_amax, d_out_global_scale, stream)
    if st == 0:
        return
    if st > 0:
        _check(st)
    _check(load_library().mxq_tensor_amax(_ptr(x), _dtype_id(x), n, _ptr(d_out_amax), _ptr(d_out_global_scale),
                                          _stream(stream, x)))


def mxq_global_scale_from_amax(amax: float) -> float:
    return float(load_library().mxq_global_scale_from_amax(amax))


def mxq_tensor_mse_workspace_bytes(n_blocks: int) -> int:
    return int(load_library().mxq_tensor_mse_workspace_bytes(n_blocks))


def mxq_tensor_mse(d_block_sse, n_blocks, n, d_out_mse, d_workspace, stream=None) -> None:
    st = (_native or _load_native()).tensor_mse(d_block_sse, n_blocks, n, d_out_mse, d_workspace, stream)
    if st == 0:
        return
    if st > 0:
        _check(st)
    ws_bytes = d_workspace.numel() * d_workspace.element_size() if d_workspace is not None else 0
    _check(load_library().mxq_tensor_mse(_ptr(d_block_sse), n_blocks, n, _ptr(d_out_mse), _ptr(d_workspace),
                                         ws_bytes, _stream(stream, d_block_sse)))


def mxq_tensor_mse_static(d_block_sse, n_blocks, n, d_out_mse, stream=None) -> None:
    """Tensor MSE with the library's built-in scratch array: no workspace argument, nothing allocated."""
    _check(load_library().mxq_tensor_mse_static(_ptr(d_block_sse), n_blocks, n, _ptr(d_out_mse), _stream(stream, d_block_sse)))


def mxq_dequantize(d_codes, d_scales, n, block_size, scale_fmt, global_scale, d_out, stream=None) -> None:
    _check(load_library().mxq_dequantize(_ptr(d_codes), _ptr(d_scales), n, block_size, scale_fmt, global_scale,
                                         _ptr(d_out), _dtype_id(d_out), _stream(stream, d_out)))


def mxq_dequantize_ex(d_codes, d_scales, n, block_size, scale_fmt, global_scale, d_global_scale, d_out, stream=None) -> None:
    st = (_native or _load_native()).dequantize_ex(d_codes, d_scales, n, block_size, scale_fmt, global_scale,
                                                   d_global_scale, d_out, stream)
    if st == 0:
        return
    if st > 0:
        _check(st)
    _check(load_library().mxq_dequantize_ex(_ptr(d_codes), _ptr(d_scales), n, block_size, scale_fmt, global_scale,
                                            _ptr(d_global_scale), _ptr(d_out), _dtype_id(d_out), _stream(stream, d_out)))


def mxq_block_clip_sse(x, n, block_size, scale_fmt, global_scale, d_global_scale, d_scales, out_clip_sse,
                       stream=None) -> None:
    st = (_native or _load_native()).block_clip_sse(x, n, block_size, scale_fmt, global_scale, d_global_scale,
                                                    d_scales, out_clip_sse, stream)
    if st == 0:
        return
    if st > 0:
        _check(st)
    _check(load_library().mxq_block_clip_sse(_ptr(x), _dtype_id(x), n, block_size, scale_fmt, global_scale,
                                             _ptr(d_global_scale), _ptr(d_scales), _ptr(out_clip_sse), _stream(stream, x)))


def mxq_histograms(d_codes, d_scales, n, block_size, d_code_hist, d_scale_hist, stream=None) -> None:
    """d_code_hist: 16 and d_scale_hist: 256 int64/uint64 CUDA counters; counts are added to them."""
    st = (_native or _load_native()).histograms(d_codes, d_scales, n, block_size, d_code_hist, d_scale_hist, stream)
    if st == 0:
        return
    if st > 0:
        _check(st)
    _check(load_library().mxq_histograms(_ptr(d_codes), _ptr(d_scales), n, block_size, _ptr(d_code_hist),
                                         _ptr(d_scale_hist), _stream(stream, d_codes)))


def mxq_segment_mse(d_block_sse, n_blocks, blocks_per_segment, elems_per_segment, d_out_mse, stream=None) -> None:
    st = (_native or _load_native()).segment_mse(d_block_sse, n_blocks, blocks_per_segment, elems_per_segment,
                                                 d_out_mse, stream)
    if st == 0:
        return
    if st > 0:
        _check(st)
    _check(load_library().mxq_segment_mse(_ptr(d_block_sse), n_blocks, blocks_per_segment, elems_per_segment,
                                          _ptr(d_out_mse), _stream(stream, d_block_sse)))


def mxq_mask_interval(x, n, lo, hi, d_out, stream=None) -> None:
    _check(load_library().mxq_mask_interval(_ptr(x), _dtype_id(x), n, lo, hi, _ptr(d_out), _stream(stream, x)))


# ---- block-scaled 8-bit activations ---------------------------------------------------------------
# Wide tensors are (..., cols), rows evenly spaced and elements of a row contiguous (a slice of a wider tensor's columns, say); rows, cols
# and strides are taken from them.  Codes (uint8 or the element format's float8 type) and scales (uint8 or float8_e8m0fnu) are contiguous.
# All tensors lie on one device, which need not be the current one.
_CODE_TYPE = {MXQ_E4M3: torch.float8_e4m3fn, MXQ_E5M2: torch.float8_e5m2}


def _check_block8(block_size) -> None:
    if isinstance(block_size, bool) or not isinstance(block_size, int) or block_size not in (16, 32, 64, 128):
        raise MxqError(f"block_size must be 16, 32, 64 or 128, got {block_size}")


class _Call8:
    """Checks the tensors of one call against each other; the first wide tensor gives rows, cols, type and device."""

    def __init__(self, first, block_size, elem_fmt):
        if not isinstance(first, torch.Tensor) or not first.is_cuda:
            raise MxqError("libmxq takes CUDA tensors only (no CPU fallback)")
        if first.dim() == 0:
            raise MxqError("a tensor of rows is expected, got a scalar")
        if first.numel() == 0:
            raise MxqError(f"at least one row and one element a row are expected, got {tuple(first.shape)}")
        _check_block8(block_size)
        self.device, self.dtype, self.elem_fmt = first.device, first.dtype, elem_fmt
        self.cols = first.shape[-1]
        self.rows = first.numel() // self.cols
        self.blocks = -(-self.cols // block_size)

    def _on_device(self, t, what):
        if not isinstance(t, torch.Tensor) or not t.is_cuda:
            raise MxqError("libmxq takes CUDA tensors only (no CPU fallback)")
        if t.device != self.device:
            raise MxqError(f"{what} lies on {t.device}, the other tensors on {self.device}")

    def wide(self, t, what, optional=False):
        """(address, row stride)"""
        if t is None and optional:
            return 0, 0
        self._on_device(t, what)
        if t.dtype != self.dtype:
            raise MxqError(f"{what} is {t.dtype}, the other tensors {self.dtype}")
        if t.dim() == 0 or t.shape[-1] != self.cols or t.numel() != self.rows * self.cols:
            raise MxqError(f"{what} is {tuple(t.shape)}, {self.rows} rows of {self.cols} are expected")
        try:
            t = t.view(self.rows, self.cols)
        except RuntimeError:
            raise MxqError(f"{what}: rows must be evenly spaced") from None
        if self.cols > 1 and t.stride(1) != 1:
            raise MxqError(f"{what}: the elements of a row must be contiguous")
        return t.data_ptr(), t.stride(0) if self.rows > 1 else self.cols

    def held(self, codes, scales, what, optional=False):
        if codes is None and scales is None and optional:
            return 0, 0
        for t, name, count, types in ((codes, what + "codes", self.rows * self.cols, (torch.uint8, _CODE_TYPE.get(self.elem_fmt))),
                                      (scales, what + "scales", self.rows * self.blocks, (torch.uint8, torch.float8_e8m0fnu))):
            self._on_device(t, name)
            if t.dtype not in types:
                raise MxqError(f"{name}: unsupported dtype {t.dtype}")
            if not t.is_contiguous() or t.numel() != count:
                raise MxqError(f"{name}: {count} contiguous bytes are expected, got {tuple(t.shape)}")
        return codes.data_ptr(), scales.data_ptr()

    def vector(self, t, what, count, dtype=torch.float32, optional=False):
        if t is None and optional:
            return 0
        self._on_device(t, what)
        if dtype is not None and t.dtype != dtype:
            raise MxqError(f"{what} is {t.dtype}, {dtype} is expected")
        if not t.is_contiguous() or t.numel() != count:
            raise MxqError(f"{what}: {count} contiguous elements are expected, got {tuple(t.shape)}")
        return t.data_ptr()


def mxq_quantize8(x, block_size, elem_fmt, out_codes, out_scales, stream=None) -> None:
    st = (_native or _load_native()).quantize8(x, block_size, elem_fmt, out_codes, out_scales, stream)
    if st == 0:
        return
    if st > 0:
        _check(st)
    c = _Call8(x, block_size, elem_fmt)
    (px, sx), out = c.wide(x, "x"), c.held(out_codes, out_scales, "out_")
    with torch.cuda.device(c.device):
        _check(load_library().mxq_quantize8(px, _dtype_id(x), c.rows, c.cols, sx, block_size, elem_fmt, *out, _stream(stream, x)))


def mxq_dequantize8(d_codes, d_scales, block_size, elem_fmt, d_out, stream=None) -> None:
    st = (_native or _load_native()).dequantize8(d_codes, d_scales, block_size, elem_fmt, d_out, stream)
    if st == 0:
        return
    if st > 0:
        _check(st)
    c = _Call8(d_out, block_size, elem_fmt)
    (po, so), held = c.wide(d_out, "d_out"), c.held(d_codes, d_scales, "d_")
    with torch.cuda.device(c.device):
        _check(load_library().mxq_dequantize8(*held, c.rows, c.cols, block_size, elem_fmt, po, _dtype_id(d_out), so, _stream(stream, d_out)))


def mxq_add_rmsnorm8(x, residual, weight, eps, block_size, elem_fmt, out_sum, out_codes, out_scales, kept_codes=None, kept_scales=None,
                     out_rstd=None, stream=None) -> None:
    st = (_native or _load_native()).add_rmsnorm8(x, residual, weight, eps, block_size, elem_fmt, out_sum, out_codes, out_scales,
                                                  kept_codes, kept_scales, out_rstd, stream)
    if st == 0:
        return
    if st > 0:
        _check(st)
    c = _Call8(x, block_size, elem_fmt)
    (px, sx), (pr, sr), (ps, ss) = c.wide(x, "x"), c.wide(residual, "residual", True), c.wide(out_sum, "out_sum", True)
    pw = c.vector(weight, "weight", c.cols, None)
    out, kept = c.held(out_codes, out_scales, "out_"), c.held(kept_codes, kept_scales, "kept_", True)
    rstd = c.vector(out_rstd, "out_rstd", c.rows, optional=True)
    with torch.cuda.device(c.device):
        _check(load_library().mxq_add_rmsnorm8(px, pr, pw, _dtype_id(x), _dtype_id(weight), c.rows, c.cols, sx, sr, eps, block_size, elem_fmt,
                                               ps, ss, *out, *kept, rstd, _stream(stream, x)))


def mxq_add_rmsnorm8_workspace_bytes(rows: int, cols: int) -> int:
    return int(load_library().mxq_add_rmsnorm8_workspace_bytes(rows, cols))


def mxq_add_rmsnorm8_backward(dy, dsum, weight, kept_codes, kept_scales, rstd, block_size, elem_fmt, dx, dweight=None, d_workspace=None,
                              stream=None) -> None:
    st = (_native or _load_native()).add_rmsnorm8_backward(dy, dsum, weight, kept_codes, kept_scales, rstd, block_size, elem_fmt, dx, dweight,
                                                           d_workspace, stream)
    if st == 0:
        return
    if st > 0:
        _check(st)
    c = _Call8(dy, block_size, elem_fmt)
    (py, sy), (ps, ss), (px, sx) = c.wide(dy, "dy"), c.wide(dsum, "dsum", True), c.wide(dx, "dx")
    pw = c.vector(weight, "weight", c.cols, None)
    kept, prs = c.held(kept_codes, kept_scales, "kept_"), c.vector(rstd, "rstd", c.rows)
    pdw = c.vector(dweight, "dweight", c.cols, optional=True)
    if d_workspace is not None:
        c._on_device(d_workspace, "d_workspace")
    pws = c.vector(d_workspace, "d_workspace", d_workspace.numel(), None) if d_workspace is not None else 0
    ws_bytes = d_workspace.numel() * d_workspace.element_size() if d_workspace is not None else 0
    with torch.cuda.device(c.device):
        _check(load_library().mxq_add_rmsnorm8_backward(py, ps, pw, _dtype_id(dy), _dtype_id(weight), c.rows, c.cols, sy, ss, *kept, prs,
                                                        block_size, elem_fmt, px, sx, pdw, pws, ws_bytes, _stream(stream, dy)))


def mxq_swiglu8(gate, up, block_size, elem_fmt, out_codes, out_scales, gate_codes=None, gate_scales=None, up_codes=None, up_scales=None,
                stream=None) -> None:
    st = (_native or _load_native()).swiglu8(gate, up, block_size, elem_fmt, out_codes, out_scales, gate_codes, gate_scales, up_codes,
                                             up_scales, stream)
    if st == 0:
        return
    if st > 0:
        _check(st)
    c = _Call8(gate, block_size, elem_fmt)
    (pg, sg), (pu, su) = c.wide(gate, "gate"), c.wide(up, "up")
    out = c.held(out_codes, out_scales, "out_")
    kept = (*c.held(gate_codes, gate_scales, "gate_", True), *c.held(up_codes, up_scales, "up_", True))
    with torch.cuda.device(c.device):
        _check(load_library().mxq_swiglu8(pg, pu, _dtype_id(gate), c.rows, c.cols, sg, su, block_size, elem_fmt, *out, *kept,
                                          _stream(stream, gate)))


def mxq_swiglu8_backward(dy, gate_codes, gate_scales, up_codes, up_scales, block_size, elem_fmt, dgate, dup, stream=None) -> None:
    st = (_native or _load_native()).swiglu8_backward(dy, gate_codes, gate_scales, up_codes, up_scales, block_size, elem_fmt, dgate, dup,
                                                      stream)
    if st == 0:
        return
    if st > 0:
        _check(st)
    c = _Call8(dy, block_size, elem_fmt)
    (py, sy), (pg, sg), (pu, su) = c.wide(dy, "dy"), c.wide(dgate, "dgate"), c.wide(dup, "dup")
    kept = (*c.held(gate_codes, gate_scales, "gate_"), *c.held(up_codes, up_scales, "up_"))
    with torch.cuda.device(c.device):
        _check(load_library().mxq_swiglu8_backward(py, _dtype_id(dy), c.rows, c.cols, sy, *kept, block_size, elem_fmt, pg, sg, pu, su,
                                                   _stream(stream, dy)))


def mxq_set_option(option: int, value: int) -> None:
    st = (_native or _load_native()).set_option(int(option), int(value))
    if st == 0:
        return
    if st > 0:
        _check(st)
    _check(load_library().mxq_set_option(int(option), int(value)))


def mxq_get_option(option: int) -> int:
    out = ctypes.c_int(0)
    _check(load_library().mxq_get_option(int(option), ctypes.byref(out)))
    return int(out.value)


def mxq_launch_count() -> int:
    return int(load_library().mxq_launch_count())


def mxq_version() -> int:
    return int(load_library().mxq_version())


# ---- convenience: allocate outputs with torch, then call the C-ABI -----------------------------
def alloc_outputs(n: int, block_size: int, device, with_sse: bool = True):
    codes = torch.empty(n // 2, dtype=torch.uint8, device=device)
    scales = torch.empty(n // block_size, dtype=torch.uint8, device=device)
    sse = torch.empty(n // block_size, dtype=torch.float32, device=device) if with_sse else None
    return codes, scales, sse


def quantize(x: torch.Tensor, block_size: int, scale_fmt: int, recipe: int, global_scale: float = 1.0,
             d_global_scale=None, with_sse: bool = True, stream=None):
    """Allocates (codes, scales, block_sse) and runs mxq_quantize_ex on the flat tensor."""
    x = x.reshape(-1)
    codes, scales, sse = alloc_outputs(x.numel(), block_size, x.device, with_sse)
    mxq_quantize_ex(x, x.numel(), block_size, scale_fmt, recipe, global_scale, d_global_scale, codes, scales, sse,
                    stream)
    return codes, scales, sse


def tensor_mse(block_sse: torch.Tensor, n: int, stream=None) -> torch.Tensor:
    ws = torch.empty(mxq_tensor_mse_workspace_bytes(block_sse.numel()) // 8, dtype=torch.float64,
                     device=block_sse.device)
    out = torch.empty(1, dtype=torch.float64, device=block_sse.device)
    mxq_tensor_mse(block_sse, block_sse.numel(), n, out, ws, stream)
    return out


def alloc_outputs8(rows: int, cols: int, block_size: int, elem_fmt: int, device):
    """Codes and scales of one 8-bit tensor, as the float8 types that torch has for them."""
    _check_block8(block_size)
    if elem_fmt not in _CODE_TYPE:
        raise MxqError(f"elem_fmt must be MXQ_E4M3 or MXQ_E5M2, got {elem_fmt}")
    codes = torch.empty(rows, cols, dtype=_CODE_TYPE[elem_fmt], device=device)
    scales = torch.empty(rows, -(-cols // block_size), dtype=torch.float8_e8m0fnu, device=device)
    return codes, scales


def quantize8(x: torch.Tensor, block_size: int = 32, elem_fmt: int = MXQ_E4M3, stream=None):
    """Allocates (codes, scales) and runs mxq_quantize8 on the rows of x."""
    c = _Call8(x, block_size, elem_fmt)
    codes, scales = alloc_outputs8(c.rows, c.cols, block_size, elem_fmt, c.device)
    mxq_quantize8(x, block_size, elem_fmt, codes, scales, stream)
    return codes, scales
