"""GB300-native (sm_103a) H-Scale hot path: Python binding of ``libhscale.so``.

The functions here have the names of the C entry points in ``include/hscale.h`` and
only marshal arguments: they take torch CUDA tensors, check dtype/shape/device, pass
raw device pointers and the current CUDA stream through ctypes, and raise
``HScaleError`` on a non-zero status.  Every step of the path runs in the CUDA
kernels; there is no CPU fallback: if the compiled library is missing, loading it
raises.

Paper map: ``hscale_hessian_diag_accumulate`` is h = diag(X^T X) (Sec. 3.2, Eq. 4);
``hscale_rtn_scales`` the global scale and RTN codes (Sec. 3.3, Eq. 7);
``hscale_refine_scales`` Algorithm 1 (Eqs. 6-13); ``hscale_pack_nvfp4`` the final
re-quantization (Sec. 3.3); ``hscale_fourover6_codes`` the 4over6 start of Algorithm 2.
"""
from __future__ import annotations

import ctypes
import pathlib
import threading

import torch

__all__ = [
    "HScaleError", "load", "library_path", "hscale_status_string", "hscale_abi_version",
    "hscale_device_error_flags",
    "hscale_hessian_diag_accumulate", "hscale_hessian_diag_accumulate_ex", "HSCALE_HESSIAN_X_READY",
    "hscale_hessian_sum_partials", "hscale_amax_bits", "hscale_global_scale_from_amax",
    "hscale_rtn_workspace_bytes", "hscale_rtn_scales",
    "hscale_rtn_scales_noalloc",
    "hscale_refine_scales", "hscale_refine_scales_ex", "hscale_refine_scales_4over6",
    "hscale_refine_scales_strided", "hscale_refine_workspace_bytes", "hscale_refine_scales_ws",
    "hscale_pack_nvfp4", "hscale_fourover6_codes",
    "hscale_dequant_residual", "hscale_output_error_workspace_bytes", "hscale_output_error",
    "residual_ld", "hscale_selftest_bounded_wait", "hscale_hessian_full_workspace_bytes",
    "hscale_hessian_full_accumulate", "hscale_gptq_factor_workspace_bytes", "hscale_gptq_factor",
    "hscale_gptq_workspace_bytes", "hscale_gptq_hscale",
    "HSCALE_CHECKPOINT_INT8", "HSCALE_CHECKPOINT_E4M3", "hscale_checkpoint_save", "hscale_checkpoint_load",
    "hscale_project_workspace_bytes", "hscale_project", "hscale_project_backward_workspace_bytes",
    "hscale_project_backward",
    "HSCALE_ACT_SILU", "HSCALE_ACT_GELU_TANH", "hscale_route", "hscale_route_backward", "hscale_experts_workspace_bytes",
    "hscale_experts", "hscale_experts_backward_workspace_bytes", "hscale_experts_backward", "TensorList", "hscale_tensors",
    "hscale_grad_norm_workspace_bytes", "hscale_grad_norm", "hscale_grad_clip", "EXPORTED_SYMBOLS",
]

_PKG = pathlib.Path(__file__).resolve().parent
_LIB_PATH = _PKG / "_build" / "libhscale.so"
_lock = threading.Lock()
_lib = None

# every entry point of include/hscale.h, with its ctypes signature
_P, _I64, _I32, _SZ = ctypes.c_void_p, ctypes.c_int64, ctypes.c_int32, ctypes.c_size_t
_SIGNATURES = {
    "hscale_status_string": (ctypes.c_char_p, [ctypes.c_int]),
    "hscale_abi_version": (ctypes.c_int, []),
    "hscale_device_error_flags": (ctypes.c_int, [_P]),
    "hscale_selftest_bounded_wait": (ctypes.c_int, [ctypes.c_uint32, _P]),
    "hscale_hessian_diag_accumulate": (ctypes.c_int, [_P, _I64, _I64, _I64, _P, _P]),
    "hscale_hessian_diag_accumulate_ex": (ctypes.c_int, [_P, _I64, _I64, _I64, _P, ctypes.c_uint32, _P]),
    "hscale_hessian_sum_partials": (ctypes.c_int, [_P, _I64, _I64, _I64, _P, _P]),
    "hscale_amax_bits": (ctypes.c_int, [_P, _I64, _I64, _P, _P]),
    "hscale_global_scale_from_amax": (ctypes.c_int, [_P, _P, _P]),
    "hscale_rtn_workspace_bytes": (_SZ, []),
    "hscale_rtn_scales": (ctypes.c_int, [_P, _I64, _I64, _P, _P, _P, _SZ, _P]),
    "hscale_rtn_scales_noalloc": (ctypes.c_int, [_P, _I64, _I64, _P, _P, _P]),
    "hscale_refine_scales": (ctypes.c_int, [_P, _P, _I64, _I64, _P, _P, _I32, _I32, _P, _P, _P]),
    "hscale_refine_scales_ex": (ctypes.c_int, [_P, _P, _I64, _I64, _P, _P, _I32, _I32, _P, _P, _I32, _P]),
    "hscale_refine_scales_4over6": (ctypes.c_int, [_P, _P, _I64, _I64, _P, _I32, _I32, _P, _P, _I32, _P]),
    "hscale_refine_scales_strided": (ctypes.c_int, [_P, _I64, _P, _I64, _I64, _P, _P, _I64, _I32, _I32, _I32,
                                                    _P, _I64, _P, _I64, _I32, _P]),
    "hscale_refine_workspace_bytes": (_SZ, []),
    "hscale_refine_scales_ws": (ctypes.c_int, [_P, _P, _I64, _I64, _P, _P, _I32, _I32, _I32, _P, _P, _I32, _P, _SZ,
                                               _P]),
    "hscale_pack_nvfp4": (ctypes.c_int, [_P, _I64, _I64, _P, _P, _P, _P]),
    "hscale_fourover6_codes": (ctypes.c_int, [_P, _I64, _I64, _P, _P, _P]),
    "hscale_dequant_residual": (ctypes.c_int, [_P, _I64, _I64, _P, _P, _P, _P, _I64, _P]),
    "hscale_output_error_workspace_bytes": (ctypes.c_size_t, [_I64, _I64]),
    "hscale_output_error": (ctypes.c_int, [_P, _I64, _I64, _I64, _P, _I64, _I64, _P, _P, ctypes.c_size_t, _P]),
    "hscale_hessian_full_workspace_bytes": (ctypes.c_size_t, [_I64, _I64]),
    "hscale_hessian_full_accumulate": (ctypes.c_int, [_P, _I64, _I64, _I64, _P, _I64, _P, ctypes.c_size_t, _P]),
    "hscale_gptq_factor_workspace_bytes": (ctypes.c_size_t, [_I64]),
    "hscale_gptq_factor": (ctypes.c_int, [_P, _I64, _I64, ctypes.c_float, _P, _P, _P, _P, ctypes.c_size_t, _P]),
    "hscale_gptq_workspace_bytes": (ctypes.c_size_t, [_I64, _I64, _I32]),
    "hscale_gptq_hscale": (ctypes.c_int, [_P, _I64, _I64, _P, _P, _P, _P, _I32, _I32, _I32, _P, _P, _P,
                                          ctypes.c_size_t, _P]),
    "hscale_checkpoint_save": (ctypes.c_int, [_P, _I64, _I64, _I64, _I32, _P, _I64, _P, _I64, _P]),
    "hscale_checkpoint_load": (ctypes.c_int, [_P, _I64, _P, _I64, _I64, _I64, _I32, _P, _I64, _P]),
    "hscale_project_workspace_bytes": (_SZ, [_I64, _I64, _I64, _I64, _I64]),
    "hscale_project": (ctypes.c_int, [_P, _I64, _I64, _I64, _P, _P, _P, _I64, _P, _P, _P, _I64, _I64, _P, _P, _I64,
                                      _P, _SZ, _P]),
    "hscale_project_backward_workspace_bytes": (_SZ, [_I64, _I64, _I64, _I64, _I64]),
    "hscale_project_backward": (ctypes.c_int, [_P, _I64, _I64, _I64, _P, _I64, _P, _I64, _I32, _I64, _P, _P, _P, _P,
                                               _P, _P, _I64, _I64, _P, _P, _I64, _P, _P, _P, _SZ, _P]),
    "hscale_route": (ctypes.c_int, [_P, _I32, _I64, _I64, _I64, _I64, _I32, _P, _P, _P]),
    "hscale_route_backward": (ctypes.c_int, [_P, _I32, _I64, _I64, _I64, _P, _P, _P, _I64, _I32, _P, _I64, _P]),
    "hscale_experts_workspace_bytes": (_SZ, [_I64, _I64, _I64, _I64, _I64]),
    "hscale_experts": (ctypes.c_int, [_P, _I64, _I64, _I64, _P, _P, _I64, _P, _P, _P, _P, _P, _P, _P, _P, _P, _I64, _I64,
                                      _I32, _P, _I64, _P, _SZ, _P]),
    "hscale_experts_backward_workspace_bytes": (_SZ, [_I64, _I64, _I64, _I64, _I64]),
    "hscale_experts_backward": (ctypes.c_int, [_P, _I64, _I64, _I64, _P, _I64, _P, _P, _I64, _P, _P, _P, _P, _P, _P, _P, _P,
                                               _P, _I64, _I64, _I32, _P, _I64, _P, _P, _SZ, _P]),
    "hscale_grad_norm_workspace_bytes": (_SZ, []),
    "hscale_grad_norm": (ctypes.c_int, [_P, _P, _P, _I64, _P, _P, _SZ, _P]),
    "hscale_grad_clip": (ctypes.c_int, [_P, _P, _P, _I64, ctypes.c_float, _P, _P, _P, _SZ, _P]),
}
EXPORTED_SYMBOLS = tuple(_SIGNATURES)


class HScaleError(RuntimeError):
    def __init__(self, fn: str, status: int):
        super().__init__(f"{fn} failed with status {status}: {hscale_status_string(status)}")
        self.status = status


def library_path() -> pathlib.Path:
    return _LIB_PATH


def load(build_if_missing: bool = False) -> ctypes.CDLL:
    """The loaded CUDA library.  Raises if it has not been built."""
    global _lib
    lib = _lib  # set once, complete: every later call passes without the lock
    if lib is not None:
        return lib
    with _lock:
        if _lib is not None:
            return _lib
        if not _LIB_PATH.exists():
            if not build_if_missing:
                raise ImportError(f"{_LIB_PATH} is missing: build it with "
                                  "`python -c 'import __graft_entry__ as g; g.build()'`")
            from . import build as _build
            _build.build()
        lib = ctypes.CDLL(str(_LIB_PATH))
        for name, (res, args) in _SIGNATURES.items():
            fn = getattr(lib, name)
            fn.restype = res
            fn.argtypes = args
        _lib = lib
        return lib


def hscale_status_string(status: int) -> str:
    return load().hscale_status_string(int(status)).decode()


def hscale_abi_version() -> int:
    return int(load().hscale_abi_version())


def hscale_selftest_bounded_wait(polls: int, stream=None) -> None:
    """Launch the bounded-wait self-test (the wait runs out and sets device flag bit 0)."""
    _check("hscale_selftest_bounded_wait", load().hscale_selftest_bounded_wait(int(polls), _stream_ptr(stream)))


def hscale_device_error_flags() -> int:
    """Synchronise and return (then clear) the device failure flags; 0 = none."""
    v = ctypes.c_uint32(0)
    _check("hscale_device_error_flags", load().hscale_device_error_flags(ctypes.byref(v)))
    return int(v.value)


# the current stream's handle without building a Stream object on every call
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)


def _stream_ptr(stream, device: int | None = None) -> int:
    """device: the current one, where the caller knows it."""
    if stream is None:
        if _raw_stream is not None:
            return _raw_stream(torch.cuda.current_device() if device is None else device)
        stream = torch.cuda.current_stream()
    return int(stream.cuda_stream) if hasattr(stream, "cuda_stream") else int(stream)


def _check(fn: str, status: int) -> None:
    if status != 0:
        raise HScaleError(fn, status)


def _ptr(t: torch.Tensor | None):
    return None if t is None else t.data_ptr()


def _need(t: torch.Tensor, dtype, name: str):
    if not isinstance(t, torch.Tensor) or t.dtype != dtype or not t.is_cuda:
        raise TypeError(f"{name} must be a CUDA tensor of dtype {dtype}")


HSCALE_HESSIAN_X_READY = 1


def hscale_hessian_diag_accumulate(x: torch.Tensor, h: torch.Tensor, stream=None) -> torch.Tensor:
    """h[j] += sum_t x[t, j]^2 for a bf16 chunk x [tokens, n] (row stride >= n)."""
    return hscale_hessian_diag_accumulate_ex(x, h, 0, stream)


def hscale_hessian_diag_accumulate_ex(x: torch.Tensor, h: torch.Tensor, flags: int = 0,
                                      stream=None) -> torch.Tensor:
    """hscale_hessian_diag_accumulate with flags; HSCALE_HESSIAN_X_READY declares that nothing
    still running writes x, so the kernel may overlap the previous kernel on the stream."""
    _need(x, torch.bfloat16, "x")
    _need(h, torch.float32, "h")
    if x.dim() != 2 or x.stride(1) != 1:
        raise ValueError("x must be 2-D with unit column stride")
    tokens, n = x.shape
    if h.numel() != n or not h.is_contiguous():
        raise ValueError("h must be a contiguous float32 vector of length n")
    ld = x.stride(0) if tokens > 1 else n
    _check("hscale_hessian_diag_accumulate_ex",
           load().hscale_hessian_diag_accumulate_ex(_ptr(x), tokens, n, ld, _ptr(h), int(flags),
                                                    _stream_ptr(stream)))
    return h


def hscale_hessian_sum_partials(partials: torch.Tensor, h: torch.Tensor, stream=None) -> torch.Tensor:
    """h = rank-order fp32 sum of the rows of partials [parts, n] (each a rank's partial h)."""
    _need(partials, torch.float32, "partials")
    _need(h, torch.float32, "h")
    if partials.dim() != 2 or partials.stride(1) != 1:
        raise ValueError("partials must be 2-D [parts, n] with unit column stride")
    parts, n = partials.shape
    if h.numel() != n or not h.is_contiguous():
        raise ValueError("h must be a contiguous float32 vector of length n")
    ld = partials.stride(0) if parts > 1 else n
    _check("hscale_hessian_sum_partials",
           load().hscale_hessian_sum_partials(_ptr(partials), parts, n, ld, _ptr(h), _stream_ptr(stream)))
    return h


def hscale_amax_bits(w: torch.Tensor, amax_bits: torch.Tensor, stream=None) -> torch.Tensor:
    """amax_bits (int32 [1], device) = bf16 bit pattern of max|W| (for an all-reduce MAX)."""
    _need(w, torch.bfloat16, "w")
    _need(amax_bits, torch.int32, "amax_bits")
    if not w.is_contiguous() or w.dim() != 2:
        raise ValueError("w must be a contiguous 2-D tensor")
    m, n = w.shape
    _check("hscale_amax_bits", load().hscale_amax_bits(_ptr(w), m, n, _ptr(amax_bits), _stream_ptr(stream)))
    return amax_bits


def hscale_global_scale_from_amax(amax_bits: torch.Tensor, global_scale: torch.Tensor, stream=None) -> None:
    """global_scale[0] = s_g of a matrix whose amax word is amax_bits[0]."""
    _need(amax_bits, torch.int32, "amax_bits")
    _need(global_scale, torch.float32, "global_scale")
    _check("hscale_global_scale_from_amax",
           load().hscale_global_scale_from_amax(_ptr(amax_bits), _ptr(global_scale), _stream_ptr(stream)))


def hscale_rtn_workspace_bytes() -> int:
    return int(load().hscale_rtn_workspace_bytes())


def hscale_rtn_scales(w: torch.Tensor, global_scale: torch.Tensor, codes: torch.Tensor | None,
                      workspace: torch.Tensor, stream=None) -> None:
    """s_g = amax|W| / 2688 into global_scale[0]; RTN codes [m, n/16] into codes."""
    _need(w, torch.bfloat16, "w")
    _need(global_scale, torch.float32, "global_scale")
    if not w.is_contiguous() or w.dim() != 2:
        raise ValueError("w must be a contiguous 2-D tensor")
    m, n = w.shape
    if codes is not None:
        _need(codes, torch.uint8, "codes")
        if codes.numel() != m * (n // 16) or not codes.is_contiguous():
            raise ValueError("codes must be contiguous [m, n/16]")
    if not workspace.is_cuda:
        raise TypeError("workspace must live on the GPU")
    nbytes = workspace.numel() * workspace.element_size()
    _check("hscale_rtn_scales",
           load().hscale_rtn_scales(_ptr(w), m, n, _ptr(global_scale), _ptr(codes),
                                    _ptr(workspace), nbytes, _stream_ptr(stream)))


def hscale_rtn_scales_noalloc(w: torch.Tensor, global_scale: torch.Tensor,
                              codes: torch.Tensor | None, stream=None) -> None:
    """hscale_rtn_scales for callers that cannot allocate: no workspace argument; the
    library's fixed per-GPU scratch array is used instead (calls must not overlap)."""
    _need(w, torch.bfloat16, "w")
    _need(global_scale, torch.float32, "global_scale")
    if not w.is_contiguous() or w.dim() != 2:
        raise ValueError("w must be a contiguous 2-D tensor")
    m, n = w.shape
    if codes is not None:
        _need(codes, torch.uint8, "codes")
        if codes.numel() != m * (n // 16) or not codes.is_contiguous():
            raise ValueError("codes must be contiguous [m, n/16]")
    _check("hscale_rtn_scales_noalloc",
           load().hscale_rtn_scales_noalloc(_ptr(w), m, n, _ptr(global_scale), _ptr(codes),
                                            _stream_ptr(stream)))


def hscale_refine_scales(w: torch.Tensor, h: torch.Tensor | None, global_scale: torch.Tensor,
                         init_codes: torch.Tensor | None, down: int, up: int,
                         codes_out: torch.Tensor, packed_out: torch.Tensor | None,
                         stream=None) -> None:
    """Algorithm 1 over every group of W, with the final re-quantization and packing."""
    hscale_refine_scales_ex(w, h, global_scale, init_codes, down, up, codes_out, packed_out, 0, stream)


def hscale_refine_scales_ex(w: torch.Tensor, h: torch.Tensor | None, global_scale: torch.Tensor,
                            init_codes: torch.Tensor | None, down: int, up: int,
                            codes_out: torch.Tensor, packed_out: torch.Tensor | None,
                            ctas_per_sm: int, stream=None) -> None:
    """hscale_refine_scales with at most ``ctas_per_sm`` resident CTAs per SM (0: all)."""
    _need(w, torch.bfloat16, "w")
    _need(global_scale, torch.float32, "global_scale")
    _need(codes_out, torch.uint8, "codes_out")
    if not w.is_contiguous() or w.dim() != 2:
        raise ValueError("w must be a contiguous 2-D tensor")
    m, n = w.shape
    if h is not None:
        _need(h, torch.float32, "h")
        if h.numel() != n or not h.is_contiguous():
            raise ValueError("h must be a contiguous float32 vector of length n")
    for name, t, size in (("init_codes", init_codes, m * (n // 16)),
                          ("codes_out", codes_out, m * (n // 16)),
                          ("packed_out", packed_out, m * (n // 2))):
        if t is not None:
            _need(t, torch.uint8, name)
            if t.numel() != size or not t.is_contiguous():
                raise ValueError(f"{name} must be contiguous with {size} bytes")
    _check("hscale_refine_scales_ex",
           load().hscale_refine_scales_ex(_ptr(w), _ptr(h), m, n, _ptr(global_scale), _ptr(init_codes),
                                          int(down), int(up), _ptr(codes_out), _ptr(packed_out),
                                          int(ctas_per_sm), _stream_ptr(stream)))


def hscale_refine_workspace_bytes() -> int:
    return int(load().hscale_refine_workspace_bytes())


def hscale_refine_scales_ws(w: torch.Tensor, h: torch.Tensor | None, global_scale: torch.Tensor,
                            init_codes: torch.Tensor | None, fourover6: int, down: int, up: int,
                            codes_out: torch.Tensor, packed_out: torch.Tensor | None, ctas_per_sm: int,
                            workspace: torch.Tensor | None, stream=None) -> None:
    """hscale_refine_scales_ex (fourover6 = 0) or _4over6 (fourover6 = 1) with long searches'
    units shared out at run time through ``workspace`` (a device uint8 tensor of at least
    hscale_refine_workspace_bytes() bytes, or None for the static deal)."""
    _need(w, torch.bfloat16, "w")
    _need(global_scale, torch.float32, "global_scale")
    _need(codes_out, torch.uint8, "codes_out")
    if not w.is_contiguous() or w.dim() != 2:
        raise ValueError("w must be a contiguous 2-D tensor")
    m, n = w.shape
    if h is not None:
        _need(h, torch.float32, "h")
        if h.numel() != n or not h.is_contiguous():
            raise ValueError("h must be a contiguous float32 vector of length n")
    for name, t, size in (("init_codes", init_codes, m * (n // 16)),
                          ("codes_out", codes_out, m * (n // 16)),
                          ("packed_out", packed_out, m * (n // 2))):
        if t is not None:
            _need(t, torch.uint8, name)
            if t.numel() != size or not t.is_contiguous():
                raise ValueError(f"{name} must be contiguous with {size} bytes")
    nbytes = 0
    if workspace is not None:
        _need(workspace, torch.uint8, "workspace")
        nbytes = workspace.numel()
    _check("hscale_refine_scales_ws",
           load().hscale_refine_scales_ws(_ptr(w), _ptr(h), m, n, _ptr(global_scale), _ptr(init_codes),
                                          int(fourover6), int(down), int(up), _ptr(codes_out), _ptr(packed_out),
                                          int(ctas_per_sm), _ptr(workspace), nbytes, _stream_ptr(stream)))


def hscale_refine_scales_4over6(w: torch.Tensor, h: torch.Tensor | None, global_scale: torch.Tensor,
                                down: int, up: int, codes_out: torch.Tensor, packed_out: torch.Tensor | None,
                                ctas_per_sm: int = 0, stream=None) -> None:
    """Algorithm 2 in one pass: 4over6 initial codes decided in the search, then the search."""
    _need(w, torch.bfloat16, "w")
    _need(global_scale, torch.float32, "global_scale")
    _need(codes_out, torch.uint8, "codes_out")
    if not w.is_contiguous() or w.dim() != 2:
        raise ValueError("w must be a contiguous 2-D tensor")
    m, n = w.shape
    if h is not None:
        _need(h, torch.float32, "h")
        if h.numel() != n or not h.is_contiguous():
            raise ValueError("h must be a contiguous float32 vector of length n")
    for name, t, size in (("codes_out", codes_out, m * (n // 16)),
                          ("packed_out", packed_out, m * (n // 2))):
        if t is not None:
            _need(t, torch.uint8, name)
            if t.numel() != size or not t.is_contiguous():
                raise ValueError(f"{name} must be contiguous with {size} bytes")
    _check("hscale_refine_scales_4over6",
           load().hscale_refine_scales_4over6(_ptr(w), _ptr(h), m, n, _ptr(global_scale), int(down), int(up),
                                              _ptr(codes_out), _ptr(packed_out), int(ctas_per_sm),
                                              _stream_ptr(stream)))


def _row_view(t: torch.Tensor, name: str, dtype, rows: int, cols: int) -> int:
    """Row stride (elements) of a 2-D view with unit column stride; checks its shape."""
    _need(t, dtype, name)
    if t.dim() != 2 or tuple(t.shape) != (rows, cols) or (cols > 1 and t.stride(1) != 1):
        raise ValueError(f"{name} must be a [{rows}, {cols}] view with contiguous rows")
    return t.stride(0) if rows > 1 else max(cols, t.stride(0))


def hscale_refine_scales_strided(w: torch.Tensor, h: torch.Tensor | None, global_scale: torch.Tensor,
                                 init_codes: torch.Tensor | None, fourover6: bool, down: int, up: int,
                                 codes_out: torch.Tensor, packed_out: torch.Tensor | None,
                                 ctas_per_sm: int = 0, stream=None) -> None:
    """The search on 2-D views (e.g. ``W[:, c0:c1]``, ``codes[:, c0/16:c1/16]``,
    ``packed[:, c0/2:c1/2]``)."""
    if w.dim() != 2:
        raise ValueError("w must be a 2-D view")
    m, n = w.shape
    ld_w = _row_view(w, "w", torch.bfloat16, m, n)
    _need(global_scale, torch.float32, "global_scale")
    if h is not None:
        _need(h, torch.float32, "h")
        if h.numel() != n or not h.is_contiguous():
            raise ValueError("h must be a contiguous float32 vector of length n")
    ld_c = _row_view(codes_out, "codes_out", torch.uint8, m, n // 16)
    ld_i = 0 if init_codes is None else _row_view(init_codes, "init_codes", torch.uint8, m, n // 16)
    ld_p = 0 if packed_out is None else _row_view(packed_out, "packed_out", torch.uint8, m, n // 2)
    _check("hscale_refine_scales_strided",
           load().hscale_refine_scales_strided(_ptr(w), ld_w, _ptr(h), m, n, _ptr(global_scale), _ptr(init_codes),
                                               ld_i, int(bool(fourover6)), int(down), int(up), _ptr(codes_out), ld_c,
                                               _ptr(packed_out), ld_p, int(ctas_per_sm), _stream_ptr(stream)))


def hscale_pack_nvfp4(w: torch.Tensor, global_scale: torch.Tensor, codes: torch.Tensor,
                      packed_out: torch.Tensor, stream=None) -> None:
    """FP4 nibbles of W under the given codes."""
    _need(w, torch.bfloat16, "w")
    _need(global_scale, torch.float32, "global_scale")
    _need(codes, torch.uint8, "codes")
    _need(packed_out, torch.uint8, "packed_out")
    if not w.is_contiguous() or w.dim() != 2:
        raise ValueError("w must be a contiguous 2-D tensor")
    m, n = w.shape
    if codes.numel() != m * (n // 16) or packed_out.numel() != m * (n // 2):
        raise ValueError("codes must be [m, n/16] and packed_out [m, n/2]")
    _check("hscale_pack_nvfp4",
           load().hscale_pack_nvfp4(_ptr(w), m, n, _ptr(global_scale), _ptr(codes),
                                    _ptr(packed_out), _stream_ptr(stream)))


def hscale_fourover6_codes(w: torch.Tensor, global_scale: torch.Tensor, codes: torch.Tensor,
                           stream=None) -> None:
    """Algorithm 2's 4over6 initial codes [m, n/16] (input to hscale_refine_scales)."""
    _need(w, torch.bfloat16, "w")
    _need(global_scale, torch.float32, "global_scale")
    _need(codes, torch.uint8, "codes")
    if not w.is_contiguous() or w.dim() != 2:
        raise ValueError("w must be a contiguous 2-D tensor")
    m, n = w.shape
    if codes.numel() != m * (n // 16) or not codes.is_contiguous():
        raise ValueError("codes must be contiguous [m, n/16]")
    _check("hscale_fourover6_codes",
           load().hscale_fourover6_codes(_ptr(w), m, n, _ptr(global_scale), _ptr(codes),
                                         _stream_ptr(stream)))


def residual_ld(n: int) -> int:
    """Row length (elements) of the [hi | lo] residual matrix for n input features."""
    return 2 * 64 * ((int(n) + 63) // 64)


def hscale_dequant_residual(w: torch.Tensor, global_scale: torch.Tensor, codes: torch.Tensor,
                            packed: torch.Tensor, dw2: torch.Tensor, stream=None) -> None:
    """dW = W - W_hat of packed NVFP4 weights into dw2 [m, ld] bf16 as [hi | lo] halves."""
    _need(w, torch.bfloat16, "w")
    _need(global_scale, torch.float32, "global_scale")
    _need(codes, torch.uint8, "codes")
    _need(packed, torch.uint8, "packed")
    _need(dw2, torch.bfloat16, "dw2")
    if not w.is_contiguous() or w.dim() != 2:
        raise ValueError("w must be a contiguous 2-D tensor")
    m, n = w.shape
    if codes.numel() != m * (n // 16) or packed.numel() != m * (n // 2):
        raise ValueError("codes must be [m, n/16] and packed [m, n/2]")
    if dw2.dim() != 2 or dw2.shape[0] != m or dw2.stride(1) != 1 or dw2.shape[1] < residual_ld(n):
        raise ValueError("dw2 must be [m, >= residual_ld(n)] with unit column stride")
    _check("hscale_dequant_residual",
           load().hscale_dequant_residual(_ptr(w), m, n, _ptr(global_scale), _ptr(codes), _ptr(packed),
                                          _ptr(dw2), dw2.stride(0), _stream_ptr(stream)))


def hscale_output_error_workspace_bytes(tokens: int, m: int) -> int:
    return int(load().hscale_output_error_workspace_bytes(int(tokens), int(m)))


def hscale_output_error(x: torch.Tensor, dw2: torch.Tensor, m: int, out_sum: torch.Tensor,
                        workspace: torch.Tensor, stream=None) -> None:
    """out_sum (fp64, device) += ||X dW^T||_F^2 for x [tokens, n] (row stride ld_x)."""
    _need(x, torch.bfloat16, "x")
    _need(dw2, torch.bfloat16, "dw2")
    _need(out_sum, torch.float64, "out_sum")
    if x.dim() != 2 or x.stride(1) != 1 or dw2.dim() != 2 or dw2.stride(1) != 1:
        raise ValueError("x and dw2 must be 2-D with unit column stride")
    tokens, n = x.shape
    _check("hscale_output_error",
           load().hscale_output_error(_ptr(x), tokens, n, x.stride(0), _ptr(dw2), dw2.stride(0), int(m),
                                      _ptr(out_sum), _ptr(workspace), workspace.numel() * workspace.element_size(),
                                      _stream_ptr(stream)))


def _workspace(nbytes: int, device, stream) -> torch.Tensor:
    """Scratch memory of a call on `stream`.  It is given back when the call returns, with its kernels still to run: so it
    is that stream's memory, which goes to later work on that stream alone."""
    nbytes = max(int(nbytes), 256)
    if stream is None:
        return torch.empty(nbytes, dtype=torch.uint8, device=device)
    if not isinstance(stream, torch.cuda.Stream):
        handle = _stream_ptr(stream)  # 0 and 1 (cudaStreamLegacy): the default stream
        stream = torch.cuda.default_stream(device) if handle <= 1 else torch.cuda.ExternalStream(handle, device=device)
    with torch.cuda.stream(stream):
        return torch.empty(nbytes, dtype=torch.uint8, device=device)


def hscale_hessian_full_accumulate(x: torch.Tensor, H: torch.Tensor, workspace: torch.Tensor | None = None,
                                   stream=None) -> None:
    """Upper triangle of H (fp32 [n, n]) += X^T X for x [tokens, n] bf16 on the tensor cores.
    A workspace is needed (and allocated here if not given) only for x whose rows are not
    16-byte aligned."""
    _need(x, torch.bfloat16, "x")
    _need(H, torch.float32, "H")
    if x.dim() != 2 or x.stride(1) != 1 or H.dim() != 2 or H.stride(1) != 1:
        raise ValueError("x and H must be 2-D with unit column stride")
    tokens, n = x.shape
    direct = x.data_ptr() % 16 == 0 and x.stride(0) % 8 == 0
    if workspace is None and not direct:
        workspace = _workspace(load().hscale_hessian_full_workspace_bytes(tokens, n), x.device, stream)
    _check("hscale_hessian_full_accumulate",
           load().hscale_hessian_full_accumulate(_ptr(x), tokens, n, x.stride(0), _ptr(H), H.stride(0),
                                                 _ptr(workspace) if workspace is not None else None,
                                                 workspace.numel() if workspace is not None else 0,
                                                 _stream_ptr(stream)))


def hscale_gptq_factor(H: torch.Tensor, damp: float, U: torch.Tensor, dead: torch.Tensor | None,
                       info: torch.Tensor, workspace: torch.Tensor | None = None, stream=None) -> None:
    """U (fp32 [n, n], upper) with U^T U = (H + damp * mean(diag H) I)^-1, as GPTQ forms it."""
    _need(H, torch.float32, "H")
    _need(U, torch.float32, "U")
    _need(info, torch.int32, "info")
    n = H.shape[0]
    if U.shape != (n, n) or not U.is_contiguous() or info.numel() < 3:
        raise ValueError("U must be contiguous [n, n] and info hold 3 int32")
    if dead is not None:
        _need(dead, torch.uint8, "dead")
    if workspace is None:
        nbytes = load().hscale_gptq_factor_workspace_bytes(n)
        if nbytes == 0:
            raise HScaleError("hscale_gptq_factor_workspace_bytes", 5)
        workspace = _workspace(nbytes, H.device, stream)
    _check("hscale_gptq_factor",
           load().hscale_gptq_factor(_ptr(H), n, H.stride(0), float(damp), _ptr(U), _ptr(dead), _ptr(info),
                                     _ptr(workspace), workspace.numel(), _stream_ptr(stream)))


def hscale_gptq_hscale(w: torch.Tensor, U: torch.Tensor, h: torch.Tensor, global_scale: torch.Tensor,
                       dead: torch.Tensor | None, block: int, down: int, up: int, codes_out: torch.Tensor,
                       packed_out: torch.Tensor, workspace: torch.Tensor | None = None, stream=None) -> None:
    """Algorithm 3: GPTQ over blocks of `block` columns with H-Scale as the local quantizer."""
    _need(w, torch.bfloat16, "w")
    for name, t, dt in (("U", U, torch.float32), ("h", h, torch.float32), ("global_scale", global_scale, torch.float32),
                        ("codes_out", codes_out, torch.uint8), ("packed_out", packed_out, torch.uint8)):
        _need(t, dt, name)
    if not w.is_contiguous() or w.dim() != 2:
        raise ValueError("w must be a contiguous 2-D tensor")
    m, n = w.shape
    if workspace is None:
        workspace = _workspace(load().hscale_gptq_workspace_bytes(m, n, block), w.device, stream)
    _check("hscale_gptq_hscale",
           load().hscale_gptq_hscale(_ptr(w), m, n, _ptr(U), _ptr(h), _ptr(global_scale), _ptr(dead), int(block),
                                     int(down), int(up), _ptr(codes_out), _ptr(packed_out), _ptr(workspace),
                                     workspace.numel(), _stream_ptr(stream)))


def hscale_hessian_full_workspace_bytes(tokens: int, n: int) -> int:
    return int(load().hscale_hessian_full_workspace_bytes(int(tokens), int(n)))


def hscale_gptq_factor_workspace_bytes(n: int) -> int:
    return int(load().hscale_gptq_factor_workspace_bytes(int(n)))


def hscale_gptq_workspace_bytes(m: int, n: int, block: int) -> int:
    return int(load().hscale_gptq_workspace_bytes(int(m), int(n), int(block)))


HSCALE_CHECKPOINT_INT8, HSCALE_CHECKPOINT_E4M3 = 0, 1


def _view_ld(t: torch.Tensor, name: str, dtype, rows: int, cols: int) -> int:
    """_row_view for the calls whose cost is latency: the usual case in few steps."""
    if isinstance(t, torch.Tensor) and t.dtype is dtype and t.is_cuda and t.shape == (rows, cols):
        ld, step = t.stride()
        if step == 1 and rows > 1:
            return ld
    return _row_view(t, name, dtype, rows, cols)


def _checkpoint_views(x: torch.Tensor, codes: torch.Tensor, scales: torch.Tensor) -> tuple:
    if not isinstance(x, torch.Tensor) or x.dim() != 2:
        raise ValueError("x must be a 2-D view")
    tokens, n = x.shape
    return (tokens, n, _view_ld(x, "x", torch.bfloat16, tokens, n), _view_ld(codes, "codes", torch.uint8, tokens, n),
            _view_ld(scales, "scales", torch.uint8, tokens, (n + 31) // 32))


def hscale_checkpoint_save(x: torch.Tensor, fmt: int, codes: torch.Tensor, scales: torch.Tensor, stream=None) -> None:
    """Activations x (bf16 [tokens, n]) in 8 bits: codes [tokens, n] and one power-of-two scale byte per
    32 channels, scales [tokens, ceil(n / 32)] (uint8 views with contiguous rows)."""
    tokens, n, ld_x, ld_c, ld_s = _checkpoint_views(x, codes, scales)
    _check("hscale_checkpoint_save",
           load().hscale_checkpoint_save(x.data_ptr(), tokens, n, ld_x, int(fmt), codes.data_ptr(), ld_c,
                                         scales.data_ptr(), ld_s, _stream_ptr(stream)))


def hscale_checkpoint_load(codes: torch.Tensor, scales: torch.Tensor, fmt: int, x: torch.Tensor, stream=None) -> None:
    """x (bf16 [tokens, n]) = the values that a checkpoint stands for."""
    tokens, n, ld_x, ld_c, ld_s = _checkpoint_views(x, codes, scales)
    _check("hscale_checkpoint_load",
           load().hscale_checkpoint_load(codes.data_ptr(), ld_c, scales.data_ptr(), ld_s, tokens, n, int(fmt),
                                         x.data_ptr(), ld_x, _stream_ptr(stream)))


def _whole(t: torch.Tensor, name: str, dtype, shape: tuple) -> None:
    try:
        if t.dtype is dtype and t.is_cuda and t.shape == shape and t.is_contiguous():
            return
    except AttributeError:
        pass
    _need(t, dtype, name)
    raise ValueError(f"{name} must be contiguous {list(shape)}")


def _rows(t: torch.Tensor, name: str) -> tuple:
    """(rows, columns, row stride) of a bf16 [rows, columns] view with contiguous rows.  A single row's stride
    is free: rounded up to the alignment that the library asks for."""
    try:
        if t.dtype is torch.bfloat16 and t.is_cuda:
            rows, cols = t.shape
            ld, step = t.stride()
            if step == 1 or cols <= 1:
                return rows, cols, ld if rows > 1 else (max(cols, ld) + 7) // 8 * 8
    except (AttributeError, ValueError):
        pass
    if not isinstance(t, torch.Tensor) or t.dim() != 2:
        raise ValueError(f"{name} must be a 2-D view")
    _need(t, torch.bfloat16, name)
    raise ValueError(f"{name} must be a 2-D view with contiguous rows")


def _projection(packed, codes, global_scale, a, b, alpha, adapter_of, tokens: int, m: int, n: int):
    """Checks of a packed weight and its adapters; (adapters, rank)."""
    u8, f32, bf16 = torch.uint8, torch.float32, torch.bfloat16
    try:  # the usual case, whose cost a small call feels
        if (n % 16 == 0 and packed.dtype is u8 and codes.dtype is u8 and global_scale.dtype is f32
                and packed.shape == (m, n // 2) and codes.shape == (m, n // 16)
                and packed.is_contiguous() and codes.is_contiguous()
                and packed.is_cuda and codes.is_cuda and global_scale.is_cuda and a is not None):
            adapters, rank, width = a.shape
            if (a.dtype is bf16 and b.dtype is bf16 and alpha.dtype is f32 and width == n
                    and b.shape == (adapters, m, rank) and alpha.shape == (adapters,)
                    and a.is_contiguous() and b.is_contiguous() and alpha.is_contiguous()
                    and a.is_cuda and b.is_cuda and alpha.is_cuda
                    and (adapter_of is None or (adapter_of.dtype is torch.int32 and adapter_of.shape == (tokens,)
                                                and adapter_of.is_contiguous() and adapter_of.is_cuda))):
                return adapters, rank
    except (AttributeError, ValueError):
        pass
    if n % 16 != 0:
        raise ValueError("n must be a multiple of 16")
    _whole(packed, "packed", u8, (m, n // 2))
    _whole(codes, "codes", u8, (m, n // 16))
    _need(global_scale, f32, "global_scale")
    if a is None:
        if b is not None or alpha is not None or adapter_of is not None:
            raise ValueError("a, b, alpha and adapter_of belong together")
        return 0, 0
    _need(a, bf16, "a")
    if a.dim() != 3:
        raise ValueError("a must be [adapters, rank, n]")
    adapters, rank, _ = a.shape
    _whole(a, "a", bf16, (adapters, rank, n))
    _whole(b, "b", bf16, (adapters, m, rank))
    _whole(alpha, "alpha", f32, (adapters,))
    if adapter_of is not None:
        _whole(adapter_of, "adapter_of", torch.int32, (tokens,))
    return adapters, rank


def _project_workspace(workspace, nbytes: int, device, stream):
    if workspace is None and nbytes > 0:
        workspace = _workspace(nbytes, device, stream)
    if workspace is not None:
        _need(workspace, torch.uint8, "workspace")
    return workspace, 0 if workspace is None else workspace.numel()


def hscale_project_workspace_bytes(tokens: int, m: int, n: int, adapters: int, rank: int) -> int:
    return int(load().hscale_project_workspace_bytes(int(tokens), int(m), int(n), int(adapters), int(rank)))


def hscale_project(x: torch.Tensor, packed: torch.Tensor, codes: torch.Tensor, global_scale: torch.Tensor,
                   a: torch.Tensor | None, b: torch.Tensor | None, alpha: torch.Tensor | None,
                   adapter_of: torch.Tensor | None, y: torch.Tensor, workspace: torch.Tensor | None = None,
                   stream=None) -> None:
    """y (bf16 [tokens, m]) = x W_hat^T, plus alpha_a B_a A_a x_t with a = adapter_of[t] (int32 [tokens];
    outside [0, adapters): none; None: adapter 0 for every token).  a [adapters, rank, n] and
    b [adapters, m, rank] are bf16, alpha fp32 [adapters]; a, b, alpha None: no adapters."""
    tokens, n, ld_x = _rows(x, "x")
    y_rows, m, ld_y = _rows(y, "y")
    if y_rows != tokens:
        raise ValueError("x and y must have the same number of rows")
    adapters, rank = _projection(packed, codes, global_scale, a, b, alpha, adapter_of, tokens, m, n)
    lib = _lib or load()
    if workspace is None:
        nbytes = lib.hscale_project_workspace_bytes(tokens, m, n, adapters, rank)
        workspace = _workspace(nbytes, x.device, stream) if nbytes else None
    nbytes = 0
    if workspace is not None:
        _need(workspace, torch.uint8, "workspace")
        nbytes = workspace.numel()
    status = lib.hscale_project(
        x.data_ptr(), tokens, n, ld_x, packed.data_ptr(), codes.data_ptr(), global_scale.data_ptr(), m,
        None if a is None else a.data_ptr(), None if b is None else b.data_ptr(),
        None if alpha is None else alpha.data_ptr(), adapters, rank,
        None if adapter_of is None else adapter_of.data_ptr(), y.data_ptr(), ld_y,
        None if workspace is None else workspace.data_ptr(), nbytes, _stream_ptr(stream))
    if status:
        raise HScaleError("hscale_project", status)


def hscale_project_backward_workspace_bytes(tokens: int, m: int, n: int, adapters: int, rank: int) -> int:
    return int(load().hscale_project_backward_workspace_bytes(int(tokens), int(m), int(n), int(adapters), int(rank)))


def hscale_project_backward(dy: torch.Tensor, x_codes: torch.Tensor | None, x_scales: torch.Tensor | None,
                            x_format: int, packed: torch.Tensor, codes: torch.Tensor, global_scale: torch.Tensor,
                            a: torch.Tensor | None, b: torch.Tensor | None, alpha: torch.Tensor | None,
                            adapter_of: torch.Tensor | None, dx: torch.Tensor | None, da: torch.Tensor | None,
                            db: torch.Tensor | None, workspace: torch.Tensor | None = None, stream=None) -> None:
    """The gradients of hscale_project for dy (bf16 [tokens, m]) at the x of a checkpoint (x_codes, x_scales,
    x_format): dx (bf16 [tokens, n]), da and db (bf16, shaped like a and b); each may be None."""
    tokens, m, ld_dy = _rows(dy, "dy")
    _need(packed, torch.uint8, "packed")
    if packed.dim() != 2:
        raise ValueError("packed must be [m, n/2]")
    n = 2 * packed.shape[1]
    ld_dx = n
    if dx is not None:
        dx_rows, dx_cols, ld_dx = _rows(dx, "dx")
        if (dx_rows, dx_cols) != (tokens, n):
            raise ValueError(f"dx must be a [{tokens}, {n}] view")
    adapters, rank = _projection(packed, codes, global_scale, a, b, alpha, adapter_of, tokens, m, n)
    if adapters == 0 and (da is not None or db is not None):
        if a is None:
            raise ValueError("da and db need adapters")
    if da is not None:
        _whole(da, "da", torch.bfloat16, (adapters, rank, n))
    if db is not None:
        _whole(db, "db", torch.bfloat16, (adapters, m, rank))
    ld_c = ld_s = 0
    if adapters > 0 and (da is not None or db is not None):
        ld_c = _view_ld(x_codes, "x_codes", torch.uint8, tokens, n)
        ld_s = _view_ld(x_scales, "x_scales", torch.uint8, tokens, (n + 31) // 32)
    lib = load()
    workspace, nbytes = _project_workspace(
        workspace, lib.hscale_project_backward_workspace_bytes(tokens, m, n, adapters, rank)
        if workspace is None else 0, dy.device, stream)
    _check("hscale_project_backward",
           lib.hscale_project_backward(dy.data_ptr(), tokens, m, ld_dy, _ptr(x_codes), ld_c, _ptr(x_scales), ld_s,
                                       int(x_format), n, packed.data_ptr(), codes.data_ptr(),
                                       global_scale.data_ptr(), _ptr(a), _ptr(b), _ptr(alpha), adapters, rank,
                                       _ptr(adapter_of), _ptr(dx), ld_dx, _ptr(da), _ptr(db), _ptr(workspace),
                                       nbytes, _stream_ptr(stream)))


# ---------------------------------------------------------------- mixtures of experts
HSCALE_ACT_SILU, HSCALE_ACT_GELU_TANH = 0, 1
_TYPES = {torch.bfloat16: 0, torch.float32: 1, torch.float16: 2}


def _here(t: torch.Tensor, name: str) -> int:
    """The current device, which t is on."""
    device = torch.cuda.current_device()
    if t.get_device() != device:
        raise ValueError(f"{name} must be on the current device")
    return device


def _beside(device: int, *others) -> None:
    """The other tensors of a call (None: not given) are on the device too."""
    for t in others:
        if t is not None and t.get_device() != device:
            raise ValueError("the tensors of a call must be on one device, the current one")


def _logits(t: torch.Tensor, name: str) -> tuple:
    """(tokens, experts, row stride, type, device) of a bf16 or fp32 [tokens, experts] view with contiguous rows."""
    if not isinstance(t, torch.Tensor) or t.dim() != 2:
        raise ValueError(f"{name} must be a 2-D view")
    if t.dtype not in (torch.bfloat16, torch.float32) or not t.is_cuda:
        raise TypeError(f"{name} must be a CUDA tensor of dtype torch.bfloat16 or torch.float32")
    tokens, experts = t.shape
    if experts > 1 and t.stride(1) != 1:
        raise ValueError(f"{name} must be a 2-D view with contiguous rows")
    device = _here(t, name)
    return tokens, experts, t.stride(0) if tokens > 1 else max(experts, t.stride(0)), _TYPES[t.dtype], device


def _routing(ids: torch.Tensor, weights: torch.Tensor, tokens: int) -> int:
    """k of ids (int32) and weights (fp32) [tokens, k]."""
    if not isinstance(ids, torch.Tensor) or ids.dim() != 2:
        raise ValueError("ids must be [tokens, k]")
    k = ids.shape[1]
    _whole(ids, "ids", torch.int32, (tokens, k))
    _whole(weights, "weights", torch.float32, (tokens, k))
    return k


def hscale_route(logits: torch.Tensor, ids: torch.Tensor, weights: torch.Tensor, renormalize: bool, stream=None) -> None:
    """The k largest of each token's logits (bf16 or fp32 [tokens, experts]), ties to the lowest index: ids (int32
    [tokens, k]) and weights (fp32 [tokens, k]), softmax(logits) there, or that divided by its sum over the chosen
    ones (renormalize).  -Inf and NaN are experts that are off; where too few are on, ids are -1 and weights 0."""
    tokens, experts, ld, kind, device = _logits(logits, "logits")
    k = _routing(ids, weights, tokens)
    _beside(device, ids, weights)
    _check("hscale_route",
           (_lib or load()).hscale_route(logits.data_ptr(), kind, tokens, experts, ld, k, int(bool(renormalize)), ids.data_ptr(),
                                         weights.data_ptr(), _stream_ptr(stream, device)))


def hscale_route_backward(logits: torch.Tensor | None, ids: torch.Tensor, weights: torch.Tensor, dweights: torch.Tensor,
                          renormalize: bool, dlogits: torch.Tensor, stream=None) -> None:
    """dlogits (like logits) of dweights (fp32 [tokens, k]), with the ids and weights that hscale_route gave.  logits may
    be None where the weights are renormalized."""
    tokens, experts, ld_out, kind, device = _logits(dlogits, "dlogits")
    ld = experts
    if logits is not None:
        rows, cols, ld, logits_kind, _ = _logits(logits, "logits")
        if (rows, cols, logits_kind) != (tokens, experts, kind):
            raise ValueError("logits and dlogits must have the same shape and dtype")
    elif not renormalize:
        raise ValueError("logits are needed where the weights are not renormalized")
    k = _routing(ids, weights, tokens)
    _whole(dweights, "dweights", torch.float32, (tokens, k))
    _beside(device, ids, weights, dweights)
    _check("hscale_route_backward",
           (_lib or load()).hscale_route_backward(_ptr(logits), kind, tokens, experts, ld, ids.data_ptr(), weights.data_ptr(),
                                                  dweights.data_ptr(), k, int(bool(renormalize)), dlogits.data_ptr(), ld_out,
                                                  _stream_ptr(stream, device)))


def _expert_matrices(gate: tuple, up: tuple, down: tuple, n: int) -> tuple:
    """Checks of (packed, codes, scale) of each matrix; (experts, inner, the nine pointers)."""
    u8, f32 = torch.uint8, torch.float32
    packed = gate[0]
    if not isinstance(packed, torch.Tensor) or packed.dim() != 3:
        raise ValueError("gate's packed weight must be [experts, inner, n/2]")
    experts, inner, _ = packed.shape
    if n % 16 != 0 or inner % 16 != 0:
        raise ValueError("n and inner must be multiples of 16")
    pointers = []
    for name, (p, c, s), rows, cols in (("gate", gate, inner, n), ("up", up, inner, n), ("down", down, n, inner)):
        _whole(p, name + "'s packed weight", u8, (experts, rows, cols // 2))
        _whole(c, name + "'s codes", u8, (experts, rows, cols // 16))
        _whole(s, name + "'s scale", f32, (experts,))
        pointers += [p.data_ptr(), c.data_ptr(), s.data_ptr()]
    return experts, inner, pointers


def hscale_experts_workspace_bytes(tokens: int, k: int, n: int, inner: int, experts: int) -> int:
    return int(load().hscale_experts_workspace_bytes(int(tokens), int(k), int(n), int(inner), int(experts)))


def hscale_experts(x: torch.Tensor, ids: torch.Tensor, weights: torch.Tensor, gate: tuple, up: tuple, down: tuple,
                   activation: int, y: torch.Tensor, workspace: torch.Tensor | None = None, stream=None) -> None:
    """y_t (bf16 [tokens, n]) = sum_j weights[t, j] D (act(G x_t) * (U x_t)) of expert ids[t, j] (int32 [tokens, k]; outside
    [0, experts): none).  gate, up and down are (packed, codes, scale) of G, U [experts, inner, n] and D [experts, n,
    inner]: packed uint8 [experts, rows, cols/2], codes uint8 [experts, rows, cols/16], scale fp32 [experts]."""
    tokens, n, ld_x = _rows(x, "x")
    y_rows, y_cols, ld_y = _rows(y, "y")
    if (y_rows, y_cols) != (tokens, n):
        raise ValueError("x and y must have the same shape")
    device = _here(x, "x")
    k = _routing(ids, weights, tokens)
    experts, inner, pointers = _expert_matrices(gate, up, down, n)
    lib = _lib or load()
    workspace, nbytes = _project_workspace(
        workspace, lib.hscale_experts_workspace_bytes(tokens, k, n, inner, experts) if workspace is None else 0, x.device, stream)
    _beside(device, y, ids, weights, *gate, *up, *down, workspace)
    _check("hscale_experts",
           lib.hscale_experts(x.data_ptr(), tokens, n, ld_x, ids.data_ptr(), weights.data_ptr(), k, *pointers, experts, inner,
                              int(activation), y.data_ptr(), ld_y, _ptr(workspace), nbytes, _stream_ptr(stream, device)))


def hscale_experts_backward_workspace_bytes(tokens: int, k: int, n: int, inner: int, experts: int) -> int:
    return int(load().hscale_experts_backward_workspace_bytes(int(tokens), int(k), int(n), int(inner), int(experts)))


def hscale_experts_backward(dy: torch.Tensor, x: torch.Tensor, ids: torch.Tensor, weights: torch.Tensor, gate: tuple,
                            up: tuple, down: tuple, activation: int, dx: torch.Tensor | None,
                            dweights: torch.Tensor | None, workspace: torch.Tensor | None = None, stream=None) -> None:
    """The gradients of hscale_experts for dy (bf16 [tokens, n]): dx (bf16 [tokens, n]) and dweights (fp32 [tokens, k]); each
    may be None."""
    tokens, n, ld_dy = _rows(dy, "dy")
    x_rows, x_cols, ld_x = _rows(x, "x")
    if (x_rows, x_cols) != (tokens, n):
        raise ValueError("x and dy must have the same shape")
    ld_dx = n
    if dx is not None:
        dx_rows, dx_cols, ld_dx = _rows(dx, "dx")
        if (dx_rows, dx_cols) != (tokens, n):
            raise ValueError(f"dx must be a [{tokens}, {n}] view")
    device = _here(dy, "dy")
    k = _routing(ids, weights, tokens)
    if dweights is not None:
        _whole(dweights, "dweights", torch.float32, (tokens, k))
    experts, inner, pointers = _expert_matrices(gate, up, down, n)
    lib = _lib or load()
    workspace, nbytes = _project_workspace(
        workspace, lib.hscale_experts_backward_workspace_bytes(tokens, k, n, inner, experts) if workspace is None else 0,
        dy.device, stream)
    _beside(device, x, ids, weights, *gate, *up, *down, dx, dweights, workspace)
    _check("hscale_experts_backward",
           lib.hscale_experts_backward(dy.data_ptr(), tokens, n, ld_dy, x.data_ptr(), ld_x, ids.data_ptr(), weights.data_ptr(), k,
                                       *pointers, experts, inner, int(activation), _ptr(dx), ld_dx, _ptr(dweights),
                                       _ptr(workspace), nbytes, _stream_ptr(stream, device)))


# ---------------------------------------------------------------- gradients
class TensorList:
    """Tensors of a call that takes many, checked once: a program that keeps its gradients' memory keeps this beside
    them.  It holds the tensors; whoever moves one (``.data``, ``set_``) makes a new list."""

    def __init__(self, tensors):
        self.tensors = tuple(tensors)
        for t in self.tensors:
            if not isinstance(t, torch.Tensor) or t.dtype not in _TYPES or not t.is_cuda:
                raise TypeError("tensors must be CUDA tensors of dtype bfloat16, float16 or float32")
            if not t.is_contiguous():
                raise ValueError("tensors must be contiguous")
        count = len(self.tensors)
        self.device = self.tensors[0].get_device() if count else None
        if any(t.get_device() != self.device for t in self.tensors):
            raise ValueError("tensors must be on one device")
        pointers, sizes = [t.data_ptr() for t in self.tensors], [t.numel() for t in self.tensors]
        self.pointers = (ctypes.c_void_p * count)(*pointers)
        self.sizes = (ctypes.c_int64 * count)(*sizes)
        self.types = (ctypes.c_int32 * count)(*[_TYPES[t.dtype] for t in self.tensors])
        self.shape = tuple(zip(sizes, self.types))
        spans = sorted((p, p + s * t.element_size()) for p, s, t in zip(pointers, sizes, self.tensors) if s)
        self.disjoint = all(a[1] <= b[0] for a, b in zip(spans, spans[1:]))

    def __len__(self):
        return len(self.tensors)


def hscale_tensors(tensors) -> TensorList:
    """The tensors (or a TensorList) as a TensorList."""
    return tensors if isinstance(tensors, TensorList) else TensorList(tensors)


def _grad_arguments(tensors, norm, workspace, stream) -> tuple:
    tensors = hscale_tensors(tensors)
    _need(norm, torch.float32, "norm")
    if norm.numel() < 1:
        raise ValueError("norm must hold one float32")
    device = _here(norm, "norm")
    if len(tensors) and tensors.device != device:
        raise ValueError("tensors and norm must be on one device")
    lib = _lib or load()
    workspace, nbytes = _project_workspace(workspace, lib.hscale_grad_norm_workspace_bytes() if workspace is None else 0,
                                           norm.device, stream)
    _beside(device, workspace)
    return lib, tensors, workspace, nbytes, device


def hscale_grad_norm_workspace_bytes() -> int:
    return int(load().hscale_grad_norm_workspace_bytes())


def hscale_grad_norm(tensors, norm: torch.Tensor, workspace: torch.Tensor | None = None, stream=None) -> None:
    """norm (fp32 [1]) = the 2-norm over all elements of the tensors (bf16, fp16 and fp32; a list or a TensorList)."""
    lib, tensors, workspace, nbytes, device = _grad_arguments(tensors, norm, workspace, stream)
    _check("hscale_grad_norm", lib.hscale_grad_norm(tensors.pointers, tensors.sizes, tensors.types, len(tensors),
                                                    norm.data_ptr(), _ptr(workspace), nbytes, _stream_ptr(stream, device)))


def hscale_grad_clip(tensors, max_norm: float, norm: torch.Tensor, out=None, workspace: torch.Tensor | None = None,
                     stream=None) -> None:
    """norm as hscale_grad_norm, and out_i = tensors_i * min(1, max_norm / norm) (out None: in place).  What is written
    overlaps no other tensor (out_i may be tensors_i).  Where the norm is not finite nothing is scaled."""
    lib, tensors, workspace, nbytes, device = _grad_arguments(tensors, norm, workspace, stream)
    into = tensors if out is None else hscale_tensors(out)
    if into.shape != tensors.shape or into.device != tensors.device:
        raise ValueError("out must have the tensors' sizes, dtypes and device")
    if not into.disjoint:
        raise ValueError("tensors that are written must not overlap")
    _check("hscale_grad_clip", lib.hscale_grad_clip(tensors.pointers, tensors.sizes, tensors.types, len(tensors),
                                                    float(max_norm), norm.data_ptr(), None if out is None else into.pointers,
                                                    _ptr(workspace), nbytes, _stream_ptr(stream, device)))
