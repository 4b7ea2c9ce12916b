"""ctypes binding of libmsda (argument marshalling only).

The functions mirror the C ABI in ``include/msda.h`` and take torch tensors for device memory:
every step of the computation runs in the library's HIP kernels. There is no fallback: if
``libmsda.so`` has not been built, or the GPU is missing, the calls raise.
"""
from __future__ import annotations

import contextlib
import ctypes
import os
from typing import Optional, Sequence, Tuple

import numpy as np

_PKG = os.path.dirname(os.path.abspath(__file__))
# MSDA_LIBRARY names another build of the same library (the ablation builds of microbench/ablation.py)
LIB_PATH = os.environ.get("MSDA_LIBRARY") or os.path.join(_PKG, "_lib", "libmsda.so")

MSDA_SUCCESS = 0
MSDA_ERROR_INVALID_VALUE = 1
MSDA_ERROR_NOT_SUPPORTED = 2
MSDA_ERROR_LAUNCH_FAILED = 3
MSDA_F32 = 0
MSDA_F16 = 1
MSDA_BF16 = 2
MSDA_MAX_LEVELS = 16
MSDA_LAYERNORM_MAX_C = 16384
MSDA_ROTARY_MAX_D = 1024
MSDA_ATTENTION_MAX_D = 128
MSDA_QUANTIZED_MAX_K = 131071
MSDA_CACHE_MAX_D = 128
MSDA_WORKSPACE_PREFERRED = 0
MSDA_WORKSPACE_OWNER = 1
MSDA_WORKSPACE_DETERMINISTIC = 2

EXPORTED = ["msda_check_args", "msda_forward", "msda_backward", "msda_backward_atomic",
            "msda_backward_deterministic", "msda_backward_workspace_size",
            "msda_forward_fused", "msda_backward_fused_workspace_size", "msda_backward_fused",
            "msda_status_string", "msda_last_error", "msda_version", "msda_release", "msda_backward_noalloc",
            "msda_layernorm_forward", "msda_layernorm_backward", "msda_layernorm_backward_workspace_size",
            "msda_rotary_forward", "msda_rotary_backward",
            "msda_attention_forward", "msda_attention_backward", "msda_attention_workspace_size",
            "msda_rmsnorm_forward", "msda_rmsnorm_quantize", "msda_rmsnorm_backward", "msda_rmsnorm_backward_workspace_size",
            "msda_quantize_rows", "msda_quantized_matmul", "msda_cache_append", "msda_cache_attention",
            "msda_cache_attention_workspace_size"]
MSDA_NOALLOC_SCRATCH_BYTES = 128 << 20


class MsdaError(RuntimeError):
    def __init__(self, status: int, where: str, detail: str):
        self.status = status
        super().__init__(f"{where}: {status_string(status)}: {detail}")


class AttentionDescription(ctypes.Structure):
    """msda_attention_t."""
    _fields_ = [(name, ctypes.c_int64) for name in ("N", "Lq", "Lk", "M", "Mkv", "D")] + \
        [("dtype", ctypes.c_int), ("causal", ctypes.c_int), ("unaligned", ctypes.c_int), ("scale", ctypes.c_float), ("softcap", ctypes.c_float)] + \
        [(name, ctypes.c_int64 * 3) for name in ("q_stride", "k_stride", "v_stride")] + \
        [(name, ctypes.c_void_p) for name in ("slopes", "q_pos", "k_pos", "q_doc", "k_doc", "prefix")]


class CacheDescription(ctypes.Structure):
    """msda_cache_t."""
    _fields_ = [(name, ctypes.c_int64) for name in ("N", "pages", "page_size", "Mkv", "D", "width", "table_stride")] + \
        [(name, ctypes.c_void_p) for name in ("k", "v", "k_scale", "v_scale", "table", "length", "start")]


_lib = None


def lib():
    """The loaded libmsda (raises if it has not been built)."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(f"{LIB_PATH} is missing: build it with `python -m paper_2505_14022_amd.build`")
        L = ctypes.CDLL(LIB_PATH)
        i64, vp, ip = ctypes.c_int64, ctypes.c_void_p, ctypes.POINTER(ctypes.c_int64)
        L.msda_check_args.argtypes = [ip, ip] + [i64] * 7 + [ctypes.c_int]
        L.msda_check_args.restype = ctypes.c_int
        L.msda_forward.argtypes = [vp, ip, ip, vp, vp, vp] + [i64] * 7 + [ctypes.c_int, vp]
        L.msda_forward.restype = ctypes.c_int
        L.msda_backward.argtypes = [vp, ip, ip, vp, vp, vp, vp, vp, vp, vp, ctypes.c_size_t] + [i64] * 7 + \
            [ctypes.c_int, vp]
        L.msda_backward.restype = ctypes.c_int
        L.msda_backward_atomic.argtypes = [vp, ip, ip, vp, vp, vp, vp, vp, vp] + [i64] * 7 + [ctypes.c_int, vp]
        L.msda_backward_atomic.restype = ctypes.c_int
        L.msda_backward_noalloc.argtypes = L.msda_backward_atomic.argtypes
        L.msda_backward_noalloc.restype = ctypes.c_int
        L.msda_backward_deterministic.argtypes = L.msda_backward.argtypes
        L.msda_backward_deterministic.restype = ctypes.c_int
        L.msda_backward_workspace_size.argtypes = [ip, ip] + [i64] * 7 + [ctypes.c_int, ctypes.c_int,
                                                                         ctypes.POINTER(ctypes.c_size_t)]
        L.msda_backward_workspace_size.restype = ctypes.c_int
        L.msda_forward_fused.argtypes = [vp, ip, ip, vp, vp, vp, vp] + [i64] * 7 + [ctypes.c_int, vp]
        L.msda_forward_fused.restype = ctypes.c_int
        L.msda_backward_fused_workspace_size.argtypes = L.msda_backward_workspace_size.argtypes
        L.msda_backward_fused_workspace_size.restype = ctypes.c_int
        L.msda_backward_fused.argtypes = [vp, ip, ip] + [vp] * 9 + [ctypes.c_size_t] + [i64] * 7 + \
            [ctypes.c_int, vp]
        L.msda_backward_fused.restype = ctypes.c_int
        L.msda_status_string.argtypes = [ctypes.c_int]
        L.msda_status_string.restype = ctypes.c_char_p
        L.msda_last_error.argtypes = []
        L.msda_last_error.restype = ctypes.c_char_p
        L.msda_version.argtypes = []
        L.msda_version.restype = ctypes.c_int
        L.msda_release.argtypes = []
        L.msda_release.restype = ctypes.c_int
        f32, size, sizep = ctypes.c_float, ctypes.c_size_t, ctypes.POINTER(ctypes.c_size_t)
        L.msda_layernorm_forward.argtypes = [vp] * 8 + [i64, i64, f32, ctypes.c_int, vp]
        L.msda_layernorm_forward.restype = ctypes.c_int
        L.msda_layernorm_backward_workspace_size.argtypes = [i64, i64, ctypes.c_int, sizep]
        L.msda_layernorm_backward_workspace_size.restype = ctypes.c_int
        L.msda_layernorm_backward.argtypes = [vp] * 11 + [size, i64, i64, ctypes.c_int, vp]
        L.msda_layernorm_backward.restype = ctypes.c_int
        L.msda_rotary_forward.argtypes = [vp, ip, vp, vp, vp, ip] + [i64] * 7 + [ctypes.c_int, ctypes.c_int, vp]
        L.msda_rotary_forward.restype = ctypes.c_int
        L.msda_rotary_backward.argtypes = L.msda_rotary_forward.argtypes
        L.msda_rotary_backward.restype = ctypes.c_int
        desc = ctypes.POINTER(AttentionDescription)
        L.msda_attention_workspace_size.argtypes = [desc, ctypes.c_int, sizep]
        L.msda_attention_workspace_size.restype = ctypes.c_int
        L.msda_attention_forward.argtypes = [desc] + [vp] * 6 + [size, vp]
        L.msda_attention_forward.restype = ctypes.c_int
        L.msda_attention_backward.argtypes = [desc] + [vp] * 10 + [size, vp]
        L.msda_attention_backward.restype = ctypes.c_int
        L.msda_rmsnorm_forward.argtypes = [vp] * 6 + [i64, i64, f32, ctypes.c_int, vp]
        L.msda_rmsnorm_quantize.argtypes = [vp] * 6 + [i64, i64, f32, ctypes.c_int, vp]
        L.msda_rmsnorm_backward_workspace_size.argtypes = [i64, i64, ctypes.c_int, sizep]
        L.msda_rmsnorm_backward.argtypes = [vp] * 9 + [size, i64, i64, ctypes.c_int, vp]
        L.msda_quantize_rows.argtypes = [vp] * 3 + [i64, i64, ctypes.c_int, vp]
        L.msda_quantized_matmul.argtypes = [vp] * 6 + [i64, i64, i64, ctypes.c_int, vp]
        cache = ctypes.POINTER(CacheDescription)
        L.msda_cache_append.argtypes = [cache, vp, ip, vp, ip, vp, vp, i64, i64, i64, ctypes.c_int, ctypes.c_int, vp]
        L.msda_cache_attention_workspace_size.argtypes = [cache, i64, i64, ctypes.c_int, sizep]
        L.msda_cache_attention.argtypes = [cache, vp, ip, vp, vp, i64, i64, f32, f32, ctypes.c_int, ctypes.c_int, vp, size, vp]
        for name in EXPORTED[-9:]:
            getattr(L, name).restype = ctypes.c_int
        _lib = L
    return _lib


def status_string(status: int) -> str:
    return lib().msda_status_string(int(status)).decode()


def last_error() -> str:
    return lib().msda_last_error().decode()


def release():
    """msda_release: destroy the library's side streams and events (after their work is done)."""
    _raise(lib().msda_release(), "msda_release")


def _host_tables(spatial_shapes, level_start_index) -> Tuple[np.ndarray, np.ndarray]:
    def to_np(x):
        if type(x) is np.ndarray and x.dtype == np.int64 and x.flags.c_contiguous:
            return x
        if hasattr(x, "detach"):
            x = x.detach().cpu().numpy()
        return np.ascontiguousarray(np.asarray(x), dtype=np.int64)

    return to_np(spatial_shapes).reshape(-1), to_np(level_start_index).reshape(-1)


_I64P = ctypes.POINTER(ctypes.c_int64)


def _iptr(a: np.ndarray):
    return ctypes.cast(a.__array_interface__["data"][0], _I64P) if a.size else a.ctypes.data_as(_I64P)


def _dptr(t) -> Optional[int]:
    if t is None:
        return None
    if not t.is_cuda:
        raise ValueError("tensor arguments must be device tensors")
    if not t.is_contiguous():
        raise ValueError("tensor arguments must be contiguous")
    return t.data_ptr()


def _stream(stream) -> Optional[int]:
    if stream is None:
        import torch

        return torch.cuda.current_stream().cuda_stream
    return int(getattr(stream, "cuda_stream", stream))


_NO_CONTEXT = contextlib.nullcontext()


def _on(stream):
    """A context under which torch allocates memory for use on `stream` (torch's current stream when
    it is None). Outputs and workspaces the binding allocates are used by the kernels enqueued on
    `stream`: allocated under another stream, the caching allocator could hand their memory to a
    later allocation on that stream as soon as the binding returns, while the kernels still run."""
    import torch

    if stream is None:
        return _NO_CONTEXT  # torch allocates under its current stream anyway (entering it anew costs 7 us)
    if isinstance(stream, torch.cuda.Stream):
        return torch.cuda.stream(stream)
    return torch.cuda.stream(torch.cuda.ExternalStream(_stream(stream)))


def _dtype_code(t) -> int:
    import torch

    if t.dtype == torch.float32:
        return MSDA_F32
    if t.dtype == torch.float16:
        return MSDA_F16
    raise ValueError(f"value dtype must be float32 or float16, got {t.dtype}")


def _raise(st: int, where: str):
    if st != MSDA_SUCCESS:
        raise MsdaError(st, where, last_error())


def check_args(spatial_shapes, level_start_index, N, S, M, D, Lq, L, P, dtype) -> int:
    """msda_check_args: returns the status code (host-only, needs no GPU)."""
    sh, st = _host_tables(spatial_shapes, level_start_index)
    return lib().msda_check_args(_iptr(sh) if sh.size else None, _iptr(st) if st.size else None,
                                 N, S, M, D, Lq, L, P, int(dtype))


def _dims(value, sampling_loc):
    N, S, M, D = value.shape
    _, Lq, M2, L, P, two = sampling_loc.shape
    if M2 != M or two != 2:
        raise ValueError(f"sampling_loc shape {tuple(sampling_loc.shape)} does not match value {tuple(value.shape)}")
    return N, S, M, D, Lq, L, P


def workspace_size(spatial_shapes, level_start_index, N, S, M, D, Lq, L, P, dtype,
                   mode: int = MSDA_WORKSPACE_PREFERRED) -> int:
    """msda_backward_workspace_size: bytes of device workspace for the owner-computes grad_value
    (MSDA_WORKSPACE_PREFERRED: 0 where the library prefers atomics; MSDA_WORKSPACE_OWNER: the
    owner-computes size wherever that path applies)."""
    sh, st = _host_tables(spatial_shapes, level_start_index)
    out = ctypes.c_size_t(0)
    r = lib().msda_backward_workspace_size(_iptr(sh), _iptr(st), N, S, M, D, Lq, L, P, int(dtype), int(mode),
                                           ctypes.byref(out))
    _raise(r, "msda_backward_workspace_size")
    return int(out.value)


def forward(value, spatial_shapes, level_start_index, sampling_loc, attn_weight, out=None, stream=None):
    """out[N, Lq, M*D] = MSDA(value, sampling_loc, attn_weight), computed by msda_forward."""
    import torch

    N, S, M, D, Lq, L, P = _dims(value, sampling_loc)
    if out is None:
        with _on(stream):
            out = torch.empty((N, Lq, M * D), dtype=value.dtype, device=value.device)
    sh, st = _host_tables(spatial_shapes, level_start_index)
    r = lib().msda_forward(_dptr(value), _iptr(sh), _iptr(st), _dptr(sampling_loc), _dptr(attn_weight),
                           _dptr(out), N, S, M, D, Lq, L, P, _dtype_code(value), _stream(stream))
    _raise(r, "msda_forward")
    return out


def backward(value, spatial_shapes, level_start_index, sampling_loc, attn_weight, grad_out,
             grad_value=None, grad_loc=None, grad_attn=None, workspace="auto", stream=None):
    """(grad_value fp32, grad_loc, grad_attn) from msda_backward.

    workspace: "auto" allocates the workspace the library prefers for this problem (none where
    atomics are faster), "owner" the owner-computes workspace wherever that path applies, or a
    caller-owned uint8 device tensor; None calls msda_backward_atomic (grad_value by fp32 atomics,
    no workspace).
    """
    import torch

    N, S, M, D, Lq, L, P = _dims(value, sampling_loc)
    dev = value.device
    sh, st = _host_tables(spatial_shapes, level_start_index)
    with _on(stream):
        if grad_value is None:
            grad_value = torch.empty((N, S, M, D), dtype=torch.float32, device=dev)
        if grad_loc is None:
            grad_loc = torch.empty(tuple(sampling_loc.shape), dtype=torch.float32, device=dev)
        if grad_attn is None:
            grad_attn = torch.empty(tuple(attn_weight.shape), dtype=torch.float32, device=dev)
        atomic = workspace is None
        if isinstance(workspace, str):
            if workspace not in ("auto", "owner"):
                raise ValueError(f"workspace must be 'auto', 'owner', None or a tensor, not {workspace!r}")
            mode = MSDA_WORKSPACE_PREFERRED if workspace == "auto" else MSDA_WORKSPACE_OWNER
            nbytes = workspace_size(sh.reshape(-1, 2), st, N, S, M, D, Lq, L, P, _dtype_code(value), mode)
            workspace = torch.empty(max(nbytes, 1), dtype=torch.uint8, device=dev) if nbytes else None
    if atomic:
        r = lib().msda_backward_atomic(_dptr(value), _iptr(sh), _iptr(st), _dptr(sampling_loc), _dptr(attn_weight),
                                       _dptr(grad_out), _dptr(grad_value), _dptr(grad_loc), _dptr(grad_attn),
                                       N, S, M, D, Lq, L, P, _dtype_code(value), _stream(stream))
        _raise(r, "msda_backward_atomic")
        return grad_value, grad_loc, grad_attn
    ws_ptr = _dptr(workspace) if workspace is not None else None
    ws_bytes = workspace.numel() * workspace.element_size() if workspace is not None else 0
    r = lib().msda_backward(_dptr(value), _iptr(sh), _iptr(st), _dptr(sampling_loc), _dptr(attn_weight),
                            _dptr(grad_out), _dptr(grad_value), _dptr(grad_loc), _dptr(grad_attn), ws_ptr, ws_bytes,
                            N, S, M, D, Lq, L, P, _dtype_code(value), _stream(stream))
    _raise(r, "msda_backward")
    return grad_value, grad_loc, grad_attn


def backward_noalloc(value, spatial_shapes, level_start_index, sampling_loc, attn_weight, grad_out,
                     grad_value, grad_loc, grad_attn, stream=None):
    """msda_backward_noalloc into caller-allocated outputs: the library allocates nothing (its
    owner-computes scratch is a static device array of MSDA_NOALLOC_SCRATCH_BYTES per GPU)."""
    N, S, M, D, Lq, L, P = _dims(value, sampling_loc)
    sh, st = _host_tables(spatial_shapes, level_start_index)
    r = lib().msda_backward_noalloc(_dptr(value), _iptr(sh), _iptr(st), _dptr(sampling_loc), _dptr(attn_weight),
                                    _dptr(grad_out), _dptr(grad_value), _dptr(grad_loc), _dptr(grad_attn),
                                    N, S, M, D, Lq, L, P, _dtype_code(value), _stream(stream))
    _raise(r, "msda_backward_noalloc")
    return grad_value, grad_loc, grad_attn


def backward_deterministic(value, spatial_shapes, level_start_index, sampling_loc, attn_weight, grad_out,
                           grad_value=None, grad_loc=None, grad_attn=None, workspace=None, stream=None):
    """(grad_value fp32, grad_loc, grad_attn) from msda_backward_deterministic (bitwise reproducible
    grad_value). workspace: a caller-owned uint8 device tensor, or None to allocate one of the size
    msda_backward_workspace_size(..., MSDA_WORKSPACE_DETERMINISTIC) reports."""
    import torch

    N, S, M, D, Lq, L, P = _dims(value, sampling_loc)
    dev = value.device
    sh, st = _host_tables(spatial_shapes, level_start_index)
    with _on(stream):
        if grad_value is None:
            grad_value = torch.empty((N, S, M, D), dtype=torch.float32, device=dev)
        if grad_loc is None:
            grad_loc = torch.empty(tuple(sampling_loc.shape), dtype=torch.float32, device=dev)
        if grad_attn is None:
            grad_attn = torch.empty(tuple(attn_weight.shape), dtype=torch.float32, device=dev)
        if workspace is None:
            nbytes = workspace_size(sh.reshape(-1, 2), st, N, S, M, D, Lq, L, P, _dtype_code(value),
                                    MSDA_WORKSPACE_DETERMINISTIC)
            workspace = torch.empty(max(nbytes, 1), dtype=torch.uint8, device=dev)
    ws_bytes = workspace.numel() * workspace.element_size()
    r = lib().msda_backward_deterministic(_dptr(value), _iptr(sh), _iptr(st), _dptr(sampling_loc),
                                          _dptr(attn_weight), _dptr(grad_out), _dptr(grad_value), _dptr(grad_loc),
                                          _dptr(grad_attn), _dptr(workspace), ws_bytes, N, S, M, D, Lq, L, P,
                                          _dtype_code(value), _stream(stream))
    _raise(r, "msda_backward_deterministic")
    return grad_value, grad_loc, grad_attn


def _fused_dims(value, ref_points, offsets, logits):
    N, S, M, D = value.shape
    if offsets.dim() != 6 or offsets.shape[-1] != 2:
        raise ValueError(f"offsets must be [N, Lq, M, L, P, 2], not {tuple(offsets.shape)}")
    _, Lq, M2, L, P, _ = offsets.shape
    if (M2 != M or tuple(ref_points.shape) != (N, Lq, L, 2) or tuple(logits.shape) != (N, Lq, M, L * P)
            or offsets.shape[0] != N):
        raise ValueError(f"value {tuple(value.shape)}, ref_points {tuple(ref_points.shape)}, offsets "
                         f"{tuple(offsets.shape)} and logits {tuple(logits.shape)} do not match")
    return N, S, M, D, Lq, L, P


def fused_workspace_size(spatial_shapes, level_start_index, N, S, M, D, Lq, L, P, dtype,
                         mode: int = MSDA_WORKSPACE_PREFERRED) -> int:
    """msda_backward_fused_workspace_size: staging of the locations, weights and their gradients
    plus the owner-computes workspace (as workspace_size with the same mode)."""
    sh, st = _host_tables(spatial_shapes, level_start_index)
    out = ctypes.c_size_t(0)
    r = lib().msda_backward_fused_workspace_size(_iptr(sh), _iptr(st), N, S, M, D, Lq, L, P, int(dtype),
                                                 int(mode), ctypes.byref(out))
    _raise(r, "msda_backward_fused_workspace_size")
    return int(out.value)


def forward_fused(value, spatial_shapes, level_start_index, ref_points, offsets, logits, out=None, stream=None):
    """out[N, Lq, M*D] from msda_forward_fused: locations ref_points + offsets / (W_l, H_l) and
    weights softmax(logits) are formed inside the kernel."""
    import torch

    N, S, M, D, Lq, L, P = _fused_dims(value, ref_points, offsets, logits)
    if out is None:
        with _on(stream):
            out = torch.empty((N, Lq, M * D), dtype=value.dtype, device=value.device)
    sh, st = _host_tables(spatial_shapes, level_start_index)
    r = lib().msda_forward_fused(_dptr(value), _iptr(sh), _iptr(st), _dptr(ref_points), _dptr(offsets),
                                 _dptr(logits), _dptr(out), N, S, M, D, Lq, L, P, _dtype_code(value),
                                 _stream(stream))
    _raise(r, "msda_forward_fused")
    return out


def backward_fused(value, spatial_shapes, level_start_index, ref_points, offsets, logits, grad_out,
                   grad_value=None, grad_ref=None, grad_offsets=None, grad_logits=None, workspace="auto",
                   want_grad_ref: bool = True, stream=None):
    """(grad_value fp32, grad_ref or None, grad_offsets, grad_logits) from msda_backward_fused.

    workspace: "auto" (the size the library prefers), "owner" (with the owner-computes grad_value
    wherever it applies) or a caller-owned uint8 device tensor of at least the staging size.
    """
    import torch

    N, S, M, D, Lq, L, P = _fused_dims(value, ref_points, offsets, logits)
    dev = value.device
    sh, st = _host_tables(spatial_shapes, level_start_index)
    with _on(stream):
        if grad_value is None:
            grad_value = torch.empty((N, S, M, D), dtype=torch.float32, device=dev)
        if grad_ref is None and want_grad_ref:
            grad_ref = torch.empty(tuple(ref_points.shape), dtype=torch.float32, device=dev)
        if grad_offsets is None:
            grad_offsets = torch.empty(tuple(offsets.shape), dtype=torch.float32, device=dev)
        if grad_logits is None:
            grad_logits = torch.empty(tuple(logits.shape), dtype=torch.float32, device=dev)
        if isinstance(workspace, str):
            if workspace not in ("auto", "owner"):
                raise ValueError(f"workspace must be 'auto', 'owner' or a tensor, not {workspace!r}")
            mode = MSDA_WORKSPACE_PREFERRED if workspace == "auto" else MSDA_WORKSPACE_OWNER
            nbytes = fused_workspace_size(sh.reshape(-1, 2), st, N, S, M, D, Lq, L, P, _dtype_code(value), mode)
            workspace = torch.empty(max(nbytes, 1), dtype=torch.uint8, device=dev)
    ws_bytes = workspace.numel() * workspace.element_size()
    r = lib().msda_backward_fused(_dptr(value), _iptr(sh), _iptr(st), _dptr(ref_points), _dptr(offsets),
                                  _dptr(logits), _dptr(grad_out), _dptr(grad_value),
                                  _dptr(grad_ref) if grad_ref is not None else None, _dptr(grad_offsets),
                                  _dptr(grad_logits), _dptr(workspace), ws_bytes, N, S, M, D, Lq, L, P,
                                  _dtype_code(value), _stream(stream))
    _raise(r, "msda_backward_fused")
    return grad_value, grad_ref, grad_offsets, grad_logits


def forward_raw(value_ptr: int, shapes: np.ndarray, starts: np.ndarray, loc_ptr: int, attn_ptr: int,
                out_ptr: int, dims: Sequence[int], dtype: int, stream: int) -> int:
    """msda_forward on raw device addresses; returns the status (used by the benchmark loop)."""
    return lib().msda_forward(value_ptr, _iptr(shapes), _iptr(starts), loc_ptr, attn_ptr, out_ptr,
                              *dims, dtype, stream)


def backward_raw(value_ptr: int, shapes: np.ndarray, starts: np.ndarray, loc_ptr: int, attn_ptr: int,
                 gout_ptr: int, gv_ptr: int, gl_ptr: int, ga_ptr: int, ws_ptr: Optional[int], ws_bytes: int,
                 dims: Sequence[int], dtype: int, stream: int, deterministic: bool = False) -> int:
    """msda_backward (msda_backward_deterministic; msda_backward_atomic when ws_ptr is None) on raw
    device addresses; returns the status (used by the benchmark loop)."""
    if ws_ptr is None and not deterministic:
        return lib().msda_backward_atomic(value_ptr, _iptr(shapes), _iptr(starts), loc_ptr, attn_ptr, gout_ptr,
                                          gv_ptr, gl_ptr, ga_ptr, *dims, dtype, stream)
    fn = lib().msda_backward_deterministic if deterministic else lib().msda_backward
    return fn(value_ptr, _iptr(shapes), _iptr(starts), loc_ptr, attn_ptr, gout_ptr, gv_ptr, gl_ptr, ga_ptr, ws_ptr,
              ws_bytes, *dims, dtype, stream)


def forward_fused_raw(value_ptr: int, shapes: np.ndarray, starts: np.ndarray, ref_ptr: int, off_ptr: int,
                      logit_ptr: int, out_ptr: int, dims: Sequence[int], dtype: int, stream: int) -> int:
    """msda_forward_fused on raw device addresses; returns the status (used by the benchmark loop)."""
    return lib().msda_forward_fused(value_ptr, _iptr(shapes), _iptr(starts), ref_ptr, off_ptr, logit_ptr, out_ptr,
                                    *dims, dtype, stream)


def backward_fused_raw(value_ptr: int, shapes: np.ndarray, starts: np.ndarray, ref_ptr: int, off_ptr: int,
                       logit_ptr: int, gout_ptr: int, gv_ptr: int, gref_ptr: Optional[int], goff_ptr: int,
                       glog_ptr: int, ws_ptr: int, ws_bytes: int, dims: Sequence[int], dtype: int,
                       stream: int) -> int:
    """msda_backward_fused on raw device addresses; returns the status (used by the benchmark loop)."""
    return lib().msda_backward_fused(value_ptr, _iptr(shapes), _iptr(starts), ref_ptr, off_ptr, logit_ptr,
                                     gout_ptr, gv_ptr, gref_ptr, goff_ptr, glog_ptr, ws_ptr, ws_bytes, *dims,
                                     dtype, stream)


# ---------------------------------------------------------------- layer operators


def _layer_dtype(t) -> int:
    import torch

    if t.dtype == torch.bfloat16:
        return MSDA_BF16
    if t.dtype in (torch.float32, torch.float16):
        return _dtype_code(t)
    raise ValueError(f"dtype must be float32, float16 or bfloat16, got {t.dtype}")


def _expect(name, t, shape, dtype, like, strided=False):
    """Checks one tensor argument: its shape and dtype, the device of `like`, and contiguity (with
    `strided`, of the channels alone). None passes."""
    if t is None or (t.shape == shape and t.dtype is dtype and t.get_device() == like.get_device() >= 0 and
                     (t.is_contiguous() or (strided and t.stride(-1) == 1))):
        return  # get_device() is negative of what is not on a GPU
    if tuple(t.shape) != tuple(shape) or t.dtype != dtype:
        raise ValueError(f"{name} must be {dtype} of shape {tuple(shape)}, got {t.dtype} of {tuple(t.shape)}")
    if t.device != like.device:
        raise ValueError(f"{name} is on {t.device}, expected {like.device}")
    if not t.is_cuda:
        raise ValueError("tensor arguments must be device tensors")
    if not strided:
        raise ValueError(f"{name} must be contiguous")
    if t.shape[-1] > 1:
        raise ValueError(f"the channels of {name} must be contiguous")


def _launching(t, stream):
    """A context in which the device of `t` is current and torch allocates memory for use on the call's
    stream, and that stream's handle: `stream`, or torch's current stream of the device."""
    import torch

    index = t.get_device()
    here = index == torch.cuda.current_device()
    if stream is None:
        handle = torch._C._cuda_getCurrentRawStream(index)  # current_stream(index).cuda_stream, without the 3 us object
        return _NO_CONTEXT if here else torch.cuda.device(index), handle
    if isinstance(stream, torch.cuda.Stream) and stream.device != t.device:
        raise ValueError(f"the stream is of {stream.device}, the tensors are on {t.device}")
    context = contextlib.ExitStack()
    if not here:
        context.enter_context(torch.cuda.device(index))
    context.enter_context(_on(stream))
    return context, _stream(stream)


def _address(t) -> Optional[int]:
    return None if t is None else t.data_ptr()


def _strides(t):
    return (ctypes.c_int64 * 3)(*t.stride()[:3])


def _workspace(workspace, nbytes, like):
    """The workspace tensor of a call: one of `nbytes` for "auto", or the caller's."""
    import torch

    if isinstance(workspace, str):
        if workspace != "auto":
            raise ValueError(f"workspace must be 'auto' or a tensor, not {workspace!r}")
        return like.new_empty(nbytes, dtype=torch.uint8) if nbytes else None
    if workspace is not None and (workspace.device != like.device or not workspace.is_contiguous()):
        raise ValueError(f"the workspace must be contiguous and on {like.device}")
    return workspace


def _bytes(t) -> int:
    return 0 if t is None else t.numel() * t.element_size()


def layernorm_workspace_size(rows, C, dtype) -> int:
    """msda_layernorm_backward_workspace_size: bytes of device workspace for the sums over rows."""
    out = ctypes.c_size_t(0)
    _raise(lib().msda_layernorm_backward_workspace_size(rows, C, int(dtype), ctypes.byref(out)),
           "msda_layernorm_backward_workspace_size")
    return int(out.value)


def _rows(x):
    if x.dim() < 1:
        raise ValueError("x must have a channel dimension")
    C = x.shape[-1]
    rows = 1
    for n in x.shape[:-1]:
        rows *= n
    return rows, C


def layernorm_forward(x, weight=None, bias=None, residual=None, eps=1e-5, want_sum: bool = False, out=None, mean=None,
                      rstd=None, sum=None, stream=None):
    """(out, mean, rstd) from msda_layernorm_forward: layer norm of x + residual over the last dimension; with
    want_sum (or a `sum` tensor) also x + residual itself, as a fourth result. weight and bias are fp32."""
    import torch

    rows, C = _rows(x)
    code = _layer_dtype(x)
    _expect("x", x, x.shape, x.dtype, x)
    for name, t in (("residual", residual), ("out", out), ("sum", sum)):
        _expect(name, t, x.shape, x.dtype, x)
    for name, t in (("weight", weight), ("bias", bias)):
        _expect(name, t, (C,), torch.float32, x)
    for name, t in (("mean", mean), ("rstd", rstd)):
        _expect(name, t, x.shape[:-1], torch.float32, x)
    context, s = _launching(x, stream)
    with context:
        out = torch.empty_like(x) if out is None else out
        mean = torch.empty(x.shape[:-1], dtype=torch.float32, device=x.device) if mean is None else mean
        rstd = torch.empty(x.shape[:-1], dtype=torch.float32, device=x.device) if rstd is None else rstd
        sum = torch.empty_like(x) if sum is None and want_sum else sum
        r = lib().msda_layernorm_forward(_address(x), _address(residual), _address(weight), _address(bias), _address(out),
                                         _address(sum), _address(mean), _address(rstd), rows, C, float(eps), code, s)
    _raise(r, "msda_layernorm_forward")
    return (out, mean, rstd) if sum is None else (out, mean, rstd, sum)


def layernorm_backward(x, grad_out, mean, rstd, weight=None, residual=None, grad_sum=None,
                       want_weight_grads: bool = True, grad_x=None, grad_weight=None, grad_bias=None, workspace="auto",
                       stream=None):
    """(grad_x, grad_weight, grad_bias) from msda_layernorm_backward; grad_x is the gradient of x and of residual.
    Without want_weight_grads the last two are None (or the tensors given). grad_sum: the gradient of the
    forward's `sum`."""
    import torch

    rows, C = _rows(x)
    code = _layer_dtype(x)
    _expect("x", x, x.shape, x.dtype, x)
    for name, t in (("residual", residual), ("grad_out", grad_out), ("grad_sum", grad_sum), ("grad_x", grad_x)):
        _expect(name, t, x.shape, x.dtype, x)
    for name, t in (("weight", weight), ("grad_weight", grad_weight), ("grad_bias", grad_bias)):
        _expect(name, t, (C,), torch.float32, x)
    for name, t in (("mean", mean), ("rstd", rstd)):
        _expect(name, t, x.shape[:-1], torch.float32, x)
    context, s = _launching(x, stream)
    with context:
        grad_x = torch.empty_like(x) if grad_x is None else grad_x
        if want_weight_grads:
            grad_weight = torch.empty(C, dtype=torch.float32, device=x.device) if grad_weight is None else grad_weight
            grad_bias = torch.empty(C, dtype=torch.float32, device=x.device) if grad_bias is None else grad_bias
        wanted = grad_weight is not None or grad_bias is not None
        ws = _workspace(workspace, layernorm_workspace_size(rows, C, code) if wanted else 0, x)
        r = lib().msda_layernorm_backward(_address(x), _address(residual), _address(weight), _address(grad_out),
                                          _address(grad_sum), _address(mean), _address(rstd), _address(grad_x),
                                          _address(grad_weight), _address(grad_bias), _address(ws), _bytes(ws), rows, C,
                                          code, s)
    _raise(r, "msda_layernorm_backward")
    return grad_x, grad_weight, grad_bias


def _rotate(entry, in_name, x, pos, freqs, interleaved, out_name, out, stream):
    import torch

    if x.dim() != 4 or freqs.dim() != 2:
        raise ValueError(f"{in_name} must be [N, T, M, D] and freqs [A, R], not {tuple(x.shape)} and {tuple(freqs.shape)}")
    N, T, M, D = x.shape
    A, R = freqs.shape
    code = _layer_dtype(x)
    shared = pos.dim() == 2
    _expect(in_name, x, x.shape, x.dtype, x, strided=True)
    _expect(out_name, out, x.shape, x.dtype, x, strided=True)
    _expect("pos", pos, (T, A) if shared else (N, T, A), torch.float32, x)
    _expect("freqs", freqs, (A, R), torch.float32, x)
    context, s = _launching(x, stream)
    with context:
        out = torch.empty((N, T, M, D), dtype=x.dtype, device=x.device) if out is None else out
        r = getattr(lib(), entry)(_address(x), _strides(x), _address(pos), _address(freqs), _address(out), _strides(out),
                                  N, T, M, D, A, R, 1 if shared else N, int(bool(interleaved)), code, s)
    _raise(r, entry)
    return out


def rotary_forward(x, pos, freqs, interleaved: bool = False, out=None, stream=None):
    """x [N, T, M, D] with its channel pairs turned by the angles pos . freqs, from msda_rotary_forward. pos is
    [N, T, A], or [T, A] for the same positions in every batch item; freqs is [A, R]. x may be a view whose channels
    are contiguous (the queries and keys of a packed projection); out=x rotates in place."""
    return _rotate("msda_rotary_forward", "x", x, pos, freqs, interleaved, "out", out, stream)


def rotary_backward(grad_out, pos, freqs, interleaved: bool = False, grad_x=None, stream=None):
    """The gradient of rotary_forward's x from msda_rotary_backward: grad_out turned back. grad_x=grad_out turns in
    place."""
    return _rotate("msda_rotary_backward", "grad_out", grad_out, pos, freqs, interleaved, "grad_x", grad_x, stream)


def _attention(q, k, v, scale, softcap, slopes, q_pos, k_pos, q_doc, k_doc, prefix, causal):
    """The call's msda_attention_t, after the checks of its tensors."""
    import torch

    if q.dim() != 4 or k.dim() != 4:
        raise ValueError(f"q must be [N, Lq, M, D] and k [N, Lk, Mkv, D], not {tuple(q.shape)} and {tuple(k.shape)}")
    N, Lq, M, D = q.shape
    _, Lk, Mkv, _ = k.shape
    code = _layer_dtype(q)
    _expect("q", q, q.shape, q.dtype, q, strided=True)
    for name, t in (("k", k), ("v", v)):
        _expect(name, t, (N, Lk, Mkv, D), q.dtype, q, strided=True)
    _expect("slopes", slopes, (M,), torch.float32, q)
    _expect("q_pos", q_pos, (N, Lq, 2), torch.float32, q)
    _expect("k_pos", k_pos, (N, Lk, 2), torch.float32, q)
    _expect("q_doc", q_doc, (N, Lq), torch.int32, q)
    _expect("k_doc", k_doc, (N, Lk), torch.int32, q)
    _expect("prefix", prefix, (N,), torch.int32, q)
    if (q_doc is None) != (k_doc is None):
        raise ValueError("q_doc and k_doc must be given both or neither")
    if slopes is not None and (q_pos is None or k_pos is None):
        raise ValueError("slopes need q_pos and k_pos")
    unaligned = int(any(t.data_ptr() % 16 for t in (q, k, v)))
    return AttentionDescription(N, Lq, Lk, M, Mkv, D, code, int(bool(causal)), unaligned,
                                D ** -0.5 if scale is None else float(scale), float(softcap), _strides(q), _strides(k),
                                _strides(v), *(_address(t) for t in (slopes, q_pos, k_pos, q_doc, k_doc, prefix)))


def _attention_workspace(a, backward: bool) -> int:
    out = ctypes.c_size_t(0)
    _raise(lib().msda_attention_workspace_size(ctypes.byref(a), int(backward), ctypes.byref(out)),
           "msda_attention_workspace_size")
    return int(out.value)


def attention_workspace_size(q, k, v, backward: bool = False, scale=None, softcap: float = 0.0, slopes=None, q_pos=None,
                             k_pos=None, q_doc=None, k_doc=None, prefix=None, causal: bool = False) -> int:
    """msda_attention_workspace_size of the call with these arguments."""
    return _attention_workspace(_attention(q, k, v, scale, softcap, slopes, q_pos, k_pos, q_doc, k_doc, prefix, causal),
                                backward)


def attention_forward(q, k, v, scale=None, softcap: float = 0.0, slopes=None, q_pos=None, k_pos=None, q_doc=None,
                      k_doc=None, prefix=None, causal: bool = False, want_lse: bool = True, out=None, lse=None,
                      workspace="auto", stream=None):
    """(out [N, Lq, M, D], lse [N, M, Lq] or None) from msda_attention_forward.

    q [N, Lq, M, D], k and v [N, Lk, Mkv, D], M a multiple of Mkv; views whose channels are contiguous are
    taken. scale: D ** -0.5 when None. softcap: cap of the scores (0: none). slopes [M], q_pos [N, Lq, 2] and
    k_pos [N, Lk, 2] (fp32): a bias of -slope times the distance. q_doc [N, Lq] and k_doc [N, Lk] (int32): queries see
    the keys of their own document, negative ones are padding. prefix [N] (int32): the first keys, common to all documents
    and exempt from the order. causal: the last query sees every key, each one before it one fewer.
    workspace: "auto" allocates it, or a caller-owned uint8 tensor of attention_workspace_size bytes.
    """
    import torch

    a = _attention(q, k, v, scale, softcap, slopes, q_pos, k_pos, q_doc, k_doc, prefix, causal)
    _expect("out", out, q.shape, q.dtype, q)
    _expect("lse", lse, (a.N, a.M, a.Lq), torch.float32, q)
    context, s = _launching(q, stream)
    with context:
        out = torch.empty(q.shape, dtype=q.dtype, device=q.device) if out is None else out
        if lse is None and want_lse:
            lse = torch.empty((a.N, a.M, a.Lq), dtype=torch.float32, device=q.device)
        ws = _workspace(workspace, _attention_workspace(a, False), q)
        r = lib().msda_attention_forward(ctypes.byref(a), _address(q), _address(k), _address(v), _address(out),
                                         _address(lse), _address(ws), _bytes(ws), s)
    _raise(r, "msda_attention_forward")
    return out, lse


def attention_backward(q, k, v, out, lse, grad_out, scale=None, softcap: float = 0.0, slopes=None, q_pos=None, k_pos=None,
                       q_doc=None, k_doc=None, prefix=None, causal: bool = False, grad_q=None, grad_k=None, grad_v=None,
                       workspace="auto", stream=None):
    """(grad_q, grad_k, grad_v) from msda_attention_backward, with the forward's arguments and its out and lse."""
    import torch

    a = _attention(q, k, v, scale, softcap, slopes, q_pos, k_pos, q_doc, k_doc, prefix, causal)
    for name, t in (("out", out), ("grad_out", grad_out), ("grad_q", grad_q)):
        _expect(name, t, q.shape, q.dtype, q)
    _expect("lse", lse, (a.N, a.M, a.Lq), torch.float32, q)
    for name, t in (("grad_k", grad_k), ("grad_v", grad_v)):
        _expect(name, t, k.shape, q.dtype, q)
    context, s = _launching(q, stream)
    with context:
        grad_q = torch.empty(q.shape, dtype=q.dtype, device=q.device) if grad_q is None else grad_q
        grad_k = torch.empty(k.shape, dtype=q.dtype, device=q.device) if grad_k is None else grad_k
        grad_v = torch.empty(k.shape, dtype=q.dtype, device=q.device) if grad_v is None else grad_v
        ws = _workspace(workspace, _attention_workspace(a, True), q)
        r = lib().msda_attention_backward(ctypes.byref(a), _address(q), _address(k), _address(v), _address(out),
                                          _address(lse), _address(grad_out), _address(grad_q), _address(grad_k),
                                          _address(grad_v), _address(ws), _bytes(ws), s)
    _raise(r, "msda_attention_backward")
    return grad_q, grad_k, grad_v


# ---------------------------------------------------------------- serving operators


def rmsnorm_workspace_size(rows, C, dtype) -> int:
    """msda_rmsnorm_backward_workspace_size: bytes of device workspace for the sums over rows."""
    out = ctypes.c_size_t(0)
    _raise(lib().msda_rmsnorm_backward_workspace_size(rows, C, int(dtype), ctypes.byref(out)),
           "msda_rmsnorm_backward_workspace_size")
    return int(out.value)


def rmsnorm_forward(x, weight=None, residual=None, eps=1e-6, want_sum: bool = False, out=None, rstd=None, sum=None,
                    stream=None):
    """(out, rstd) from msda_rmsnorm_forward: root-mean-square norm of x + residual over the last dimension; with
    want_sum (or a `sum` tensor) also x + residual itself, as a third result. weight is fp32."""
    import torch

    rows, C = _rows(x)
    code = _layer_dtype(x)
    _expect("x", x, x.shape, x.dtype, x)
    for name, t in (("residual", residual), ("out", out), ("sum", sum)):
        _expect(name, t, x.shape, x.dtype, x)
    _expect("weight", weight, (C,), torch.float32, x)
    _expect("rstd", rstd, x.shape[:-1], torch.float32, x)
    context, s = _launching(x, stream)
    with context:
        out = torch.empty_like(x) if out is None else out
        rstd = x.new_empty(x.shape[:-1], dtype=torch.float32) if rstd is None else rstd
        sum = torch.empty_like(x) if sum is None and want_sum else sum
        r = lib().msda_rmsnorm_forward(_address(x), _address(residual), _address(weight), _address(out), _address(sum),
                                       _address(rstd), rows, C, float(eps), code, s)
    _raise(r, "msda_rmsnorm_forward")
    return (out, rstd) if sum is None else (out, rstd, sum)


def rmsnorm_quantize(x, weight=None, residual=None, eps=1e-6, want_sum: bool = False, codes=None, scale=None, sum=None,
                     stream=None):
    """(codes, scale) from msda_rmsnorm_quantize: rmsnorm_forward's result in 8 bits, codes (int8, x's shape) times scale
    (fp32, one for each row); with want_sum (or a `sum` tensor) also x + residual, as a third result."""
    import torch

    rows, C = _rows(x)
    code = _layer_dtype(x)
    _expect("x", x, x.shape, x.dtype, x)
    for name, t in (("residual", residual), ("sum", sum)):
        _expect(name, t, x.shape, x.dtype, x)
    _expect("weight", weight, (C,), torch.float32, x)
    _expect("codes", codes, x.shape, torch.int8, x)
    _expect("scale", scale, x.shape[:-1], torch.float32, x)
    context, s = _launching(x, stream)
    with context:
        codes = torch.empty_like(x, dtype=torch.int8) if codes is None else codes
        scale = x.new_empty(x.shape[:-1], dtype=torch.float32) if scale is None else scale
        sum = torch.empty_like(x) if sum is None and want_sum else sum
        r = lib().msda_rmsnorm_quantize(_address(x), _address(residual), _address(weight), _address(codes), _address(scale),
                                        _address(sum), rows, C, float(eps), code, s)
    _raise(r, "msda_rmsnorm_quantize")
    return (codes, scale) if sum is None else (codes, scale, sum)


def rmsnorm_backward(x, grad_out, rstd, weight=None, residual=None, grad_sum=None, want_weight_grad: bool = True, grad_x=None,
                     grad_weight=None, workspace="auto", stream=None):
    """(grad_x, grad_weight) from msda_rmsnorm_backward; grad_x is the gradient of x and of residual. Without
    want_weight_grad the last is None (or the tensor given). grad_sum: the gradient of the forward's `sum`."""
    import torch

    rows, C = _rows(x)
    code = _layer_dtype(x)
    _expect("x", x, x.shape, x.dtype, x)
    for name, t in (("residual", residual), ("grad_out", grad_out), ("grad_sum", grad_sum), ("grad_x", grad_x)):
        _expect(name, t, x.shape, x.dtype, x)
    for name, t in (("weight", weight), ("grad_weight", grad_weight)):
        _expect(name, t, (C,), torch.float32, x)
    _expect("rstd", rstd, x.shape[:-1], torch.float32, x)
    context, s = _launching(x, stream)
    with context:
        grad_x = torch.empty_like(x) if grad_x is None else grad_x
        if want_weight_grad and grad_weight is None:
            grad_weight = x.new_empty(C, dtype=torch.float32)
        ws = _workspace(workspace, 0 if grad_weight is None else rmsnorm_workspace_size(rows, C, code), x)
        r = lib().msda_rmsnorm_backward(_address(x), _address(residual), _address(weight), _address(grad_out),
                                        _address(grad_sum), _address(rstd), _address(grad_x), _address(grad_weight),
                                        _address(ws), _bytes(ws), rows, C, code, s)
    _raise(r, "msda_rmsnorm_backward")
    return grad_x, grad_weight


def quantize_rows(x, codes=None, scale=None, stream=None):
    """(codes, scale) from msda_quantize_rows: x in 8 bits, codes (int8, x's shape) times scale (fp32, one for each row of the
    last dimension)."""
    import torch

    rows, C = _rows(x)
    code = _layer_dtype(x)
    _expect("x", x, x.shape, x.dtype, x)
    _expect("codes", codes, x.shape, torch.int8, x)
    _expect("scale", scale, x.shape[:-1], torch.float32, x)
    context, s = _launching(x, stream)
    with context:
        codes = torch.empty_like(x, dtype=torch.int8) if codes is None else codes
        scale = x.new_empty(x.shape[:-1], dtype=torch.float32) if scale is None else scale
        r = lib().msda_quantize_rows(_address(x), _address(codes), _address(scale), rows, C, code, s)
    _raise(r, "msda_quantize_rows")
    return codes, scale


def quantized_matmul(a, b, a_scale, b_scale, bias=None, dtype=None, out=None, stream=None):
    """out [..., O] from msda_quantized_matmul: codes a [..., K] (int8) times codes b [O, K] (int8), with scales a_scale [...]
    and b_scale [O] and a bias [O] (fp32). dtype of the result: float32, float16 or bfloat16 (`out`'s, or bfloat16)."""
    import torch

    rows, K = _rows(a)
    if b.dim() != 2:
        raise ValueError(f"b must be [O, K], not {tuple(b.shape)}")
    O = b.shape[0]
    dtype = (torch.bfloat16 if out is None else out.dtype) if dtype is None else dtype
    shape = a.shape[:-1] + (O,)
    _expect("a", a, a.shape, torch.int8, a)
    _expect("b", b, (O, K), torch.int8, a)
    _expect("a_scale", a_scale, a.shape[:-1], torch.float32, a)
    for name, t in (("b_scale", b_scale), ("bias", bias)):
        _expect(name, t, (O,), torch.float32, a)
    _expect("out", out, shape, dtype, a)
    context, s = _launching(a, stream)
    with context:
        out = a.new_empty(shape, dtype=dtype) if out is None else out
        r = lib().msda_quantized_matmul(_address(a), _address(b), _address(a_scale), _address(b_scale), _address(bias),
                                        _address(out), rows, K, O, _layer_dtype(out), s)
    _raise(r, "msda_quantized_matmul")
    return out


_TwoStrides = ctypes.c_int64 * 2


def _two_strides(t):
    return _TwoStrides(*t.stride()[:2])


def _cache(T, k_cache, v_cache, k_scale, v_scale, table, length, start):
    """The call's msda_cache_t, after the checks of its tensors."""
    import torch

    if k_cache.dim() != 4 or table.dim() != 2:
        raise ValueError(f"k_cache must be [pages, Mkv, page_size, D] and table [N, width], not {tuple(k_cache.shape)} and "
                         f"{tuple(table.shape)}")
    pages, Mkv, page_size, D = k_cache.shape
    N, width = table.shape
    _expect("k_cache", k_cache, k_cache.shape, torch.int8, k_cache)
    _expect("v_cache", v_cache, k_cache.shape, torch.int8, k_cache)
    for name, t in (("k_scale", k_scale), ("v_scale", v_scale)):
        _expect(name, t, (pages, Mkv), torch.float32, k_cache)
    _expect("table", table, (N, width), torch.int32, k_cache, strided=True)
    _expect("length", length, (N,), torch.int32, k_cache)
    _expect("start", start, (N + 1,), torch.int32, k_cache)
    return CacheDescription(N, pages, page_size, Mkv, D, width, table.stride(0),
                            *(_address(t) for t in (k_cache, v_cache, k_scale, v_scale, table, length, start)))


def cache_append(k, v, k_cache, v_cache, k_scale, v_scale, table, length, start=None, pos=None, freqs=None,
                 interleaved: bool = False, stream=None):
    """Appends k and v [T, Mkv, D] to a paged cache in place, from msda_cache_append.

    k_cache and v_cache [pages, Mkv, page_size, D] (int8) with k_scale and v_scale [pages, Mkv] (fp32); table [N, width]
    (int32): the pages of each sequence, a view of a wider table's first columns is taken; length [N] (int32): tokens of each
    sequence, the new ones included; start [N + 1] (int32): the first of each sequence's new tokens among the T, or None: one
    each. freqs [A, R] (fp32): k is turned by pos [T, A] (fp32; None: a token's place in its sequence, A == 1) on the way,
    as by rotary_forward. k and v may be views whose channels are contiguous.
    """
    import torch

    if k.dim() != 3 or (freqs is not None and freqs.dim() != 2):
        raise ValueError(f"k must be [T, Mkv, D] and freqs [A, R], not {tuple(k.shape)} and "
                         f"{None if freqs is None else tuple(freqs.shape)}")
    if freqs is None and pos is not None:
        raise ValueError("pos needs freqs")
    T = k.shape[0]
    A, R = (1, 0) if freqs is None else freqs.shape
    code = _layer_dtype(k)
    c = _cache(T, k_cache, v_cache, k_scale, v_scale, table, length, start)
    _expect("k", k, (T, c.Mkv, c.D), k.dtype, k_cache, strided=True)
    _expect("v", v, (T, c.Mkv, c.D), k.dtype, k_cache, strided=True)
    _expect("pos", pos, (T, A), torch.float32, k_cache)
    _expect("freqs", freqs, (A, R), torch.float32, k_cache)
    context, s = _launching(k_cache, stream)
    with context:
        r = lib().msda_cache_append(ctypes.byref(c), _address(k), _two_strides(k), _address(v), _two_strides(v), _address(pos),
                                    _address(freqs), T, A, R, int(bool(interleaved)), code, s)
    _raise(r, "msda_cache_append")


def _cache_attention_workspace(c, T, M, code) -> int:
    out = ctypes.c_size_t(0)
    _raise(lib().msda_cache_attention_workspace_size(ctypes.byref(c), T, M, code, ctypes.byref(out)),
           "msda_cache_attention_workspace_size")
    return int(out.value)


def cache_attention_workspace_size(q, k_cache, v_cache, k_scale, v_scale, table, length, start=None) -> int:
    """msda_cache_attention_workspace_size of the call with these arguments."""
    c = _cache(q.shape[0], k_cache, v_cache, k_scale, v_scale, table, length, start)
    return _cache_attention_workspace(c, q.shape[0], q.shape[1], _layer_dtype(q))


def cache_attention(q, k_cache, v_cache, k_scale, v_scale, table, length, start=None, scale=None, softcap: float = 0.0,
                    causal: bool = True, want_lse: bool = True, out=None, lse=None, workspace="auto", stream=None):
    """(out [T, M, D], lse [T, M] or None) of the new tokens' queries q [T, M, D] over a paged cache, from
    msda_cache_attention.

    The cache's arguments as in cache_append, which has stored the new tokens' keys and values already; M is a multiple of Mkv;
    q may be a view whose channels are contiguous. Long sequences are split by the table's width: a view of the columns that
    they reach is faster than a table that is several times wider. scale: D ** -0.5 when None. softcap: cap of the scores (0: none). causal:
    a token sees those up to itself, otherwise all of its sequence. workspace: "auto" allocates it, or a caller-owned uint8
    tensor of cache_attention_workspace_size bytes.
    """
    import torch

    if q.dim() != 3:
        raise ValueError(f"q must be [T, M, D], not {tuple(q.shape)}")
    T, M, D = q.shape
    code = _layer_dtype(q)
    c = _cache(T, k_cache, v_cache, k_scale, v_scale, table, length, start)
    _expect("q", q, (T, M, c.D), q.dtype, k_cache, strided=True)
    _expect("out", out, q.shape, q.dtype, k_cache)
    _expect("lse", lse, (T, M), torch.float32, k_cache)
    context, s = _launching(k_cache, stream)
    with context:
        out = q.new_empty(q.shape) if out is None else out
        if lse is None and want_lse:
            lse = q.new_empty((T, M), dtype=torch.float32)
        ws = _workspace(workspace, _cache_attention_workspace(c, T, M, code), k_cache)
        r = lib().msda_cache_attention(ctypes.byref(c), _address(q), _two_strides(q), _address(out), _address(lse), T, M,
                                       D ** -0.5 if scale is None else float(scale), float(softcap), int(bool(causal)), code,
                                       _address(ws), _bytes(ws), s)
    _raise(r, "msda_cache_attention")
    return out, lse
