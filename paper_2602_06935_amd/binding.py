"""Thin ctypes binding of libcotten_attn.so (same names as include/cotten_attn.h).

Argument marshalling only: every arithmetic step runs in the HIP kernels.  torch is
used for device memory (`torch.empty`, `.data_ptr()`) and for the current stream.
There is no CPU fallback: if the library cannot be loaded, or a tensor is not on
the GPU, the call raises.

The library allocates nothing.  Calls that need a workspace get one from here when the caller
passes none: a `torch.empty` buffer of the call's own, given back when the call has enqueued its
launches.  Several threads may call on one stream at a time; a workspace (or `kept` buffer) that
they pass themselves must not be shared by calls that may overlap on the host: the launches of
two calls could alternate on the stream.
"""
from __future__ import annotations

import ctypes
import functools
import os
from typing import Optional, Tuple

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libcotten_attn.so")

COTTEN_F32 = 0
COTTEN_BF16 = 1
COTTEN_F16 = 2
COTTEN_BHND = 0
COTTEN_BNHD = 1
COTTEN_MAP_COSINE = 0
COTTEN_MAP_ELU1 = 1

EXPORTS = (
    "cotten_attn_fwd", "cotten_attn_bwd", "cotten_attn_fwd_ex", "cotten_attn_bwd_ex",
    "cotten_attn_workspace_bytes", "cotten_status_string",
    "cotten_normaliser_fwd", "cotten_normaliser_bwd", "cotten_attn_bwd_static",
    "cotten_attn_workspace_bytes_ex",
    "cotten_delta_fwd", "cotten_delta_bwd", "cotten_delta_kept_bytes", "cotten_delta_workspace_bytes",
    "cotten_embed_fwd", "cotten_embed_bwd", "cotten_embed_workspace_bytes",
    "cotten_dropout", "cotten_residual_fwd", "cotten_residual_bwd", "cotten_residual_workspace_bytes",
    "cotten_beam_select", "cotten_beam_reorder", "cotten_beam_workspace_bytes",
    "cotten_decay_fwd", "cotten_decay_bwd", "cotten_decay_workspace_bytes",
)


class CottenParams(ctypes.Structure):
    _fields_ = [("dtype", ctypes.c_int), ("scale", ctypes.c_float), ("eps", ctypes.c_float),
                ("workspace", ctypes.c_void_p), ("workspace_bytes", ctypes.c_size_t),
                ("slice_scale", ctypes.c_void_p), ("dlog_scale", ctypes.c_void_p),
                ("layout", ctypes.c_int), ("causal", ctypes.c_int),
                ("saved_state", ctypes.c_void_p), ("feature_map", ctypes.c_int)]


class CottenDeltaParams(ctypes.Structure):
    _fields_ = [("dtype", ctypes.c_int), ("scale", ctypes.c_float), ("eps", ctypes.c_float),
                ("layout", ctypes.c_int), ("workspace", ctypes.c_void_p), ("workspace_bytes", ctypes.c_size_t),
                ("initial_state", ctypes.c_void_p), ("final_state", ctypes.c_void_p),
                ("dfinal_state", ctypes.c_void_p), ("dinitial_state", ctypes.c_void_p),
                ("kept", ctypes.c_void_p), ("kept_bytes", ctypes.c_size_t)]


class CottenEmbedParams(ctypes.Structure):
    _fields_ = [("dtype", ctypes.c_int), ("id_bytes", ctypes.c_int), ("scale", ctypes.c_float),
                ("padding_idx", ctypes.c_int), ("positions", ctypes.c_int), ("position_offset", ctypes.c_int),
                ("workspace", ctypes.c_void_p), ("workspace_bytes", ctypes.c_size_t)]


class CottenDecayParams(ctypes.Structure):
    _fields_ = [("dtype", ctypes.c_int), ("scale", ctypes.c_float), ("eps", ctypes.c_float),
                ("layout", ctypes.c_int), ("workspace", ctypes.c_void_p), ("workspace_bytes", ctypes.c_size_t),
                ("initial_state", ctypes.c_void_p), ("final_state", ctypes.c_void_p),
                ("dfinal_state", ctypes.c_void_p), ("dinitial_state", ctypes.c_void_p)]


class CottenDropoutParams(ctypes.Structure):
    _fields_ = [("dtype", ctypes.c_int), ("p", ctypes.c_double), ("seed", ctypes.c_uint64), ("offset", ctypes.c_uint64),
                ("step", ctypes.c_void_p)]


class CottenResidualParams(ctypes.Structure):
    _fields_ = [("dtype", ctypes.c_int), ("norm", ctypes.c_int), ("post_weight", ctypes.c_void_p),
                ("post_bias", ctypes.c_void_p), ("gate", ctypes.c_void_p), ("next_weight", ctypes.c_void_p),
                ("next_bias", ctypes.c_void_p), ("gate_per_sequence", ctypes.c_int), ("alpha", ctypes.c_float),
                ("eps", ctypes.c_float), ("p", ctypes.c_double), ("seed", ctypes.c_uint64), ("offset", ctypes.c_uint64),
                ("step", ctypes.c_void_p), ("workspace", ctypes.c_void_p), ("workspace_bytes", ctypes.c_size_t)]


class CottenResidualGrads(ctypes.Structure):
    _fields_ = [("post_weight", ctypes.c_void_p), ("post_bias", ctypes.c_void_p), ("gate", ctypes.c_void_p),
                ("next_weight", ctypes.c_void_p), ("next_bias", ctypes.c_void_p)]


class CottenBeamParams(ctypes.Structure):
    _fields_ = [("dtype", ctypes.c_int), ("pad", ctypes.c_int), ("workspace", ctypes.c_void_p),
                ("workspace_bytes", ctypes.c_size_t)]


class CottenError(RuntimeError):
    def __init__(self, status: int, message: str):
        super().__init__(f"cotten_attn status {status}: {message}")
        self.status = status


_lib = None


def load_library(build_if_missing: bool = True) -> ctypes.CDLL:
    """dlopen the in-tree library; compile it first only when no build exists."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        if not build_if_missing:
            raise FileNotFoundError(LIB_PATH)
        from . import build as _build
        _build.build()
    lib = ctypes.CDLL(LIB_PATH)
    vp, ip = ctypes.c_void_p, ctypes.c_int
    lib.cotten_attn_fwd.argtypes = [vp, vp, vp, vp, vp, ip, ip, ip, ip, vp]
    lib.cotten_attn_bwd.argtypes = [vp, vp, vp, vp, vp, vp, vp, vp, ip, ip, ip, ip, vp]
    lib.cotten_attn_fwd_ex.argtypes = lib.cotten_attn_fwd.argtypes + [ctypes.POINTER(CottenParams)]
    lib.cotten_attn_bwd_ex.argtypes = lib.cotten_attn_bwd.argtypes + [ctypes.POINTER(CottenParams)]
    lib.cotten_attn_bwd_static.argtypes = lib.cotten_attn_bwd_ex.argtypes
    for f in (lib.cotten_attn_fwd, lib.cotten_attn_bwd, lib.cotten_attn_fwd_ex, lib.cotten_attn_bwd_ex,
              lib.cotten_attn_bwd_static):
        f.restype = ctypes.c_int
    lib.cotten_attn_workspace_bytes.argtypes = [ip, ip, ip, ip, ip, ip]
    lib.cotten_attn_workspace_bytes.restype = ctypes.c_size_t
    lib.cotten_attn_workspace_bytes_ex.argtypes = [ip, ip, ip, ip, ip, ctypes.POINTER(CottenParams)]
    lib.cotten_attn_workspace_bytes_ex.restype = ctypes.c_size_t
    lib.cotten_normaliser_fwd.argtypes = [vp, vp, vp, ip, ip, ip, vp]
    lib.cotten_normaliser_bwd.argtypes = [vp, vp, vp, ip, ip, ip, vp]
    lib.cotten_normaliser_fwd.restype = lib.cotten_normaliser_bwd.restype = ctypes.c_int
    lib.cotten_delta_fwd.argtypes = [vp] * 7 + [ip] * 4 + [vp, ctypes.POINTER(CottenDeltaParams)]
    lib.cotten_delta_bwd.argtypes = [vp] * 12 + [ip] * 4 + [vp, ctypes.POINTER(CottenDeltaParams)]
    lib.cotten_delta_fwd.restype = lib.cotten_delta_bwd.restype = ctypes.c_int
    lib.cotten_delta_kept_bytes.argtypes = [ip] * 5
    lib.cotten_delta_workspace_bytes.argtypes = [ip] * 7
    lib.cotten_delta_kept_bytes.restype = lib.cotten_delta_workspace_bytes.restype = ctypes.c_size_t
    lib.cotten_embed_fwd.argtypes = lib.cotten_embed_bwd.argtypes = \
        [vp] * 4 + [ip] * 4 + [vp, ctypes.POINTER(CottenEmbedParams)]
    lib.cotten_embed_fwd.restype = lib.cotten_embed_bwd.restype = ctypes.c_int
    lib.cotten_embed_workspace_bytes.argtypes = [ip] * 4
    lib.cotten_embed_workspace_bytes.restype = ctypes.c_size_t
    lib.cotten_decay_fwd.argtypes = [vp] * 6 + [ip] * 4 + [vp, ctypes.POINTER(CottenDecayParams)]
    lib.cotten_decay_bwd.argtypes = [vp] * 10 + [ip] * 4 + [vp, ctypes.POINTER(CottenDecayParams)]
    lib.cotten_decay_fwd.restype = lib.cotten_decay_bwd.restype = ctypes.c_int
    lib.cotten_decay_workspace_bytes.argtypes = [ip] * 7
    lib.cotten_decay_workspace_bytes.restype = ctypes.c_size_t
    lib.cotten_dropout.argtypes = [vp, vp, ctypes.c_size_t, vp, ctypes.POINTER(CottenDropoutParams)]
    lib.cotten_residual_fwd.argtypes = [vp] * 4 + [ip] * 3 + [vp, ctypes.POINTER(CottenResidualParams)]
    lib.cotten_residual_bwd.argtypes = [vp] * 6 + [ip] * 3 + [vp, ctypes.POINTER(CottenResidualParams),
                                                             ctypes.POINTER(CottenResidualGrads)]
    for f in (lib.cotten_dropout, lib.cotten_residual_fwd, lib.cotten_residual_bwd):
        f.restype = ctypes.c_int
    lib.cotten_residual_workspace_bytes.argtypes = [ip] * 4
    lib.cotten_residual_workspace_bytes.restype = ctypes.c_size_t
    lib.cotten_beam_select.argtypes = [vp] * 6 + [ip] * 3 + [vp, ctypes.POINTER(CottenBeamParams)]
    lib.cotten_beam_reorder.argtypes = [vp, vp, ip, ip, ctypes.c_size_t, vp]
    lib.cotten_beam_select.restype = lib.cotten_beam_reorder.restype = ctypes.c_int
    lib.cotten_beam_workspace_bytes.argtypes = [ip] * 3
    lib.cotten_beam_workspace_bytes.restype = ctypes.c_size_t
    lib.cotten_status_string.argtypes = [ip]
    lib.cotten_status_string.restype = ctypes.c_char_p
    _lib = lib
    return lib


def cotten_status_string(status: int) -> str:
    return load_library().cotten_status_string(int(status)).decode()


def cotten_attn_workspace_bytes(B: int, H: int, N: int, d_h: int, dtype: int, is_bwd: bool) -> int:
    return int(load_library().cotten_attn_workspace_bytes(B, H, N, d_h, dtype, int(bool(is_bwd))))


def cotten_attn_workspace_bytes_ex(B: int, H: int, N: int, d_h: int, is_bwd: bool, *, dtype: int,
                                   causal: bool = False) -> int:
    """Workspace bytes of a call with these options (the causal variant has needs of its own)."""
    prm = CottenParams()
    prm.dtype = dtype
    prm.causal = 1 if causal else 0
    return int(load_library().cotten_attn_workspace_bytes_ex(B, H, N, d_h, int(bool(is_bwd)),
                                                             ctypes.byref(prm)))


def _check(status: int) -> None:
    if status != 0:
        raise CottenError(status, cotten_status_string(status))


_DTYPE_CODES = {torch.float32: COTTEN_F32, torch.bfloat16: COTTEN_BF16, torch.float16: COTTEN_F16}


def _dtype_code(t: torch.Tensor) -> int:
    code = _DTYPE_CODES.get(t.dtype)
    if code is None:
        raise TypeError(f"unsupported I/O dtype {t.dtype}")
    return code


def _prep(name: str, t: torch.Tensor, like: Optional[torch.Tensor] = None) -> torch.Tensor:
    if not t.is_cuda:
        raise ValueError(f"{name} must be a GPU tensor (there is no CPU path)")
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous [B,H,N,d_h]")
    if like is not None and (t.shape != like.shape or t.dtype != like.dtype or t.device != like.device):
        raise ValueError(f"{name} must match Q in shape, dtype and device")
    return t


def _prep_like(Q: torch.Tensor, others) -> None:
    """The checks of _prep on Q and on the (name, tensor) pairs that must match it.  Attributes of Q are read once and
    the checks written as one condition: the attribute reads are most of what a check costs."""
    if not (Q.is_cuda and Q.is_contiguous()):
        _prep("Q", Q)
    shape, dtype, device = Q.shape, Q.dtype, Q.device
    for name, t in others:
        if not (t.shape == shape and t.dtype is dtype and t.device == device and t.is_contiguous()):
            _prep(name, t, Q)


def _mask_ptr(mask: Optional[torch.Tensor], B: int, N: int, dev) -> Optional[int]:
    if mask is None:
        return None
    if mask.dtype is not torch.uint8 or mask.shape != (B, N) or not mask.is_contiguous() or mask.device != dev:
        raise ValueError("mask must be a contiguous uint8 [B,N] tensor on the same device")
    return mask.data_ptr()


def _f32_vector(name: str, t: Optional[torch.Tensor], numel: int, dev) -> Optional[int]:
    if t is None:
        return None
    if t.dtype != torch.float32 or t.numel() != numel or not t.is_contiguous() or t.device != dev:
        raise ValueError(f"{name} must be a contiguous float32 GPU tensor of {numel} elements")
    return t.data_ptr()


def _dims(Q: torch.Tensor, layout: str) -> Tuple[int, int, int, int]:
    """(B, H, N, d_h) of a tensor stored as `layout` ("bhnd" or "bnhd")."""
    if Q.dim() != 4:
        raise ValueError("expected a 4-d tensor")
    if layout == "bhnd":
        B, H, N, d = Q.shape
    elif layout == "bnhd":
        B, N, H, d = Q.shape
    else:
        raise ValueError("layout must be 'bhnd' or 'bnhd'")
    return B, H, N, d


_FEATURE_MAPS = {"cosine": COTTEN_MAP_COSINE, "elu1": COTTEN_MAP_ELU1}


def _params(Q: torch.Tensor, scale, eps, workspace: Optional[torch.Tensor],
            slice_scale: Optional[torch.Tensor] = None,
            dlog_scale: Optional[torch.Tensor] = None, layout: str = "bhnd",
            causal: bool = False, saved_state: Optional[torch.Tensor] = None,
            feature_map: str = "cosine") -> CottenParams:
    fmap = _FEATURE_MAPS.get(feature_map)
    if fmap is None:
        raise ValueError("feature_map must be 'cosine' or 'elu1'")
    kept = scales = dlog = space = None
    if saved_state is not None or slice_scale is not None or dlog_scale is not None:
        B, H, _, d = _dims(Q, layout)
        kept = _f32_vector("saved_state", saved_state, B * H * d * d, Q.device)
        scales = _f32_vector("slice_scale", slice_scale, B * H, Q.device)
        dlog = _f32_vector("dlog_scale", dlog_scale, B * H, Q.device)
    dtype = _dtype_code(Q)
    space_bytes = 0
    if workspace is not None:
        if not workspace.is_cuda or not workspace.is_contiguous():
            raise ValueError("workspace must be a contiguous GPU tensor")
        space = workspace.data_ptr()
        space_bytes = workspace.numel() * workspace.element_size()
    return CottenParams(dtype, 0.0 if scale is None else float(scale), -1.0 if eps is None else float(eps),
                        space, space_bytes, scales, dlog, COTTEN_BNHD if layout == "bnhd" else COTTEN_BHND,
                        1 if causal else 0, kept, fmap)


@functools.lru_cache(maxsize=1024)
def _workspace_need(B: int, H: int, N: int, d: int, is_bwd: bool, dtype: int, causal: bool) -> int:
    return cotten_attn_workspace_bytes_ex(B, H, N, d, is_bwd, dtype=dtype, causal=causal)


def _workspace(like: torch.Tensor, need: int, stream_handle: int) -> torch.Tensor:
    """A workspace for one call that needs one and was given none.  It is that call's alone: the lock of the interpreter is
    not held while the library enqueues, so another thread's launches may come between this call's on the same stream.
    torch hands a buffer that was freed on again in the order of the stream it was allocated on, so the buffer comes
    from the stream of the call (while that is captured, from the graph's pool) and may be dropped as soon as the call returns."""
    device = like.device
    if stream_handle == _current_stream_handle(device.index):
        return torch.empty(need, dtype=torch.uint8, device=device)
    with torch.cuda.device(device), torch.cuda.stream(torch.cuda.ExternalStream(stream_handle, device)):
        return torch.empty(need, dtype=torch.uint8, device=device)


# Handle of the current stream of a device: straight from torch's extension module where that has it (0.1 us; a
# Stream object, made for its handle, 2.9).
_current_stream_handle = getattr(torch._C, "_cuda_getCurrentRawStream",
                                 lambda device: torch.cuda.current_stream(device).cuda_stream)


# The current device likewise (a GPU tensor is at hand wherever it is asked for: the runtime is up).
_current_device = getattr(torch._C, "_cuda_getDevice", torch.cuda.current_device)


def _stream_handle(stream, device: torch.device) -> int:
    if stream is None:  # the current one of the device that the tensors are on
        return _current_stream_handle(device.index)
    if isinstance(stream, torch.cuda.Stream):
        return stream.cuda_stream
    return int(stream)


def _on_device(device: torch.device, entry, *args) -> None:
    """One call into the library with `device` current."""
    if device.index == _current_device():
        status = entry(*args)
        if status != 0:
            _check(status)
    else:
        with torch.cuda.device(device):
            _check(entry(*args))


def cotten_attn_fwd(Q: torch.Tensor, K: torch.Tensor, V: torch.Tensor,
                    mask: Optional[torch.Tensor], O: Optional[torch.Tensor] = None, *,
                    scale: Optional[float] = None, eps: Optional[float] = None,
                    stream=None, workspace: Optional[torch.Tensor] = None,
                    slice_scale: Optional[torch.Tensor] = None,
                    layout: str = "bhnd", causal: bool = False,
                    saved_state: Optional[torch.Tensor] = None,
                    feature_map: str = "cosine") -> torch.Tensor:
    """O = scale * Qhat (Khat^T V) under the key mask; enqueues on the stream and returns O.
    `slice_scale` ([B,H] float32) gives every slice its own scale instead of `scale`;
    `layout` "bnhd" means all tensors are [B,N,H,d_h] instead of [B,H,N,d_h];
    `saved_state` ([B,H,d_h,d_h] float32) receives the state S of every slice for the
    backward call."""
    lib = _lib or load_library()
    _prep_like(Q, (("K", K), ("V", V)))
    B, H, N, d = _dims(Q, layout)
    O = torch.empty_like(Q) if O is None else _prep("O", O, Q)
    handle = _stream_handle(stream, Q.device)
    if workspace is None:
        need = _workspace_need(B, H, N, d, False, _dtype_code(Q), bool(causal))
        if need != 0:
            workspace = _workspace(Q, need, handle)
    prm = _params(Q, scale, eps, workspace, slice_scale, None, layout, causal, saved_state, feature_map)
    _on_device(Q.device, lib.cotten_attn_fwd_ex, Q.data_ptr(), K.data_ptr(), V.data_ptr(),
               _mask_ptr(mask, B, N, Q.device), O.data_ptr(), B, H, N, d, handle, ctypes.byref(prm))
    return O


def cotten_attn_bwd(Q: torch.Tensor, K: torch.Tensor, V: torch.Tensor,
                    mask: Optional[torch.Tensor], dO: torch.Tensor,
                    dQ: Optional[torch.Tensor] = None, dK: Optional[torch.Tensor] = None,
                    dV: Optional[torch.Tensor] = None, *, scale: Optional[float] = None,
                    eps: Optional[float] = None, stream=None,
                    workspace: Optional[torch.Tensor] = None,
                    slice_scale: Optional[torch.Tensor] = None,
                    dlog_scale: Optional[torch.Tensor] = None, layout: str = "bhnd",
                    causal: bool = False, static_scratch: bool = False,
                    saved_state: Optional[torch.Tensor] = None, feature_map: str = "cosine"
                    ) -> Tuple[torch.Tensor, torch.Tensor, torch.Tensor]:
    """(dQ, dK, dV) for upstream gradient dO; enqueues on the stream and returns the tensors.
    `slice_scale` as in the forward; `dlog_scale` ([B,H] float32), when given, receives
    d loss / d log(scale) of every slice.  With `static_scratch` the call goes to
    cotten_attn_bwd_static: no workspace is passed or allocated, the library's own static
    scratch array serves (the output tensors must then be given, nothing is allocated here).
    `saved_state`: the state the forward call of the same inputs wrote; read instead of being
    rebuilt from K, V."""
    lib = _lib or load_library()
    _prep_like(Q, (("K", K), ("V", V), ("dO", dO)))
    B, H, N, d = _dims(Q, layout)
    dQ = torch.empty_like(Q) if dQ is None else _prep("dQ", dQ, Q)
    dK = torch.empty_like(Q) if dK is None else _prep("dK", dK, Q)
    dV = torch.empty_like(Q) if dV is None else _prep("dV", dV, Q)
    handle = _stream_handle(stream, Q.device)
    if static_scratch:
        workspace = None
    elif workspace is None:
        need = _workspace_need(B, H, N, d, True, _dtype_code(Q), bool(causal))
        if need != 0:
            workspace = _workspace(Q, need, handle)
    prm = _params(Q, scale, eps, workspace, slice_scale, dlog_scale, layout, causal, saved_state,
                  feature_map)
    entry = lib.cotten_attn_bwd_static if static_scratch else lib.cotten_attn_bwd_ex
    _on_device(Q.device, entry, Q.data_ptr(), K.data_ptr(), V.data_ptr(), _mask_ptr(mask, B, N, Q.device),
               dO.data_ptr(), dQ.data_ptr(), dK.data_ptr(), dV.data_ptr(), B, H, N, d, handle, ctypes.byref(prm))
    return dQ, dK, dV


def _lengths_ptr(n: Optional[torch.Tensor], B: int, dev) -> Optional[int]:
    if n is None:
        return None
    if n.dtype != torch.int32 or n.numel() != B or not n.is_contiguous() or n.device != dev:
        raise ValueError("n must be a contiguous int32 GPU tensor of B elements")
    return n.data_ptr()


def cotten_normaliser_fwd(m: torch.Tensor, n: Optional[torch.Tensor], B: int, N: int,
                          slice_scale: Optional[torch.Tensor] = None, *, stream=None) -> torch.Tensor:
    """slice_scale[b,h] = n_b ** (-m_h) (n = None: the padded length N for every sequence)."""
    lib = load_library()
    if not m.is_cuda or m.dtype != torch.float32 or not m.is_contiguous() or m.dim() != 1:
        raise ValueError("m must be a contiguous float32 GPU vector [H]")
    H = m.numel()
    if slice_scale is None:
        slice_scale = torch.empty(B, H, device=m.device, dtype=torch.float32)
    with torch.cuda.device(m.device):
        _check(lib.cotten_normaliser_fwd(m.data_ptr(), _lengths_ptr(n, B, m.device),
                                         _f32_vector("slice_scale", slice_scale, B * H, m.device),
                                         B, H, N, _stream_handle(stream, m.device)))
    return slice_scale


def cotten_normaliser_bwd(dlog_scale: torch.Tensor, n: Optional[torch.Tensor], N: int,
                          dm: Optional[torch.Tensor] = None, *, stream=None) -> torch.Tensor:
    """dm[h] = -sum_b ln(n_b) * dlog_scale[b,h]."""
    lib = load_library()
    if not dlog_scale.is_cuda or dlog_scale.dim() != 2:
        raise ValueError("dlog_scale must be a GPU tensor [B,H]")
    B, H = dlog_scale.shape
    dev = dlog_scale.device
    if dm is None:
        dm = torch.empty(H, device=dev, dtype=torch.float32)
    with torch.cuda.device(dev):
        _check(lib.cotten_normaliser_bwd(_f32_vector("dlog_scale", dlog_scale, B * H, dev),
                                         _lengths_ptr(n, B, dev), _f32_vector("dm", dm, H, dev),
                                         B, H, N, _stream_handle(stream, dev)))
    return dm


# ---- gated delta rule -----------------------------------------------------------------------------

_LAYOUTS = {"bhnd": COTTEN_BHND, "bnhd": COTTEN_BNHD}


@functools.lru_cache(maxsize=1024)
def cotten_delta_kept_bytes(B: int, H: int, N: int, d_h: int, dtype: int) -> int:
    return int(load_library().cotten_delta_kept_bytes(B, H, N, d_h, dtype))


@functools.lru_cache(maxsize=1024)
def cotten_delta_workspace_bytes(B: int, H: int, N: int, d_h: int, dtype: int, is_bwd: bool,
                                 with_kept: bool = False) -> int:
    return int(load_library().cotten_delta_workspace_bytes(B, H, N, d_h, dtype, int(bool(is_bwd)),
                                                           int(bool(with_kept))))


def cotten_delta_kept(Q: torch.Tensor, *, layout: str = "bhnd") -> torch.Tensor:
    """A buffer for what the forward of Q's shape hands to its backward (`kept` of the two calls)."""
    B, H, N, d = _dims(Q, layout)
    return torch.empty(cotten_delta_kept_bytes(B, H, N, d, _dtype_code(Q)), dtype=torch.uint8, device=Q.device)


def _buffer(name: str, t: Optional[torch.Tensor], dev) -> Tuple[Optional[int], int]:
    if t is None:
        return None, 0
    if not t.is_contiguous() or t.device != dev:
        raise ValueError(f"{name} must be a contiguous tensor on the device of Q")
    return t.data_ptr(), t.numel() * t.element_size()


def _check_gate(name: str, t: torch.Tensor, lead, dev) -> None:
    if not (t.dtype is torch.float32 and t.shape == lead and t.device == dev and t.is_contiguous()):
        raise ValueError(f"{name} must be a contiguous float32 tensor of shape {tuple(lead)} on the device of Q")


_LEAST_SCALE = torch.finfo(torch.float32).tiny


def _state_ptr(name: str, t: Optional[torch.Tensor], shape, dev) -> Optional[int]:
    if t is None:
        return None
    if t.shape != shape and t.shape != (shape[0] * shape[1], *shape[2:]):    # (another order of as many elements would be read as this one)
        raise ValueError(f"{name} must be of shape {shape} or {(shape[0] * shape[1], *shape[2:])}, not {tuple(t.shape)}")
    if t.dtype is not torch.float32 or not t.is_contiguous() or t.device != dev:
        raise ValueError(f"{name} must be a contiguous float32 tensor on the device of Q")
    return t.data_ptr()


def _delta_params(Q, dims, gates, scale, eps, layout, workspace, kept, initial_state=None, final_state=None,
                  dfinal_state=None, dinitial_state=None) -> CottenDeltaParams:
    """The checks of what the two calls share besides Q, K and V, and their parameters."""
    B, H, _, d = dims
    dev, lead, shape = Q.device, Q.shape[:3], (B, H, d, d)
    if scale is not None and scale < _LEAST_SCALE:    # (the library takes 0 and below for 1)
        raise ValueError(f"scale must be None for 1, or {_LEAST_SCALE} at least")
    for name, t in gates:
        _check_gate(name, t, lead, dev)
    first = _state_ptr("initial_state", initial_state, shape, dev)
    return CottenDeltaParams(
        _DTYPE_CODES[Q.dtype], 0.0 if scale is None else scale, -1.0 if eps is None else eps, _LAYOUTS[layout],
        *_buffer("workspace", workspace, dev), first,
        first if final_state is initial_state else _state_ptr("final_state", final_state, shape, dev),
        _state_ptr("dfinal_state", dfinal_state, shape, dev), _state_ptr("dinitial_state", dinitial_state, shape, dev),
        *_buffer("kept", kept, dev))


def cotten_delta_fwd(Q: torch.Tensor, K: torch.Tensor, V: torch.Tensor, g: torch.Tensor, beta: torch.Tensor,
                     mask: Optional[torch.Tensor], O: Optional[torch.Tensor] = None, *,
                     scale: Optional[float] = None, eps: Optional[float] = None, stream=None,
                     workspace: Optional[torch.Tensor] = None, layout: str = "bhnd",
                     initial_state: Optional[torch.Tensor] = None,
                     final_state: Optional[torch.Tensor] = None,
                     kept: Optional[torch.Tensor] = None) -> torch.Tensor:
    """Gated delta rule: S_t = a_t S_{t-1} + khat_t u_t^T with u_t = beta_t (v_t - a_t S_{t-1}^T khat_t) and a_t =
    exp(g_t); O_t = scale * S_t^T qhat_t.  Enqueues on the stream and returns O.
    `g` (log decays) and `beta` are float32, [B,H,N] ([B,N,H] with layout "bnhd"); a masked token leaves the state as it is;
    `scale` is positive and defaults to 1.  `initial_state` and `final_state` ([B,H,d_h,d_h] float32) may be the same tensor: with N = 1 that
    is a server's step.  `kept` (see cotten_delta_kept) receives what the backward needs of this call."""
    lib = _lib or load_library()
    _prep_like(Q, (("K", K), ("V", V)))
    dims = _dims(Q, layout)
    dtype = _dtype_code(Q)
    O = torch.empty_like(Q) if O is None else _prep("O", O, Q)
    handle = _stream_handle(stream, Q.device)
    if workspace is None and kept is None:
        need = cotten_delta_workspace_bytes(*dims, dtype, False)
        if need != 0:
            workspace = _workspace(Q, need, handle)
    prm = _delta_params(Q, dims, (("g", g), ("beta", beta)), scale, eps, layout, workspace, kept, initial_state,
                        final_state)
    _on_device(Q.device, lib.cotten_delta_fwd, Q.data_ptr(), K.data_ptr(), V.data_ptr(), g.data_ptr(),
               beta.data_ptr(), _mask_ptr(mask, dims[0], dims[2], Q.device), O.data_ptr(), *dims, handle,
               ctypes.byref(prm))
    return O


def cotten_delta_bwd(Q: torch.Tensor, K: torch.Tensor, V: torch.Tensor, g: torch.Tensor, beta: torch.Tensor,
                     mask: Optional[torch.Tensor], dO: torch.Tensor, dQ: Optional[torch.Tensor] = None,
                     dK: Optional[torch.Tensor] = None, dV: Optional[torch.Tensor] = None,
                     dg: Optional[torch.Tensor] = None, dbeta: Optional[torch.Tensor] = None, *,
                     scale: Optional[float] = None, eps: Optional[float] = None, stream=None,
                     workspace: Optional[torch.Tensor] = None, layout: str = "bhnd",
                     initial_state: Optional[torch.Tensor] = None, dfinal_state: Optional[torch.Tensor] = None,
                     dinitial_state: Optional[torch.Tensor] = None, kept: Optional[torch.Tensor] = None):
    """(dQ, dK, dV, dg, dbeta) for the upstream gradients dO and, when given, `dfinal_state`; `dinitial_state`, when
    given, receives the gradient of the initial state.  `kept`: what the forward call of the same inputs wrote (without it
    `initial_state` has to hold what that call saw, and the sequence is walked forwards once more)."""
    lib = _lib or load_library()
    _prep_like(Q, (("K", K), ("V", V), ("dO", dO)))
    dims = _dims(Q, layout)
    dQ = torch.empty_like(Q) if dQ is None else _prep("dQ", dQ, Q)
    dK = torch.empty_like(Q) if dK is None else _prep("dK", dK, Q)
    dV = torch.empty_like(Q) if dV is None else _prep("dV", dV, Q)
    dg = torch.empty_like(g) if dg is None else dg
    dbeta = torch.empty_like(beta) if dbeta is None else dbeta
    handle = _stream_handle(stream, Q.device)
    if workspace is None:
        workspace = _workspace(Q, cotten_delta_workspace_bytes(*dims, _dtype_code(Q), True, kept is not None), handle)
    prm = _delta_params(Q, dims, (("g", g), ("beta", beta), ("dg", dg), ("dbeta", dbeta)), scale, eps, layout, workspace,
                        kept, initial_state, None, dfinal_state, dinitial_state)
    return _delta_backward(prm, dims, handle, Q, K, V, g, beta, _mask_ptr(mask, dims[0], dims[2], Q.device), dO, dQ, dK, dV,
                           dg, dbeta)


def _delta_backward(prm, dims, handle, Q, K, V, g, beta, mask, dO, dQ, dK, dV, dg, dbeta):
    """The call itself: everything is checked."""
    _on_device(Q.device, _lib.cotten_delta_bwd, Q.data_ptr(), K.data_ptr(), V.data_ptr(), g.data_ptr(), beta.data_ptr(),
               mask, dO.data_ptr(), dQ.data_ptr(), dK.data_ptr(), dV.data_ptr(), dg.data_ptr(), dbeta.data_ptr(), *dims,
               handle, ctypes.byref(prm))
    return dQ, dK, dV, dg, dbeta


def _delta_backward_of(prm, dims, Q, K, V, g, beta, mask, dO, initial_state, dfinal_state, dinitial_state, kept):
    """The gradients of a forward call that has checked its tensors (the differentiable function's): `prm` holds its type,
    scale, eps and layout, the rest of it is filled in here."""
    handle = _stream_handle(None, Q.device)
    workspace = _workspace(Q, cotten_delta_workspace_bytes(*dims, prm.dtype, True, kept is not None), handle)
    prm.workspace, prm.workspace_bytes = workspace.data_ptr(), workspace.numel()
    if kept is not None:
        prm.kept, prm.kept_bytes = kept.data_ptr(), kept.numel()
    if initial_state is not None:
        prm.initial_state = initial_state.data_ptr()
    if dfinal_state is not None:
        prm.dfinal_state = dfinal_state.data_ptr()
    if dinitial_state is not None:
        prm.dinitial_state = dinitial_state.data_ptr()
    new = torch.empty_like
    return _delta_backward(prm, dims, handle, Q, K, V, g, beta, None if mask is None else mask.data_ptr(), dO, new(Q),
                           new(Q), new(Q), new(g), new(beta))


# ---- decay attention ------------------------------------------------------------------------------

@functools.lru_cache(maxsize=1024)
def cotten_decay_workspace_bytes(B: int, H: int, N: int, d_h: int, dtype: int, is_bwd: bool, with_dg: bool = False) -> int:
    return int(load_library().cotten_decay_workspace_bytes(B, H, N, d_h, dtype, int(bool(is_bwd)), int(bool(with_dg))))


def _check_decays(name: str, t: torch.Tensor, H: int, dev) -> int:
    if not (t.dtype is torch.float32 and t.shape == (H,) and t.device == dev and t.is_contiguous()):
        raise ValueError(f"{name} must be a contiguous float32 tensor of shape ({H},) on the device of Q")
    return t.data_ptr()


def _decay_params(Q, dims, scale, eps, layout, workspace, initial_state=None, final_state=None, dfinal_state=None,
                  dinitial_state=None) -> CottenDecayParams:
    """The checks of what the two calls share besides Q, K, V and g, and their parameters."""
    B, H, _, d = dims
    dev, shape = Q.device, (B, H, d, d)
    if scale is not None and scale < _LEAST_SCALE:    # (the library takes 0 and below for 1)
        raise ValueError(f"scale must be None for 1, or {_LEAST_SCALE} at least")
    first = _state_ptr("initial_state", initial_state, shape, dev)
    return CottenDecayParams(
        _dtype_code(Q), 0.0 if scale is None else scale, -1.0 if eps is None else eps, _LAYOUTS[layout],
        *_buffer("workspace", workspace, dev), first,
        first if final_state is initial_state else _state_ptr("final_state", final_state, shape, dev),
        _state_ptr("dfinal_state", dfinal_state, shape, dev), _state_ptr("dinitial_state", dinitial_state, shape, dev))


def cotten_decay_fwd(Q: torch.Tensor, K: torch.Tensor, V: torch.Tensor, g: torch.Tensor, mask: Optional[torch.Tensor],
                     O: Optional[torch.Tensor] = None, *, scale: Optional[float] = None, eps: Optional[float] = None,
                     stream=None, workspace: Optional[torch.Tensor] = None, layout: str = "bhnd",
                     initial_state: Optional[torch.Tensor] = None, final_state: Optional[torch.Tensor] = None) -> torch.Tensor:
    """Linear attention with a decay for each head: S_t = exp(g_h) S_{t-1} + khat_t v_t^T; O_t = scale * S_t^T qhat_t.  Enqueues on
    the stream and returns O.  `g` (log decays) is float32 [H]; a masked token leaves the state as it is; `scale` is positive and
    defaults to 1.  `initial_state` and `final_state` ([B,H,d_h,d_h] float32) may be the same tensor: with N = 1 that is a server's
    step."""
    lib = _lib or load_library()
    _prep_like(Q, (("K", K), ("V", V)))
    dims = _dims(Q, layout)
    decays = _check_decays("g", g, dims[1], Q.device)
    O = torch.empty_like(Q) if O is None else _prep("O", O, Q)
    handle = _stream_handle(stream, Q.device)
    if workspace is None:
        need = cotten_decay_workspace_bytes(*dims, _dtype_code(Q), False)
        if need != 0:
            workspace = _workspace(Q, need, handle)
    prm = _decay_params(Q, dims, scale, eps, layout, workspace, initial_state, final_state)
    _on_device(Q.device, lib.cotten_decay_fwd, Q.data_ptr(), K.data_ptr(), V.data_ptr(), decays,
               _mask_ptr(mask, dims[0], dims[2], Q.device), O.data_ptr(), *dims, handle, ctypes.byref(prm))
    return O


def cotten_decay_bwd(Q: torch.Tensor, K: torch.Tensor, V: torch.Tensor, g: torch.Tensor, mask: Optional[torch.Tensor],
                     dO: torch.Tensor, dQ: Optional[torch.Tensor] = None, dK: Optional[torch.Tensor] = None,
                     dV: Optional[torch.Tensor] = None, *, dg: Optional[torch.Tensor] = None, scale: Optional[float] = None,
                     eps: Optional[float] = None, stream=None, workspace: Optional[torch.Tensor] = None, layout: str = "bhnd",
                     initial_state: Optional[torch.Tensor] = None, dfinal_state: Optional[torch.Tensor] = None,
                     dinitial_state: Optional[torch.Tensor] = None) -> Tuple[torch.Tensor, torch.Tensor, torch.Tensor]:
    """(dQ, dK, dV) for the upstream gradients dO and, when given, `dfinal_state`; `dg` ([H] float32) and `dinitial_state`, when
    given, receive the gradients of the decays and of the initial state.  The inputs and `initial_state` have to hold what the
    forward call saw: nothing else is kept of it."""
    lib = _lib or load_library()
    _prep_like(Q, (("K", K), ("V", V), ("dO", dO)))
    dims = _dims(Q, layout)
    decays = _check_decays("g", g, dims[1], Q.device)
    of_decays = None if dg is None else _check_decays("dg", dg, dims[1], Q.device)
    dQ = torch.empty_like(Q) if dQ is None else _prep("dQ", dQ, Q)
    dK = torch.empty_like(Q) if dK is None else _prep("dK", dK, Q)
    dV = torch.empty_like(Q) if dV is None else _prep("dV", dV, Q)
    handle = _stream_handle(stream, Q.device)
    if workspace is None:
        need = cotten_decay_workspace_bytes(*dims, _dtype_code(Q), True, dg is not None)
        if need != 0:
            workspace = _workspace(Q, need, handle)
    prm = _decay_params(Q, dims, scale, eps, layout, workspace, initial_state, None, dfinal_state, dinitial_state)
    _on_device(Q.device, lib.cotten_decay_bwd, Q.data_ptr(), K.data_ptr(), V.data_ptr(), decays,
               _mask_ptr(mask, dims[0], dims[2], Q.device), dO.data_ptr(), dQ.data_ptr(), dK.data_ptr(), dV.data_ptr(), of_decays,
               *dims, handle, ctypes.byref(prm))
    return dQ, dK, dV


def _decay_backward_of(prm, dims, Q, K, V, g, mask, dO, initial_state, dfinal_state, dinitial_state, dg):
    """The gradients of a forward call that has checked its tensors (the differentiable function's): `prm` holds its type,
    scale, eps and layout, the rest of it is filled in here."""
    handle = _stream_handle(None, Q.device)
    need = cotten_decay_workspace_bytes(*dims, prm.dtype, True, dg is not None)
    if need != 0:
        workspace = _workspace(Q, need, handle)
        prm.workspace, prm.workspace_bytes = workspace.data_ptr(), need
    if initial_state is not None:
        prm.initial_state = initial_state.data_ptr()
    if dfinal_state is not None:
        prm.dfinal_state = dfinal_state.data_ptr()
    if dinitial_state is not None:
        prm.dinitial_state = dinitial_state.data_ptr()
    dQ, dK, dV = torch.empty_like(Q), torch.empty_like(Q), torch.empty_like(Q)
    _on_device(Q.device, _lib.cotten_decay_bwd, Q.data_ptr(), K.data_ptr(), V.data_ptr(), g.data_ptr(),
               None if mask is None else mask.data_ptr(), dO.data_ptr(), dQ.data_ptr(), dK.data_ptr(), dV.data_ptr(),
               None if dg is None else dg.data_ptr(), *dims, handle, ctypes.byref(prm))
    return dQ, dK, dV


# ---- embedding of item ids -----------------------------------------------------------------------

@functools.lru_cache(maxsize=1024)
def cotten_embed_workspace_bytes(B: int, N: int, D: int, V: int) -> int:
    return int(load_library().cotten_embed_workspace_bytes(B, N, D, V))


_MOST_INT = 2 ** 31 - 1    # (ctypes takes the lower 32 bits of a larger number)
_ID_BYTES = {torch.int32: 4, torch.int64: 8}


def _embed_params(ids: torch.Tensor, like: torch.Tensor, scale: float, padding_idx: Optional[int], positions: int,
                  position_offset: int) -> CottenEmbedParams:
    width = _ID_BYTES.get(ids.dtype)
    if width is None or ids.dim() != 2 or not ids.is_contiguous() or ids.device != like.device:
        raise ValueError("ids must be a contiguous int32 or int64 [B,N] tensor on the same device")
    if padding_idx is None:
        padding_idx = -1
    elif not 0 <= padding_idx <= _MOST_INT:
        raise ValueError("padding_idx must be None or an id, counted from 0, of 31 bits")
    if abs(position_offset) > _MOST_INT or positions > _MOST_INT:
        raise ValueError("position_offset and the rows of the positions must be numbers of 31 bits")
    return CottenEmbedParams(_dtype_code(like), width, scale, padding_idx, positions, position_offset)


def _check_table(name: str, t: torch.Tensor, dims: int, like: Optional[torch.Tensor] = None) -> None:
    if t.is_cuda and t.dim() == dims and t.is_contiguous():
        if like is None or (t.dtype is like.dtype and t.shape[-1] == like.shape[-1] and t.device == like.device):
            return
        raise ValueError(f"{name} must match the other tensors in width, dtype and device")
    if not t.is_cuda:
        raise ValueError(f"{name} must be a GPU tensor (there is no CPU path)")
    raise ValueError(f"{name} must be a contiguous {dims}-d tensor")


def cotten_embed_fwd(ids: torch.Tensor, W: torch.Tensor, positions: Optional[torch.Tensor] = None,
                     E: Optional[torch.Tensor] = None, *, scale: float = 1.0, padding_idx: Optional[int] = None,
                     position_offset: int = 0, stream=None) -> torch.Tensor:
    """E[b,n] = scale * W[ids[b,n]] + positions[position_offset + n]; enqueues on the stream and returns E [B,N,D].
    `ids` int32 or int64 [B,N]; a token with `padding_idx`, or an id that W has no row for, gets no row of W."""
    lib = _lib or load_library()
    _check_table("W", W, 2)
    table = rows = None
    if positions is not None:
        _check_table("positions", positions, 2, W)
        table, rows = positions.data_ptr(), positions.shape[0]
    prm = _embed_params(ids, W, scale, padding_idx, rows or 0, position_offset)
    (B, N), (V, D) = ids.shape, W.shape
    if V > _MOST_INT:
        raise ValueError("W must have fewer than 2^31 rows")
    if E is None:
        E = W.new_empty((B, N, D))
    else:
        _check_table("E", E, 3, W)
        if E.shape != (B, N, D):
            raise ValueError("E must be [B,N,D]")
    _on_device(W.device, lib.cotten_embed_fwd, ids.data_ptr(), W.data_ptr(), table, E.data_ptr(), B, N, D, V,
               _stream_handle(stream, W.device), ctypes.byref(prm))
    return E


def cotten_embed_bwd(ids: torch.Tensor, dE: torch.Tensor, V: int, dW: Optional[torch.Tensor] = None,
                     dP: Optional[torch.Tensor] = None, *, scale: float = 1.0, padding_idx: Optional[int] = None,
                     position_offset: int = 0, stream=None, workspace: Optional[torch.Tensor] = None,
                     of_table: bool = True) -> Optional[torch.Tensor]:
    """The gradient dW [V,D] of the table (written whole) for the upstream gradient dE; `dP`, the shape of the table of
    positions, receives its gradient when given.  `of_table=False`: dP alone (a table that is not trained), and None comes back."""
    lib = _lib or load_library()
    _check_table("dE", dE, 3)
    B, N, D = dE.shape
    if ids.shape != (B, N):
        raise ValueError("ids must be [B,N] and dE [B,N,D]")
    if V > _MOST_INT:
        raise ValueError("V, the rows of the table, must be fewer than 2^31")
    if not of_table:
        if dW is not None or dP is None:
            raise ValueError("of_table=False: dP is wanted, and no dW")
    elif dW is None:
        dW = dE.new_empty((V, D))
    else:
        _check_table("dW", dW, 2, dE)
        if dW.shape[0] != V:
            raise ValueError("dW must be [V,D]")
    positions = rows = None
    if dP is not None:
        _check_table("dP", dP, 2, dE)
        positions, rows = dP.data_ptr(), dP.shape[0]
    handle = _stream_handle(stream, dE.device)
    prm = _embed_params(ids, dE, scale, padding_idx, rows or 0, position_offset)
    if workspace is None:
        need = cotten_embed_workspace_bytes(B, N, D, V)
        if need != 0:
            workspace = _workspace(dE, need, handle)
    if workspace is not None:
        prm.workspace, prm.workspace_bytes = _buffer("workspace", workspace, dE.device)
    _on_device(dE.device, lib.cotten_embed_bwd, ids.data_ptr(), dE.data_ptr(), None if dW is None else dW.data_ptr(), positions,
               B, N, D, V, handle, ctypes.byref(prm))
    return dW


def _embed_backward_of(prm, ids, dE, W_shape, P_shape, of_table):
    """(dW, dP) of a forward call that has checked its tensors (the differentiable function's): `prm` holds all but the
    workspace.  `P_shape` None: dW alone; not `of_table`: dP alone."""
    B, N, D = dE.shape
    handle = _stream_handle(None, dE.device)
    workspace = _workspace(dE, cotten_embed_workspace_bytes(B, N, D, W_shape[0]), handle)
    prm.workspace, prm.workspace_bytes = workspace.data_ptr(), workspace.numel()
    dW = dE.new_empty(W_shape) if of_table else None
    dP = None if P_shape is None else dE.new_empty(P_shape)
    _on_device(dE.device, _lib.cotten_embed_bwd, ids.data_ptr(), dE.data_ptr(),
               None if dW is None else dW.data_ptr(), None if dP is None else dP.data_ptr(), B, N, D, W_shape[0], handle, ctypes.byref(prm))
    return dW, dP


# ---- dropout, and the seam between two blocks --------------------------------------------------------

_NORMS = {"rms": 0, "layer": 1}
_MOST_UINT64 = 2 ** 64 - 1


def _check_generator(p: float, seed: int, offset: int, step: Optional[torch.Tensor], dev) -> Optional[int]:
    """Refuses what the C call would not see; returns the address of `step`."""
    if not 0.0 <= p < 1.0:
        raise ValueError("p must be from 0 on and below 1")
    if not (0 <= seed <= _MOST_UINT64 and 0 <= offset <= _MOST_UINT64):    # (ctypes takes the lower 64 bits of other numbers)
        raise ValueError("seed and offset must be from 0 on, and of 64 bits")
    if step is None:
        return None
    if step.dtype is not torch.int64 or step.numel() != 1 or step.device != dev:
        raise ValueError("step must be one int64 number on the device of the other tensors")
    return step.data_ptr()


def cotten_dropout(x: torch.Tensor, p: float, *, seed: int, offset: int = 0, step: Optional[torch.Tensor] = None,
                   out: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """x / (1 - p) where the generator keeps an element and 0 elsewhere; p counts in multiples of 2^-16.  The same seed and
    offset (the number of the call) give the same decisions: the backward is this call on the upstream gradient.  `step`, one
    int64 number on the device, is added to the offset when the kernel runs: a captured graph draws anew when the program
    changes it between replays.  `out` may be x."""
    lib = _lib or load_library()
    if not (x.is_cuda and x.is_contiguous()):
        raise ValueError("x must be a contiguous GPU tensor (there is no CPU path)")
    prm = CottenDropoutParams(_dtype_code(x), p, seed, offset, _check_generator(p, seed, offset, step, x.device))
    if out is None:
        out = torch.empty_like(x)
    elif out.shape != x.shape or out.dtype is not x.dtype or out.device != x.device or not out.is_contiguous():
        raise ValueError("out must be a contiguous tensor like x")
    if x.numel() == 0:
        return out
    _on_device(x.device, lib.cotten_dropout, x.data_ptr(), out.data_ptr(), x.numel(), _stream_handle(stream, x.device),
               ctypes.byref(prm))
    return out


@functools.lru_cache(maxsize=1024)
def cotten_residual_workspace_bytes(B: int, N: int, D: int, gate_per_sequence: bool = False) -> int:
    return int(load_library().cotten_residual_workspace_bytes(B, N, D, int(bool(gate_per_sequence))))


def _seam_vector(name: str, t: torch.Tensor, dtype: torch.dtype, shape, dev) -> int:
    if t.dtype is not dtype or t.shape != shape or t.device != dev or not t.is_contiguous():
        raise ValueError(f"{name} must be a contiguous {list(shape)} tensor of the type and on the device of X")
    return t.data_ptr()


def _residual_params(X, F, norm, post_weight, post_bias, gate, alpha, next_weight, next_bias, eps, p, seed, offset,
                     step) -> CottenResidualParams:
    """The checks of what the two calls share, and their parameters."""
    shape, dtype, dev = X.shape, X.dtype, X.device   # (looked up once: every one of them is a call)
    if len(shape) != 3:
        raise ValueError("X must be [B,N,D]")
    _check_like("X", X, shape, dtype, dev)
    _check_like("F", F, shape, dtype, dev)
    kind = _NORMS.get(norm)
    if kind is None:
        raise ValueError("norm must be 'rms' or 'layer'")
    if (post_bias is not None and post_weight is None) or (next_bias is not None and next_weight is None):
        raise ValueError("a norm's bias goes with its weight")
    width = shape[2:]
    per_sequence, gates = False, None
    if gate is not None:
        per_sequence = gate.dim() == 2
        gates = _seam_vector("gate", gate, dtype, (shape[0], shape[2]) if per_sequence else width, dev)
    return CottenResidualParams(
        _dtype_code(X), kind,
        None if post_weight is None else _seam_vector("post_weight", post_weight, dtype, width, dev),
        None if post_bias is None else _seam_vector("post_bias", post_bias, dtype, width, dev), gates,
        None if next_weight is None else _seam_vector("next_weight", next_weight, dtype, width, dev),
        None if next_bias is None else _seam_vector("next_bias", next_bias, dtype, width, dev), int(per_sequence), alpha,
        -1.0 if eps is None else eps, p, seed, offset, _check_generator(p, seed, offset, step, dev))


def _check_like(name: str, t: torch.Tensor, shape, dtype: torch.dtype, dev) -> None:
    if not (t.is_cuda and t.is_contiguous() and t.shape == shape and t.dtype is dtype and t.device == dev):
        raise ValueError(f"{name} must be a contiguous GPU tensor [B,N,D], like X (there is no CPU path)")


def cotten_residual_fwd(X: torch.Tensor, F: torch.Tensor, Y: Optional[torch.Tensor] = None, H: Optional[torch.Tensor] = None, *,
                        norm: str = "rms", post_weight: Optional[torch.Tensor] = None,
                        post_bias: Optional[torch.Tensor] = None, gate: Optional[torch.Tensor] = None, alpha: float = 1.0,
                        next_weight: Optional[torch.Tensor] = None, next_bias: Optional[torch.Tensor] = None,
                        eps: Optional[float] = None, p: float = 0.0, seed: int = 0, offset: int = 0,
                        step: Optional[torch.Tensor] = None, stream=None):
    """(Y, H): Y = X + alpha * gate * drop(N(F; post_weight, post_bias)), H = N(Y; next_weight, next_bias), with `norm` "rms" or
    "layer" for both; enqueues on the stream.  F is not normalised without `post_weight`, H is None without `next_weight`; `gate`
    is [D], or [B,D] for a row per sequence; `p`, `seed`, `offset` and `step` are those of cotten_dropout.  Y may be X and H may be F."""
    lib = _lib or load_library()
    prm = _residual_params(X, F, norm, post_weight, post_bias, gate, alpha, next_weight, next_bias, eps, p, seed, offset, step)
    if Y is None:
        Y = torch.empty_like(X)
    else:
        _check_like("Y", Y, X.shape, X.dtype, X.device)
    if next_weight is None:
        if H is not None:
            raise ValueError("H comes from next_weight")
    elif H is None:
        H = torch.empty_like(X)
    else:
        _check_like("H", H, X.shape, X.dtype, X.device)
    dev = X.device
    _on_device(dev, lib.cotten_residual_fwd, X.data_ptr(), F.data_ptr(), Y.data_ptr(), None if H is None else H.data_ptr(),
               *X.shape, _stream_handle(stream, dev), ctypes.byref(prm))
    return Y, H


def cotten_residual_bwd(X: torch.Tensor, F: torch.Tensor, dY: Optional[torch.Tensor], dH: Optional[torch.Tensor], *,
                        norm: str = "rms", post_weight: Optional[torch.Tensor] = None,
                        post_bias: Optional[torch.Tensor] = None, gate: Optional[torch.Tensor] = None, alpha: float = 1.0,
                        next_weight: Optional[torch.Tensor] = None, next_bias: Optional[torch.Tensor] = None,
                        eps: Optional[float] = None, p: float = 0.0, seed: int = 0, offset: int = 0,
                        step: Optional[torch.Tensor] = None, stream=None, workspace: Optional[torch.Tensor] = None,
                        wanted: Tuple[bool, bool, bool, bool, bool] = (True,) * 5):
    """(dX, dF, dpost_weight, dpost_bias, dgate, dnext_weight, dnext_bias) of the forward call with the same arguments for the
    upstream gradients dY and dH (None: zeros; not both); None for what the call does not have.  `wanted`: which of the
    last five are."""
    lib = _lib or load_library()
    prm = _residual_params(X, F, norm, post_weight, post_bias, gate, alpha, next_weight, next_bias, eps, p, seed, offset, step)
    if dY is None and dH is None:
        raise ValueError("dY or dH must be given")
    if dH is not None and next_weight is None:
        raise ValueError("dH goes with next_weight")
    for name, t in (("dY", dY), ("dH", dH)):
        if t is not None:
            _check_like(name, t, X.shape, X.dtype, X.device)
    return _residual_backward(prm, _stream_handle(stream, X.device), workspace, X, F, dY, dH,
                              (post_weight, post_bias, gate, next_weight, next_bias), wanted)


def _residual_backward_of(call, X, F, dY, dH, vectors, step, wanted):
    """The gradients of a forward call that has checked its tensors (the differentiable function's): `call` is its norm, alpha,
    eps, p, seed and offset."""
    norm, alpha, eps, p, seed, offset = call
    gate = vectors[2]
    prm = CottenResidualParams(_dtype_code(X), _NORMS[norm], *(None if t is None else t.data_ptr() for t in vectors),
                               int(gate is not None and gate.dim() == 2), alpha, -1.0 if eps is None else eps, p, seed, offset,
                               None if step is None else step.data_ptr())
    return _residual_backward(prm, _stream_handle(None, X.device), None, X, F, dY, dH, vectors, wanted)


def _residual_backward(prm, handle, workspace, X, F, dY, dH, vectors, wanted):
    """The call itself: everything but the workspace is checked."""
    if workspace is None:
        workspace = _workspace(X, cotten_residual_workspace_bytes(*X.shape, bool(prm.gate_per_sequence)), handle)
    prm.workspace, prm.workspace_bytes = _buffer("workspace", workspace, X.device)
    dX, dF = torch.empty_like(X), torch.empty_like(X)
    grads = [torch.empty_like(t) if t is not None and w else None for t, w in zip(vectors, wanted)]
    to = CottenResidualGrads(*(None if t is None else t.data_ptr() for t in grads))
    _on_device(X.device, _lib.cotten_residual_bwd, X.data_ptr(), F.data_ptr(), None if dY is None else dY.data_ptr(),
               None if dH is None else dH.data_ptr(), dX.data_ptr(), dF.data_ptr(), *X.shape, handle, ctypes.byref(prm),
               ctypes.byref(to))
    return (dX, dF, *grads)


# ---- a step of a beam search -----------------------------------------------------------------------------

@functools.lru_cache(maxsize=1024)
def cotten_beam_workspace_bytes(B: int, K: int, V: int) -> int:
    return int(load_library().cotten_beam_workspace_bytes(B, K, V))


def _of_beams(name: str, t: torch.Tensor, dtype: torch.dtype, shape, dev) -> int:
    if t.dtype is not dtype or t.shape != shape or t.device != dev or not t.is_contiguous():
        raise ValueError(f"{name} must be a contiguous {dtype} tensor of shape {tuple(shape)} on the same device")
    return t.data_ptr()


def cotten_beam_select(logits: torch.Tensor, scores: torch.Tensor, *, finished: Optional[torch.Tensor] = None, pad: int = 0,
                       new_scores: Optional[torch.Tensor] = None, parents: Optional[torch.Tensor] = None,
                       tokens: Optional[torch.Tensor] = None, stream=None, workspace: Optional[torch.Tensor] = None
                       ) -> Tuple[torch.Tensor, torch.Tensor, torch.Tensor]:
    """(new_scores, parents, tokens), each [B,K]: of every sequence the K best of scores[k] + log_softmax(logits[k])[v], in falling
    order, the lower k * V + v of equal ones first; parents says which beam is continued, tokens with which item (int32).  `logits`
    [B,K,V], `scores` [B,K] float32; a beam that is not 0 in `finished` ([B,K] uint8) goes on with the item `pad` alone, at its
    score.  `new_scores` may be `scores`."""
    lib = _lib or load_library()
    if not (logits.is_cuda and logits.is_contiguous()):
        raise ValueError("logits must be a contiguous GPU tensor (there is no CPU path)")
    if logits.dim() != 3:
        raise ValueError("logits must be [B,K,V]")
    B, K, V = logits.shape
    if max(B, K, V) > _MOST_INT or not 0 <= pad <= _MOST_INT:
        raise ValueError("sizes and pad must be numbers of 31 bits")
    dev, shape, dtype = logits.device, logits.shape[:2], _dtype_code(logits)
    given = [_of_beams("scores", scores, torch.float32, shape, dev),
             None if finished is None else _of_beams("finished", finished, torch.uint8, shape, dev)]
    results = []
    for name, t, of in (("new_scores", new_scores, torch.float32), ("parents", parents, torch.int32), ("tokens", tokens, torch.int32)):
        if t is None:
            t = torch.empty_like(scores) if of is torch.float32 else torch.empty_like(scores, dtype=of)
            given.append(t.data_ptr())
        else:
            given.append(_of_beams(name, t, of, shape, dev))
        results.append(t)
    handle = _stream_handle(stream, dev)
    if workspace is None:
        workspace = _workspace(logits, cotten_beam_workspace_bytes(B, K, V), handle)
        prm = CottenBeamParams(dtype, pad, workspace.data_ptr(), workspace.numel())
    else:
        prm = CottenBeamParams(dtype, pad, *_buffer("workspace", workspace, dev))
    _on_device(dev, lib.cotten_beam_select, logits.data_ptr(), *given, B, K, V, handle, ctypes.byref(prm))
    return tuple(results)


def cotten_beam_reorder(state: torch.Tensor, parents: torch.Tensor, *, stream=None) -> torch.Tensor:
    """state[b,k] <- state[b,parents[b,k]] in place, for any contiguous [B,K,...] tensor (or [B*K,...]): states of the gated delta
    rule and of the decay attention, histories, flags.  `parents` [B,K] int32, as cotten_beam_select writes it."""
    lib = _lib or load_library()
    if not (state.is_cuda and state.is_contiguous()):
        raise ValueError("state must be a contiguous GPU tensor (there is no CPU path)")
    if parents.dim() != 2:
        raise ValueError("parents must be [B,K]")
    B, K = parents.shape
    _of_beams("parents", parents, torch.int32, parents.shape, state.device)
    if state.shape[:2] != parents.shape and state.shape[:1] != (B * K,):
        raise ValueError(f"state must be [{B},{K},...] or [{B * K},...]")
    if state.numel() == 0:
        return state
    _on_device(state.device, lib.cotten_beam_reorder, state.data_ptr(), parents.data_ptr(), B, K,
               state.numel() // (B * K) * state.element_size(), _stream_handle(stream, state.device))
    return state
