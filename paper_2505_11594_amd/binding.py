"""Thin ctypes binding over ``libsage_mi355x.so`` (declared in include/sage_mi355x.h).

Argument marshalling only: every step of the attention path runs in the HIP
kernels.  torch supplies device memory and the current stream.  If the
library has not been built, ``lib()`` raises: there is no fallback path.
"""
from __future__ import annotations

import ctypes
import functools
import os
import struct

HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(HERE, "libsage_mi355x.so")

SAGE_OK, SAGE_ERR_INVALID_ARG, SAGE_ERR_UNSUPPORTED, SAGE_ERR_HIP, SAGE_ERR_WORKSPACE = 0, 1, 2, 3, 4
SAGE_FMT_MXFP4, SAGE_FMT_NV16_E4M3 = 0x0, 0x1
SAGE_IN_FP16, SAGE_IN_BF16 = 0x0, 0x4
SAGE_OUT_F32 = 0x8
SAGE_NO_SMOOTH_K = 0x10
SAGE_SMOOTH_Q = 0x20
SAGE_BKV64 = 0x40
SAGE_BKV256 = 0x80
SAGE_KV_FP4, SAGE_ROPE_PAIRS = 0x200, 0x400
SAGE_WG256 = 0x100       # 256 queries per workgroup (MXFP4, 256-key tiles, non-causal, no smoothing Q)


def bkv_flag(bkv: int) -> int:
    """The fmt bit that selects a KV tile of ``bkv`` keys (64, 128 or 256)."""
    return {64: SAGE_BKV64, 128: 0, 256: SAGE_BKV256}[bkv]
SAGE_ROLE_Q, SAGE_ROLE_K, SAGE_ROLE_V = 0, 1, 2

_lib = None


_strides = struct.Struct("@3q").pack      # sage_strides
_cache = struct.Struct("@4P6q4i").pack    # sage_kv_cache


class SageError(RuntimeError):
    def __init__(self, fn: str, status: int):
        super().__init__("%s failed: %s" % (fn, status_string(status)))
        self.status = status


def lib():
    """Load the in-tree HIP library (raises if it has not been built).

    torch is imported first: its wheel carries its own HIP runtime under the
    same soname as ROCm's, and the runtime loaded first is the one every
    later library binds to.  Loading this library before torch would map
    ROCm's runtime next to torch's, and device pointers and streams would
    cross between the two."""
    global _lib
    if _lib is None:
        import torch  # noqa: F401  (see above)
        if not os.path.exists(LIB_PATH):
            raise RuntimeError("libsage_mi355x.so is not built; run __graft_entry__.build() "
                               "or python paper_2505_11594_amd/build.py")
        L = ctypes.CDLL(LIB_PATH)
        vp, i, u, sz = ctypes.c_void_p, ctypes.c_int, ctypes.c_uint, ctypes.c_size_t
        L.sage_quant_sizes.argtypes = [i, i, i, i, i, u, ctypes.POINTER(sz), ctypes.POINTER(sz)]
        L.sage_quant_workspace_size.argtypes = [i, i, i, i, i, u]
        L.sage_quant_workspace_size.restype = sz
        L.sage_quant_fp4.argtypes = [vp, i, i, i, i, i, u, vp, vp, vp, vp, sz, vp]
        L.sage_attn_fp4_workspace_size.argtypes = [i, i, i, i, u]
        L.sage_attn_fp4_workspace_size.restype = sz
        L.sage_attn_fp4_fwd.argtypes = [vp, vp, vp, vp, i, i, i, i, i, u, vp]
        L.sage_attn_fp4_fwd_ws.argtypes = [vp, vp, vp, vp, i, i, i, i, i, u, vp, sz, vp]
        L.sage_attn_fp4_fwd_noalloc.argtypes = [vp, vp, vp, vp, i, i, i, i, i, u, vp]
        L.sage_attn_fp4_fwd_prequant.argtypes = [vp] * 7 + [i, i, i, i, i, u, vp]
        L.sage_attn_bf16_fwd.argtypes = [vp, vp, vp, vp, i, i, i, i, i, u, vp]
        L.sage_quant_int8_sizes.argtypes = [i, i, i, i, i, u, ctypes.POINTER(sz), ctypes.POINTER(sz)]
        L.sage_quant_int8.argtypes = [vp, i, i, i, i, i, u, vp, vp, vp, vp, sz, vp]
        L.sage_attn_int8_workspace_size.argtypes = [i, i, i, i, u]
        L.sage_attn_int8_workspace_size.restype = sz
        L.sage_attn_int8_fwd.argtypes = [vp, vp, vp, vp, vp, i, i, i, i, i, u, vp]
        L.sage_attn_int8_fwd_ws.argtypes = [vp, vp, vp, vp, vp, i, i, i, i, i, u, vp, sz, vp]
        L.sage_attn_int8_fwd_prequant.argtypes = [vp] * 8 + [i, i, i, i, i, u, vp]
        L.sage_attn_int8_bwd.argtypes = [vp] * 9 + [i, i, i, i, i, u, vp]
        L.sage_attn_int8_bwd_ws.argtypes = [vp] * 9 + [i, i, i, i, i, u, vp, sz, vp]
        L.sage_attn_int8_bwd_workspace_size.argtypes = [i, i, i, i, u]
        L.sage_attn_int8_bwd_workspace_size.restype = sz
        L.sage_attn_int8_bwd_min_workspace_size.argtypes = [i, i, i, i, u]
        L.sage_attn_int8_bwd_min_workspace_size.restype = sz
        i64, st, ca = ctypes.c_int64, vp, vp           # (sage_strides and sage_kv_cache by address)
        L.sage_attn_window_fwd.argtypes = [vp] * 6 + [i] * 7 + [u] + [st] * 4 + [vp]
        L.sage_attn_window_bwd_workspace_size.argtypes = [i] * 7
        L.sage_attn_window_bwd_workspace_size.restype = sz
        L.sage_attn_window_bwd.argtypes = [vp] * 10 + [i] * 7 + [u] + [st] * 5 + [vp, sz, vp]
        L.sage_kv_append.argtypes = [ca, vp, vp, st, st, vp, i, vp, vp, vp, i64, i, i, u, vp]
        L.sage_kv_append_slots.argtypes = [ca, vp, vp, st, st, vp, i, i, u, vp]
        f = ctypes.c_float
        L.sage_qk_norm_rope_fwd.argtypes = [vp] * 5 + [i, vp, i, vp, vp, vp] + [i] * 5 + [f, u] + [st] * 4 + [vp]
        L.sage_qk_norm_rope_bwd_workspace_size.argtypes = [i] * 5
        L.sage_qk_norm_rope_bwd_workspace_size.restype = sz
        L.sage_qk_norm_rope_bwd.argtypes = [vp] * 5 + [i, vp, i] + [vp] * 7 + [i] * 5 + [f, u] + [st] * 6 + [vp, sz, vp]
        L.sage_kv_plan.argtypes = [vp, i, vp, vp, vp, i, vp, i, vp, vp, vp, vp, i, i, vp]
        L.sage_attn_paged_decode_workspace_size.argtypes = [i] * 7
        L.sage_attn_paged_decode_workspace_size.restype = sz
        L.sage_attn_paged_decode.argtypes = [ca, vp, i64, i64, vp, vp, vp, i, vp, i, i, i, i, vp, i64, u, vp, sz, vp]
        L.sage_kv_evict_workspace_size.argtypes = [i] * 4
        L.sage_kv_evict_workspace_size.restype = sz
        L.sage_kv_evict.argtypes = [ca, vp, i, vp, vp, i64, vp, i, i, i, i, vp, vp, vp, i, vp, sz, vp]
        L.sage_kv_evict_fp4.argtypes = L.sage_kv_evict.argtypes
        L.sage_status_string.argtypes = [i]
        L.sage_status_string.restype = ctypes.c_char_p
        L.sage_version.restype = ctypes.c_char_p
        for name in ("sage_quant_sizes", "sage_quant_fp4", "sage_attn_fp4_fwd", "sage_attn_fp4_fwd_ws",
                     "sage_attn_fp4_fwd_noalloc", "sage_attn_fp4_fwd_prequant", "sage_attn_bf16_fwd", "sage_quant_int8_sizes",
                     "sage_quant_int8", "sage_attn_int8_fwd", "sage_attn_int8_fwd_ws",
                     "sage_attn_int8_fwd_prequant", "sage_attn_int8_bwd", "sage_attn_int8_bwd_ws",
                     "sage_attn_window_fwd", "sage_attn_window_bwd", "sage_kv_append", "sage_attn_paged_decode", "sage_kv_evict",
                     "sage_kv_evict_fp4", "sage_kv_append_slots", "sage_qk_norm_rope_fwd", "sage_qk_norm_rope_bwd", "sage_kv_plan"):
            getattr(L, name).restype = i
        _lib = L
    return _lib


def status_string(status: int) -> str:
    return lib().sage_status_string(int(status)).decode()


def _check(fn: str, rc: int):
    if rc != SAGE_OK:
        raise SageError(fn, rc)


def _stream():
    import torch
    return ctypes.c_void_p(torch.cuda.current_stream().cuda_stream)


def _ptr(t):
    return ctypes.c_void_p(t.data_ptr()) if t is not None else None


_in_flags = {}


def _in_flag(t) -> int:
    flag = _in_flags.get(t.dtype)
    if flag is None:
        import torch
        _in_flags.update({torch.bfloat16: SAGE_IN_BF16, torch.float16: SAGE_IN_FP16})
        if t.dtype not in _in_flags:
            raise TypeError("inputs must be bf16 or fp16, got %s" % t.dtype)
        flag = _in_flags[t.dtype]
    return flag


def _shape(t):
    if t.dim() != 4 or not t.is_contiguous() or not t.is_cuda:
        raise ValueError("expected a contiguous 4-d [B, H, N, D] device tensor")
    return tuple(int(s) for s in t.shape)


def _check_qkv(q, k, v):
    """q, k and v must share shape, 16-bit dtype and device: the kernels read
    all three with q's element type and size."""
    shp = _shape(q)
    _in_flag(q)
    for t, what in ((k, "k"), (v, "v")):
        if _shape(t) != shp or t.dtype != q.dtype or t.device != q.device:
            raise ValueError("%s must match q: shape %s, dtype %s, device %s; got %s, %s, %s"
                             % (what, shp, q.dtype, q.device, tuple(t.shape), t.dtype, t.device))
    return shp


def _check_tensor(t, what: str, shape, dtype, device):
    """A caller-supplied buffer must match what the kernels will write or read
    (the C ABI receives bare pointers and cannot check it)."""
    if type(shape) is not tuple:                         # a caller's list never equals a torch.Size
        shape = tuple(shape)
    if t.dtype is not dtype or t.shape != shape or t.get_device() != device.index or not t.is_contiguous():
        raise ValueError("%s must be a contiguous %s tensor of shape %s on %s, got %s %s on %s"
                         % (what, dtype, tuple(shape), device, t.dtype, tuple(t.shape), t.device))


def _check_workspace(ws, device):
    import torch
    if ws.dtype != torch.uint8 or ws.dim() != 1 or not ws.is_contiguous() or ws.device != device:
        raise ValueError("workspace must be a contiguous 1-d uint8 tensor on %s" % device)


def _check_quantized(pair, what: str, nbytes, device):
    import torch
    for t, n, part in zip(pair[:2], nbytes, ("codes", "scales")):
        if t.dtype != torch.uint8 or not t.is_contiguous() or t.device != device or t.numel() != n:
            raise ValueError("%s %s must be %d contiguous uint8 bytes on %s" % (what, part, n, device))


def quant_sizes(role: int, B: int, H: int, N: int, D: int, fmt: int):
    c, s = ctypes.c_size_t(), ctypes.c_size_t()
    _check("sage_quant_sizes", lib().sage_quant_sizes(role, B, H, N, D, fmt, ctypes.byref(c), ctypes.byref(s)))
    return c.value, s.value


def sage_quant_fp4(x, role: int, fmt: int = SAGE_FMT_MXFP4):
    """Quantize one tensor; returns (codes uint8, scales uint8, mean fp32 or None) on the device:
    role K with smoothing K: the channel mean [B,H,D]; role Q with SAGE_SMOOTH_Q: the query-block
    means [B,H,ceil(N/128),D]."""
    import torch
    B, H, N, D = _shape(x)
    fmt = fmt | _in_flag(x)
    cb, sb = quant_sizes(role, B, H, N, D, fmt)
    codes = torch.empty(cb, dtype=torch.uint8, device=x.device)
    scales = torch.empty(sb, dtype=torch.uint8, device=x.device)
    kmean = None
    ws = None
    if role == SAGE_ROLE_Q and (fmt & SAGE_SMOOTH_Q):
        kmean = torch.empty((B, H, (N + 127) // 128, D), dtype=torch.float32, device=x.device)
    if role == SAGE_ROLE_K and not (fmt & SAGE_NO_SMOOTH_K):
        kmean = torch.empty((B, H, D), dtype=torch.float32, device=x.device)
        wsb = int(lib().sage_quant_workspace_size(role, B, H, N, D, fmt))
        ws = torch.empty(max(wsb, 8), dtype=torch.uint8, device=x.device)
    _check("sage_quant_fp4", lib().sage_quant_fp4(_ptr(x), role, B, H, N, D, fmt, _ptr(codes), _ptr(scales),
                                                  _ptr(kmean), _ptr(ws), ws.numel() if ws is not None else 0,
                                                  _stream()))
    return codes, scales, kmean


def attn_fp4_workspace_size(B: int, H: int, N: int, D: int, fmt: int) -> int:
    return int(lib().sage_attn_fp4_workspace_size(B, H, N, D, fmt))


def _out(q, out_f32: bool):
    import torch
    return torch.empty(q.shape, dtype=torch.float32 if out_f32 else q.dtype, device=q.device)


def _check_o(o, q, out_f32: bool):
    import torch
    _check_tensor(o, "out", q.shape, torch.float32 if out_f32 else q.dtype, q.device)


def sage_attn_fp4_fwd(q, k, v, causal: bool = False, fmt: int = SAGE_FMT_MXFP4, out_f32: bool = True,
                      out=None, workspace=None):
    """O = attention(Q, K, V) through the FP4 path.  With ``workspace`` (a uint8 device
    tensor of at least attn_fp4_workspace_size bytes) no allocation happens inside."""
    B, H, N, D = _check_qkv(q, k, v)
    fmt = fmt | _in_flag(q) | (SAGE_OUT_F32 if out_f32 else 0)
    o = _out(q, out_f32) if out is None else out
    _check_o(o, q, out_f32)
    if workspace is not None:
        _check_workspace(workspace, q.device)
    if workspace is None:
        rc = lib().sage_attn_fp4_fwd(_ptr(q), _ptr(k), _ptr(v), _ptr(o), B, H, N, D, int(bool(causal)), fmt, _stream())
        _check("sage_attn_fp4_fwd", rc)
    else:
        rc = lib().sage_attn_fp4_fwd_ws(_ptr(q), _ptr(k), _ptr(v), _ptr(o), B, H, N, D, int(bool(causal)), fmt,
                                        _ptr(workspace), workspace.numel(), _stream())
        _check("sage_attn_fp4_fwd_ws", rc)
    return o


def sage_attn_fp4_fwd_noalloc(q, k, v, causal: bool = False, fmt: int = SAGE_FMT_MXFP4, out_f32: bool = True,
                              out=None):
    """sage_attn_fp4_fwd on the library's fixed per-GPU scratch (no device allocation
    inside the C call; ``out`` may be preallocated).  Calls that overlap on one GPU race."""
    B, H, N, D = _check_qkv(q, k, v)
    fmt = fmt | _in_flag(q) | (SAGE_OUT_F32 if out_f32 else 0)
    o = _out(q, out_f32) if out is None else out
    _check_o(o, q, out_f32)
    rc = lib().sage_attn_fp4_fwd_noalloc(_ptr(q), _ptr(k), _ptr(v), _ptr(o), B, H, N, D, int(bool(causal)), fmt,
                                         _stream())
    _check("sage_attn_fp4_fwd_noalloc", rc)
    return o


def sage_attn_fp4_fwd_prequant(qq, kq, vq, shape, causal: bool = False, fmt: int = SAGE_FMT_MXFP4,
                               in_bf16: bool = True, out_f32: bool = True, out=None):
    """Attention kernel alone on (codes, scales) pairs from sage_quant_fp4."""
    import torch
    B, H, N, D = shape
    fmt = fmt | (SAGE_IN_BF16 if in_bf16 else SAGE_IN_FP16) | (SAGE_OUT_F32 if out_f32 else 0)
    dev = qq[0].device
    for pair, role, what in ((qq, SAGE_ROLE_Q, "q"), (kq, SAGE_ROLE_K, "k"), (vq, SAGE_ROLE_V, "v")):
        _check_quantized(pair, what, quant_sizes(role, B, H, N, D, fmt), dev)
    odt = torch.float32 if out_f32 else (torch.bfloat16 if in_bf16 else torch.float16)
    if out is None:
        out = torch.empty(shape, dtype=odt, device=dev)
    _check_tensor(out, "out", shape, odt, dev)
    rc = lib().sage_attn_fp4_fwd_prequant(_ptr(qq[0]), _ptr(qq[1]), _ptr(kq[0]), _ptr(kq[1]), _ptr(vq[0]),
                                          _ptr(vq[1]), _ptr(out), B, H, N, D, int(bool(causal)), fmt, _stream())
    _check("sage_attn_fp4_fwd_prequant", rc)
    return out


def sage_attn_bf16_fwd(q, k, v, causal: bool = False, out_f32: bool = True, out=None):
    """bf16-MFMA comparison kernel of the same structure."""
    B, H, N, D = _check_qkv(q, k, v)
    flags = _in_flag(q) | (SAGE_OUT_F32 if out_f32 else 0)
    o = _out(q, out_f32) if out is None else out
    _check_o(o, q, out_f32)
    rc = lib().sage_attn_bf16_fwd(_ptr(q), _ptr(k), _ptr(v), _ptr(o), B, H, N, D, int(bool(causal)), flags, _stream())
    _check("sage_attn_bf16_fwd", rc)
    return o


# ---------------------------------------------------------------- 8-bit attention
def quant_int8_sizes(role: int, B: int, H: int, N: int, D: int, flags: int = 0):
    c, s = ctypes.c_size_t(), ctypes.c_size_t()
    _check("sage_quant_int8_sizes",
           lib().sage_quant_int8_sizes(role, B, H, N, D, flags, ctypes.byref(c), ctypes.byref(s)))
    return c.value, s.value


def sage_quant_int8(x, role: int, flags: int = 0):
    """psi for one role; returns (codes int8, scales fp32, mean fp32 or None) on the device
    (role K with smoothing K: the channel mean [B,H,D])."""
    import torch
    B, H, N, D = _shape(x)
    flags = flags | _in_flag(x)
    cb, sb = quant_int8_sizes(role, B, H, N, D, flags)
    codes = torch.empty(cb, dtype=torch.int8, device=x.device)
    scales = torch.empty(sb // 4, dtype=torch.float32, device=x.device)
    kmean, ws = None, None
    if role == SAGE_ROLE_K and not (flags & SAGE_NO_SMOOTH_K):
        kmean = torch.empty((B, H, D), dtype=torch.float32, device=x.device)
        wsb = int(lib().sage_quant_workspace_size(role, B, H, N, D, 0))
        ws = torch.empty(max(wsb, 8), dtype=torch.uint8, device=x.device)
    _check("sage_quant_int8", lib().sage_quant_int8(_ptr(x), role, B, H, N, D, flags, _ptr(codes), _ptr(scales),
                                                    _ptr(kmean), _ptr(ws), ws.numel() if ws is not None else 0,
                                                    _stream()))
    return codes, scales, kmean


def attn_int8_workspace_size(B: int, H: int, N: int, D: int, flags: int = 0) -> int:
    return int(lib().sage_attn_int8_workspace_size(B, H, N, D, flags))


def sage_attn_int8_fwd(q, k, v, causal: bool = False, flags: int = 0, out_f32: bool = True, lse: bool = True,
                       out=None, lse_out=None, workspace=None):
    """Algorithm 2's 8-bit attention forward.  Returns (O, L) with L = m + log l
    [B,H,N] fp32 (None when ``lse`` is False).  With ``workspace`` (uint8, at
    least attn_int8_workspace_size bytes) no allocation happens inside."""
    import torch
    B, H, N, D = _check_qkv(q, k, v)
    flags = flags | _in_flag(q) | (SAGE_OUT_F32 if out_f32 else 0)
    o = _out(q, out_f32) if out is None else out
    _check_o(o, q, out_f32)
    L = None
    if lse:
        L = torch.empty((B, H, N), dtype=torch.float32, device=q.device) if lse_out is None else lse_out
        _check_tensor(L, "lse_out", (B, H, N), torch.float32, q.device)
    if workspace is not None:
        _check_workspace(workspace, q.device)
    if workspace is None:
        rc = lib().sage_attn_int8_fwd(_ptr(q), _ptr(k), _ptr(v), _ptr(o), _ptr(L), B, H, N, D, int(bool(causal)),
                                      flags, _stream())
        _check("sage_attn_int8_fwd", rc)
    else:
        rc = lib().sage_attn_int8_fwd_ws(_ptr(q), _ptr(k), _ptr(v), _ptr(o), _ptr(L), B, H, N, D, int(bool(causal)),
                                         flags, _ptr(workspace), workspace.numel(), _stream())
        _check("sage_attn_int8_fwd_ws", rc)
    return o, L


def sage_attn_int8_fwd_prequant(qq, kq, vq, shape, causal: bool = False, in_bf16: bool = True,
                                out_f32: bool = True, lse: bool = True, flags: int = 0):
    """The 8-bit attention kernel alone on (codes, scales) pairs from sage_quant_int8
    (flags: SAGE_BKV64 as given to sage_quant_int8)."""
    import torch
    B, H, N, D = shape
    flags = flags | (SAGE_IN_BF16 if in_bf16 else SAGE_IN_FP16) | (SAGE_OUT_F32 if out_f32 else 0)
    dev = qq[0].device
    for pair, role, what in ((qq, SAGE_ROLE_Q, "q"), (kq, SAGE_ROLE_K, "k"), (vq, SAGE_ROLE_V, "v")):
        cb, sb = quant_int8_sizes(role, B, H, N, D, flags & SAGE_BKV64)
        for t, n, part, dt in ((pair[0], cb, "codes", torch.int8), (pair[1], sb // 4, "scales", torch.float32)):
            if t.dtype != dt or not t.is_contiguous() or t.device != dev or t.numel() != n:
                raise ValueError("%s %s must be %d contiguous %s elements on %s" % (what, part, n, dt, dev))
    out = torch.empty(shape, dtype=torch.float32 if out_f32 else (torch.bfloat16 if in_bf16 else torch.float16),
                      device=dev)
    L = torch.empty((B, H, N), dtype=torch.float32, device=dev) if lse else None
    rc = lib().sage_attn_int8_fwd_prequant(_ptr(qq[0]), _ptr(qq[1]), _ptr(kq[0]), _ptr(kq[1]), _ptr(vq[0]),
                                           _ptr(vq[1]), _ptr(out), _ptr(L), B, H, N, D, int(bool(causal)), flags,
                                           _stream())
    _check("sage_attn_int8_fwd_prequant", rc)
    return out, L


def attn_int8_bwd_workspace_size(B: int, H: int, N: int, D: int, flags: int = 0) -> int:
    return int(lib().sage_attn_int8_bwd_workspace_size(B, H, N, D, flags))


def attn_int8_bwd_min_workspace_size(B: int, H: int, N: int, D: int, flags: int = 0) -> int:
    return int(lib().sage_attn_int8_bwd_min_workspace_size(B, H, N, D, flags))


def sage_attn_int8_bwd(q, k, v, o, lse, dout, causal: bool = False, flags: int = 0, workspace=None, out=None):
    """Algorithm 3's 8-bit attention backward: returns (dQ, dK, dV) fp32 [B,H,N,D].
    o, lse: the forward's fp32 output and L.  ``out``: three preallocated fp32
    tensors; with ``workspace`` nothing is allocated inside."""
    import torch
    B, H, N, D = _shape(q)
    for t in (k, v, dout):
        if _shape(t) != (B, H, N, D) or t.dtype != q.dtype:
            raise ValueError("q, k, v, dout must have the same shape and dtype")
    if _shape(o) != (B, H, N, D) or o.dtype != torch.float32:
        raise ValueError("o must be the fp32 forward output")
    if tuple(lse.shape) != (B, H, N) or lse.dtype != torch.float32 or not lse.is_contiguous():
        raise ValueError("lse must be fp32 [B,H,N]")
    for t, what in ((k, "k"), (v, "v"), (dout, "dout"), (o, "o"), (lse, "lse")):
        if t.device != q.device:
            raise ValueError("%s must be on %s" % (what, q.device))
    flags = flags | _in_flag(q)
    dq, dk, dv = out if out is not None else [torch.empty((B, H, N, D), dtype=torch.float32, device=q.device)
                                              for _ in range(3)]
    for t, what in ((dq, "dq"), (dk, "dk"), (dv, "dv")):
        _check_tensor(t, what, (B, H, N, D), torch.float32, q.device)
    if workspace is not None:
        _check_workspace(workspace, q.device)
    ptrs = [_ptr(t) for t in (q, k, v, o, lse, dout, dq, dk, dv)]
    if workspace is None:
        _check("sage_attn_int8_bwd", lib().sage_attn_int8_bwd(*ptrs, B, H, N, D, int(bool(causal)), flags, _stream()))
    else:
        _check("sage_attn_int8_bwd_ws", lib().sage_attn_int8_bwd_ws(*ptrs, B, H, N, D, int(bool(causal)), flags,
                                                                  _ptr(workspace), workspace.numel(), _stream()))
    return dq, dk, dv


# ------------------------------------------------- sliding window, paged cache, one-token attention
_NO_WINDOW = 2 ** 31 - 1


_calls = {}


def _call(fn: str, device, *args):
    """The C call on ``device`` and its current stream."""
    f = _calls.get(fn)
    if f is None:
        import torch
        _calls[""] = torch                               # first: who finds the function takes this too
        f = _calls[fn] = getattr(lib(), fn)
    torch = _calls[""]
    index = device.index
    stream = torch._C._cuda_getCurrentRawStream(index)
    if torch._C._cuda_getDevice() == index:
        rc = f(*args, stream)
    else:
        with torch.cuda.device(device):
            rc = f(*args, stream)
    if rc != SAGE_OK:
        raise SageError(fn, rc)


def _adr(t):
    return t.data_ptr() if t is not None else None


def _rows(t, what: str, ndim: int = 4):
    """A strided tensor with contiguous channels whose rows start on 16 bytes: its strides but the
    last (of a dimension of size 1, whose stride is never used, 0)."""
    n, s = t.shape, t.stride()
    if len(n) != ndim or not t.is_cuda or 0 in n:
        raise ValueError("%s must be a non-empty %d-d device tensor, got shape %s on %s"
                         % (what, ndim, tuple(n), t.device))
    if ndim == 4:
        x, y, z, c = s
        if n[2] == 1:
            z = 0
    else:
        (x, y, c), z = s, 0
    if n[0] == 1:
        x = 0
    if n[1] == 1:
        y = 0
    if c != 1 or t.data_ptr() & 15 or (x | y | z) & (16 // t.itemsize - 1):
        raise ValueError("%s must have contiguous channels and rows on 16-byte addresses, got strides %s"
                         % (what, tuple(s)))
    return (x, y, z) if ndim == 4 else (x, y)


def _same(t, like, what: str, shape):
    if t.dtype is not like.dtype or t.shape != shape or t.get_device() != like.get_device():
        raise ValueError("%s must be a %s tensor of shape %s on %s, got %s %s on %s"
                         % (what, like.dtype, tuple(shape), like.device, t.dtype, tuple(t.shape), t.device))


def _window_of(window, sinks: int):
    window = _NO_WINDOW if window is None else int(window)
    if window < 1 or sinks < 0:
        raise ValueError("window must be at least 1 (None: no window) and sinks at least 0")
    return min(window, _NO_WINDOW), min(int(sinks), _NO_WINDOW)


def _check_window_args(q, k, v, lens):
    import torch
    qs, ks, vs = _rows(q, "q"), _rows(k, "k"), _rows(v, "v")
    B, Hq, N, D = q.shape
    Hkv = k.shape[1]
    if Hq % Hkv:
        raise ValueError("q's %d heads are no multiple of k's %d" % (Hq, Hkv))
    for t, what in ((k, "k"), (v, "v")):
        _same(t, q, what, (B, Hkv, N, D))
    if lens is not None:
        _check_tensor(lens, "lens", (B,), torch.int32, q.device)
    return (B, Hq, Hkv, N, D), [_strides(*x) for x in (qs, ks, vs)]


def sage_attn_window_fwd(q, k, v, window=None, sinks: int = 0, lens=None, lse: bool = True, out=None, lse_out=None):
    """Causal attention in which a query sees the last ``window`` keys (its own among them; None:
    all) and the first ``sinks``.  q [B, Hq, N, D], k and v [B, Hkv, N, D] 16-bit, any strides with
    contiguous channels; Hq a multiple of Hkv.  ``lens``: int32 [B], the tokens of a padded batch's
    sequences.  Returns (O, L): O like q (``out`` may have other strides), L fp32 [B, Hq, N] (None
    when ``lse`` is False); rows behind a sequence's end are 0 and -inf."""
    import torch
    flags = _in_flag(q)
    (B, Hq, Hkv, N, D), st = _check_window_args(q, k, v, lens)
    window, sinks = _window_of(window, sinks)
    o = torch.empty((B, Hq, N, D), dtype=q.dtype, device=q.device) if out is None else out
    _same(o, q, "out", (B, Hq, N, D))
    st.append(_strides(*_rows(o, "out")))
    L = None
    if lse:
        L = torch.empty((B, Hq, N), dtype=torch.float32, device=q.device) if lse_out is None else lse_out
        _check_tensor(L, "lse_out", (B, Hq, N), torch.float32, q.device)
    _call("sage_attn_window_fwd", q.device, _adr(q), _adr(k), _adr(v), _adr(o), _adr(L), _adr(lens), B, Hq, Hkv, N, D,
          window, sinks, flags, *st)
    return o, L


def attn_window_bwd_workspace_size(B: int, Hq: int, Hkv: int, N: int, D: int, window=None, sinks: int = 0) -> int:
    return int(lib().sage_attn_window_bwd_workspace_size(B, Hq, Hkv, N, D, *_window_of(window, sinks)))


def sage_attn_window_bwd(q, k, v, o, lse, dout, window=None, sinks: int = 0, lens=None, workspace=None, out=None):
    """The gradients (dQ, dK, dV) of sage_attn_window_fwd for dout, the gradient of its O; o and lse
    are its own outputs (not joined from parts of the keys), window, sinks and lens as given to it.  q, k, v, o, dout of any strides with
    contiguous channels; the gradients are contiguous, of q's type, dK and dV summed over a group's
    query heads.  ``out``: three preallocated tensors; with ``workspace`` (uint8, at least
    attn_window_bwd_workspace_size bytes) too nothing is allocated inside."""
    import torch
    flags = _in_flag(q)
    (B, Hq, Hkv, N, D), st = _check_window_args(q, k, v, lens)
    window, sinks = _window_of(window, sinks)
    for t, what in ((o, "o"), (dout, "dout")):
        _same(t, q, what, (B, Hq, N, D))
        st.append(_strides(*_rows(t, what)))
    _check_tensor(lse, "lse", (B, Hq, N), torch.float32, q.device)
    shapes = ((B, Hq, N, D), (B, Hkv, N, D), (B, Hkv, N, D))
    dq, dk, dv = out if out is not None else [torch.empty(s, dtype=q.dtype, device=q.device) for s in shapes]
    for t, s, what in zip((dq, dk, dv), shapes, ("dq", "dk", "dv")):
        _check_tensor(t, what, s, q.dtype, q.device)
    if workspace is None:
        n = attn_window_bwd_workspace_size(B, Hq, Hkv, N, D, window, sinks)
        workspace = torch.empty(max(n, 1), dtype=torch.uint8, device=q.device)
    _check_workspace(workspace, q.device)
    _call("sage_attn_window_bwd", q.device, *[_adr(t) for t in (q, k, v, o, lse, dout, lens, dq, dk, dv)], B, Hq, Hkv, N, D,
          window, sinks, flags, *st, _adr(workspace), workspace.numel())
    return dq, dk, dv


def _check_pages(k_cache, v_cache, k_scale, v_scale):
    """The C description of a paged cache, its flag, and (page_size, Hkv, D)."""
    import torch
    ks, vs = _rows(k_cache, "k_cache"), _rows(v_cache, "v_cache")
    P, Hkv, page, D = k_cache.shape
    _same(v_cache, k_cache, "v_cache", k_cache.shape)
    dev, fp4 = k_cache.device, k_cache.dtype == torch.uint8
    if (k_scale is None) != (v_scale is None) or (k_cache.dtype in (torch.int8, torch.uint8)) != (k_scale is not None):
        raise ValueError("an int8 or uint8 (MXFP4) cache has k_scale and v_scale, a 16-bit one has neither")
    if fp4:
        D *= 2
        _check_tensor(k_scale, "k_scale", (P, Hkv, page, D // 32), torch.uint8, dev)
        _check_tensor(v_scale, "v_scale", (P, Hkv, page, D // 32), torch.uint8, dev)
    elif k_scale is not None:
        _check_tensor(k_scale, "k_scale", (P, Hkv, page), torch.float32, dev)
        _check_tensor(v_scale, "v_scale", (P, Hkv, page), torch.float32, dev)
    else:
        _in_flag(k_cache)
    return _cache(k_cache.data_ptr(), v_cache.data_ptr(), _adr(k_scale) or 0, _adr(v_scale) or 0, *ks, *vs, P, page, Hkv, D), \
        SAGE_KV_FP4 if fp4 else 0, (page, Hkv, D)


def _check_cache(k_cache, v_cache, k_scale, v_scale, table):
    """The same with its tables: the C description, the flag, and (S, max_pages, page_size, Hkv, D)."""
    import torch
    c, kind, dims = _check_pages(k_cache, v_cache, k_scale, v_scale)
    if table.dim() != 2 or table.numel() == 0:
        raise ValueError("table must be a non-empty [S, max_pages] tensor")
    S, M = table.shape
    _check_tensor(table, "table", (S, M), torch.int32, k_cache.device)
    return c, kind, (S, M) + dims


def _check_weights(w, what: str, S: int, Hkv: int, capacity: int, device):
    import torch
    if w.dim() != 3 or w.shape[2] < capacity:
        raise ValueError("%s must be [S, Hkv, at least %d]" % (what, capacity))
    _check_tensor(w, what, (S, Hkv, w.shape[2]), torch.float32, device)


def sage_kv_append(k, v, k_cache, v_cache, table, pos, counts=None, k_scale=None, v_scale=None, weights=None):
    """Store new tokens in a paged cache: token t < counts[s] (None: all) of k, v [S, Hkv, N, D] at
    position pos[s] + t of sequence s.  The cache is [pages, Hkv, page_size, D] of any strides with
    contiguous channels, of k's type or int8 with fp32 scales [pages, Hkv, page_size], or MXFP4: uint8
    [pages, Hkv, page_size, D / 2] of two codes each with uint8 scales [pages, Hkv, page_size, D / 32].
    ``table`` int32 [S, max_pages] holds the sequences' pages.  ``weights`` [S, Hkv, >= max_pages *
    page_size] is set to 0 at the new tokens."""
    import torch
    c, kind, (S, M, page, Hkv, D) = _check_cache(k_cache, v_cache, k_scale, v_scale, table)
    flags = _in_flag(k) | kind
    ks, vs = _rows(k, "k"), _rows(v, "v")
    N, dev = int(k.shape[2]), k_cache.device
    _same(v, k, "v", (S, Hkv, N, D))
    _same(k, v, "k", (S, Hkv, N, D))
    if k.device != dev or (k_scale is None and k.dtype != k_cache.dtype):
        raise ValueError("k and v must be on %s and of the cache's type" % dev)
    _check_tensor(pos, "pos", (S,), torch.int32, dev)
    if counts is not None:
        _check_tensor(counts, "counts", (S,), torch.int32, dev)
    if weights is not None:
        _check_weights(weights, "weights", S, Hkv, M * page, dev)
    _call("sage_kv_append", dev, c, _adr(k), _adr(v), _strides(*ks), _strides(*vs), _adr(table), M, _adr(pos),
          _adr(counts), _adr(weights), weights.shape[2] if weights is not None else 0, S, N, flags)


def sage_kv_append_slots(k, v, k_cache, v_cache, slots, k_scale=None, v_scale=None):
    """Store new tokens in a paged cache (as in sage_kv_append) by slots, int64 [B, N] as sage_kv_plan
    gives them (page * page_size + place in the page; negative: not stored): token t of row b of k, v
    [B, Hkv, N, D].  The tokens of several sequences behind one another are one row, B = 1."""
    import torch
    c, kind, (page, Hkv, D) = _check_pages(k_cache, v_cache, k_scale, v_scale)
    flags, dev = _in_flag(k) | kind, k_cache.device
    ks, vs = _rows(k, "k"), _rows(v, "v")
    B, N = int(k.shape[0]), int(k.shape[2])
    _same(k, k, "k", (B, Hkv, N, D))
    _same(v, k, "v", (B, Hkv, N, D))
    if k.device != dev or (k_scale is None and k.dtype != k_cache.dtype):
        raise ValueError("k and v must be on %s and of the cache's type" % dev)
    _check_tensor(slots, "slots", (B, N), torch.int64, dev)
    _call("sage_kv_append_slots", dev, c, _adr(k), _adr(v), _strides(*ks), _strides(*vs), _adr(slots), B, N, flags)


@functools.lru_cache(maxsize=256)
def attn_paged_decode_workspace_size(S: int, Hq: int, Hkv: int, D: int, max_pages: int, page_size: int,
                                     weights: bool = False) -> int:
    return int(lib().sage_attn_paged_decode_workspace_size(S, Hq, Hkv, D, max_pages, page_size, int(bool(weights))))


def sage_attn_paged_decode(q, k_cache, v_cache, table, lens, window=None, sinks: int = 0, k_scale=None, v_scale=None,
                           weights=None, lse: bool = True, out=None, lse_out=None, workspace=None):
    """Attention of each sequence's last token, q [S, Hq, D], over its lens[s] cached tokens (its own
    among them); the cache as in sage_kv_append.  ``weights`` fp32 [S, Hkv, >= max_pages * page_size]:
    the attention weights, summed over a group's query heads, are added to it (this takes a workspace
    of 4 * S * Hq * max_pages * page_size bytes).  Returns (O, L), L fp32 [S, Hq] (None when ``lse``
    is False).  With ``workspace`` (uint8, at least attn_paged_decode_workspace_size bytes) and ``out``,
    ``lse_out`` nothing is allocated inside."""
    import torch
    c, kind, (S, M, page, Hkv, D) = _check_cache(k_cache, v_cache, k_scale, v_scale, table)
    flags, dev = _in_flag(q) | kind, k_cache.device
    qs = _rows(q, "q", 3)
    Hq = int(q.shape[1])
    if tuple(q.shape) != (S, Hq, D) or q.device != dev or (k_scale is None and q.dtype != k_cache.dtype):
        raise ValueError("q must be [%d, Hq, %d] of the cache's type on %s, got %s %s on %s"
                         % (S, D, dev, q.dtype, tuple(q.shape), q.device))
    if Hq % Hkv:
        raise ValueError("q's %d heads are no multiple of the cache's %d" % (Hq, Hkv))
    window, sinks = _window_of(window, sinks)
    _check_tensor(lens, "lens", (S,), torch.int32, dev)
    if weights is not None:
        _check_weights(weights, "weights", S, Hkv, M * page, dev)
    if out is None:
        o = q.new_empty((S, Hq, D))
    else:
        o = out
        _check_tensor(o, "out", (S, Hq, D), q.dtype, dev)
    L = None
    if lse and lse_out is None:
        L = q.new_empty((S, Hq), dtype=torch.float32)
    elif lse:
        L = lse_out
        _check_tensor(L, "lse_out", (S, Hq), torch.float32, dev)
    if workspace is None:
        n = attn_paged_decode_workspace_size(S, Hq, Hkv, D, M, page, weights is not None)
        workspace = torch.empty(n, dtype=torch.uint8, device=dev) if n else None
    else:
        _check_workspace(workspace, dev)
    _call("sage_attn_paged_decode", dev, c, _adr(q), qs[0], qs[1], _adr(o), _adr(L), _adr(table), M, _adr(lens),
          S, Hq, window, sinks, _adr(weights), weights.shape[2] if weights is not None else 0, flags, _adr(workspace),
          workspace.numel() if workspace is not None else 0)
    return o, L


def kv_evict_workspace_size(S: int, Hkv: int, max_pages: int, page_size: int) -> int:
    return int(lib().sage_kv_evict_workspace_size(S, Hkv, max_pages, page_size))


def sage_kv_evict(k_cache, v_cache, table, lens, weights, new_table, budget: int, keep_first: int = 0, keep_last: int = 0,
                  k_scale=None, v_scale=None, out=None, workspace=None):
    """Shorten cached sequences to ``budget`` tokens: the first keep_first, the last keep_last and the
    heaviest of those between by ``weights`` [S, Hkv, >= max_pages * page_size], per head, in their
    order; copied to the pages of ``new_table`` (int32 [S, new_max_pages]), which hold nothing else
    that the call moves.  Returns (new_lens [S], new_weights [S, Hkv, new_max_pages * page_size],
    kept [S, Hkv, budget]: the old positions, -1 behind the last).  With ``out`` (these three) and
    ``workspace`` (uint8, at least kv_evict_workspace_size bytes) nothing is allocated inside."""
    import torch
    c, kind, (S, M, page, Hkv, D) = _check_cache(k_cache, v_cache, k_scale, v_scale, table)
    dev = k_cache.device
    _check_tensor(lens, "lens", (S,), torch.int32, dev)
    _check_weights(weights, "weights", S, Hkv, M * page, dev)
    if new_table.dim() != 2 or new_table.numel() == 0:
        raise ValueError("new_table must be a non-empty [S, new_max_pages] tensor")
    M2 = int(new_table.shape[1])
    _check_tensor(new_table, "new_table", (S, M2), torch.int32, dev)
    if not (1 <= budget <= M2 * page) or keep_first < 0 or keep_last < 0 or keep_first + keep_last > budget:
        raise ValueError("budget must be at least 1, keep_first + keep_last and at most new_table's capacity")
    shapes = ((S,), (S, Hkv, M2 * page), (S, Hkv, budget))
    types = (torch.int32, torch.float32, torch.int32)
    new_lens, new_weights, kept = out if out is not None else [torch.empty(n, dtype=d, device=dev) for n, d in zip(shapes, types)]
    for t, n, d, what in zip((new_lens, new_weights, kept), shapes, types, ("new_lens", "new_weights", "kept")):
        _check_tensor(t, what, n, d, dev)
    if workspace is None:
        n = kv_evict_workspace_size(S, Hkv, M, page)
        workspace = torch.empty(n, dtype=torch.uint8, device=dev) if n else None
    else:
        _check_workspace(workspace, dev)
    _call("sage_kv_evict_fp4" if kind else "sage_kv_evict", dev, c, _adr(table), M, _adr(lens), _adr(weights),
          weights.shape[2], _adr(new_table), M2, budget, keep_first, keep_last, _adr(new_lens), _adr(new_weights), _adr(kept), S, _adr(workspace),
          workspace.numel() if workspace is not None else 0)
    return new_lens, new_weights, kept


# ------------------------------------------------- norms with rotation, page tables
_F32 = _I32 = None


def _check_norm_rope(q, k, q_weight, k_weight, inv_freq, pos, lens, eps, interleaved):
    """What forward and backward share: the C arguments up to lens, (B, Hq, Hkv, N, D), eps and flags, and the
    strides of q and k."""
    global _F32, _I32
    if _F32 is None:
        import torch
        _I32 = torch.int32                               # first: who finds _F32 takes this too
        _F32 = torch.float32
    flags = _in_flag(q)
    if interleaved:
        flags |= SAGE_ROPE_PAIRS
    st = [_strides(*_rows(q, "q")), _strides(*_rows(k, "k"))]
    B, Hq, N, D = q.shape
    Hkv, dev = k.shape[1], q.device
    if Hq % Hkv:
        raise ValueError("q's %d heads are no multiple of k's %d" % (Hq, Hkv))
    _same(k, q, "k", (B, Hkv, N, D))
    if q_weight is not None:
        _check_tensor(q_weight, "q_weight", (D,), _F32, dev)
    if k_weight is not None:
        _check_tensor(k_weight, "k_weight", (D,), _F32, dev)
    half = inv_freq.numel()
    if half > D // 2 or half % 4:
        raise ValueError("inv_freq must have at most %d entries, a multiple of 4, got %d" % (D // 2, half))
    _check_tensor(inv_freq, "inv_freq", (half,), _F32, dev)
    each = 0
    if pos is not None:
        each = int(pos.dim() == 2)
        _check_tensor(pos, "pos", (B, N) if each else (B,), _I32, dev)
    if lens is not None:
        _check_tensor(lens, "lens", (B,), _I32, dev)
    if not 2.0 ** -100 <= eps <= 1:
        raise ValueError("eps must be 2^-100 to 1, got %r" % (eps,))
    head = (q.data_ptr(), k.data_ptr(), _adr(q_weight), _adr(k_weight), inv_freq.data_ptr(), 2 * half, _adr(pos), each, _adr(lens))
    return head, (B, Hq, Hkv, N, D, eps, flags), st


def _like(out, tensors, names, strides):
    """Outputs like tensors: new ones, contiguous (no strides for the C call), or the caller's, checked."""
    if out is None:
        strides += [None] * len(tensors)
        return [t.new_empty(t.shape) for t in tensors]
    for t, x, what in zip(out, tensors, names):
        _same(t, x, what, x.shape)
        strides.append(_strides(*_rows(t, what)))
    return out


def sage_qk_norm_rope_fwd(q, k, q_weight, k_weight, inv_freq, pos=None, lens=None, eps: float = 1e-6,
                          interleaved: bool = False, out=None):
    """Each head's row of q [B, Hq, N, D] and k [B, Hkv, N, D] (16-bit, any strides with contiguous
    channels, views of one packed projection too) normed, x * (mean(x^2) + eps)^(-1/2) * weight, and
    its first 2 * len(inv_freq) channels rotated by position * inv_freq: channel i with i +
    len(inv_freq), or 2i with 2i + 1 if ``interleaved``.  Weights fp32 [D] or None; inv_freq fp32, a
    multiple of 4 entries.  ``pos``: int32 [B, N], or [B] for rows whose positions run on from these,
    or None (from 0 on).  ``lens``: int32 [B], the tokens of a padded batch's sequences; what lies
    behind is not read, and 0 in the outputs.  Returns both like q and k; ``out``: two tensors of any
    strides, which may be q and k themselves; other rows in common are refused."""
    head, tail, st = _check_norm_rope(q, k, q_weight, k_weight, inv_freq, pos, lens, eps, interleaved)
    zq, zk = _like(out, (q, k), ("out[0]", "out[1]"), st)
    _call("sage_qk_norm_rope_fwd", q.device, *head, zq.data_ptr(), zk.data_ptr(), *tail, *st)
    return zq, zk


@functools.lru_cache(maxsize=256)
def qk_norm_rope_bwd_workspace_size(B: int, Hq: int, Hkv: int, N: int, D: int) -> int:
    return int(lib().sage_qk_norm_rope_bwd_workspace_size(B, Hq, Hkv, N, D))


def sage_qk_norm_rope_bwd(q, k, q_weight, k_weight, inv_freq, dzq, dzk, pos=None, lens=None, eps: float = 1e-6,
                          interleaved: bool = False, workspace=None, out=None):
    """The gradients (dq, dk, dq_weight, dk_weight) of sage_qk_norm_rope_fwd for dzq and dzk, those of
    its outputs; all else as given to it.  dq and dk are like q and k (0 behind a sequence's end), those
    of the weights fp32 [D] (None for a weight that is None).  ``out``: four tensors (or None for the
    weights'), dq and dk of any strides, which may be dzq and dzk themselves; with ``workspace`` (uint8,
    at least qk_norm_rope_bwd_workspace_size bytes) too nothing is allocated inside."""
    import torch
    head, tail, st = _check_norm_rope(q, k, q_weight, k_weight, inv_freq, pos, lens, eps, interleaved)
    B, Hq, Hkv, N, D = tail[:5]
    dev = q.device
    _like((dzq, dzk), (q, k), ("dzq", "dzk"), st)
    if out is None:
        dwq, dwk = (q.new_empty(D, dtype=torch.float32) if w is not None else None for w in (q_weight, k_weight))
        dq, dk = _like(None, (q, k), None, st)
    else:
        dq, dk, dwq, dwk = out
        _like((dq, dk), (q, k), ("dq", "dk"), st)
        for w, what in ((dwq, "dq_weight"), (dwk, "dk_weight")):
            if w is not None:
                _check_tensor(w, what, (D,), torch.float32, dev)
    if workspace is None:
        workspace = q.new_empty(qk_norm_rope_bwd_workspace_size(B, Hq, Hkv, N, D), dtype=torch.uint8)
    else:
        _check_workspace(workspace, dev)
    _call("sage_qk_norm_rope_bwd", dev, *head, dzq.data_ptr(), dzk.data_ptr(), dq.data_ptr(), dk.data_ptr(), _adr(dwq), _adr(dwk),
          *tail, *st, workspace.data_ptr(), workspace.numel())
    return dq, dk, dwq, dwk


def sage_kv_plan(table, lens, counts, free_pages, n_free, page_size: int, max_tokens: int, out=None):
    """Pages and slots of a batch's next tokens: request s has lens[s] cached tokens and brings
    counts[s] (negative: it has ended, and its pages go back).  ``table`` int32 [S, max_pages], ``lens``
    int32 [S], the stack ``free_pages`` int32 and its height ``n_free`` int32 [1] are brought up to date in
    place; requests are granted in order as far as pages and ``max_tokens`` go.  Returns (granted [S],
    starts [S + 1], pos [max_tokens], slots int64 [max_tokens]): the tokens granted, their sums before
    each request, and each new token's position and slot (0 and -1 behind the last), for
    sage_qk_norm_rope_fwd and sage_kv_append_slots.  Tokens of all requests lie behind one another:
    sage_attn_paged_decode, which takes a row per request, wants row starts[s + 1] - 1 for request s (and
    what it gives for a request that was granted none says nothing).  With ``out`` (these four) nothing
    is allocated."""
    import torch
    if table.dim() != 2 or table.numel() == 0 or not table.is_cuda:
        raise ValueError("table must be a non-empty [S, max_pages] device tensor")
    S, M = table.shape
    dev = table.device
    _check_tensor(table, "table", (S, M), torch.int32, dev)
    _check_tensor(lens, "lens", (S,), torch.int32, dev)
    _check_tensor(counts, "counts", (S,), torch.int32, dev)
    _check_tensor(free_pages, "free_pages", (free_pages.numel(),), torch.int32, dev)
    _check_tensor(n_free, "n_free", (1,), torch.int32, dev)
    shapes, types = ((S,), (S + 1,), (max_tokens,), (max_tokens,)), (torch.int32,) * 3 + (torch.int64,)
    if page_size < 1 or max_tokens < 1 or free_pages.numel() == 0:
        raise ValueError("page_size, max_tokens and the capacity of free_pages must be at least 1")
    if out is None:
        granted, starts, pos, slots = [table.new_empty(n, dtype=d) for n, d in zip(shapes, types)]
    else:
        granted, starts, pos, slots = out
        for t, n, d, what in zip(out, shapes, types, ("granted", "starts", "pos", "slots")):
            _check_tensor(t, what, n, d, dev)
    _call("sage_kv_plan", dev, _adr(table), M, _adr(lens), _adr(counts), _adr(free_pages), free_pages.numel(), _adr(n_free),
          page_size, _adr(granted), _adr(starts), _adr(pos), _adr(slots), max_tokens, S)
    return granted, starts, pos, slots


def version() -> str:
    return lib().sage_version().decode()
