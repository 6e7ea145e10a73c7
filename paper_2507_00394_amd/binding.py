"""Thin ctypes binding of ``libhelix_attn.so``: argument marshalling only.

Every function has the name and argument order of its C entry point (see
``include/helix_attn.h``); tensors are torch device tensors whose ``data_ptr()`` is
handed over, and work is enqueued on torch's current stream.  There is no fallback: a
missing library raises ``HelixLibraryError`` on first use.
"""
from __future__ import annotations

import ctypes
import pathlib

import torch

LIB_PATH = pathlib.Path(__file__).resolve().parent / "csrc" / "libhelix_attn.so"
EXPORTS = ("helix_attn_fwd", "helix_attn_bwd", "helix_attn_bwd_static", "helix_attn_fwd_strided", "helix_attn_bwd_strided",
           "helix_attn_check_strides", "helix_qkv_linear_fwd", "helix_qkv_linear_bwd", "helix_qkv_linear_bwd_workspace_bytes",
           "helix_attn_bwd_workspace_bytes",
           "helix_attn_bwd_preprocess", "helix_attn_bwd_delta_head", "helix_attn_bwd_dkdv", "helix_attn_bwd_dq",
           "helix_dropout_add_fwd", "helix_dropout_add_bwd", "helix_layer_norm_fwd", "helix_layer_norm_bwd", "helix_layer_norm_bwd_workspace_bytes",
           "helix_dropout_add_layer_norm_fwd", "helix_dropout_add_layer_norm_bwd",
           "helix_gated_linear_fwd", "helix_gated_linear_bwd", "helix_gated_linear_bwd_workspace_bytes",
           "helix_attn_device_info", "helix_mfma_probe", "helix_mfma_mix_probe", "helix_status_string", "helix_attn_version")
HELIX_OK = 0
_lib = None


class helix_strides(ctypes.Structure):
    """Element strides (batch, head, row) of a logical [B, H, S, D] view; see the header."""
    _fields_ = [("batch", ctypes.c_longlong), ("head", ctypes.c_longlong), ("row", ctypes.c_longlong)]


class HelixLibraryError(RuntimeError):
    pass


class HelixStatusError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        super().__init__(f"{where}: {status_string(status)} (status {status})")


def lib() -> ctypes.CDLL:
    global _lib
    if _lib is None:
        if not LIB_PATH.exists():
            raise HelixLibraryError(f"{LIB_PATH} is not built; run `python -m paper_2507_00394_amd.build`")
        L = ctypes.CDLL(str(LIB_PATH))
        vp, fp, i, f, sz = ctypes.c_void_p, ctypes.c_void_p, ctypes.c_int, ctypes.c_float, ctypes.c_size_t
        L.helix_attn_fwd.argtypes = [vp, vp, vp, vp, fp, i, i, i, i, f, i, vp]
        L.helix_attn_bwd.argtypes = [vp, vp, vp, vp, fp, vp, vp, vp, vp, vp, sz, i, i, i, i, f, i, vp]
        L.helix_attn_bwd_static.argtypes = [vp, vp, vp, vp, fp, vp, vp, vp, vp, i, i, i, i, f, i, vp]
        L.helix_attn_bwd_static.restype = i
        sp = ctypes.POINTER(helix_strides)
        L.helix_attn_fwd_strided.argtypes = [vp, sp, vp, sp, vp, sp, vp, sp, fp, i, i, i, i, f, i, vp]
        L.helix_attn_bwd_strided.argtypes = [vp, sp, vp, sp, vp, sp, vp, sp, fp, vp, sp, vp, sp, vp, sp, vp, sp,
                                             vp, sz, i, i, i, i, f, i, vp]
        L.helix_attn_check_strides.argtypes = [sp, i, i, i, i]
        L.helix_attn_check_strides.restype = i
        ll = ctypes.c_longlong
        L.helix_qkv_linear_fwd.argtypes = [vp, ll, vp, ll, vp, ll, i, i, i, vp]
        L.helix_qkv_linear_bwd.argtypes = [vp, ll, vp, ll, vp, ll, vp, ll, fp, ll, vp, sz, i, i, i, vp]
        L.helix_qkv_linear_bwd_workspace_bytes.argtypes = [i, i, i]
        L.helix_qkv_linear_bwd_workspace_bytes.restype = sz
        L.helix_qkv_linear_fwd.restype = i
        L.helix_qkv_linear_bwd.restype = i
        L.helix_dropout_add_fwd.argtypes = [vp, ll, vp, ll, vp, ll, i, i, i, f, vp, ll, vp]
        L.helix_dropout_add_bwd.argtypes = [vp, ll, vp, ll, i, i, i, f, vp, ll, vp]
        L.helix_layer_norm_fwd.argtypes = [vp, ll, fp, fp, vp, ll, fp, fp, i, i, i, f, vp]
        L.helix_layer_norm_bwd.argtypes = [vp, ll, vp, ll, fp, fp, fp, vp, ll, fp, fp, vp, sz, i, i, i, vp]
        L.helix_layer_norm_bwd_workspace_bytes.argtypes = [i, i]
        L.helix_layer_norm_bwd_workspace_bytes.restype = sz
        L.helix_dropout_add_layer_norm_fwd.argtypes = [vp, ll, vp, ll, vp, ll, fp, fp, vp, ll, fp, fp, i, i, i, f, vp, ll, f, vp]
        L.helix_dropout_add_layer_norm_bwd.argtypes = [vp, ll, vp, ll, vp, ll, fp, fp, fp, vp, ll, vp, ll, fp, fp, vp, sz, i, i, i, f, vp, ll, vp]
        L.helix_gated_linear_fwd.argtypes = [vp, ll, vp, ll, vp, ll, vp, ll, i, i, i, i, vp]
        L.helix_gated_linear_bwd.argtypes = [vp, ll, vp, ll, vp, ll, vp, ll, vp, ll, vp, ll, vp, sz, i, i, i, i, vp]
        L.helix_gated_linear_bwd_workspace_bytes.argtypes = [i, i, i]
        L.helix_gated_linear_bwd_workspace_bytes.restype = sz
        for name in ("helix_gated_linear_fwd", "helix_gated_linear_bwd", "helix_dropout_add_fwd", "helix_dropout_add_bwd", "helix_layer_norm_fwd", "helix_layer_norm_bwd",
                     "helix_dropout_add_layer_norm_fwd", "helix_dropout_add_layer_norm_bwd"):
            getattr(L, name).restype = i
        L.helix_attn_bwd_workspace_bytes.argtypes = [i, i, i, i]
        L.helix_attn_bwd_workspace_bytes.restype = sz
        L.helix_attn_bwd_preprocess.argtypes = [vp, vp, fp, vp, i, i, i, i, vp]
        L.helix_attn_bwd_delta_head.argtypes = [vp, vp, vp, vp, fp, vp, i, i, i, i, i, f, i, vp]
        L.helix_attn_bwd_dkdv.argtypes = [vp, vp, vp, vp, vp, vp, vp, i, i, i, i, f, i, vp]
        L.helix_attn_bwd_dq.argtypes = [vp, vp, vp, vp, vp, vp, i, i, i, i, f, i, vp]
        L.helix_status_string.argtypes = [i]
        L.helix_status_string.restype = ctypes.c_char_p
        L.helix_attn_version.argtypes = []
        L.helix_attn_device_info.argtypes = [ctypes.POINTER(ctypes.c_int), ctypes.POINTER(ctypes.c_int)]
        L.helix_attn_device_info.restype = i
        L.helix_mfma_probe.argtypes = [fp, i, i, i, ctypes.POINTER(ctypes.c_longlong), vp]
        L.helix_mfma_probe.restype = i
        L.helix_mfma_mix_probe.argtypes = [fp, i, i, i, ctypes.POINTER(ctypes.c_longlong), vp]
        L.helix_mfma_mix_probe.restype = i
        for name in ("helix_attn_fwd", "helix_attn_bwd", "helix_attn_fwd_strided", "helix_attn_bwd_strided",
                     "helix_attn_bwd_preprocess", "helix_attn_bwd_delta_head",
                     "helix_attn_bwd_dkdv",
                     "helix_attn_bwd_dq", "helix_attn_version"):
            getattr(L, name).restype = i
        _lib = L
    return _lib


def status_string(status: int) -> str:
    return lib().helix_status_string(int(status)).decode()


# What a call does on the host beside its launches (3 us each) is most of a short call's time, so the helpers below are plain:
# pointers and streams go to ctypes as integers, shapes are compared as they are, and the current stream comes from torch's C
# layer (0.2 us against 2.9 for a Stream object).  us a call, launches included: forward 9.8 -> 6.3, backward 15.8 -> 11.2,
# linear layer forward 9.4 -> 5.5.
_BF16, _F32 = torch.bfloat16, torch.float32
_raw_stream, _device = getattr(torch._C, "_cuda_getCurrentRawStream", None), getattr(torch._C, "_cuda_getDevice", None)


def _ptr(t):
    return None if t is None else t.data_ptr()


def _stream(stream):
    if stream is not None:
        return stream.cuda_stream
    return _raw_stream(_device()) if _raw_stream and _device else torch.cuda.current_stream().cuda_stream


def _check_bf16(name, t, shape):
    if t.dtype is not _BF16 or not t.is_cuda or not t.is_contiguous() or t.shape != shape:
        raise ValueError(f"{name}: need a contiguous CUDA bfloat16 tensor of shape {tuple(shape)}")


def _check_f32(name, t, shape):
    if t.dtype is not _F32 or not t.is_cuda or not t.is_contiguous() or t.shape != shape:
        raise ValueError(f"{name}: need a contiguous CUDA float32 tensor of shape {tuple(shape)}")


def _raise(status, where):
    if status != HELIX_OK:
        raise HelixStatusError(status, where)


def helix_attn_version() -> int:
    return lib().helix_attn_version()


def helix_attn_device_info():
    """(compute units, peak engine clock in kHz) of the current device."""
    cu, khz = ctypes.c_int(0), ctypes.c_int(0)
    _raise(lib().helix_attn_device_info(ctypes.byref(cu), ctypes.byref(khz)), "helix_attn_device_info")
    return cu.value, khz.value


def helix_mfma_probe(sink, workgroups, iters, random_operands, stream=None) -> int:
    """Enqueues the pure MFMA loop; returns the FLOPs it performs.  `sink`: a CUDA float32 tensor with one element."""
    _check_f32("sink", sink, (1,))
    flops = ctypes.c_longlong(0)
    _raise(lib().helix_mfma_probe(_ptr(sink), int(workgroups), int(iters), int(bool(random_operands)), ctypes.byref(flops),
                                  _stream(stream)), "helix_mfma_probe")
    return flops.value


def helix_mfma_mix_probe(sink, workgroups, iters, forward_mix, stream=None) -> int:
    """Enqueues the MFMA loop with LDS reads and vector work beside it; returns the FLOPs it performs."""
    _check_f32("sink", sink, (1,))
    flops = ctypes.c_longlong(0)
    _raise(lib().helix_mfma_mix_probe(_ptr(sink), int(workgroups), int(iters), int(bool(forward_mix)), ctypes.byref(flops),
                                      _stream(stream)), "helix_mfma_mix_probe")
    return flops.value


def helix_attn_bwd_workspace_bytes(B, H, S, D) -> int:
    return int(lib().helix_attn_bwd_workspace_bytes(B, H, S, D))


def helix_attn_fwd(q, k, v, o, lse, scale, causal=True, stream=None):
    """o, lse <- attention forward of q, k, v ([B,H,S,D] bf16); lse is [B,H,S] fp32."""
    shape = B, H, S, D = q.shape
    for n, t in (("q", q), ("k", k), ("v", v), ("o", o)):
        _check_bf16(n, t, shape)
    _check_f32("lse", lse, (B, H, S))
    _raise(lib().helix_attn_fwd(_ptr(q), _ptr(k), _ptr(v), _ptr(o), _ptr(lse), B, H, S, D, float(scale), int(causal),
                                _stream(stream)), "helix_attn_fwd")


def helix_attn_bwd(q, k, v, o, lse, dO, dq, dk, dv, workspace, scale, causal=True, stream=None):
    """dq, dk, dv <- attention backward; workspace is a uint8 CUDA tensor of the required size."""
    shape = B, H, S, D = q.shape
    for n, t in (("q", q), ("k", k), ("v", v), ("o", o), ("dO", dO), ("dq", dq), ("dk", dk), ("dv", dv)):
        _check_bf16(n, t, shape)
    _check_f32("lse", lse, (B, H, S))
    if workspace.dtype != torch.uint8 or not workspace.is_cuda or not workspace.is_contiguous():
        raise ValueError("workspace: need a contiguous CUDA uint8 tensor")
    _raise(lib().helix_attn_bwd(_ptr(q), _ptr(k), _ptr(v), _ptr(o), _ptr(lse), _ptr(dO), _ptr(dq), _ptr(dk), _ptr(dv),
                                _ptr(workspace), workspace.numel(), B, H, S, D, float(scale), int(causal),
                                _stream(stream)), "helix_attn_bwd")


def helix_attn_bwd_static(q, k, v, o, lse, dO, dq, dk, dv, scale, causal=True, stream=None):
    """helix_attn_bwd without a workspace argument: the statistics live in the library's built-in device array."""
    shape = B, H, S, D = q.shape
    for n, t in (("q", q), ("k", k), ("v", v), ("o", o), ("dO", dO), ("dq", dq), ("dk", dk), ("dv", dv)):
        _check_bf16(n, t, shape)
    _check_f32("lse", lse, (B, H, S))
    _raise(lib().helix_attn_bwd_static(_ptr(q), _ptr(k), _ptr(v), _ptr(o), _ptr(lse), _ptr(dO), _ptr(dq), _ptr(dk), _ptr(dv),
                                       B, H, S, D, float(scale), int(causal), _stream(stream)), "helix_attn_bwd_static")


def _view(name, t, shape):
    """(pointer, strides) of a logical [B, H, S, D] bf16 view whose last dimension is contiguous."""
    sb, sh, ss, sd = t.stride() if t.dim() == 4 else (0, 0, 0, 0)
    if t.dtype is not _BF16 or not t.is_cuda or t.shape != shape or sd != 1:
        raise ValueError(f"{name}: need a CUDA bfloat16 view of shape {tuple(shape)} with unit stride in D")
    return t.data_ptr(), ctypes.byref(helix_strides(sb, sh, ss))


def helix_attn_check_strides(strides, B, H, S, D) -> int:
    """Status for element strides (batch, head, row), or None for contiguous."""
    arg = None if strides is None else ctypes.byref(helix_strides(*strides))
    return int(lib().helix_attn_check_strides(arg, B, H, S, D))


def helix_attn_fwd_strided(q, k, v, o, lse, scale, causal=True, stream=None):
    """helix_attn_fwd on views: each of q, k, v, o has logical shape [B,H,S,D] and any strides the
    library accepts (for example ``x.permute(1, 2, 0, 3)`` of an [S,B,H,D] activation)."""
    shape = B, H, S, D = q.shape
    (pq, sq), (pk, sk), (pv, sv), (po, so) = (_view(n, t, shape) for n, t in
                                              (("q", q), ("k", k), ("v", v), ("o", o)))
    _check_f32("lse", lse, (B, H, S))
    _raise(lib().helix_attn_fwd_strided(pq, sq, pk, sk, pv, sv, po, so, _ptr(lse), B, H, S, D, float(scale),
                                        int(causal), _stream(stream)), "helix_attn_fwd_strided")


def helix_attn_bwd_strided(q, k, v, o, lse, dO, dq, dk, dv, workspace, scale, causal=True, stream=None):
    """helix_attn_bwd on views (see helix_attn_fwd_strided)."""
    shape = B, H, S, D = q.shape
    views = [_view(n, t, shape) for n, t in (("q", q), ("k", k), ("v", v), ("o", o), ("dO", dO),
                                                    ("dq", dq), ("dk", dk), ("dv", dv))]
    _check_f32("lse", lse, (B, H, S))
    if workspace.dtype != torch.uint8 or not workspace.is_cuda or not workspace.is_contiguous():
        raise ValueError("workspace: need a contiguous CUDA uint8 tensor")
    (pq, sq), (pk, sk), (pv, sv), (po, so), (pg, sg), (pdq, sdq), (pdk, sdk), (pdv, sdv) = views
    _raise(lib().helix_attn_bwd_strided(pq, sq, pk, sk, pv, sv, po, so, _ptr(lse), pg, sg, pdq, sdq, pdk, sdk,
                                        pdv, sdv, _ptr(workspace), workspace.numel(), B, H, S, D, float(scale),
                                        int(causal), _stream(stream)), "helix_attn_bwd_strided")


def _check_stats(stats, B, H, S, D):
    """The backward's workspace as the stage calls see it: a uint8 CUDA tensor of at least
    helix_attn_bwd_workspace_bytes bytes (plane 0: -delta, plane 1: lse * log2(e))."""
    if stats.dtype != torch.uint8 or not stats.is_cuda or not stats.is_contiguous() or \
            stats.numel() < helix_attn_bwd_workspace_bytes(B, H, S, D):
        raise ValueError("stats: need a contiguous CUDA uint8 tensor of helix_attn_bwd_workspace_bytes(B, H, S, D) bytes")


def helix_attn_bwd_preprocess(o, dO, lse, stats, stream=None):
    B, H, S, D = o.shape
    _check_bf16("o", o, o.shape); _check_bf16("dO", dO, o.shape); _check_f32("lse", lse, (B, H, S))
    _check_stats(stats, B, H, S, D)
    _raise(lib().helix_attn_bwd_preprocess(_ptr(o), _ptr(dO), _ptr(lse), _ptr(stats), B, H, S, D, _stream(stream)),
           "helix_attn_bwd_preprocess")


DELTA_HEAD_ROWS = 2048


def helix_attn_bwd_delta_head(q, k, v, dO, lse, stats, rows, scale, causal=True, stream=None):
    shape = B, H, S, D = q.shape
    for n, t in (("q", q), ("k", k), ("v", v), ("dO", dO)):
        _check_bf16(n, t, shape)
    _check_f32("lse", lse, (B, H, S)); _check_stats(stats, B, H, S, D)
    _raise(lib().helix_attn_bwd_delta_head(_ptr(q), _ptr(k), _ptr(v), _ptr(dO), _ptr(lse), _ptr(stats), int(rows),
                                           B, H, S, D, float(scale), int(causal), _stream(stream)),
           "helix_attn_bwd_delta_head")


def helix_attn_bwd_dkdv(q, k, v, dO, stats, dk, dv, scale, causal=True, stream=None):
    shape = B, H, S, D = q.shape
    for n, t in (("q", q), ("k", k), ("v", v), ("dO", dO), ("dk", dk), ("dv", dv)):
        _check_bf16(n, t, shape)
    _check_stats(stats, B, H, S, D)
    _raise(lib().helix_attn_bwd_dkdv(_ptr(q), _ptr(k), _ptr(v), _ptr(dO), _ptr(stats), _ptr(dk), _ptr(dv),
                                     B, H, S, D, float(scale), int(causal), _stream(stream)), "helix_attn_bwd_dkdv")


def helix_attn_bwd_dq(q, k, v, dO, stats, dq, scale, causal=True, stream=None):
    shape = B, H, S, D = q.shape
    for n, t in (("q", q), ("k", k), ("v", v), ("dO", dO), ("dq", dq)):
        _check_bf16(n, t, shape)
    _check_stats(stats, B, H, S, D)
    _raise(lib().helix_attn_bwd_dq(_ptr(q), _ptr(k), _ptr(v), _ptr(dO), _ptr(stats), _ptr(dq),
                                   B, H, S, D, float(scale), int(causal), _stream(stream)), "helix_attn_bwd_dq")


def _matrix(name, t, rows, cols, dtype=torch.bfloat16):
    """(pointer, leading dimension) of a 2-D device matrix whose rows are contiguous."""
    ld, one = t.stride() if t.dim() == 2 else (0, 0)
    if t.dtype is not dtype or not t.is_cuda or t.shape != (rows, cols) or one != 1:
        raise ValueError(f"{name}: need a CUDA {dtype} matrix of shape ({rows}, {cols}) with contiguous rows")
    return t.data_ptr(), ld


def helix_qkv_linear_fwd(a, w, qkv, stream=None):
    """qkv[M,N] <- a[M,K] @ w[K,N]; 2-D views with contiguous rows (qkv may be the [S*B, 3*H*D] view of a fused buffer)."""
    M, K = a.shape
    N = w.shape[1]
    (pa, lda), (pw, ldw), (pq, ldq) = _matrix("a", a, M, K), _matrix("w", w, K, N), _matrix("qkv", qkv, M, N)
    _raise(lib().helix_qkv_linear_fwd(pa, lda, pw, ldw, pq, ldq, M, K, N, _stream(stream)), "helix_qkv_linear_fwd")


def helix_qkv_linear_bwd_workspace_bytes(M, K, N) -> int:
    return int(lib().helix_qkv_linear_bwd_workspace_bytes(M, K, N))


def helix_qkv_linear_bwd(a, w, dqkv, da, dw, workspace=None, stream=None):
    """da[M,K] <- dqkv @ w^T (bf16), dw[K,N] <- a^T @ dqkv (fp32); workspace: uint8 CUDA tensor of
    helix_qkv_linear_bwd_workspace_bytes(M, K, N) bytes."""
    M, K = a.shape
    N = w.shape[1]
    (pa, lda), (pw, ldw), (pg, ldg) = _matrix("a", a, M, K), _matrix("w", w, K, N), _matrix("dqkv", dqkv, M, N)
    (pda, ldda), (pdw, lddw) = _matrix("da", da, M, K), _matrix("dw", dw, K, N, torch.float32)
    if workspace is not None and (workspace.dtype != torch.uint8 or not workspace.is_cuda or not workspace.is_contiguous()):
        raise ValueError("workspace: need a contiguous CUDA uint8 tensor")
    _raise(lib().helix_qkv_linear_bwd(pa, lda, pw, ldw, pg, ldg, pda, ldda, pdw, lddw, _ptr(workspace),
                                      0 if workspace is None else workspace.numel(), M, K, N, _stream(stream)),
           "helix_qkv_linear_bwd")


# ---------------------------------------------------------------- row-wise operators
# Tensors have to be on the current device, whose stream the calls go to (a tensor in host memory is on device -1).
_TYPES = {torch.bfloat16: 0, torch.float16: 1, torch.float32: 2}


def _current(t, stream):
    """The current device; `t` is the call's first tensor."""
    if not t.is_cuda:
        raise ValueError("need CUDA tensors")
    device = torch.cuda.current_device() if _device is None else _device()
    if stream is not None and stream.device_index != device:
        raise ValueError(f"stream: belongs to device {stream.device_index}, the current device is {device}")
    return device


def _refuse(name, t, device, what):
    if not t.is_cuda:
        raise ValueError(f"{name}: need a CUDA tensor")
    if t.get_device() != device:
        raise ValueError(f"{name}: is on {t.device}, the current device is cuda:{device}")
    raise ValueError(f"{name}: need {what}")


def _length(n):
    """A length for the library, whose lengths have 32 bits: one that has more is 0 there, a bad shape, and not what is left of it."""
    return n if -0x80000000 <= n <= 0x7fffffff else 0


def _row(n):
    """A first_row for the library, in 64 bits: what has more is -1 there, a bad shape."""
    n = int(n)
    return n if 0 <= n < 1 << 63 else -1


def _first(name, t, stream):
    """(device, shape, element type, pointer, elements between rows) of a call's first activation, which the others have to be like."""
    dev = _current(t, stream)
    shape, dtype = t.shape, t.dtype
    if len(shape) != 2 or dtype not in _TYPES:
        raise ValueError(f"{name}: need a matrix of bfloat16, float16 or float32")
    return dev, shape, dtype, *_activation(name, t, shape, dtype, dev)


def _activation(name, t, shape, dtype, device):
    """(pointer, elements between rows) of a 2-D device matrix whose rows are contiguous."""
    if t.dtype is not dtype or t.shape != shape or t.get_device() != device:
        _refuse(name, t, device, f"a {dtype} matrix of shape {tuple(shape)}")
    ld, one = t.stride()
    if one != 1 and shape[1] > 1:
        raise ValueError(f"{name}: need contiguous rows")
    return t.data_ptr(), ld if shape[0] > 1 else shape[1]   # a single row has no next one


def _vector(name, t, n, device):
    """Pointer of n contiguous fp32 values."""
    if t.dtype is not _F32 or t.dim() != 1 or t.numel() != n or not t.is_contiguous() or t.get_device() != device:
        _refuse(name, t, device, f"a contiguous float32 vector of {n} elements")
    return t.data_ptr()


def _generator(rng, device):
    """rng: None, or an int64 tensor with the two elements seed and offset."""
    if rng is None:
        return None
    if rng.dtype is not torch.int64 or rng.numel() != 2 or not rng.is_contiguous() or rng.get_device() != device:
        _refuse("rng", rng, device, "a contiguous int64 tensor of two elements, seed and offset")
    return rng.data_ptr()


def _workspace(workspace, device):
    if workspace.dtype is not torch.uint8 or not workspace.is_contiguous() or workspace.get_device() != device:
        _refuse("workspace", workspace, device, "a contiguous uint8 tensor")
    return workspace.data_ptr(), workspace.numel()


def helix_dropout_add_fwd(x, residual, out, p, rng, first_row=0, stream=None):
    """out[M,E] <- residual + dropout(x); residual None: dropout(x).  rng: CUDA int64 tensor [seed, offset] (None where p == 0);
    row i takes the random numbers of row first_row + i."""
    dev, shape, dtype, px, ldx = _first("x", x, stream)
    pr, ldr = (None, 0) if residual is None else _activation("residual", residual, shape, dtype, dev)
    po, ldo = _activation("out", out, shape, dtype, dev)
    _raise(lib().helix_dropout_add_fwd(px, ldx, pr, ldr, po, ldo, _length(shape[0]), _length(shape[1]), _TYPES[dtype], float(p), _generator(rng, dev), _row(first_row), _stream(stream)),
           "helix_dropout_add_fwd")


def helix_dropout_add_bwd(dout, dx, p, rng, first_row=0, stream=None):
    """dx[M,E] <- gradient of the dropped-out branch; the residual's gradient is dout itself."""
    dev, shape, dtype, pg, ldg = _first("dout", dout, stream)
    px, ldx = _activation("dx", dx, shape, dtype, dev)
    _raise(lib().helix_dropout_add_bwd(pg, ldg, px, ldx, _length(shape[0]), _length(shape[1]), _TYPES[dtype], float(p), _generator(rng, dev), _row(first_row), _stream(stream)),
           "helix_dropout_add_bwd")


def helix_layer_norm_fwd(x, gamma, beta, y, mean, rstd, eps=1e-5, stream=None):
    """y[M,E], mean[M], rstd[M] <- layer norm of the rows of x; gamma, beta: fp32 [E].  mean and rstd may be None."""
    dev, shape, dtype, px, ldx = _first("x", x, stream)
    M, E = shape
    py, ldy = _activation("y", y, shape, dtype, dev)
    _raise(lib().helix_layer_norm_fwd(px, ldx, _vector("gamma", gamma, E, dev), _vector("beta", beta, E, dev), py, ldy,
                                      None if mean is None else _vector("mean", mean, M, dev), None if rstd is None else _vector("rstd", rstd, M, dev),
                                      _length(M), _length(E), _TYPES[dtype], float(eps), _stream(stream)), "helix_layer_norm_fwd")


def helix_layer_norm_bwd_workspace_bytes(M, E) -> int:
    """Bytes for up to M rows of E columns."""
    return int(lib().helix_layer_norm_bwd_workspace_bytes(_length(M), _length(E)))


def helix_layer_norm_bwd(dy, x, gamma, mean, rstd, dx, dgamma, dbeta, workspace, stream=None):
    """dx[M,E], dgamma[E], dbeta[E] <- gradients of helix_layer_norm_fwd; workspace: uint8 CUDA tensor of
    helix_layer_norm_bwd_workspace_bytes(M, E) bytes."""
    dev, shape, dtype, px, ldx = _first("x", x, stream)
    M, E = shape
    pdy, lddy = _activation("dy", dy, shape, dtype, dev)
    pdx, lddx = _activation("dx", dx, shape, dtype, dev)
    pw, nw = _workspace(workspace, dev)
    _raise(lib().helix_layer_norm_bwd(pdy, lddy, px, ldx, _vector("gamma", gamma, E, dev), _vector("mean", mean, M, dev), _vector("rstd", rstd, M, dev), pdx, lddx,
                                      _vector("dgamma", dgamma, E, dev), _vector("dbeta", dbeta, E, dev), pw, nw, _length(M), _length(E), _TYPES[dtype], _stream(stream)),
           "helix_layer_norm_bwd")


def helix_dropout_add_layer_norm_fwd(x, residual, s, gamma, beta, y, mean, rstd, p, rng, eps=1e-5, first_row=0, stream=None):
    """s <- residual + dropout(x), y, mean, rstd <- layer norm of s (see helix_dropout_add_fwd and helix_layer_norm_fwd)."""
    dev, shape, dtype, px, ldx = _first("x", x, stream)
    M, E = shape
    pr, ldr = _activation("residual", residual, shape, dtype, dev)
    ps, lds = _activation("s", s, shape, dtype, dev)
    py, ldy = _activation("y", y, shape, dtype, dev)
    _raise(lib().helix_dropout_add_layer_norm_fwd(px, ldx, pr, ldr, ps, lds, _vector("gamma", gamma, E, dev), _vector("beta", beta, E, dev), py, ldy,
                                                  None if mean is None else _vector("mean", mean, M, dev), None if rstd is None else _vector("rstd", rstd, M, dev),
                                                  _length(M), _length(E), _TYPES[dtype], float(p), _generator(rng, dev), _row(first_row), float(eps), _stream(stream)), "helix_dropout_add_layer_norm_fwd")


def helix_dropout_add_layer_norm_bwd(dy, ds, s, gamma, mean, rstd, dx, dresidual, dgamma, dbeta, workspace, p, rng, first_row=0, stream=None):
    """dresidual <- ds + gradient of the layer norm of s, dx <- its dropped-out share, dgamma, dbeta.  ds may be None."""
    dev, shape, dtype, ps, lds = _first("s", s, stream)
    M, E = shape
    pdy, lddy = _activation("dy", dy, shape, dtype, dev)
    pds, ldds = (None, 0) if ds is None else _activation("ds", ds, shape, dtype, dev)
    pdx, lddx = _activation("dx", dx, shape, dtype, dev)
    pdr, lddr = _activation("dresidual", dresidual, shape, dtype, dev)
    pw, nw = _workspace(workspace, dev)
    _raise(lib().helix_dropout_add_layer_norm_bwd(pdy, lddy, pds, ldds, ps, lds, _vector("gamma", gamma, E, dev), _vector("mean", mean, M, dev),
                                                  _vector("rstd", rstd, M, dev), pdx, lddx, pdr, lddr, _vector("dgamma", dgamma, E, dev),
                                                  _vector("dbeta", dbeta, E, dev), pw, nw, _length(M), _length(E), _TYPES[dtype], float(p), _generator(rng, dev), _row(first_row),
                                                  _stream(stream)), "helix_dropout_add_layer_norm_bwd")


# ---------------------------------------------------------------- gated feed-forward projections
_ACTIVATIONS = {"silu": 0, "gelu": 1}


def _gated(a, w, activation):
    """(M, K, F, activation) of the gated projections."""
    if activation not in _ACTIVATIONS:
        raise ValueError(f"activation: need one of {tuple(_ACTIVATIONS)}")
    if a.dim() != 2 or w.dim() != 2 or w.shape[1] % 2:
        raise ValueError("need matrices a [M, K] and w [K, 2F]")
    return *a.shape, w.shape[1] // 2, _ACTIVATIONS[activation]


def helix_gated_linear_fwd(a, w, h, gu=None, activation="silu", stream=None):
    """h[M,F] <- act(a @ w[:, :F]) * (a @ w[:, F:]); gu[M,2F], if given, <- a @ w for the backward.  bf16, 2-D views with contiguous rows."""
    M, K, F, act = _gated(a, w, activation)
    dev = _current(a, stream)
    pa, lda = _activation("a", a, (M, K), _BF16, dev)
    pw, ldw = _activation("w", w, (K, 2 * F), _BF16, dev)
    pg, ldg = (None, 0) if gu is None else _activation("gu", gu, (M, 2 * F), _BF16, dev)
    ph, ldh = _activation("h", h, (M, F), _BF16, dev)
    _raise(lib().helix_gated_linear_fwd(pa, lda, pw, ldw, pg, ldg, ph, ldh, _length(M), _length(K), _length(F), act, _stream(stream)), "helix_gated_linear_fwd")


def helix_gated_linear_bwd_workspace_bytes(M, K, F) -> int:
    """Bytes for up to M tokens."""
    return int(lib().helix_gated_linear_bwd_workspace_bytes(_length(M), _length(K), _length(F)))


def helix_gated_linear_bwd(a, w, dh, da, dw, workspace, gu=None, activation="silu", stream=None):
    """da[M,K], dw[K,2F] <- gradients of helix_gated_linear_fwd for dh[M,F], from the gu it wrote or, without, from a and w alone; workspace:
    uint8 CUDA tensor of helix_gated_linear_bwd_workspace_bytes(M, K, F) bytes."""
    M, K, F, act = _gated(a, w, activation)
    dev = _current(a, stream)
    pa, lda = _activation("a", a, (M, K), _BF16, dev)
    pw, ldw = _activation("w", w, (K, 2 * F), _BF16, dev)
    pg, ldg = (None, 0) if gu is None else _activation("gu", gu, (M, 2 * F), _BF16, dev)
    ph, ldh = _activation("dh", dh, (M, F), _BF16, dev)
    pda, ldda = _activation("da", da, (M, K), _BF16, dev)
    pdw, lddw = _activation("dw", dw, (K, 2 * F), _BF16, dev)
    pws, nws = _workspace(workspace, dev)
    _raise(lib().helix_gated_linear_bwd(pa, lda, pw, ldw, pg, ldg, ph, ldh, pda, ldda, pdw, lddw, pws, nws, _length(M), _length(K), _length(F), act, _stream(stream)), "helix_gated_linear_bwd")
