"""ctypes binding of full attention over packed sequences, the paged cache of keys and values and the
attention of single tokens over it (include/spt_attn.h): argument marshalling only.  Tensors live on one GPU;
nothing is computed here or by torch.  Q, K, V and their kin may be views whose rows and heads lie apart (slices of a
fused projection, say) as long as the head dimension is dense and rows start at multiples of 16 bytes."""
from __future__ import annotations

import ctypes
from typing import NamedTuple, Optional

import torch

from . import spt

CACHE_BF16, CACHE_E4M3 = 0, 1

EXPORTS = ("spt_attn_prompt_fwd", "spt_attn_prompt_bwd", "spt_attn_prompt_workspace_bytes", "spt_cache_write",
           "spt_cache_read", "spt_attn_decode", "spt_attn_decode_workspace_bytes")


class AttnShape(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("B", "Tq", "Tk", "H", "Hk", "dh", "causal")] + [("scale", ctypes.c_float)]


class CacheShape(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("pages", "page", "Hk", "dh", "format", "B", "max_pages")]


class Cache(NamedTuple):
    """The pool: K, V [pages, Hk, page, dh] bf16 or 8-bit codes (uint8), ks, vs [pages, Hk, page] uint8 or None."""
    K: torch.Tensor
    V: torch.Tensor
    ks: Optional[torch.Tensor] = None
    vs: Optional[torch.Tensor] = None


_ready = False


def lib() -> ctypes.CDLL:
    global _ready
    L = spt.lib()
    if not _ready:
        vp, sz, i32, f32 = ctypes.c_void_p, ctypes.c_size_t, ctypes.c_int32, ctypes.c_float
        shp, csh = ctypes.POINTER(AttnShape), ctypes.POINTER(CacheShape)
        L.spt_attn_prompt_workspace_bytes.restype = sz
        L.spt_attn_prompt_workspace_bytes.argtypes = [shp]
        L.spt_attn_decode_workspace_bytes.restype = sz
        L.spt_attn_decode_workspace_bytes.argtypes = [csh, i32]
        L.spt_attn_prompt_fwd.argtypes = [shp] + [vp] * 9
        L.spt_attn_prompt_bwd.argtypes = [shp] + [vp] * 13 + [sz, vp]
        L.spt_cache_write.argtypes = [csh, i32] + [vp] * 11
        L.spt_cache_read.argtypes = [csh, i32] + [vp] * 11
        L.spt_attn_decode.argtypes = [csh, i32, f32] + [vp] * 10 + [sz, vp]
        for name in ("spt_attn_prompt_fwd", "spt_attn_prompt_bwd", "spt_cache_write", "spt_cache_read", "spt_attn_decode"):
            getattr(L, name).restype = ctypes.c_int
        _ready = True
    return L


def make_shape(B, Tq, Tk, H, Hk, dh, causal=True, scale=None) -> AttnShape:
    return AttnShape(B, Tq, Tk, H, Hk, dh, int(causal), dh ** -0.5 if scale is None else scale)


def make_cache_shape(pages, page, Hk, dh, B, max_pages, format=CACHE_BF16) -> CacheShape:
    return CacheShape(pages, page, Hk, dh, format, B, max_pages)


def alloc_cache(shape: CacheShape, device="cuda") -> Cache:
    """A pool whose contents are undefined until they are written."""
    s = shape
    rows = (s.pages, s.Hk, s.page)
    bf = s.format == CACHE_BF16
    kv = [torch.empty((*rows, s.dh), dtype=torch.bfloat16 if bf else torch.uint8, device=device) for _ in range(2)]
    return Cache(*kv, *(() if bf else [torch.empty(rows, dtype=torch.uint8, device=device) for _ in range(2)]))


def prompt_workspace_bytes(shape: AttnShape) -> int:
    return int(lib().spt_attn_prompt_workspace_bytes(ctypes.byref(shape)))


def decode_workspace_bytes(shape: CacheShape, H: int) -> int:
    return int(lib().spt_attn_decode_workspace_bytes(ctypes.byref(shape), H))


def _alloc(n: int, where: str, device) -> torch.Tensor:
    if n == 0:
        raise spt.SptError(-2, where)
    return torch.empty(n, dtype=torch.uint8, device=device)


def alloc_prompt_workspace(shape: AttnShape, device="cuda") -> torch.Tensor:
    return _alloc(prompt_workspace_bytes(shape), "spt_attn_prompt_workspace_bytes", device)


def alloc_decode_workspace(shape: CacheShape, H: int, device="cuda") -> torch.Tensor:
    return _alloc(decode_workspace_bytes(shape, H), "spt_attn_decode_workspace_bytes", device)


_BF16, _F32, _I32, _U8 = torch.bfloat16, torch.float32, torch.int32, torch.uint8
_byref = ctypes.byref
_current_device, _current_stream = torch._C._cuda_getDevice, torch._C._cuda_getCurrentRawStream


def _gpu(t, name: str) -> int:
    """The GPU of a call's first tensor, which all others must be on."""
    dev = t.get_device() if isinstance(t, torch.Tensor) else -1
    if dev < 0:
        raise ValueError(f"{name}: need a tensor on a GPU")
    return dev


def _dense(t, dtype, numel: int, dev: int, name: str):
    """Pointer of a dense tensor, or None."""
    if t is None:
        return None
    if t.dtype is not dtype or t.numel() != numel or not t.is_contiguous() or t.get_device() != dev:
        raise ValueError(f"{name}: need a contiguous tensor of {dtype} with {numel} elements on cuda:{dev}, "
                         f"got {t.dtype} {tuple(t.shape)} on {t.device}")
    return t.data_ptr()


def _rows(t, shape, dev: int, name: str, apart: list):
    """Pointer of rows [T, heads, dh], which may lie apart: then their name goes into `apart`."""
    if t.dtype is _BF16 and t.shape == shape and t.get_device() == dev:
        if t.is_contiguous():
            return t.data_ptr()
        if t.stride(2) == 1:
            apart.append(name)
            return t.data_ptr()
    raise ValueError(f"{name}: need a tensor of {_BF16} {shape} on cuda:{dev} with a dense last axis, "
                     f"got {t.dtype} {tuple(t.shape)} on {t.device}, strides {tuple(t.stride())}")


def _strides(apart: list, *tensors):
    """Row and head strides of all row tensors of a call, or None where all are dense."""
    if not apart:
        return None
    at = [n for t in tensors for n in ((t.shape[1] * t.shape[2], t.shape[2]) if t.is_contiguous() else (t.stride(0), t.stride(1)))]
    return (ctypes.c_int64 * len(at))(*at)


def _call(dev: int, name: str, *args):
    """Calls launch on the current device and its current stream: make it the tensors' device."""
    f = _functions.get(name) or _functions.setdefault(name, getattr(lib(), name))
    if dev == _current_device():
        rc = f(*args, _current_stream(dev))
    else:
        with torch.cuda.device(dev):
            rc = f(*args, _current_stream(dev))
    if rc != 0:
        raise spt.SptError(rc, name)


_functions: dict = {}


def prompt_fwd(shape: AttnShape, Q, K, V, cu_q, cu_k, Y=None, lse=None, save_for_backward=True):
    """Y[Tq,H,dh] bf16 and (optionally) lse[H,Tq] fp32 of Q[Tq,H,dh], K, V[Tk,Hk,dh] and the first rows cu_q, cu_k
    [B+1] int32 of the sequences.  Rows behind the last sequence stay as they are."""
    s, dev = shape, _gpu(Q, "Q")
    B, H, Tq = s.B, s.H, s.Tq
    q, k = (Tq, H, s.dh), (s.Tk, s.Hk, s.dh)
    if Y is None:
        Y = torch.empty(q, dtype=_BF16, device=Q.device)
    if lse is None and save_for_backward:
        lse = torch.empty((H, Tq), dtype=_F32, device=Q.device)
    apart = []
    y = _rows(Y, q, dev, "Y", apart)
    _call(dev, "spt_attn_prompt_fwd", _byref(s), _rows(Q, q, dev, "Q", apart), _rows(K, k, dev, "K", apart), _rows(V, k, dev, "V", apart),
          _strides(apart, Q, K, V, Y), _dense(cu_q, _I32, B + 1, dev, "cu_q"), _dense(cu_k, _I32, B + 1, dev, "cu_k"), y,
          _dense(lse, _F32, H * Tq, dev, "lse"))
    return Y, lse


def prompt_bwd(shape: AttnShape, Q, K, V, Y, dY, lse, cu_q, cu_k, ws=None, dQ=None, dK=None, dV=None):
    """dQ[Tq,H,dh], dK, dV[Tk,Hk,dh] bf16 from dY[Tq,H,dh] and the forward's Y and lse."""
    s, dev = shape, _gpu(Q, "Q")
    B, H, Tq = s.B, s.H, s.Tq
    q, k = (Tq, H, s.dh), (s.Tk, s.Hk, s.dh)
    dQ, dK, dV = (torch.empty(n, dtype=_BF16, device=Q.device) if t is None else t for t, n in ((dQ, q), (dK, k), (dV, k)))
    if ws is None:
        ws = alloc_prompt_workspace(s, Q.device)
    apart, size = [], ws.numel()
    dq, dk, dv = _rows(dQ, q, dev, "dQ", apart), _rows(dK, k, dev, "dK", apart), _rows(dV, k, dev, "dV", apart)
    _call(dev, "spt_attn_prompt_bwd", _byref(s), _rows(Q, q, dev, "Q", apart), _rows(K, k, dev, "K", apart), _rows(V, k, dev, "V", apart),
          _rows(Y, q, dev, "Y", apart), _rows(dY, q, dev, "dY", apart), _dense(lse, _F32, H * Tq, dev, "lse"),
          _strides(apart, Q, K, V, Y, dY, dQ, dK, dV), _dense(cu_q, _I32, B + 1, dev, "cu_q"), _dense(cu_k, _I32, B + 1, dev, "cu_k"),
          dq, dk, dv, _dense(ws, _U8, size, dev, "ws"), size)
    return dQ, dK, dV


def _pool(s: CacheShape, cache, dev: int):
    K, V, ks, vs = cache
    bf, rows = s.format == CACHE_BF16, s.pages * s.Hk * s.page
    if not bf and K.dtype is torch.float8_e4m3fn:
        K, V = K.view(_U8), V.view(_U8)
    dtype, n = _BF16 if bf else _U8, rows * s.dh
    return (_dense(K, dtype, n, dev, "cache.K"), _dense(V, dtype, n, dev, "cache.V"), _dense(ks, _U8, rows, dev, "cache.ks"),
            _dense(vs, _U8, rows, dev, "cache.vs"))


def _move_rows(name: str, s: CacheShape, K, V, cache, table, start, cu, dev: int):
    n, B, apart = (K.shape[0], s.Hk, s.dh), s.B, []
    _call(dev, name, _byref(s), n[0], _rows(K, n, dev, "K", apart), _rows(V, n, dev, "V", apart), _strides(apart, K, V),
          _dense(table, _I32, B * s.max_pages, dev, "table"), _dense(start, _I32, B, dev, "start"), _dense(cu, _I32, B + 1, dev, "cu"),
          *_pool(s, cache, dev))


def cache_write(shape: CacheShape, K, V, cache, table, start, cu):
    """Rows cu[b] .. cu[b+1]-1 of K, V [T,Hk,dh] bf16 become tokens start[b], start[b] + 1, ... of sequence b, whose
    pages table[b] names."""
    _move_rows("spt_cache_write", shape, K, V, cache, table, start, cu, _gpu(K, "K"))
    return cache


def cache_read(shape: CacheShape, cache, table, start, cu, T=None, K=None, V=None):
    """K, V [T,Hk,dh] bf16: what the cache holds for tokens start[b], start[b] + 1, ... of sequence b, in rows
    cu[b] .. cu[b+1]-1.  Give T, or K and V."""
    dev = _gpu(cache[0], "cache.K")
    if K is None or V is None:
        T = next((t.shape[0] for t in (K, V) if t is not None), T)
        if T is None:
            raise ValueError("cache_read: need T, or K and V")
        K, V = (torch.empty((T, shape.Hk, shape.dh), dtype=_BF16, device=cache[0].device) if t is None else t for t in (K, V))
    _move_rows("spt_cache_read", shape, K, V, cache, table, start, cu, dev)
    return K, V


def decode(shape: CacheShape, Q, cache, table, lens, scale=None, ws=None, Y=None):
    """Y[B,H,dh] bf16: attention of one query for each sequence, Q[B,H,dh], over the first lens[b] tokens of its pages."""
    s, dev = shape, _gpu(Q, "Q")
    B, H, dh = s.B, Q.shape[1], s.dh
    n = (B, H, dh)
    if Y is None:
        Y = torch.empty(n, dtype=_BF16, device=Q.device)
    if ws is None:
        ws = alloc_decode_workspace(s, H, Q.device)
    apart, size = [], ws.numel()
    y = _rows(Y, n, dev, "Y", apart)
    _call(dev, "spt_attn_decode", _byref(s), H, dh ** -0.5 if scale is None else scale, _rows(Q, n, dev, "Q", apart), _strides(apart, Q, Y),
          *_pool(s, cache, dev), _dense(table, _I32, B * s.max_pages, dev, "table"), _dense(lens, _I32, B, dev, "lens"), y,
          _dense(ws, _U8, size, dev, "ws"), size)
    return Y
