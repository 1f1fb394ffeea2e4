"""ctypes binding of full attention over packed sequences, the paged cache of keys and values and the
attention of single tokens over it (include/spt_attn.h): argument marshalling only.  Tensors live on one GPU;
nothing is computed here or by torch.  Q, K, V and their kin may be views whose rows and heads lie apart (slices of a
fused projection, say) as long as the head dimension is dense and rows start at multiples of 16 bytes."""
from __future__ import annotations

import contextlib
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


class _Args:
    """Pointers of a call's tensors, which must all be on the GPU of the first, and the strides of those that
    may be views (None where all of them are dense)."""

    def __init__(self, first):
        if not isinstance(first, torch.Tensor) or not first.is_cuda:
            raise ValueError("need tensors on a GPU")
        self.device, self.at, self.dense, self.keep = first.device, [], True, None

    def plain(self, t, dtype, numel, name):
        if t is None:
            return None
        if t.device != self.device:
            raise ValueError(f"{name}: on {t.device}, the other tensors are on {self.device}")
        return spt._ptr(t, dtype, numel, name)

    def rows(self, t, shape, name):
        if t.dtype is not _BF16 or tuple(t.shape) != shape or t.device != self.device or (t.stride(2) != 1 and shape[2] != 1):
            raise ValueError(f"{name}: need a tensor of {_BF16} {shape} on {self.device} with a dense last axis, "
                             f"got {t.dtype} {tuple(t.shape)} on {t.device}, strides {tuple(t.stride())}")
        if t.is_contiguous():
            self.at += (shape[1] * shape[2], shape[2])
        else:
            self.dense = False
            self.at += (t.stride(0), t.stride(1))
        return t.data_ptr()

    def strides(self):
        if self.dense:
            return None
        self.keep = (ctypes.c_int64 * len(self.at))(*self.at)
        return ctypes.cast(self.keep, ctypes.c_void_p)

    def here(self):
        """The calls launch on the current device: make it the tensors'."""
        if self.device.index == torch._C._cuda_getDevice():
            return contextlib.nullcontext()
        return torch.cuda.device(self.device)


def _run(a: _Args, name: str, *args):
    with a.here():
        spt._check(getattr(lib(), name)(*args, spt._stream()), name)


def prompt_fwd(shape: AttnShape, Q, K, V, cu_q, cu_k, Y=None, lse=None, save_for_backward=True):
    """Y[Tq,H,dh] bf16 and (optionally) lse[H,Tq] fp32 of Q[Tq,H,dh], K, V[Tk,Hk,dh] and the first rows cu_q, cu_k
    [B+1] int32 of the sequences.  Rows behind the last sequence stay as they are."""
    s, a = shape, _Args(Q)
    q, k = (s.Tq, s.H, s.dh), (s.Tk, s.Hk, s.dh)
    Y = torch.empty(q, dtype=_BF16, device=a.device) if Y is None else Y
    if lse is None and save_for_backward:
        lse = torch.empty((s.H, s.Tq), dtype=_F32, device=a.device)
    ptrs = [a.rows(Q, q, "Q"), a.rows(K, k, "K"), a.rows(V, k, "V")]
    y = a.rows(Y, q, "Y")
    _run(a, "spt_attn_prompt_fwd", ctypes.byref(s), *ptrs, a.strides(), a.plain(cu_q, _I32, s.B + 1, "cu_q"),
         a.plain(cu_k, _I32, s.B + 1, "cu_k"), y, a.plain(lse, _F32, s.H * s.Tq, "lse"))
    return Y, lse


def prompt_bwd(shape: AttnShape, Q, K, V, Y, dY, lse, cu_q, cu_k, ws=None, dQ=None, dK=None, dV=None):
    """dQ[Tq,H,dh], dK, dV[Tk,Hk,dh] bf16 from dY[Tq,H,dh] and the forward's Y and lse."""
    s, a = shape, _Args(Q)
    q, k = (s.Tq, s.H, s.dh), (s.Tk, s.Hk, s.dh)
    dQ, dK, dV = (torch.empty(n, dtype=_BF16, device=a.device) if t is None else t for t, n in ((dQ, q), (dK, k), (dV, k)))
    ws = alloc_prompt_workspace(s, a.device) if ws is None else ws
    ins = [a.rows(t, n, name) for t, n, name in ((Q, q, "Q"), (K, k, "K"), (V, k, "V"), (Y, q, "Y"), (dY, q, "dY"))]
    outs = [a.rows(t, n, name) for t, n, name in ((dQ, q, "dQ"), (dK, k, "dK"), (dV, k, "dV"))]
    _run(a, "spt_attn_prompt_bwd", ctypes.byref(s), *ins, a.plain(lse, _F32, s.H * s.Tq, "lse"), a.strides(),
         a.plain(cu_q, _I32, s.B + 1, "cu_q"), a.plain(cu_k, _I32, s.B + 1, "cu_k"), *outs,
         a.plain(ws, _U8, ws.numel(), "ws"), ws.numel())
    return dQ, dK, dV


def _cache_ptrs(a: _Args, s: CacheShape, cache):
    K, V, ks, vs = cache
    dtype, rows = (_BF16 if s.format == CACHE_BF16 else _U8), s.pages * s.Hk * s.page
    if dtype is _U8 and K.dtype is torch.float8_e4m3fn:
        K, V = K.view(_U8), V.view(_U8)
    return [a.plain(K, dtype, rows * s.dh, "cache.K"), a.plain(V, dtype, rows * s.dh, "cache.V"),
            a.plain(ks, _U8, rows, "cache.ks"), a.plain(vs, _U8, rows, "cache.vs")]


def _seq_ptrs(a: _Args, s: CacheShape, table, start, cu):
    return [a.plain(table, _I32, s.B * s.max_pages, "table"), a.plain(start, _I32, s.B, "start"), a.plain(cu, _I32, s.B + 1, "cu")]


def cache_write(shape: CacheShape, K, V, cache, table, start, cu):
    """Rows cu[b] .. cu[b+1]-1 of K, V [T,Hk,dh] bf16 become tokens start[b], start[b] + 1, ... of sequence b, whose
    pages table[b] names."""
    s, a = shape, _Args(K)
    n = (K.shape[0], s.Hk, s.dh)
    kv = [a.rows(K, n, "K"), a.rows(V, n, "V")]
    _run(a, "spt_cache_write", ctypes.byref(s), n[0], *kv, a.strides(), *_seq_ptrs(a, s, table, start, cu), *_cache_ptrs(a, s, cache))
    return cache


def cache_read(shape: CacheShape, cache, table, start, cu, T=None, K=None, V=None):
    """K, V [T,Hk,dh] bf16: what the cache holds for tokens start[b], start[b] + 1, ... of sequence b, in rows
    cu[b] .. cu[b+1]-1.  Give T, or K and V."""
    s, a = shape, _Args(cache[0])
    if K is None or V is None:
        if T is None and K is None and V is None:
            raise ValueError("cache_read: need T, or K and V")
        T = T if T is not None else (V if K is None else K).shape[0]
    n = (T if T is not None else K.shape[0], s.Hk, s.dh)
    K, V = (torch.empty(n, dtype=_BF16, device=a.device) if t is None else t for t in (K, V))
    kv = [a.rows(K, n, "K"), a.rows(V, n, "V")]
    _run(a, "spt_cache_read", ctypes.byref(s), n[0], *kv, a.strides(), *_seq_ptrs(a, s, table, start, cu), *_cache_ptrs(a, s, cache))
    return K, V


def decode(shape: CacheShape, Q, cache, table, lens, scale=None, ws=None, Y=None):
    """Y[B,H,dh] bf16: attention of one query for each sequence, Q[B,H,dh], over the first lens[b] tokens of its pages."""
    s, a = shape, _Args(Q)
    n = (s.B, Q.shape[1], s.dh)
    Y = torch.empty(n, dtype=_BF16, device=a.device) if Y is None else Y
    ws = alloc_decode_workspace(s, n[1], a.device) if ws is None else ws
    q, y = a.rows(Q, n, "Q"), a.rows(Y, n, "Y")
    _run(a, "spt_attn_decode", ctypes.byref(s), n[1], s.dh ** -0.5 if scale is None else scale, q, a.strides(),
         *_cache_ptrs(a, s, cache), a.plain(table, _I32, s.B * s.max_pages, "table"), a.plain(lens, _I32, s.B, "lens"), y,
         a.plain(ws, _U8, ws.numel(), "ws"), ws.numel())
    return Y
