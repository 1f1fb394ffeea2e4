"""What full attention, the paged cache and single-token attention refuse, on the host and without a GPU, and what
the binding refuses before it calls them; the reference itself against torch's own derivatives."""
import ctypes
import os
import re

import numpy as np
import pytest
import torch

import attn_ref as ref
from paper_2312_10365_amd import attn, spt

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
OK, ODD, BYTE = (ctypes.c_void_p(x) for x in (1 << 20, (1 << 20) + 8, (1 << 20) + 2))
ARG, UNSUPPORTED, WORKSPACE = -1, -2, -3


def test_library_exports_every_declared_function():
    text = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", "spt_attn.h")).read(), flags=re.S)
    names = set(re.findall(r"\b(spt_[a-z_]+)\s*\(", text))
    assert names == set(attn.EXPORTS)
    L = attn.lib()
    assert all(hasattr(L, n) for n in names)


def fwd(shape, Q=OK, K=OK, V=OK, strides=None, cu_q=OK, cu_k=OK, Y=OK, lse=None):
    s = None if strides is None else (ctypes.c_int64 * 8)(*strides)
    return attn.lib().spt_attn_prompt_fwd(None if shape is None else ctypes.byref(shape), Q, K, V, s, cu_q, cu_k, Y, lse, None)


def bwd(shape, strides=None, ws=OK, ws_bytes=1 << 40, **other):
    s = None if strides is None else (ctypes.c_int64 * 16)(*strides)
    p = {n: OK for n in ("Q", "K", "V", "Y", "dY", "lse", "cu_q", "cu_k", "dQ", "dK", "dV")} | other
    return attn.lib().spt_attn_prompt_bwd(ctypes.byref(shape), p["Q"], p["K"], p["V"], p["Y"], p["dY"], p["lse"], s, p["cu_q"], p["cu_k"],
                                          p["dQ"], p["dK"], p["dV"], ws, ws_bytes, None)


@pytest.mark.parametrize("change,code", [
    (dict(B=0), ARG), (dict(Tq=0), ARG), (dict(Tk=0), ARG), (dict(H=0), ARG), (dict(Hk=0), ARG), (dict(Hk=3), ARG), (dict(dh=0), ARG),
    (dict(causal=2), ARG), (dict(scale=0.0), ARG), (dict(scale=-1.0), ARG), (dict(scale=float("nan")), ARG), (dict(scale=float("inf")), ARG), (dict(scale=3e38), ARG),
    (dict(dh=32), UNSUPPORTED), (dict(dh=96), UNSUPPORTED), (dict(B=4097), UNSUPPORTED), (dict(H=1 << 17, Hk=1), UNSUPPORTED),
    (dict(Tq=2 ** 31 - 1, H=64, Hk=1), UNSUPPORTED), (dict(Tk=2 ** 31 - 1, H=64, Hk=1), UNSUPPORTED)])
def test_prompt_shapes(change, code):
    good = dict(B=2, Tq=10, Tk=12, H=4, Hk=2, dh=64, causal=True, scale=0.1)
    s = attn.make_shape(**(good | {k: v for k, v in change.items() if k != "causal"}))
    s.causal = change.get("causal", 1)
    assert fwd(s) == code and bwd(s) == code
    assert attn.prompt_workspace_bytes(s) == 0
    assert attn.prompt_workspace_bytes(attn.make_shape(**good)) >= 10 * 4 * 4


def test_prompt_pointers_and_strides():
    s = attn.make_shape(2, 10, 12, 4, 2, 64)
    assert fwd(None) == ARG
    for name in ("Q", "K", "V", "Y", "cu_q", "cu_k"):
        assert fwd(s, **{name: None}) == ARG, name
    for name in ("Q", "K", "V", "Y"):
        assert fwd(s, **{name: ODD}) == ARG, name
    assert fwd(s, cu_q=BYTE) == ARG and fwd(s, lse=BYTE) == ARG
    dense = [256, 64, 128, 64, 128, 64, 256, 64]
    for at, value, code in ((0, 260, ARG), (1, 4, ARG), (2, -128, ARG), (3, 1 << 23, UNSUPPORTED), (6, 0, ARG), (7, 0, ARG), (6, 192, ARG), (7, 32, ARG)):
        assert fwd(s, strides=dense[:at] + [value] + dense[at + 1:]) == code, (at, value)
    # heads in front of rows: 10 rows of 64, then the next head, but not 9
    assert fwd(s, strides=dense[:6] + [64, 576]) == ARG
    for name in ("Q", "K", "V", "Y", "dY", "lse", "cu_q", "cu_k", "dQ", "dK", "dV"):
        assert bwd(s, **{name: None}) == ARG, name
    assert bwd(s, ws=None) == ARG and bwd(s, ws=ODD) == ARG and bwd(s, ws_bytes=16) == WORKSPACE
    all8 = dense + [256, 64] * 2 + [128, 64] * 2
    for at, code in ((8, ARG), (10, ARG), (12, ARG), (14, ARG)):
        assert bwd(s, strides=all8[:at] + [-8] + all8[at + 1:]) == code
    assert bwd(s, strides=all8[:12] + [0] + all8[13:]) == ARG                     # a gradient of a broadcast K has rows of its own


def pool(change=None):
    return attn.make_cache_shape(**(dict(pages=9, page=16, Hk=2, dh=64, B=3, max_pages=4, format=0) | (change or {})))


def write(shape, T=5, strides=None, read=False, **other):
    p = {n: OK for n in ("K", "V", "table", "start", "cu", "Kc", "Vc")} | {"ks": None, "vs": None} | other
    s = None if strides is None else (ctypes.c_int64 * 4)(*strides)
    f = attn.lib().spt_cache_read if read else attn.lib().spt_cache_write
    return f(None if shape is None else ctypes.byref(shape), T, p["K"], p["V"], s, p["table"], p["start"], p["cu"], p["Kc"], p["Vc"], p["ks"], p["vs"], None)


def decode(shape, H=4, scale=0.1, strides=None, ws_bytes=1 << 40, **other):
    p = {n: OK for n in ("Q", "Kc", "Vc", "table", "lens", "Y", "ws")} | {"ks": None, "vs": None} | other
    s = None if strides is None else (ctypes.c_int64 * 4)(*strides)
    return attn.lib().spt_attn_decode(ctypes.byref(shape), H, scale, p["Q"], s, p["Kc"], p["Vc"], p["ks"], p["vs"], p["table"], p["lens"], p["Y"],
                                      p["ws"], ws_bytes, None)


@pytest.mark.parametrize("change,code", [
    (dict(pages=0), ARG), (dict(page=0), ARG), (dict(Hk=0), ARG), (dict(dh=0), ARG), (dict(B=0), ARG), (dict(max_pages=0), ARG),
    (dict(max_pages=1 << 27), ARG), (dict(page=8), UNSUPPORTED), (dict(page=48), UNSUPPORTED), (dict(page=512), UNSUPPORTED),
    (dict(dh=80), UNSUPPORTED), (dict(format=2), UNSUPPORTED), (dict(format=-1), UNSUPPORTED), (dict(B=65536), UNSUPPORTED)])
def test_cache_shapes(change, code):
    s = pool(change)
    assert write(s) == code and write(s, read=True) == code and decode(s) == code
    assert attn.decode_workspace_bytes(s, 4) == 0


def test_cache_pointers_and_strides():
    s, s8 = pool(), pool(dict(format=attn.CACHE_E4M3))
    for read in (False, True):
        assert write(None, read=read) == ARG and write(s, T=0, read=read) == ARG and write(s, T=-1, read=read) == ARG
        for name in ("K", "V", "table", "start", "cu", "Kc", "Vc"):
            assert write(s, read=read, **{name: None}) == ARG, name
            assert write(s, read=read, **{name: BYTE}) == ARG, name
        assert write(s, read=read, ks=OK, vs=OK) == ARG                           # exponents of a cache that has none
        assert write(s8, read=read) == ARG and write(s8, read=read, ks=OK) == ARG and write(s8, read=read, ks=OK, vs=ODD) == ARG
        assert write(s, read=read, strides=[128, 64, 128, 60]) == ARG
        assert write(s, read=read, strides=[1 << 23, 64, 128, 64]) == UNSUPPORTED
    assert write(s, read=True, strides=[128, 64, 64, 64]) == ARG                  # rows that overlap, of an output


def test_decode_arguments():
    s, s8 = pool(), pool(dict(format=attn.CACHE_E4M3))
    assert decode(s, H=0) == ARG and decode(s, H=3) == ARG and decode(s, H=1 << 17) == UNSUPPORTED
    for scale in (0.0, -1.0, float("nan"), float("inf"), 3e38):
        assert decode(s, scale=scale) == ARG
    for name in ("Q", "Kc", "Vc", "table", "lens", "Y", "ws"):
        assert decode(s, **{name: None}) == ARG, name
        assert decode(s, **{name: BYTE}) == ARG, name
    assert decode(s8) == ARG and decode(s, ks=OK, vs=OK) == ARG
    assert decode(s, ws_bytes=16) == WORKSPACE
    assert decode(s, strides=[256, 64, 128, 64]) == ARG and decode(s, strides=[256, 12, 256, 64]) == ARG
    assert decode(pool(dict(max_pages=1 << 26, B=1024)), ws_bytes=1 << 40) == UNSUPPORTED
    small, large = attn.decode_workspace_bytes(s, 2), attn.decode_workspace_bytes(s, 64)
    assert 0 < small < large


def test_no_launch_of_2_to_32_threads():
    """A launch counts its threads in 32 bits: refused on the host, workspace sizes included."""
    s = pool(dict(B=65535))
    assert attn.decode_workspace_bytes(s, 128) > 0
    assert decode(s, H=130) == UNSUPPORTED and attn.decode_workspace_bytes(s, 130) == 0
    for read in (False, True):
        assert write(pool(), T=1 << 26, read=read) == UNSUPPORTED and write(pool(), T=2 ** 31 - 1, read=read) == UNSUPPORTED
    assert attn.prompt_workspace_bytes(attn.make_shape(4096, 1 << 20, 1 << 20, 128, 8, 64)) > 0
    for n in (dict(B=4096, Tq=1, Tk=1, H=2048, Hk=2048), dict(B=1, Tq=2 ** 31 - 1, Tk=1, H=1, Hk=1), dict(B=1, Tq=1, Tk=1 << 30, H=1, Hk=1),
              dict(B=1, Tq=1 << 28, Tk=1, H=4, Hk=1)):
        shape = attn.make_shape(dh=64, **n)
        assert fwd(shape) == UNSUPPORTED and bwd(shape) == UNSUPPORTED and attn.prompt_workspace_bytes(shape) == 0, n


def test_binding_refuses_before_it_calls():
    s = attn.make_shape(1, 4, 4, 2, 1, 64)
    q, k = ref.bf16(4, 2, 64, seed=1), ref.bf16(4, 1, 64, seed=2)
    cu = ref.sums([4])
    with pytest.raises(ValueError):
        attn.prompt_fwd(s, q, k, k, cu, cu)                                       # on the CPU
    with pytest.raises(ValueError):
        attn.decode(pool(), q, attn.Cache(k, k), cu, cu)
    with pytest.raises(spt.SptError):
        attn.alloc_prompt_workspace(attn.make_shape(1, 4, 4, 2, 1, 80), "cpu")
    with pytest.raises(spt.SptError):
        attn.alloc_decode_workspace(pool(dict(page=5)), 4, "cpu")
    assert attn.alloc_prompt_workspace(s, "cpu").numel() >= 4 * 2 * 4
    c = attn.alloc_cache(pool(dict(format=attn.CACHE_E4M3)), "cpu")
    assert c.K.shape == (9, 2, 16, 64) and c.K.dtype is torch.uint8 and c.ks.shape == (9, 2, 16)
    c = attn.alloc_cache(pool(), "cpu")
    assert c.V.dtype is torch.bfloat16 and c.ks is None and c.vs is None


@pytest.mark.parametrize("nq,nk,causal", [(7, 7, True), (5, 9, True), (9, 4, True), (6, 3, False)])
def test_reference_gradients_are_torch_autograd_s(nq, nk, causal):
    g = torch.Generator().manual_seed(3)
    q, k, v, dy = (torch.randn(n, h, 64, dtype=torch.float64, generator=g) for n, h in ((nq, 2), (nk, 1), (nk, 1), (nq, 2)))
    leaves = [t.clone().requires_grad_() for t in (q, k, v)]
    s = 0.1 * torch.matmul(leaves[0].transpose(0, 1), leaves[1].permute(1, 2, 0))
    seen = torch.from_numpy(ref.visible(nq, nk, causal))
    some = seen.any(1)
    p = torch.softmax(s.masked_fill(~seen, -1e300), -1) * some[None, :, None]
    y = torch.matmul(p, leaves[2].transpose(0, 1)).transpose(0, 1)
    y.backward(dy)
    out = ref.prompt(q.numpy(), k.numpy(), v.numpy(), [nq], [nk], causal, 0.1, dy.numpy())
    for name, t in (("Y", y), ("dQ", leaves[0].grad), ("dK", leaves[1].grad), ("dV", leaves[2].grad)):
        np.testing.assert_allclose(out[name][0], t.detach().numpy(), rtol=1e-10, atol=1e-12)


def test_reference_codes_are_torch_s():
    """Where torch's own conversion does not saturate it rounds alike."""
    x = torch.cat([torch.linspace(-448, 448, 4097), torch.tensor([2.0 ** -9, 2.0 ** -10, 1.5 * 2.0 ** -9, 0.0])]).double()
    codes, e = ref.quantise(x.numpy()[None])
    assert e[0] == 127
    assert np.array_equal(codes[0] & 0x7F, x.float().to(torch.float8_e4m3fn).view(torch.uint8).numpy() & 0x7F)
    assert np.array_equal(ref.values(codes, e)[0], x.float().to(torch.float8_e4m3fn).double().numpy())
