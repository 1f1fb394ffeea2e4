"""Attention of packed sequences, the paged cache and single tokens over it in 64 bits, one sequence and head at a time,
and how far bf16 results may be from it, element by element.

U is bf16's half step relative to a value.  Y: P and the result are rounded, each by U; dV the same with P, dK and dQ with
dS, whose D comes from a Y that is rounded too.  A score is a sum of dh products in 32 bits, off by S32 times the sum of their
magnitudes, and an exponential of it by as much relatively; 2^-18 covers the other operations of 32 bits (sums of up to
a few thousand weights of one sign, exponential, logarithm, division)."""
import numpy as np
import torch

U = 2.0 ** -8
E32 = 2.0 ** -18


def s32(dh):
    return (dh + 4) * 2.0 ** -24


def visible(nq, nk, causal):
    i, j = np.arange(nq)[:, None], np.arange(nk)[None, :]
    return (j <= i + nk - nq) if causal else np.ones((nq, nk), bool)


def softmax(s, seen):
    """Weights over the seen scores (rows without any above -inf: zeros) and log-sum-exp."""
    s = np.where(seen, s, -np.inf)
    top = s.max(-1, initial=-np.inf, keepdims=True)
    e = np.where(seen & (s > -np.inf), np.exp(s - np.where(top == -np.inf, 0.0, top)), 0.0)
    total = e.sum(-1, keepdims=True)
    with np.errstate(divide="ignore"):
        return e / np.where(total == 0, 1.0, total), (np.where(total == 0, -np.inf, top + np.log(total)))[..., 0]


def head(q, k, v, scale, seen, dy=None):
    """One head of one sequence: {name: (value, how far off a bf16 result may be)}; lse has its own bound."""
    dh = q.shape[1]
    k, v = (np.where(seen.any(0)[:, None], x, 0.0) for x in (k, v))     # what no query sees does not matter
    p, lse = softmax(scale * (q @ k.T), seen)
    mag = scale * (np.abs(q) @ np.abs(k).T)
    ds32 = np.where(seen, mag, 0.0) * s32(dh) + E32
    wide = ds32.max(-1, initial=0.0, keepdims=True)                     # the sum's error too
    y = p @ v
    yt = U * np.abs(y) + (p * (U * 1.01 + ds32 + wide)) @ np.abs(v)
    out = {"Y": (y, yt * 1.02 + 1e-30), "lse": (lse, wide[:, 0] + E32 * np.where(np.isfinite(lse), np.abs(lse), 0.0))}
    if dy is None:
        return out
    D = (dy * y).sum(-1, keepdims=True)
    dP = dy @ v.T
    dS = p * (dP - D)
    p_off = p * (ds32 + wide)
    D_off = (np.abs(dy) * (U * np.abs(y))).sum(-1, keepdims=True) + s32(dh) * (np.abs(dy) * np.abs(y)).sum(-1, keepdims=True)
    dS_off = (U * 1.01) * np.abs(dS) + p * (D_off + s32(dh) * (np.abs(dy) @ np.abs(v).T)) + p_off * np.abs(dP - D)
    out["dQ"] = scale * dS @ k, U * np.abs(scale * dS @ k) + scale * dS_off @ np.abs(k)
    out["dK"] = scale * dS.T @ q, scale * dS_off.T @ np.abs(q)          # (rounded once, after the sum over heads)
    out["dV"] = p.T @ dy, (p * (U * 1.01) + p_off).T @ np.abs(dy)
    return out


def prompt(Q, K, V, lens_q, lens_k, causal, scale, dY=None):
    """All sequences and heads: {name: (value, bound)}, packed as the library packs them (float64 numpy)."""
    H, Hk, dh = Q.shape[1], K.shape[1], Q.shape[2]
    names = {"Y": Q.shape, "lse": (H, Q.shape[0])} | ({} if dY is None else {"dQ": Q.shape, "dK": K.shape, "dV": K.shape})
    out = {n: (np.zeros(s), np.zeros(s)) for n, s in names.items()}
    a = b = 0
    for nq, nk in zip(lens_q, lens_k):
        rq, rk = slice(a, a + nq), slice(b, b + nk)
        seen = visible(nq, nk, causal)
        for h in range(H):
            kh = h // (H // Hk)
            one = head(Q[rq, h], K[rk, kh], V[rk, kh], scale, seen, None if dY is None else dY[rq, h])
            for n, (x, t) in one.items():
                if n == "lse":
                    out[n][0][h, rq], out[n][1][h, rq] = x, t
                elif n in ("dK", "dV"):
                    out[n][0][rk, kh] += x
                    out[n][1][rk, kh] += t
                else:
                    out[n][0][rq, h], out[n][1][rq, h] = x, t
        a, b = a + nq, b + nk
    for n in ("dQ", "dK", "dV"):
        if n in out:
            x, t = out[n]
            out[n] = x, t * 1.02 + (0.0 if n == "dQ" else U * 1.02 * np.abs(x)) + 1e-30
    return out


# e4m3: sign, 4 exponent bits (bias 7), 3 fraction bits; the all-ones code is NaN
def _e4m3():
    c = np.arange(128)
    e, f = c >> 3, c & 7
    x = np.where(e == 0, f * 2.0 ** -9, (8 + f) * 2.0 ** (e.astype(float) - 10))
    return x[:127]                                                      # 0 .. 448, ascending


CODES = _e4m3()


def quantise(x):
    """Codes and exponent bytes of rows x (float64 numpy, last axis): the definition, by search."""
    finite = np.isfinite(x)
    top = np.where(finite, np.abs(x), 0.0).max(-1)
    e = np.full(top.shape, -127)
    for n in range(-127, 121):                                          # the least exponent that holds the row
        e = np.where(top > 448 * 2.0 ** n, n + 1, e)
    a = np.where(finite, np.abs(x), 0.0) * 2.0 ** -e[..., None].astype(float)
    lo = np.clip(np.searchsorted(CODES, a, side="right") - 1, 0, 126)
    hi = np.minimum(lo + 1, 126)
    dl, dh_ = a - CODES[lo], CODES[hi] - a
    code = np.where((dl < dh_) | ((dl == dh_) & (lo % 2 == 0)) | (lo == hi), lo, hi)
    code = np.where(e[..., None] == 120, np.minimum(code, 119), code)   # (240 2^120 is the largest that bf16 has)
    code = np.where(finite, code, 127) | np.where(np.signbit(x), 128, 0)
    return code.astype(np.uint8), (e + 127).astype(np.uint8)


def values(codes, bytes_):
    table = np.concatenate([CODES, [np.nan], -CODES, [np.nan]])
    return table[codes] * 2.0 ** (bytes_.astype(float) - 127)[..., None]


def f64(t):
    return t.detach().double().cpu().numpy()


def bf16(*shape, seed, std=1.0):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(*shape, generator=g) * std).to(torch.bfloat16)


def sums(x):
    return torch.tensor(np.concatenate([[0], np.cumsum(x)]), dtype=torch.int32)


def check(name, got, want, bound):
    """Every element within its bound; what is not finite in one is the same in the other."""
    g = f64(got) if isinstance(got, torch.Tensor) else got
    assert g.shape == want.shape, (name, g.shape, want.shape)
    same = (g == want) | (np.isnan(g) & np.isnan(want))
    fine = np.isfinite(want) & np.isfinite(g)
    off = np.where(fine, np.abs(np.where(fine, g, 0.0) - np.where(fine, want, 0.0)) - bound, 0.0)
    wrong = ~same & (~fine | (off > 0))
    assert not wrong.any(), (f"{name}: {wrong.sum()} of {wrong.size} off, first at {tuple(np.argwhere(wrong)[0])}: "
                             f"{g[tuple(np.argwhere(wrong)[0])]} for {want[tuple(np.argwhere(wrong)[0])]}, bound {bound[tuple(np.argwhere(wrong)[0])]}")
