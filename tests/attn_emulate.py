"""The kernels' own arithmetic in 64 bits with their roundings to bf16 at the places where they make them, one sequence at a
time: how far off a result is to be as a whole (2-norm), where the bounds of attn_ref.py, which add up the worst of every
element, would not tell one rounding from two.

A rounding's error is even over half a step, so errors of other inputs, another order of sums or other maxima to which weights are scaled have
the same second moment; the norm over n values fluctuates by about 1 / sqrt(n) of it.  FACTOR leaves 25 % for that and for
the operations of 32 bits (2^-24 each, against 2^-9).  `mistake` leaves out or turns round what the kernels do about their roundings: a test of
the limits, which must not hold then."""
import numpy as np
import torch

import attn_ref as ref

FACTOR = 1.25


def bf(x):
    return torch.from_numpy(np.ascontiguousarray(x)).to(torch.bfloat16).double().numpy()


def two(x):
    hi = bf(x)
    return hi + bf(x - hi)


def forward(q, k, v, scale, seen, mistake=None):
    """Y of one head: weights, scaled to their row's largest, go into their product as one bf16."""
    s = np.where(seen, scale * (q @ k.T), -np.inf)
    top = s.max(-1, initial=-np.inf, keepdims=True)
    w = np.where(seen, np.exp(s - np.where(top == -np.inf, 0.0, top)), 0.0)
    total = w.sum(-1, keepdims=True)
    return bf(bf(w) @ v / np.where(total == 0, 1.0, total))


def backward(q, k, v, dy, scale, seen, exact_ds, mistake=None):
    """dQ, and dK, dV before their rounding, of one head.  Y is rounded, so D is off: the sum of a row's dS, which is 0 but for
    that, is taken off.  dS is the sum of two bf16 (`exact_ds`) or one."""
    p, _ = ref.softmax(scale * (q @ k.T), seen)
    D = (dy * forward(q, k, v, scale, seen)).sum(-1, keepdims=True)
    dP = dy @ v.T
    rounded = two if exact_ds and mistake != "one dS" else bf
    sign = {"no correction": 0.0, "correction turned round": -1.0}.get(mistake, 1.0)
    dS = p * (dP - D)
    left, dS_in, p_in = dS.sum(-1, keepdims=True), rounded(dS), bf(p)
    mass = p_in.sum(-1, keepdims=True)
    off_by = sign * (left / np.where(mass == 0, 1.0, mass) if exact_ds else dS_in.sum(-1, keepdims=True))
    dQ = bf(scale * (dS_in @ k - off_by * (p_in @ k)))
    return dQ, scale * rounded(p * (dP - (D + sign * left))).T @ q, p_in.T @ dy


def prompt(Q, K, V, lens_q, lens_k, causal, scale, dY, exact_ds, mistake=None):
    """All sequences and heads, packed: {name: value}."""
    G = Q.shape[1] // K.shape[1]
    out = {"Y": np.zeros(Q.shape), "dQ": np.zeros(Q.shape), "dK": np.zeros(K.shape), "dV": np.zeros(K.shape)}
    a = b = 0
    for nq, nk in zip(lens_q, lens_k):
        rq, rk, seen = slice(a, a + nq), slice(b, b + nk), ref.visible(nq, nk, causal)
        for h in range(Q.shape[1]):
            one = Q[rq, h], K[rk, h // G], V[rk, h // G]
            out["Y"][rq, h] = forward(*one, scale, seen)
            dQ, dK, dV = backward(*one, dY[rq, h], scale, seen, exact_ds, mistake)
            out["dQ"][rq, h] = dQ
            out["dK"][rk, h // G] += dK
            out["dV"][rk, h // G] += dV
        a, b = a + nq, b + nk
    return out | {n: bf(out[n]) for n in ("dK", "dV")}


def decode(q, k, v, scale, mistake=None):
    """One query head over its keys: weights go into their product as the sum of two bf16."""
    s = scale * (k @ q)
    w = np.exp(s - s.max())
    return bf(((bf if mistake == "one weight" else two)(w) @ v) / w.sum())


def off(got, want):
    """2-norm of the error, relative."""
    return np.linalg.norm(got - want) / np.linalg.norm(want)
