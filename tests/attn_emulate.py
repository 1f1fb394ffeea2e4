"""The kernels' own arithmetic in 64 bits with their roundings to bf16 at the places where they make them: how far off a
result is to be as a whole (2-norm), where the bounds of attn_ref.py, which add up the worst of every element, would not
tell one rounding from two.

A rounding's error is even over half a step, so errors of another order of sums, or of weights scaled to another maximum,
have the same second moment; the norm over n values fluctuates by about 1 / sqrt(n) of itself, here a few percent.  FACTOR leaves 20 % for that and
for the operations of 32 bits (2^-24 each, against 2^-9).  `mistake` leaves out or turns round what the kernels do about
their roundings: the limits must not hold then."""
import numpy as np
import torch

import attn_ref as ref

FACTOR = 1.2

# Passes that reach every form of the gradients' kernels: lengths of queries, of keys, H, Hk, head dimensions, causal, whether dS is the sum
# of two bf16, rows of Q and of K behind the last sequence (forms are chosen by the rows of the tensors); behind each the
# wavefronts of a workgroup that own 32 rows, on the side of the queries and of the keys
PASSES = {
    "short": ([2 + i % 8 for i in range(40)], None, 4, 2, (64, 128), True, True, 0, 0),                   # 4, 4
    "short_full": ([9 - i % 8 for i in range(40)], None, 3, 3, (64, 128), False, True, 0, 0),             # 4, 4
    "few": ([170, 330], None, 4, 2, (64, 128), True, True, 0, 0),                                         # 1, 1
    "few_full": ([330, 170], None, 2, 2, (64, 128), False, True, 0, 0),                                   # 1, 1
    "parts": ([100] * 12, [300] * 12, 8, 8, (64, 128), True, True, 0, 0),                                 # 2, 4
    "more_keys": ([200], [1200], 8, 8, (64, 128), False, True, 0, 0),                                     # 1, 2
    "rows_in_64s": ([300, 250], None, 16, 16, (64, 128), True, False, 0, 0),                              # 2, 2
    "grouped": ([130] * 4, None, 32, 8, (64, 128), True, False, 0, 0),                                    # 4, 1
    "rows_in_128s": ([150] * 8, None, 8, 8, (64, 128), True, False, 0, 0),                                # 4, 4
    "rows_in_128s_full": ([150] * 8, None, 8, 8, (64, 128), False, False, 0, 0),                          # 4, 4
    "keys_in_256s": ([300, 270], None, 4, 4, (128,), False, False, 9000, 16000),                          # 4, 8
    "keys_in_256s_exact": ([300, 270], None, 4, 4, (128,), False, True, 0, 16000),                        # 1, 8
}
# single tokens: lengths, H, Hk, dh, tokens of a page
TOKENS = {
    "four_heads": ([300, 100, 2000], 8, 2, 128, 16),
    "twenty_heads": ([500, 1300], 40, 2, 64, 64),
    "own_keys": ([900, 333], 6, 6, 64, 256),
}


def inputs(lens_q, lens_k, H, Hk, dh, sharp, seed=1):
    Q, K, V, dY = (ref.bf16(sum(n), h, dh, seed=seed + i) for i, (n, h) in enumerate(((lens_q, H), (lens_k, Hk), (lens_k, Hk), (lens_q, H))))
    return (Q.float() * sharp).to(torch.bfloat16), K, V, dY


def bf(x):
    return torch.from_numpy(np.ascontiguousarray(x)).to(torch.bfloat16).double().numpy()


def two(x):
    hi = bf(x)
    return hi + bf(x - hi)


def forward(q, k, v, scale, seen):
    """Y of one head: weights go into their product as one bf16, scaled to a maximum that may be one of the row's earlier
    ones: to any number, here another for every row, evenly over a power of two."""
    s = np.where(seen, scale * (q @ k.T), -np.inf)
    top = s.max(-1, initial=-np.inf, keepdims=True)
    w = np.where(seen, np.exp(s - np.where(top == -np.inf, 0.0, top)), 0.0) * 2.0 ** (np.arange(len(q)) * 0.618034 % 1.0)[:, None]
    total = w.sum(-1, keepdims=True)
    return bf(bf(w) @ v / np.where(total == 0, 1.0, total))


def backward(q, k, v, dy, scale, seen, exact_ds, mistake):
    """dQ, and dK, dV before their rounding, of one head.  Y is rounded, so D is off: the sum of a row's dS, which is 0 but
    for that, is taken off.  dS is the sum of two bf16 (`exact_ds`) or one."""
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


def _heads(f, Q, K, V, lens_q, lens_k, causal, dY, gone):
    """f's {name: values} of all sequences and heads, packed.  `gone`: rows of K whose scores are -inf."""
    G = Q.shape[1] // K.shape[1]
    out = {"Y": np.zeros(Q.shape), "dQ": np.zeros(Q.shape), "dK": np.zeros(K.shape), "dV": np.zeros(K.shape)}
    there = ~np.isin(np.arange(len(K)), gone)
    K = np.where(there[:, None, None], K, 0.0)
    a = b = 0
    for nq, nk in zip(lens_q, lens_k):
        rq, rk = slice(a, a + nq), slice(b, b + nk)
        seen = ref.visible(nq, nk, causal) & there[None, rk]
        for h in range(Q.shape[1]):
            one = f(Q[rq, h], K[rk, h // G], V[rk, h // G], dY[rq, h], seen)
            for n, x in one.items():
                if n in ("dK", "dV"):
                    out[n][rk, h // G] += x
                else:
                    out[n][rq, h] = x
        a, b = a + nq, b + nk
    return out


def prompt(Q, K, V, lens_q, lens_k, causal, scale, dY, exact_ds, mistake=None, gone=()):
    """{name: value} of a backward pass and its forward, with the kernels' roundings."""
    def f(q, k, v, dy, seen):
        return {"Y": forward(q, k, v, scale, seen)} | dict(zip(("dQ", "dK", "dV"), backward(q, k, v, dy, scale, seen, exact_ds, mistake)))
    out = _heads(f, Q, K, V, lens_q, lens_k, causal, dY, gone)
    return out | {n: bf(out[n]) for n in ("dK", "dV")}


def exact(Q, K, V, lens_q, lens_k, causal, scale, dY, gone=()):
    """The same without roundings."""
    def f(q, k, v, dy, seen):
        return {n: x for n, (x, _) in ref.head(q, k, v, scale, seen, dy).items() if n != "lse"}
    return _heads(f, Q, K, V, lens_q, lens_k, causal, dY, gone)


def decode(Q, K, V, lens, scale, mistake=None, exact=False):
    """Y [B, H, dh] of single tokens: weights go into their product as the sum of two bf16."""
    G, ends, Y = Q.shape[1] // K.shape[1], np.cumsum([0] + list(lens)), np.zeros(Q.shape)
    for b in range(len(lens)):
        rows = slice(ends[b], ends[b + 1])
        for h in range(Q.shape[1]):
            s = scale * (K[rows, h // G] @ Q[b, h])
            w = np.exp(s - s.max())
            Y[b, h] = (w if exact else bf(w) if mistake == "one weight" else two(w)) @ V[rows, h // G] / w.sum()
    return Y if exact else bf(Y)


def off(got, want):
    """2-norm of the error, relative."""
    return np.linalg.norm(got - want) / np.linalg.norm(want)
