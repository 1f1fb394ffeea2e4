"""The attention of a decoder that is trained and served, as a list of timed cases: attention over packed
prompts, a paged cache of keys and values, and attention of one new token over that cache (`attn`).

A case is a dict of plain values.  `prepare` makes what a program holds before a pass, `run` is one pass:
with `own` through the library's calls, without it in plain operations of 32 bits.  `exact` is the
definition in 64 bits.  Four kinds of pass:

  prompt  attention of packed sequences, forward: prompts before the first answer, or a part of a
          prompt behind what was read before ("past"); an encoder's when not causal
  train   the same with its backward pass
  cache   new rows written into the pages of their sequences, and rows read back as the attention of a
          later part of the prompt takes them
  decode  one new token for each sequence over its pages

Lengths of the sequences of a case run evenly, over their logarithm, from the shortest to the longest."""
import math
import random

import torch

own = False

BF16, F32, I32, U8 = torch.bfloat16, torch.float32, torch.int32, torch.uint8


def prompt_case(kind, B, lo, hi, H, Hk, dh, causal=True, past_lo=0, past_hi=0, **name):
    return dict(kind=kind, B=B, lo=lo, hi=hi, H=H, Hk=Hk, dh=dh, causal=causal, past_lo=past_lo, past_hi=past_hi, **name)


def cache_case(B, lo, hi, Hk, dh, page, e4m3, past_lo=0, past_hi=0, **name):
    return dict(kind="cache", B=B, lo=lo, hi=hi, Hk=Hk, dh=dh, page=page, e4m3=e4m3, past_lo=past_lo, past_hi=past_hi, **name)


def decode_case(B, lo, hi, H, Hk, dh, page, e4m3, **name):
    return dict(kind="decode", B=B, lo=lo, hi=hi, H=H, Hk=Hk, dh=dh, page=page, e4m3=e4m3, **name)


def listed():
    return [
        # A question of one short sequence to a small model: the call and its launches are what the user waits for.
        prompt_case("prompt", 1, 77, 77, 12, 12, 64, name="prompt_short"),
        # Prompts of a serving batch, packed: a few words beside a document, four query heads to a key head.
        prompt_case("prompt", 16, 33, 2000, 32, 8, 128, name="prompt_packed"),
        # One long document: the largest forward pass.
        prompt_case("prompt", 1, 8192, 8192, 32, 8, 128, name="prompt_long"),
        # Parts of four prompts, behind 700 to 5000 tokens that were read before.
        prompt_case("prompt", 4, 512, 512, 32, 8, 128, past_lo=700, past_hi=5000, name="prompt_part"),
        # An encoder's batch of sentences: every token sees every other.
        prompt_case("train", 32, 20, 510, 16, 16, 64, causal=False, name="train_encoder"),
        # The block that the sparse attention is timed on, with all keys: 16 sequences of 512 tokens, 32 heads.
        prompt_case("train", 16, 512, 512, 32, 32, 64, name="train_opt2048"),
        # The larger block with grouped heads, documents of mixed lengths packed: the largest training pass.
        prompt_case("train", 6, 500, 4000, 32, 8, 128, name="train_packed"),
        # The next token's keys and values of a batch of 24 sequences: rows of a decoding step.
        cache_case(24, 1, 1, 8, 128, 16, True, past_lo=100, past_hi=4000, name="cache_step"),
        # Prompts of a batch of 16 written behind what their sequences hold, and read back for their attention.
        cache_case(16, 33, 4000, 8, 128, 64, True, past_lo=16, past_hi=1000, name="cache_prompts"),
        # One sequence with a short history, every head with keys of its own.
        decode_case(1, 700, 700, 32, 32, 64, 16, False, name="decode_one"),
        # A serving batch of mixed lengths on a cache of 8 bits.
        decode_case(48, 100, 8000, 32, 8, 128, 64, True, name="decode_batch"),
        # A few long documents on a cache of 16 bits: the largest decoding step.
        decode_case(6, 30000, 32700, 32, 8, 128, 256, False, name="decode_long"),
    ]


MOST_SCORES = 32 * 8192 * 8192        # entries of all score matrices of the listed long prompt, padded
MOST_TRAIN_SCORES = 6 * 32 * 4000 * 4000
MOST_ROWS = 16 * 4000 * 8 * 128       # values written
MOST_CACHE = 6 * 32700 * 8 * 128      # values of K that a decoding step reads


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case: every kind, lengths from one token to the longest, odd ones throughout, every grouping."""
    kind = rng.choice(["prompt", "prompt", "train", "train", "cache", "decode", "decode"])
    dh = rng.choice([64, 128])
    Hk = rng.choice([1, 2, 4, 8, 12, 16])
    H = Hk * rng.choice([1, 2, 3, 4, 8] if Hk <= 4 else [1, 2, 4])
    if kind in ("prompt", "train"):
        # (sequences of one token alone have no gradient of Q and K: there is nothing to compare)
        hi = _log(rng, 1, 8192) if kind == "prompt" else _log(rng, 2, 4096)
        lo = _log(rng, 1, hi)
        past = _log(rng, 1, 4096) if kind == "prompt" and rng.random() < 0.3 else 0
        most = MOST_SCORES if kind == "prompt" else MOST_TRAIN_SCORES
        B = max(1, min(_log(rng, 1, 32), most // (H * hi * (hi + past))))
        return prompt_case(kind, B, lo, hi, H, Hk, dh, causal=rng.random() < 0.75,
                           past_lo=_log(rng, 1, past) if past else 0, past_hi=past)
    page, e4m3 = rng.choice([16, 32, 64, 128, 256]), rng.random() < 0.5
    if kind == "cache":
        hi = 1 if rng.random() < 0.3 else _log(rng, 1, 8192)
        past = _log(rng, 1, 4096) if rng.random() < 0.7 else 0
        B = max(1, min(_log(rng, 1, 64), MOST_ROWS // ((hi + past) * Hk * dh)))
        return cache_case(B, _log(rng, 1, hi), hi, Hk, dh, page, e4m3, past_lo=_log(rng, 1, past) if past else 0, past_hi=past)
    hi = _log(rng, 1, 32768)
    B = max(1, min(_log(rng, 1, 64), MOST_CACHE // (hi * Hk * dh)))
    return decode_case(B, _log(rng, 1, hi), hi, H, Hk, dh, page, e4m3)


def _spread(lo, hi, B, salt):
    """B whole numbers from lo to hi, even over their logarithm, in an order of their own (one: hi)."""
    if hi == 0 or B == 1:
        return [hi] * B
    x = [int(round(math.exp(math.log(lo) + (math.log(hi) - math.log(lo)) * i / (B - 1)))) for i in range(B)]
    random.Random(salt).shuffle(x)
    return x


def _lengths(case):
    """(new rows, rows before them) of every sequence."""
    new = _spread(case["lo"], case["hi"], case["B"], 1)
    return new, _spread(case.get("past_lo", 0), case.get("past_hi", 0), case["B"], 2)


def _sums(x):
    out = [0]
    for v in x:
        out.append(out[-1] + v)
    return out


def _prefers(K, rows, H, g):
    """Queries as a trained model has them: each an even mix of a key that it may look at (`rows` of K) and noise."""
    T, Hk, dh = rows.shape[0], K.shape[1], K.shape[2]
    liked = K[rows].float().repeat_interleave(H // Hk, 1)
    return (0.7071 * (liked + torch.randn(T, H, dh, generator=g, device="cuda"))).to(BF16)


def _quantise(x):
    """Rows of x (last axis) as 8-bit codes and the exponent of a power of two for each row, biased by 127."""
    m, e = torch.frexp(x.abs().amax(-1))                     # amax = m 2^e, m in [1/2, 1); 448 = 7/8 2^9
    e = torch.clamp(torch.where(m <= 0.875, e - 9, e - 8), min=-127)
    return torch.ldexp(x, -e[..., None]).to(torch.float8_e4m3fn).view(U8), (e + 127).to(U8)


def _values(codes, exponents):
    return torch.ldexp(codes.view(torch.float8_e4m3fn).float(), exponents[..., None].int() - 127)


def _pages(case, lengths, g):
    """A pool of pages and the page numbers of every sequence, in no order; -1 behind a sequence's last page."""
    page = case["page"]
    need = [-(-n // page) for n in lengths]
    pages, width = sum(need) + 3, max(need)
    order = torch.randperm(pages, generator=g, device="cuda").to(I32)
    at = torch.arange(width, device="cuda")[None, :]
    count = torch.tensor(need, device="cuda")[:, None]
    first = torch.tensor(_sums(need)[:-1], device="cuda")[:, None]
    table = torch.where(at < count, order[torch.where(at < count, first + at, 0)], -1).to(I32).contiguous()
    return pages, width, table


def _new_cache(case, pages, g):
    """Pages full of what their last users left there."""
    shape = (pages, case["Hk"], case["page"], case["dh"])
    K, V = (torch.randn(shape, generator=g, device="cuda").to(BF16) for _ in range(2))
    if not case["e4m3"]:
        return K, V, None, None
    (kc, ks), (vc, vs) = _quantise(K.float()), _quantise(V.float())
    return kc, vc, ks, vs


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    kind, B, Hk, dh = (case[x] for x in ("kind", "B", "Hk", "dh"))
    ints = lambda x: torch.tensor(x, dtype=I32, device="cuda")
    normal = lambda *shape: torch.randn(*shape, generator=g, device="cuda").to(BF16)
    empty = lambda *shape, dtype=BF16: torch.empty(shape, dtype=dtype, device="cuda")
    new, past = _lengths(case)
    if kind in ("prompt", "train"):
        H, keys = case["H"], [n + p for n, p in zip(new, past)]
        Tq, Tk = sum(new), sum(keys)
        cu_q, cu_k = ints(_sums(new)), ints(_sums(keys))
        K, V = normal(Tk, Hk, dh), normal(Tk, Hk, dh)
        # the key that a query prefers: any of its sequence up to its own place
        seq = torch.repeat_interleave(torch.arange(B, device="cuda"), ints(new))
        place = torch.arange(Tq, device="cuda") - cu_q[seq] + ints(past)[seq]
        liked = cu_k[seq] + (torch.rand(Tq, generator=g, device="cuda") * (place + 1)).long().clamp(max=place)
        s = dict(case=case, new=new, keys=keys, cu_q=cu_q, cu_k=cu_k, Q=_prefers(K, liked, H, g), K=K, V=V,
                 Y=empty(Tq, H, dh), scale=dh ** -0.5)
        if kind == "train":
            s.update(dY=normal(Tq, H, dh), lse=empty(H, Tq, dtype=F32), dQ=empty(Tq, H, dh), dK=empty(Tk, Hk, dh), dV=empty(Tk, Hk, dh))
        if own:
            from paper_2312_10365_amd import attn
            s["shape"] = attn.make_shape(B, Tq, Tk, H, Hk, dh, causal=case["causal"], scale=s["scale"])
            if kind == "train":
                s["ws"] = attn.alloc_prompt_workspace(s["shape"])
        return s
    whole = [n + p for n, p in zip(new, past)]
    pages, width, table = _pages(case, whole, g)
    cache = _new_cache(case, pages, g)
    s = dict(case=case, table=table, cache=cache, new=new, whole=whole)
    if own:
        from paper_2312_10365_amd import attn
        s["shape"] = attn.make_cache_shape(pages, case["page"], Hk, dh, B, width, attn.CACHE_E4M3 if case["e4m3"] else attn.CACHE_BF16)
    if kind == "cache":
        # a decoding step's rows are read back alone, a prompt's with all that its sequence holds
        back, first = (new, past) if max(new) == 1 else (whole, [0] * B)
        s.update(K=normal(sum(new), Hk, dh), V=normal(sum(new), Hk, dh), start=ints(past), cu=ints(_sums(new)),
                 back=back, back_cu=ints(_sums(back)), back_start=ints(first), Kr=empty(sum(back), Hk, dh), Vr=empty(sum(back), Hk, dh))
        return s
    H, page = case["H"], case["page"]
    lens = ints(whole)
    pos = (torch.rand(B, generator=g, device="cuda") * lens).long().clamp(max=lens - 1)
    rows = cache[0][table[torch.arange(B, device="cuda"), pos // page].long(), :, pos % page]
    K = _values(rows, cache[2][table[torch.arange(B, device="cuda"), pos // page].long(), :, pos % page]) if case["e4m3"] else rows
    s.update(lens=lens, Q=_prefers(K, torch.arange(B, device="cuda"), H, g), Y=empty(B, H, dh), scale=dh ** -0.5)
    if own:
        s["ws"] = attn.alloc_decode_workspace(s["shape"], H)
    return s


def _padded(x, cu, most):
    """Packed rows x [T, heads, dh] as [B, heads, most, dh], zero behind a sequence's end; and which rows are there."""
    at = torch.arange(most, device=x.device)
    first, end = cu[:-1, None].long(), cu[1:, None].long()
    there = at[None, :] < end - first
    rows = torch.where(there, first + at[None, :], 0)
    return (x[rows].float() * there[..., None, None]).transpose(1, 2), there


def _visible(there_q, there_k, causal):
    """Which keys each query sees, [B, queries, keys]."""
    seen = there_q[:, :, None] & there_k[:, None, :]
    if causal:
        i = torch.arange(there_q.shape[1], device=seen.device)[None, :, None]
        j = torch.arange(there_k.shape[1], device=seen.device)[None, None, :]
        seen = seen & (j <= i + (there_k.sum(1) - there_q.sum(1))[:, None, None])
    return seen


def _softmax(scores, seen):
    """Softmax over the seen entries of the last axis (a row that sees nothing: zeros), and its log-sum-exp."""
    scores = scores.masked_fill_(~seen, -math.inf)
    top = scores.amax(-1, keepdim=True)
    weights = torch.exp_(scores.sub_(torch.where(top == -math.inf, 0.0, top)))
    total = weights.sum(-1, keepdim=True)
    return weights.div_(torch.where(total == 0, 1.0, total)), (top + torch.log(total)).squeeze(-1)


def _plain_prompt(s):
    c = s["case"]
    B, H, Hk, dh, G = c["B"], c["H"], c["Hk"], c["dh"], c["H"] // c["Hk"]
    nq, nk = max(s["new"]), max(s["keys"])
    q, there_q = _padded(s["Q"], s["cu_q"], nq)
    k, there_k = _padded(s["K"], s["cu_k"], nk)
    v, _ = _padded(s["V"], s["cu_k"], nk)
    seen = _visible(there_q, there_k, c["causal"])[:, None, None]
    grouped = lambda x: x.reshape(B, Hk, G * nq, dh)           # a group's heads and queries in one axis
    apart = lambda x: x.reshape(B, Hk, G, nq, -1)
    packed = lambda x, there: x.transpose(1, 2)[there]
    q = grouped(q)
    p, lse = _softmax(apart(torch.matmul(q, k.transpose(-1, -2))).mul_(s["scale"]), seen)
    p = p.reshape(B, Hk, G * nq, nk)
    y = torch.matmul(p, v)
    heads = lambda x: packed(x.reshape(B, H, nq, dh), there_q)
    out = dict(Y=heads(y).to(BF16))
    if c["kind"] == "prompt":
        return out
    dy = grouped(_padded(s["dY"], s["cu_q"], nq)[0])
    dv = torch.matmul(p.transpose(-1, -2), dy)
    ds = torch.matmul(dy, v.transpose(-1, -2)).sub_((dy * y).sum(-1, keepdim=True)).mul_(p).mul_(s["scale"])
    dq, dk = torch.matmul(ds, k), torch.matmul(ds.transpose(-1, -2), q)
    out.update(lse=lse.reshape(B, H, nq).permute(1, 0, 2)[:, there_q], dQ=heads(dq).to(BF16),
               dK=packed(dk, there_k).to(BF16), dV=packed(dv, there_k).to(BF16))
    return out


def _places(table, page, cu, start, lengths):
    """Page, and place in it, of every packed row: row r of sequence b is token start[b] + r - cu[b]."""
    T = sum(lengths)
    seq = torch.repeat_interleave(torch.arange(len(lengths), device=table.device), (cu[1:] - cu[:-1]).long(), output_size=T)
    pos = start[seq].long() + torch.arange(T, device=table.device) - cu[seq].long()
    return table[seq, pos // page].long(), pos % page


def _plain_cache(s):
    c, (kc, vc, ks, vs) = s["case"], s["cache"]
    page, at = _places(s["table"], c["page"], s["cu"], s["start"], s["new"])
    if c["e4m3"]:
        (kc[page, :, at], ks[page, :, at]), (vc[page, :, at], vs[page, :, at]) = _quantise(s["K"].float()), _quantise(s["V"].float())
    else:
        kc[page, :, at], vc[page, :, at] = s["K"], s["V"]
    page, at = _places(s["table"], c["page"], s["back_cu"], s["back_start"], s["back"])
    if not c["e4m3"]:
        return dict(K=kc[page, :, at], V=vc[page, :, at])
    return dict(K=_values(kc[page, :, at], ks[page, :, at]).to(BF16), V=_values(vc[page, :, at], vs[page, :, at]).to(BF16))


def _plain_decode(s):
    c, (kc, vc, ks, vs) = s["case"], s["cache"]
    B, H, Hk, dh, page = (c[x] for x in ("B", "H", "Hk", "dh", "page"))
    n = max(s["whole"])
    pos = torch.arange(n, device="cuda")
    number = s["table"][:, pos // page].long()
    seen = pos[None, :] < s["lens"][:, None]
    number, at = torch.where(seen, number, 0), (pos % page)[None, :].expand(B, n)
    rows = lambda codes, e: (codes[number, :, at].float() if e is None else _values(codes[number, :, at], e[number, :, at])).transpose(1, 2)
    k, v = rows(kc, ks), rows(vc, vs)
    scores = torch.matmul(s["Q"].float().reshape(B, Hk, H // Hk, dh), k.transpose(-1, -2)).mul_(s["scale"])
    p, _ = _softmax(scores, seen[:, None, None, :])
    return dict(Y=torch.matmul(p, v * seen[:, None, :, None]).reshape(B, H, dh).to(BF16))


def run(s):
    kind = s["case"]["kind"]
    if not own:
        return (_plain_cache if kind == "cache" else _plain_decode if kind == "decode" else _plain_prompt)(s)
    from paper_2312_10365_amd import attn
    if kind == "decode":
        attn.decode(s["shape"], s["Q"], s["cache"], s["table"], s["lens"], scale=s["scale"], ws=s["ws"], Y=s["Y"])
        return dict(Y=s["Y"])
    if kind == "cache":
        attn.cache_write(s["shape"], s["K"], s["V"], s["cache"], s["table"], s["start"], s["cu"])
        attn.cache_read(s["shape"], s["cache"], s["table"], s["back_start"], s["back_cu"], K=s["Kr"], V=s["Vr"])
        return dict(K=s["Kr"], V=s["Vr"])
    rows = (s["Q"], s["K"], s["V"])
    if kind == "prompt":
        attn.prompt_fwd(s["shape"], *rows, s["cu_q"], s["cu_k"], Y=s["Y"], save_for_backward=False)
        return dict(Y=s["Y"])
    attn.prompt_fwd(s["shape"], *rows, s["cu_q"], s["cu_k"], Y=s["Y"], lse=s["lse"])
    attn.prompt_bwd(s["shape"], *rows, s["Y"], s["dY"], s["lse"], s["cu_q"], s["cu_k"], ws=s["ws"], dQ=s["dQ"], dK=s["dK"], dV=s["dV"])
    return {x: s[x] for x in ("Y", "lse", "dQ", "dK", "dV")}


def _pairs(nq, nk, causal):
    """Pairs of a query and a key that it sees."""
    return sum(min(nk, max(0, i + 1 + nk - nq)) for i in range(nq)) if causal else nq * nk


def work(case):
    new, past = _lengths(case)
    keys = [n + p for n, p in zip(new, past)]
    kind, Hk, dh = case["kind"], case["Hk"], case["dh"]
    if kind in ("prompt", "train"):
        H, Tq, Tk = case["H"], sum(new), sum(keys)
        pairs = H * sum(_pairs(n, m, case["causal"]) for n, m in zip(new, keys))
        rows = 2 * dh * (2 * Tq * H + 2 * Tk * Hk)             # Q, Y; K, V
        if kind == "prompt":
            return {"bytes": rows, "flops": 4 * dh * pairs}
        return {"bytes": 2 * rows + 4 * H * Tq, "flops": 14 * dh * pairs}     # and dQ, dY, dK, dV, lse
    held = (dh + 1) if case["e4m3"] else 2 * dh                # bytes of a row in the cache
    if kind == "cache":
        back = new if max(new) == 1 else keys
        return {"bytes": 2 * Hk * (sum(new) + sum(back)) * (2 * dh + held), "flops": 0}
    H = case["H"]
    return {"bytes": 2 * Hk * sum(keys) * held + 2 * case["B"] * H * 2 * dh, "flops": 4 * dh * H * sum(keys)}


# ---- the definition in 64 bits: one sequence at a time, nothing shared with the plain form


def _one(q, k, v, scale, causal):
    """Attention of one sequence, q [nq, H, dh], k, v [nk, H, dh] (float64): y, lse [H, nq]."""
    nq, nk = q.shape[0], k.shape[0]
    s = scale * torch.bmm(q.transpose(0, 1).contiguous(), k.permute(1, 2, 0).contiguous())
    if causal:
        i, j = torch.arange(nq, device=q.device), torch.arange(nk, device=q.device)
        s = s + torch.where(j[None, :] > i[:, None] + (nk - nq), -math.inf, 0.0)
    lse = torch.logsumexp(s, -1)
    return torch.bmm(torch.exp(s - lse[..., None]), v.transpose(0, 1).contiguous()).transpose(0, 1), lse


def _exact_prompt(s):
    c, G, parts = s["case"], s["case"]["H"] // s["case"]["Hk"], []
    cq, ck = s["cu_q"].tolist(), s["cu_k"].tolist()
    for b in range(c["B"]):
        q, k, v = (s[x][lo[b]:lo[b + 1]].double() for x, lo in (("Q", cq), ("K", ck), ("V", ck)))
        heads = []
        for h in range(c["Hk"]):                               # a key head at a time: the score matrices are large
            qh, kh, vh = q[:, h * G:(h + 1) * G], k[:, h:h + 1], v[:, h:h + 1]
            if c["kind"] == "train":
                leaves = [x.clone().requires_grad_() for x in (qh, kh, vh)]
                y, lse = _one(leaves[0], leaves[1].expand(-1, G, -1), leaves[2].expand(-1, G, -1), s["scale"], c["causal"])
                dy = s["dY"][cq[b]:cq[b + 1], h * G:(h + 1) * G].double()
                heads.append((y.detach(), *torch.autograd.grad(y, leaves, dy), lse.detach()))
            else:
                heads.append(_one(qh, kh.expand(-1, G, -1), vh.expand(-1, G, -1), s["scale"], c["causal"])[:1])
        parts.append([torch.cat(x, 0 if n == 4 else 1) for n, x in enumerate(zip(*heads))])
    parts = [torch.cat(x, 1 if n == 4 else 0) for n, x in enumerate(zip(*parts))]
    return dict(zip(("Y", "dQ", "dK", "dV", "lse"), parts))


def _nearest_e4m3(x):
    """Nearest number of three fraction bits, from 2^-6 (below it: multiples of 2^-9) to 448; ties to even."""
    step = torch.exp2(torch.floor(torch.log2(x.abs().clamp(min=2.0 ** -6))) - 3)
    return torch.round(x / step) * step


def _held(x, e4m3):
    """What a row of the cache stands for."""
    if not e4m3:
        return x
    top = x.abs().amax(-1, keepdim=True)
    unit = torch.exp2(torch.ceil(torch.log2(top.clamp(min=448 * 2.0 ** -127) / 448)))
    return _nearest_e4m3(x / unit) * unit


def _cached(s, which, b, lo, hi):
    """Rows lo to hi of sequence b as the pages hold them."""
    page, codes, e = s["case"]["page"], s["cache"][which], s["cache"][which + 2]
    at = torch.arange(lo, hi, device="cuda")
    number = s["table"][b].long()[at // page]
    x = codes[number, :, at % page]
    return x.double() if e is None else x.view(torch.float8_e4m3fn).double() * torch.exp2(e[number, :, at % page].double() - 127)[..., None]


def exact(case, seed):
    s = prepare(case, seed)
    if case["kind"] in ("prompt", "train"):
        return _exact_prompt(s)
    if case["kind"] == "cache":
        cu, out = s["cu"].tolist(), {}
        for which, x in enumerate(("K", "V")):
            rows = []
            for b in range(case["B"]):
                past, first = s["whole"][b] - s["new"][b], s["back_start"][b].item()
                rows += [_cached(s, which, b, first, past), _held(s[x][cu[b]:cu[b + 1]].double(), case["e4m3"])]
            out[x] = torch.cat(rows)
        return out
    out, G = [], case["H"] // case["Hk"]
    for b in range(case["B"]):
        k, v = (_cached(s, which, b, 0, s["whole"][b]).repeat_interleave(G, 1) for which in (0, 1))
        out.append(_one(s["Q"][b:b + 1].double(), k, v, s["scale"], False)[0])
    return dict(Y=torch.cat(out))
