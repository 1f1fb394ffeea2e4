"""Attention over packed sequences, the paged cache and single tokens over it, through the C ABI, against the definition in
64 bits (attn_ref.py), every element within what the roundings allow."""
import numpy as np
import pytest
import torch

import attn_ref as ref
from paper_2312_10365_amd import attn

pytestmark = pytest.mark.gpu

MIXED = [0, 1, 2, 31, 32, 33, 63, 64, 65, 127, 128, 129, 200]
# lengths of queries, of keys, H, Hk, dh, causal
PROMPTS = {
    "one_token": ([1], [1], 1, 1, 64, True),
    "two_tokens": ([2], [2], 2, 1, 128, True),
    "tile_edges_64": (MIXED, MIXED, 2, 2, 64, True),
    "tile_edges_128": (MIXED, MIXED, 4, 1, 128, True),
    "tile_edges_full": (MIXED, MIXED, 2, 1, 128, False),
    "full_64": ([70, 0, 5, 161], [70, 0, 5, 161], 3, 3, 64, False),
    "three_heads_a_key_head": ([77, 130], [77, 130], 6, 2, 64, True),
    "six_heads_a_key_head": ([33, 95], [33, 95], 6, 1, 128, True),
    "eight_heads_a_key_head": ([50, 19, 140], [50, 19, 140], 16, 2, 64, True),
    "part_of_a_prompt": ([1, 7, 64, 100, 3], [300, 7, 65, 517, 1000], 4, 2, 128, True),
    "part_64": ([5, 128, 40], [133, 700, 41], 4, 1, 64, True),
    "more_queries_than_keys": ([40, 130, 65, 9], [7, 64, 1, 9], 2, 1, 128, True),
    "more_queries_64": ([200, 3], [70, 2], 4, 2, 64, True),
    "no_keys": ([5, 70, 3], [0, 0, 3], 2, 2, 64, True),
    "no_keys_full": ([5, 70, 3], [0, 0, 3], 2, 1, 128, False),
    "no_queries": ([0, 4, 0], [150, 4, 33], 2, 1, 128, True),
    "cross": ([17, 90], [140, 3], 4, 2, 64, False),
    "many_short": ([(7 * n) % 11 for n in range(150)], [(7 * n) % 11 for n in range(150)], 2, 1, 64, True),
    "longer": ([1000, 30], [1000, 30], 2, 1, 128, True),
}


def prompt_inputs(lens_q, lens_k, H, Hk, dh, seed=1, spare=5, sharp=1.0):
    """Rows behind the last sequence: NaN in what goes in."""
    Tq, Tk = sum(lens_q) + spare, sum(lens_k) + spare
    Q, K, V, dY = (ref.bf16(T, h, dh, seed=seed + n) for n, (T, h) in enumerate(((Tq, H), (Tk, Hk), (Tk, Hk), (Tq, H))))
    Q = (Q.float() * sharp).to(torch.bfloat16)
    for t, n in ((Q, sum(lens_q)), (K, sum(lens_k)), (V, sum(lens_k)), (dY, sum(lens_q))):
        t[n:] = float("nan")
    return Q, K, V, dY


def run_prompt(lens_q, lens_k, causal, Q, K, V, dY=None, scale=None, lse_in=None, Y_in=None, ws=None):
    H, Hk, dh = Q.shape[1], K.shape[1], Q.shape[2]
    shape = attn.make_shape(len(lens_q), Q.shape[0], K.shape[0], H, Hk, dh, causal, scale)
    cu_q, cu_k = ref.sums(lens_q).cuda(), ref.sums(lens_k).cuda()
    fill = lambda t, dtype=torch.bfloat16: torch.full(t, 7.0, dtype=dtype, device="cuda")
    Y, lse = fill(Q.shape), fill((H, Q.shape[0]), torch.float32)
    attn.prompt_fwd(shape, Q, K, V, cu_q, cu_k, Y=Y, lse=lse)
    out = {"Y": Y, "lse": lse}
    if dY is not None:
        dQ, dK, dV = fill(Q.shape), fill(K.shape), fill(K.shape)
        attn.prompt_bwd(shape, Q, K, V, Y, dY, lse, cu_q, cu_k, ws=ws, dQ=dQ, dK=dK, dV=dV)
        out.update(dQ=dQ, dK=dK, dV=dV)
    return out


def check_prompt(out, want, nq, nk):
    for name, (x, t) in want.items():
        n = nk if name in ("dK", "dV") else nq
        got, rows = ref.f64(out[name]), (slice(None), slice(0, n)) if name == "lse" else slice(0, n)
        ref.check(name, got[rows], x, t)
        behind = got[:, n:] if name == "lse" else got[n:]
        assert (behind == 7.0).all(), f"{name}: rows behind the last sequence were written"


def want_prompt(lens_q, lens_k, causal, Q, K, V, dY, scale=None):
    nq, nk = sum(lens_q), sum(lens_k)
    scale = Q.shape[2] ** -0.5 if scale is None else scale
    q, k, v, dy = (ref.f64(t)[:n] for t, n in ((Q, nq), (K, nk), (V, nk), (dY, nq)))
    return ref.prompt(q, k, v, lens_q, lens_k, causal, float(np.float32(scale)), dy)


@pytest.mark.parametrize("name", PROMPTS)
def test_prompt(name):
    lens_q, lens_k, H, Hk, dh, causal = PROMPTS[name]
    Q, K, V, dY = prompt_inputs(lens_q, lens_k, H, Hk, dh)
    out = run_prompt(lens_q, lens_k, causal, *(t.cuda() for t in (Q, K, V, dY)))
    check_prompt(out, want_prompt(lens_q, lens_k, causal, Q, K, V, dY), sum(lens_q), sum(lens_k))


FEW = {   # few workgroups with much to read: rows in 32s, or on one side only
    "two_heads": ([300, 0, 451], [300, 0, 451], 2, 2, True),
    "two_heads_full": ([1, 640], [70, 640], 2, 2, False),
    "one_key_head": ([500, 233], [500, 233], 12, 1, True),
    "one_key_head_full": ([129, 400], [400, 129], 6, 1, False),
    "part_of_a_prompt": ([40, 1], [1000, 700], 4, 2, True),
    "more_queries": ([700, 31], [50, 300], 3, 3, True),
    "rows_in_64s": ([300, 0, 451], [300, 0, 451], 16, 16, True),
    "rows_in_64s_full": ([300, 1, 451], [290, 0, 461], 16, 16, False),
    "rows_in_64s_groups_of_4": ([300, 0, 451], [300, 0, 451], 16, 4, True),
    "rows_in_64s_groups_of_2": ([300, 33, 420], [300, 33, 420], 16, 8, True),
    "a_few_tokens_each": ([3, 1, 2] * 5, [203, 301, 150] * 5, 64, 16, True),
    "eight_tokens_each": ([8] * 16, [208] * 16, 12, 12, True),
    "two_rounds_of_64s": ([1500, 3], [1500, 3], 16, 16, True),
    "two_rounds_of_64s_full": ([30, 1400], [70, 1400], 20, 10, False),
    "keys_in_64s": ([300, 33, 420], [300, 33, 420], 32, 16, True),
    "keys_in_64s_full": ([400, 352], [400, 352], 32, 16, False),
}


@pytest.mark.parametrize("dh", [64, 128])
@pytest.mark.parametrize("name", FEW)
def test_prompt_few(name, dh):
    lens_q, lens_k, H, Hk, causal = FEW[name]
    Q, K, V, dY = prompt_inputs(lens_q, lens_k, H, Hk, dh, seed=71)
    out = run_prompt(lens_q, lens_k, causal, *(t.cuda() for t in (Q, K, V, dY)))
    check_prompt(out, want_prompt(lens_q, lens_k, causal, Q, K, V, dY), sum(lens_q), sum(lens_k))


LARGE = {   # more workgroups than are resident at once; gradients summed over many rows
    "many_heads_64": ([333, 65, 0, 200, 500], [333, 65, 0, 200, 500], 64, 64, 64, True),
    "many_heads_128": ([333, 65, 0, 200, 500], [333, 65, 0, 200, 500], 64, 16, 128, True),
    "many_heads_full": ([300, 127, 640], [300, 127, 640], 32, 32, 64, False),
    "many_heads_part": ([130, 257, 64], [700, 300, 1], 48, 16, 128, True),
    "twelve_key_heads": ([400, 95, 33], [400, 95, 33], 24, 12, 128, True),
    "rounds_64": ([333, 65, 0, 200, 500], [333, 65, 0, 200, 500], 256, 256, 64, True),
    "keys_in_256s": ([520, 700, 33, 290], [520, 700, 33, 290], 176, 176, 128, True),
    "keys_in_256s_full": ([300, 0, 512, 200], [300, 1, 511, 255], 128, 64, 128, False),
    "rounds_128": ([300, 0, 200, 77], [300, 0, 410, 77], 256, 256, 128, True),
    "most_sequences": ([(5 * i) % 3 for i in range(4096)], [(5 * i) % 3 for i in range(4096)], 4, 2, 64, True),
    "many_sequences": ([(7 * i) % 61 for i in range(150)], [(7 * i) % 61 + (5 * i) % 23 for i in range(150)], 128, 64, 64, True),
}


@pytest.mark.parametrize("name", LARGE)
def test_prompt_large(name):
    lens_q, lens_k, H, Hk, dh, causal = LARGE[name]
    Q, K, V, dY = prompt_inputs(lens_q, lens_k, H, Hk, dh, seed=61)
    out = run_prompt(lens_q, lens_k, causal, *(t.cuda() for t in (Q, K, V, dY)))
    check_prompt(out, want_prompt(lens_q, lens_k, causal, Q, K, V, dY), sum(lens_q), sum(lens_k))


@pytest.mark.parametrize("dh", [64, 128])
@pytest.mark.parametrize("sharp,scale", [(12.0, None), (1.0, 1.0), (1.0, 1e-6)])
def test_prompt_sharp_and_flat(dh, sharp, scale):
    """Weights on single keys, maxima that rise late, and all keys alike."""
    lens = [150, 70]
    Q, K, V, dY = prompt_inputs(lens, lens, 2, 1, dh, seed=5, sharp=sharp)
    out = run_prompt(lens, lens, True, *(t.cuda() for t in (Q, K, V, dY)), scale=scale)
    check_prompt(out, want_prompt(lens, lens, True, Q, K, V, dY, scale), 220, 220)


@pytest.mark.parametrize("dh", [64, 128])
def test_prompt_views(dh):
    """Q, K, V as slices of one projection, gradients into slices of its gradient; heads in front of rows."""
    lens, H, Hk = [90, 41, 64], 4, 2
    T = sum(lens)
    Q, K, V, dY = prompt_inputs(lens, lens, H, Hk, dh, seed=9, spare=0)
    fused = torch.cat([Q, K, V], 1).cuda()
    q, k, v = fused[:, :H], fused[:, H:H + Hk], fused[:, H + Hk:]
    dy = dY.transpose(0, 1).contiguous().cuda().transpose(0, 1)
    grads = torch.full((T, H + 2 * Hk + 1, dh), 7.0, dtype=torch.bfloat16, device="cuda")
    shape = attn.make_shape(len(lens), T, T, H, Hk, dh)
    cu = ref.sums(lens).cuda()
    Y = torch.empty(H, T, dh, dtype=torch.bfloat16, device="cuda").transpose(0, 1)
    _, lse = attn.prompt_fwd(shape, q, k, v, cu, cu, Y=Y)
    attn.prompt_bwd(shape, q, k, v, Y, dy, lse, cu, cu, dQ=grads[:, :H], dK=grads[:, H:H + Hk], dV=grads[:, H + Hk:H + 2 * Hk])
    dense = run_prompt(lens, lens, True, *(t.cuda() for t in (Q, K, V, dY)))
    assert (grads[:, -1] == 7.0).all()
    for name, got in dict(Y=Y, lse=lse, dQ=grads[:, :H], dK=grads[:, H:H + Hk], dV=grads[:, H + Hk:H + 2 * Hk]).items():
        assert torch.equal(got, dense[name]), name
    # a key head that all heads share, by a stride of zero
    one = K[:, :1].cuda().expand(-1, Hk, -1)
    a = attn.prompt_fwd(shape, q, one, v, cu, cu)[0]
    assert torch.equal(a, attn.prompt_fwd(shape, q, one.contiguous(), v, cu, cu)[0])


def check_not_seen(dh, value, H, Hk, lens):
    """A key (a query) that is not finite touches only the queries (the keys) of its own pairs."""
    at = 70
    Q, K, V, dY = prompt_inputs(lens, lens, H, Hk, dh, seed=21)
    clean = want_prompt(lens, lens, True, Q, K, V, dY)
    K2, V2 = K.clone(), V.clone()
    K2[at, :, 3] = value
    V2[at, :, 5] = value
    out = run_prompt(lens, lens, True, *(t.cuda() for t in (Q, K2, V2, dY)))
    T = sum(lens)
    other = np.r_[0:at, lens[0]:T]                                # queries in front of the key, and the other sequence
    for name in ("Y", "dQ"):
        ref.check(name, ref.f64(out[name])[other], *(x[other] for x in clean[name]))
    ref.check("lse", ref.f64(out["lse"])[:, other], *(x[:, other] for x in clean["lse"]))
    assert not torch.isfinite(out["Y"][at:lens[0]].float()).all(-1).any()
    for name in ("dK", "dV"):
        ref.check(name, ref.f64(out[name])[lens[0]:T], *(x[lens[0]:T] for x in clean[name]))
    # and a query: its gradients go to the keys that it sees
    Q2, dY2, q_at = Q.clone(), dY.clone(), 40
    Q2[q_at, :, 2] = value
    dY2[q_at, :, 7] = value
    out = run_prompt(lens, lens, True, *(t.cuda() for t in (Q2, K, V, dY2)))
    other = np.r_[q_at + 1:T]
    for name in ("dK", "dV"):
        ref.check(name, ref.f64(out[name])[other], *(x[other] for x in clean[name]))
        assert not np.isfinite(ref.f64(out[name])[:q_at + 1]).all(-1).any(), name
    other = np.r_[0:q_at, q_at + 1:T]
    for name in ("Y", "dQ"):
        ref.check(name, ref.f64(out[name])[other], *(x[other] for x in clean[name]))


@pytest.mark.parametrize("dh", [64, 128])
@pytest.mark.parametrize("value", [float("inf"), float("-inf"), float("nan")])
@pytest.mark.parametrize("H,Hk,lens", [(2, 1, [100, 90]), (64, 64, [100, 90]), (2, 1, [300, 250]), (16, 16, [300, 250])])
def test_prompt_what_is_not_seen_does_not_matter(dh, value, H, Hk, lens):
    check_not_seen(dh, value, H, Hk, lens)


def test_prompt_what_is_not_seen_does_not_matter_keys_in_256s():
    check_not_seen(128, float("nan"), 256, 256, [530, 520])


def test_prompt_gradients_are_those_of_differences():
    """d(sum of Y dY) along random directions, by central differences of the definition in 64 bits."""
    lens, H, Hk, dh = [37, 70], 4, 2, 64
    Q, K, V, dY = prompt_inputs(lens, lens, H, Hk, dh, seed=31, spare=0)
    out = run_prompt(lens, lens, True, *(t.cuda() for t in (Q, K, V, dY)))
    x = [ref.f64(t) for t in (Q, K, V)]
    dy, rng, step = ref.f64(dY), np.random.default_rng(3), 1e-4
    bounds = want_prompt(lens, lens, True, Q, K, V, dY)
    for n, name in enumerate(("dQ", "dK", "dV")):
        way = rng.standard_normal(x[n].shape)
        at = lambda f: (ref.prompt(*(t + f * step * way if m == n else t for m, t in enumerate(x)), lens, lens, True, dh ** -0.5)["Y"][0] * dy).sum()
        slope, got = (at(1) - at(-1)) / (2 * step), (ref.f64(out[name]) * way).sum()
        # the elements' bounds add up, and the difference's own error is of the order of step^2
        assert abs(got - slope) <= (bounds[name][1] * np.abs(way)).sum() + 1e-5 * abs(slope) + 1e-4, (name, got, slope)


@pytest.mark.parametrize("lens,H,Hk,dh", [([300, 17, 0, 129], 8, 2, 128), ([333, 65, 0, 500], 64, 64, 64), ([400, 300], 2, 1, 64),
                                          ([300, 0, 451], 16, 16, 128)])
def test_prompt_same_results_again_on_another_stream_and_in_a_graph(lens, H, Hk, dh):
    Q, K, V, dY = (t.cuda() for t in prompt_inputs(lens, lens, H, Hk, dh, seed=41))
    first = run_prompt(lens, lens, True, Q, K, V, dY)
    shape = attn.make_shape(len(lens), Q.shape[0], K.shape[0], H, Hk, dh)
    cu = ref.sums(lens).cuda()
    n = sum(lens)
    ws = attn.alloc_prompt_workspace(shape)
    ws.fill_(255)                                                 # (NaN where a value of the workspace were used unwritten)
    out = {x: torch.empty_like(t) for x, t in first.items()}

    def step():
        attn.prompt_fwd(shape, Q, K, V, cu, cu, Y=out["Y"], lse=out["lse"])
        attn.prompt_bwd(shape, Q, K, V, out["Y"], dY, out["lse"], cu, cu, ws=ws, dQ=out["dQ"], dK=out["dK"], dV=out["dV"])

    def same():
        torch.cuda.synchronize()
        for x in first:
            a, b = (out[x][:, :n], first[x][:, :n]) if x == "lse" else (out[x][:n], first[x][:n])
            assert torch.equal(a, b), x

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    same()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for _ in range(3):
        for t in out.values():
            t.zero_()
        graph.replay()
        same()
        run_prompt([5], [5], True, Q[:5].contiguous(), K[:5].contiguous(), V[:5].contiguous())


def test_prompt_long_rows_pass_32_bits():
    """Row 700000 of a tensor with 3200 values a row lies behind 2^31 values (2^32 bytes)."""
    T, H, Hk, dh = 700000, 1, 1, 64
    lens = [T - 70, 70]
    wide = torch.zeros(T, 3200, dtype=torch.bfloat16, device="cuda")
    view = lambda n: wide[:, n * dh:(n + 1) * dh].unflatten(1, (1, dh))
    parts = prompt_inputs([70], [70], H, Hk, dh, seed=51, spare=0)[:3]
    for n, t in enumerate(parts):
        view(n)[T - 70:] = t.cuda()
    # the long sequence has one query: its last rows only
    shape = attn.make_shape(2, 71, T, H, Hk, dh)
    q = torch.zeros(71, 1, dh, dtype=torch.bfloat16, device="cuda")
    q[1:] = parts[0].cuda()
    Y, _ = attn.prompt_fwd(shape, q, view(1), view(2), ref.sums([1, 70]).cuda(), ref.sums(lens).cuda())
    want = ref.prompt(*(ref.f64(t) for t in parts), [70], [70], True, dh ** -0.5)["Y"]
    ref.check("Y", ref.f64(Y)[1:], *want)
    assert (Y[0] == 0).all()


# ---- the cache

FORMATS = {"bf16": attn.CACHE_BF16, "e4m3": attn.CACHE_E4M3}


def make_cache(shape, seed=1):
    """A pool full of NaN."""
    cache = attn.alloc_cache(shape)
    if shape.format == attn.CACHE_BF16:
        for t in cache[:2]:
            t.fill_(float("nan"))
    else:
        for t in cache:
            t.fill_(255)
    return cache


def make_table(lens, page, seed=1, width=None, spare=2):
    """Pages in no order; -1 behind a sequence's last."""
    need = [-(-n // page) for n in lens]
    width = max(1, max(need)) if width is None else width
    order = np.random.default_rng(seed).permutation(sum(need) + spare)
    table, at = np.full((len(lens), width), -1, np.int32), 0
    for b, n in enumerate(need):
        table[b, :n] = order[at:at + n]
        at += n
    return torch.from_numpy(table), sum(need) + spare


def ints(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def held(x, fmt):
    x = ref.f64(x)
    return x if fmt == "bf16" else ref.values(*ref.quantise(x))


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("dh,Hk,page", [(64, 1, 16), (64, 3, 32), (128, 8, 64), (128, 2, 256), (64, 16, 128), (128, 5, 16)])
def test_cache_write_and_read(fmt, dh, Hk, page):
    past, new = [0, 5, 16, 0, 300, 31], [17, 1, 0, 1, 40, 300]
    whole = [p + n for p, n in zip(past, new)]
    table, pages = make_table(whole, page)
    shape = attn.make_cache_shape(pages, page, Hk, dh, len(new), table.shape[1], FORMATS[fmt])
    cache, T = make_cache(shape), sum(new)
    before = [None if t is None else t.clone() for t in cache]
    K, V = ref.bf16(T + 3, Hk, dh, seed=1), ref.bf16(T + 3, Hk, dh, seed=2, std=30.0)
    cu = ref.sums(new).cuda()
    attn.cache_write(shape, K.cuda(), V.cuda(), cache, table.cuda(), ints(past), cu)
    # every byte of the pool: the rows' tokens hold them, all others are as they were
    place = {(int(table[b, t // page]), t % page): r for b in range(len(new)) for r, t in
             zip(range(int(cu[b]), int(cu[b + 1])), range(past[b], whole[b]))}
    for n, x in enumerate((K, V)):
        codes, e = (x.view(torch.int16).numpy(), None) if fmt == "bf16" else ref.quantise(ref.f64(x))
        got, was = ((t[n].view(torch.int16) if fmt == "bf16" else t[n]).cpu().numpy().copy() for t in (cache, before))
        for (p, at), r in place.items():
            was[p, :, at] = codes[r]
        assert np.array_equal(got, was)
        if e is not None:
            was = before[2 + n].cpu().numpy().copy()
            for (p, at), r in place.items():
                was[p, :, at] = e[r]
            assert np.array_equal(cache[2 + n].cpu().numpy(), was)
    for start, lens in ((past, new), ([0] * 6, whole), ([3, 0, 2, 0, 299, 100], [9, 2, 5, 1, 3, 120])):
        n = sum(lens)
        Kr, Vr = (torch.full((n + 2, Hk, dh), 7.0, dtype=torch.bfloat16, device="cuda") for _ in range(2))
        attn.cache_read(shape, cache, table.cuda(), ints(start), ref.sums(lens).cuda(), K=Kr, V=Vr)
        for got, x in ((Kr, K), (Vr, V)):
            h, r = held(x, fmt), 0
            got = ref.f64(got)
            assert (got[n:] == 7.0).all()
            for b, m in enumerate(lens):
                for t in range(start[b], start[b] + m):
                    if past[b] <= t < whole[b]:
                        assert np.array_equal(got[r], h[int(cu[b]) + t - past[b]]), (b, t)
                    r += 1


def test_cache_every_bf16():
    """Every finite bf16 in a row whose largest magnitude it is or half to a thousandth of it, zeros, the smallest, what is not finite."""
    bits = np.arange(0x8000, dtype=np.uint32)
    top = bits[bits < 0x7F80].astype(np.uint16)
    rows = []
    for shift in (0, 0x40, 0x7F, 0x80, 0x155, 0x233, 0x300, 0x3FF, 0x500):
        rows.append(np.maximum(top.astype(int) - shift, 0).astype(np.uint16) | np.uint16(0x8000 if shift & 1 else 0))
    x = np.stack([top] + rows + [top * 0] * (64 - 1 - len(rows)), 1)
    extra = np.zeros((4, 64), np.uint16)
    extra[0, :3] = 0x7F80, 0xFF80, 0x3F80                    # infinities beside 1
    extra[1, :3] = 0x7FC0, 0xFFC1, 0x4049                    # NaN beside 3.14
    extra[2, :] = 0x7F80                                     # nothing finite
    x = np.concatenate([x, extra])
    T = x.shape[0]
    K = torch.from_numpy(x.view(np.int16)).view(torch.bfloat16).view(T, 1, 64)
    page = 256
    table = torch.arange(-(-T // page), dtype=torch.int32).view(1, -1)
    shape = attn.make_cache_shape(table.shape[1], page, 1, 64, 1, table.shape[1], attn.CACHE_E4M3)
    cache = make_cache(shape)
    V = K.flip(2).contiguous()
    attn.cache_write(shape, K.cuda(), V.cuda(), cache, table.cuda(), ints([0]), ints([0, T]))
    f = ref.f64(K)[:, 0]
    codes, e = ref.quantise(f)
    got = cache.K.cpu().numpy().reshape(-1, 64)[:T]
    nan = ~np.isfinite(f)
    assert np.array_equal(cache.ks.cpu().numpy().reshape(-1)[:T], e)
    assert ((got[nan] & 0x7F) == 0x7F).all() and np.array_equal(got[~nan], codes[~nan])
    Kr, Vr = attn.cache_read(shape, cache, table.cuda(), ints([0]), ints([0, T]), T)
    for got, flip in ((Kr, False), (Vr, True)):
        got = ref.f64(got)[:, 0]
        assert np.array_equal(got[:, ::-1] if flip else got, ref.values(codes, e), equal_nan=True)


@pytest.mark.parametrize("fmt", FORMATS)
def test_cache_tokens_without_a_page(fmt):
    """Tokens in front of 0, behind the table or in no page of the pool are not written, and read as zeros."""
    page, Hk, dh = 16, 2, 64
    table = torch.tensor([[0, -1, 2], [1, 5, 1 << 30], [3, -(1 << 31), 4]], dtype=torch.int32)
    shape = attn.make_cache_shape(5, page, Hk, dh, 3, 3, FORMATS[fmt])
    cache = make_cache(shape)
    K = ref.bf16(3 * 60, Hk, dh, seed=3)
    start, cu = ints([-5, 0, 20]), ints([0, 60, 120, 180])
    attn.cache_write(shape, K.cuda(), K.cuda(), cache, table.cuda(), start, cu)
    Kr, Vr = attn.cache_read(shape, cache, table.cuda(), start, cu, 180)
    want = held(K, fmt).copy()
    for r in range(180):
        t = (-5, 0, 20)[r // 60] + r % 60
        if t < 0 or t >= 48 or not 0 <= int(table[r // 60, t // page]) < 5:
            want[r] = 0.0
    assert np.array_equal(ref.f64(Kr), want) and np.array_equal(ref.f64(Vr), want)


def test_cache_views():
    page, Hk, dh, T = 32, 2, 128, 50
    table, pages = make_table([T], page)
    shape = attn.make_cache_shape(pages, page, Hk, dh, 1, table.shape[1], attn.CACHE_E4M3)
    fused = ref.bf16(T, 4 + 2 * Hk, dh, seed=8).cuda()
    K, V = fused[:, 4:4 + Hk], fused[:, 4 + Hk:]
    args = (table.cuda(), ints([0]), ints([0, T]))
    a = attn.cache_write(shape, K, V, make_cache(shape), *args)
    b = attn.cache_write(shape, K.contiguous(), V.contiguous(), make_cache(shape), *args)
    assert all(torch.equal(x, y) for x, y in zip(a, b))
    out = torch.zeros(Hk, T, 3, dh, dtype=torch.bfloat16, device="cuda")
    attn.cache_read(shape, a, *args, K=out[:, :, 0].transpose(0, 1), V=out[:, :, 2].transpose(0, 1))
    Kr, Vr = attn.cache_read(shape, a, *args, T)
    assert torch.equal(out[:, :, 0].transpose(0, 1), Kr) and torch.equal(out[:, :, 2].transpose(0, 1), Vr) and (out[:, :, 1] == 0).all()


# ---- single tokens

def decode_inputs(fmt, lens, H, Hk, dh, page, seed=1, width=None, std=1.0):
    table, pages = make_table(lens, page, seed, width)
    shape = attn.make_cache_shape(pages, page, Hk, dh, len(lens), table.shape[1], FORMATS[fmt])
    cache = make_cache(shape)
    T = max(1, sum(lens))
    K, V = ref.bf16(T, Hk, dh, seed=seed, std=std), ref.bf16(T, Hk, dh, seed=seed + 1, std=std)
    if sum(lens):
        attn.cache_write(shape, K.cuda(), V.cuda(), cache, table.cuda(), ints([0] * len(lens)), ref.sums(lens).cuda())
    Q = ref.bf16(len(lens), H, dh, seed=seed + 2)
    return shape, cache, table.cuda(), Q, held(K, fmt), held(V, fmt)


def want_decode(Q, K, V, lens, scale=None):
    q, B = ref.f64(Q), len(lens)
    return ref.prompt(q, K[:sum(lens)], V[:sum(lens)], [1] * B, lens, False, Q.shape[2] ** -0.5 if scale is None else scale)["Y"]


DECODES = {
    "one": ([1], 1, 1, 64, 16),
    "none": ([0, 0], 2, 1, 128, 16),
    "edges": ([0, 1, 15, 16, 17, 31, 32, 33, 47, 64, 65, 128, 129, 0], 4, 2, 128, 16),
    "edges_64": ([33, 0, 1, 63, 300, 16, 31, 500], 8, 1, 64, 32),
    "every_head_its_keys": ([700, 3], 12, 12, 64, 16),
    "five_heads_a_key_head": ([100, 260], 10, 2, 128, 256),
    "sixteen": ([70, 400], 16, 1, 128, 64),
    "twenty": ([70, 400, 1], 40, 2, 64, 128),
    "fifty": ([333], 50, 1, 128, 16),
    "one_long": ([20011], 8, 2, 128, 64),
    "long_and_short": ([9000, 1, 0, 5, 2500], 4, 4, 64, 256),
    "many": ([(37 * n) % 130 for n in range(150)], 2, 1, 64, 16),
    "thousands": ([(7 * n) % 41 for n in range(3000)], 2, 2, 64, 16),
}


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("wide", [False, True])
@pytest.mark.parametrize("name", DECODES)
def test_decode(fmt, name, wide):
    """Short sequences in a table made for them, and in one that could hold long ones."""
    lens, H, Hk, dh, page = DECODES[name]
    shape, cache, table, Q, K, V = decode_inputs(fmt, lens, H, Hk, dh, page, width=-(-max(max(lens), 3000) // page) if wide else None)
    Y = attn.decode(shape, Q.cuda(), cache, table, ints(lens))
    ref.check("Y", Y, *want_decode(Q, K, V, lens))


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("width", [17, 100])
@pytest.mark.parametrize("std,scale", [(8.0, None), (1.0, 3.0), (1e-30, None), (1e30, 1e-30)])
def test_decode_sharp_and_flat(fmt, width, std, scale):
    lens = [513, 40]
    shape, cache, table, Q, K, V = decode_inputs(fmt, lens, 4, 1, 128, 32, seed=7, std=std, width=width)
    Y = attn.decode(shape, Q.cuda(), cache, table, ints(lens), scale=scale)
    ref.check("Y", Y, *want_decode(Q, K, V, lens, None if scale is None else float(np.float32(scale))))


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("width", [7, 200])
def test_decode_lengths_and_pages_that_are_not_there(fmt, width):
    """Lengths below 0 and behind the table; tokens whose page is no page of the pool are left out."""
    lens, page = [100, 40, 64], 16
    shape, cache, table, Q, K, V = decode_inputs(fmt, lens, 4, 2, 64, page, width=width)
    Y = attn.decode(shape, Q.cuda(), cache, table, ints([-3, 40, 1000000]))
    assert (Y[0] == 0).all()
    keep = want_decode(Q, K, V, lens)
    ref.check("Y", Y[1:], *(x[1:] for x in keep))              # (sequence 2: behind its 64 tokens there are no pages)
    gone = table.clone()
    gone[0, 2], gone[0, 6], gone[1, 0] = -7, shape.pages, 1 << 30
    Y = attn.decode(shape, Q.cuda(), cache, gone, ints(lens))
    drop = lambda x: np.concatenate([x[:32], x[48:96], x[116:140], x[140:]])
    ref.check("Y", Y, *want_decode(Q, drop(K), drop(V), [80, 24, 64]))


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("longest", [1500, 500])
def test_decode_same_results_again_views_and_graph(fmt, longest):
    lens = [longest, 3, 0, 260]
    shape, cache, table, Q, K, V = decode_inputs(fmt, lens, 8, 2, 128, 64, seed=11)
    n, q = ints(lens), Q.cuda()
    first = attn.decode(shape, q, cache, table, n)
    ws = attn.alloc_decode_workspace(shape, 8)
    ws.fill_(255)
    fused = torch.zeros(4, 12, 128, dtype=torch.bfloat16, device="cuda")
    fused[:, 2:10] = q
    Y = torch.zeros(8, 4, 128, dtype=torch.bfloat16, device="cuda").transpose(0, 1)
    attn.decode(shape, fused[:, 2:10], cache, table, n, ws=ws, Y=Y)
    assert torch.equal(Y, first)
    graph, out = torch.cuda.CUDAGraph(), torch.empty_like(first)
    side = torch.cuda.Stream()
    with torch.cuda.graph(graph, stream=side):
        attn.decode(shape, q, cache, table, n, ws=ws, Y=out)
    for changed in (lens, [longest - 1, 2, 70, 1], lens):
        m = [min(a, b) for a, b in zip(changed, lens)]
        n.copy_(ints(m))
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        cut = [np.arange(a) + o for a, o in zip(m, np.cumsum([0] + lens))]
        rows = np.concatenate(cut).astype(int)
        ref.check("Y", out, *want_decode(Q, K[rows], V[rows], m))
        assert torch.equal(out, attn.decode(shape, q, cache, table, n))


@pytest.mark.parametrize("fmt", FORMATS)
def test_pages_behind_32_bits(fmt):
    """A pool of more than 2^32 bytes of K, of which the last pages are used."""
    page, Hk, dh, lens = 256, 8, 128, [300, 513]
    pages = (1 << 32) // (page * Hk * dh * (2 if fmt == "bf16" else 1)) + 10
    shape = attn.make_cache_shape(pages, page, Hk, dh, 2, 3, FORMATS[fmt])
    cache = attn.alloc_cache(shape)
    table = torch.tensor([[pages - 1, pages - 4, -1], [pages - 2, pages - 3, pages - 5]], dtype=torch.int32, device="cuda")
    T = sum(lens)
    K, V, Q = ref.bf16(T, Hk, dh, seed=1), ref.bf16(T, Hk, dh, seed=2), ref.bf16(2, Hk, dh, seed=3)
    cu = ref.sums(lens).cuda()
    attn.cache_write(shape, K.cuda(), V.cuda(), cache, table, ints([0, 0]), cu)
    Kr, Vr = attn.cache_read(shape, cache, table, ints([0, 0]), cu, T)
    assert np.array_equal(ref.f64(Kr), held(K, fmt)) and np.array_equal(ref.f64(Vr), held(V, fmt))
    ref.check("Y", attn.decode(shape, Q.cuda(), cache, table, ints(lens)), *want_decode(Q, held(K, fmt), held(V, fmt), lens))


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("width", [20, 200])
def test_decode_a_head_that_is_not_finite(fmt, width):
    """NaN in one query touches the output of that query alone."""
    lens = [300, 77]
    shape, cache, table, Q, K, V = decode_inputs(fmt, lens, 8, 2, 64, 16, seed=13, width=width)
    first = attn.decode(shape, Q.cuda(), cache, table, ints(lens))
    bad = Q.clone()
    bad[0, 5, 7] = float("nan")
    Y = attn.decode(shape, bad.cuda(), cache, table, ints(lens))
    assert torch.isnan(Y[0, 5]).all()
    Y[0, 5] = first[0, 5]
    assert torch.equal(Y, first)


# ---- together

def test_calls_at_once():
    """Calls on two streams, each with a workspace of its own, do not see one another."""
    lens, H, Hk, dh = [300, 17, 129], 8, 2, 128
    inputs = [tuple(t.cuda() for t in prompt_inputs(lens, lens, H, Hk, dh, seed=80 + n)) for n in range(2)]
    decodes = [decode_inputs("e4m3", [2000, 30, 700], H, Hk, dh, 64, seed=90 + n, width=40) for n in range(2)]
    n = ints([2000, 30, 700])
    alone = [(run_prompt(lens, lens, True, *x), attn.decode(d[0], d[3].cuda(), d[1], d[2], n)) for x, d in zip(inputs, decodes)]
    queries = [d[3].cuda() for d in decodes]
    streams, got = [torch.cuda.Stream() for _ in range(2)], [[], []]
    torch.cuda.synchronize()
    for _ in range(5):
        for k, stream in enumerate(streams):
            with torch.cuda.stream(stream):
                got[k].append((run_prompt(lens, lens, True, *inputs[k]), attn.decode(decodes[k][0], queries[k], decodes[k][1], decodes[k][2], n)))
    torch.cuda.synchronize()
    for k in range(2):
        for out, Y in got[k]:
            assert torch.equal(Y, alone[k][1])
            for x in out:
                a, b = (out[x][:, :sum(lens)], alone[k][0][x][:, :sum(lens)]) if x == "lse" else (out[x][:sum(lens)], alone[k][0][x][:sum(lens)])
                assert torch.equal(a, b), x


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("H,Hk,dh,page", [(8, 2, 128, 16), (4, 4, 64, 64)])
def test_prompts_in_parts_then_tokens(fmt, H, Hk, dh, page):
    """Three prompts read in two parts and continued by four tokens: what the cache holds is what every query sees."""
    parts, steps = [[30, 0, 65], [41, 7, 1]], 4
    total = [sum(x) + steps for x in zip(*parts)]
    table, pages = make_table(total, page)
    shape = attn.make_cache_shape(pages, page, Hk, dh, 3, table.shape[1], FORMATS[fmt])
    cache, table, have = make_cache(shape), table.cuda(), [0, 0, 0]
    K, V, Q = ref.bf16(sum(total), Hk, dh, seed=1), ref.bf16(sum(total), Hk, dh, seed=2), ref.bf16(sum(total), H, dh, seed=3)
    first = np.cumsum([0] + total)[:3]
    want, bound = ref.prompt(ref.f64(Q), held(K, fmt), held(V, fmt), total, total, True, dh ** -0.5)["Y"]
    for new in parts + [[1, 1, 1]] * steps:
        rows = np.concatenate([f + h + np.arange(n) for f, h, n in zip(first, have, new)]).astype(int)
        k, v, q, cu = K[rows].cuda(), V[rows].cuda(), Q[rows].cuda(), ref.sums(new).cuda()
        attn.cache_write(shape, k, v, cache, table, ints(have), cu)
        have = [h + n for h, n in zip(have, new)]
        if max(new) == 1 and min(new) == 1:
            Y = attn.decode(shape, q, cache, table, ints(have))
        else:
            cu_k = ref.sums(have).cuda()
            Kr, Vr = attn.cache_read(shape, cache, table, ints([0, 0, 0]), cu_k, sum(have))
            Y, _ = attn.prompt_fwd(attn.make_shape(3, len(rows), sum(have), H, Hk, dh), q, Kr, Vr, cu, cu_k, save_for_backward=False)
        ref.check("Y", Y, want[rows], bound[rows])
