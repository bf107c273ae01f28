"""Decode of a batch behind a shared prefix against a softmax over both parts in 64 bits.

Tolerance, element by element: the probabilities (times v_scale) are rounded to bf16 once and so is the result, each off by at most
2^-8 relative, so that |error| <= 2^-8 sum_t p_t |v^_t| + 2^-8 |o| (1 + 2^-8); sums, exponentials and merges in fp32 add less than
2^-14 sum_t p_t |v^_t| for scores up to some 2^6 (a score's own rounding is 2^-24 of it, and it is the exponent of a probability).
"""
import ctypes
import math
import os

import numpy as np
import pytest
import torch

BF16, F32, I8, I32 = torch.bfloat16, torch.float32, torch.int8, torch.int32
gpu = pytest.mark.gpu


@pytest.fixture(scope="module")
def sa():
    from paper_2407_07304_amd import build, slimattn
    if not (os.path.exists(slimattn.LIB_PATH) and os.path.exists(slimattn.BINDING_PATH)):
        build.build()
    slimattn.load()
    return slimattn


def cache(rng, *shape):
    """codes and scales of N(0, 1) rows"""
    x = rng.standard_normal(shape, dtype=np.float32)
    scale = (np.abs(x).max(-1) / np.float32(127)).astype(np.float32)
    return torch.from_numpy(np.rint(x / scale[..., None]).astype(np.int8)), torch.from_numpy(scale)


def queries(rng, B, Hq, D, scale=1.0):
    return torch.from_numpy(rng.standard_normal((B, Hq, 1, D), dtype=np.float32) * np.float32(scale)).to(BF16)


def reference(q, prefix, own, lens, scale):
    """(o, the bound of its error) in 64 bits; prefix and own on the CPU"""
    B, Hq, _, D = q.shape
    Hkv = own[0].shape[1]
    q = q.double().view(B, Hkv, Hq // Hkv, D)
    pk, pv = (prefix[i][0].double() * prefix[i + 1][0].double()[..., None] for i in (0, 2))
    o, bound = torch.empty_like(q), torch.empty_like(q)
    for b in range(B):
        n = int(lens[b])
        for g in range(Hkv):
            k, v = (torch.cat([p[g], own[i][b, g, :n].double() * own[i + 1][b, g, :n].double()[:, None]])
                    for p, i in ((pk, 0), (pv, 2)))
            s = (q[b, g] @ k.T) * scale
            p = torch.softmax(s, 1)
            o[b, g] = p @ v
            bound[b, g] = p @ v.abs()
    bound = (2.0 ** -8 + 2.0 ** -14) * bound + 2.0 ** -8 * (1 + 2.0 ** -8) * o.abs()
    return o.view(B, Hq, 1, D), bound.view(B, Hq, 1, D)


def past_the_end(own, lens):
    """The same caches with numbers past every length that would show in any result."""
    own = [t.clone() for t in own]
    for b, n in enumerate(lens.tolist()):
        for t, x in zip(own, (127, math.nan, -127, math.inf)):
            t[b, :, n:] = x
    return own


def on_gpu(ts):
    return [t.cuda() for t in ts]


def check(sa, q, prefix, own, lens, scale, what, workspace=True):
    B, Hq, _, D = q.shape
    want, bound = reference(q, prefix, own, lens, scale)
    P, (T, Hkv) = prefix[0].shape[2], (own[0].shape[2], own[0].shape[1])
    n = sa.slim_attn_decode_int8_shared_prefix_workspace_bytes(B, Hq, Hkv, P, T, D)
    assert n > 0
    ws = torch.full((n + 64,), 255, dtype=torch.uint8, device="cuda") if workspace else None     # (NaN in 32 bits)
    got = sa.slim_attn_decode_int8_shared_prefix(q.cuda(), *on_gpu(prefix), *on_gpu(past_the_end(own, lens)), lens.cuda(), scale,
                                                 workspace=None if ws is None else ws[:n])
    off = (got.double().cpu() - want).abs()
    assert torch.isfinite(off).all(), what
    assert (off <= bound).all(), "%s: %.3g of its bound" % (what, (off / bound).max())
    if ws is not None:
        assert (ws[n:] == 255).all(), "written past the workspace"
    return got


# rows of the prefix (batch x heads of a KV head): up to 16, 32, 64, 128, and several blocks of 128
ROWS = [(1, 1, 1), (1, 8, 8), (3, 10, 2), (4, 8, 2), (5, 4, 1), (8, 16, 4), (2, 32, 1), (11, 12, 3), (16, 32, 8), (31, 8, 2), (33, 8, 2),
        (43, 9, 3), (3, 40, 1), (130, 2, 2), (70, 4, 1), (2, 70, 1)]


@gpu
@pytest.mark.parametrize("B,Hq,Hkv", ROWS)
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("P,T", [(1, 1), (31, 40), (33, 300), (600, 33), (1100, 700)])
def test_shared_prefix_small_shapes(sa, B, Hq, Hkv, D, P, T):
    print("shared prefix", B, Hq, Hkv, D, P, T, flush=True)
    rng = np.random.default_rng(B * Hq + P + T + D)
    prefix, own = [*cache(rng, 1, Hkv, P, D), *cache(rng, 1, Hkv, P, D)], [*cache(rng, B, Hkv, T, D), *cache(rng, B, Hkv, T, D)]
    lens = torch.from_numpy(rng.integers(0, T + 1, B).astype(np.int32))
    lens[0] = T
    if B > 1:
        lens[1] = 0
    check(sa, queries(rng, B, Hq, D), prefix, own, lens, 1 / math.sqrt(D), "B%d Hq%d Hkv%d D%d P%d T%d" % (B, Hq, Hkv, D, P, T), P != 33)


@gpu
@pytest.mark.parametrize("B,Hq,Hkv,P,T", [(1, 4, 4, 700, 64), (4, 32, 8, 1000, 64), (2, 40, 8, 33, 900), (3, 16, 4, 9000, 5), (16, 2, 2, 300, 500), (1, 16, 1, 500, 70)])
@pytest.mark.parametrize("D", [64, 128])
def test_shared_prefix_of_few_rows_has_the_bits_of_fp32(sa, B, Hq, Hkv, P, T, D):
    """Up to 16 rows a KV head: a probability times its v_scale enters the second product as two bf16, off by 2^-16.  What is left of the
    file's bound is 2^-16 + 2^-14 of sum_t p_t |v^_t| and the result's own rounding."""
    print("shared prefix", B, Hq, Hkv, D, P, T, flush=True)
    rng = np.random.default_rng(B + Hq + P + T + D)
    prefix, own = [*cache(rng, 1, Hkv, P, D), *cache(rng, 1, Hkv, P, D)], [*cache(rng, B, Hkv, T, D), *cache(rng, B, Hkv, T, D)]
    lens = torch.from_numpy(rng.integers(0, T + 1, B).astype(np.int32))
    lens[0] = T
    q = queries(rng, B, Hq, D)
    want, bound = reference(q, prefix, own, lens, 1 / math.sqrt(D))
    last = 2.0 ** -8 * (1 + 2.0 ** -8) * want.abs()
    bound = last + (bound - last) * (2.0 ** -16 + 2.0 ** -14) / (2.0 ** -8 + 2.0 ** -14)
    got = sa.slim_attn_decode_int8_shared_prefix(q.cuda(), *on_gpu(prefix), *on_gpu(own), lens.cuda(), 1 / math.sqrt(D))
    off = (got.double().cpu() - want).abs()
    assert (off <= bound).all(), "%.3g of its bound" % (off / bound).max()


@gpu
@pytest.mark.parametrize("B,Hq,Hkv,D,P,T", [(4, 32, 8, 128, 9000, 64), (48, 32, 8, 128, 5000, 1000), (24, 64, 8, 64, 7001, 513),
                                            (1, 32, 32, 128, 20000, 1), (12, 16, 2, 64, 12345, 2000)])
def test_shared_prefix_many_splits(sa, B, Hq, Hkv, D, P, T):
    print("shared prefix", B, Hq, Hkv, D, P, T, flush=True)
    rng = np.random.default_rng(P)
    prefix, own = [*cache(rng, 1, Hkv, P, D), *cache(rng, 1, Hkv, P, D)], [*cache(rng, B, Hkv, T, D), *cache(rng, B, Hkv, T, D)]
    lens = torch.from_numpy(rng.integers(1, T + 1, B).astype(np.int32))
    check(sa, queries(rng, B, Hq, D), prefix, own, lens, 1 / math.sqrt(D), "P%d T%d" % (P, T))


@gpu
@pytest.mark.parametrize("B,Hq,Hkv,D,P,T,records", [(130, 128, 128, 64, 4200, 3, 3), (70, 256, 256, 128, 4097, 2, 3), (40, 256, 256, 128, 4300, 1, 5),
                                                    (20, 512, 256, 64, 5000, 2, 5)])
def test_shared_prefix_in_twice_as_many_splits(sa, B, Hq, Hkv, D, P, T, records):
    """A workgroup a compute unit has 64 stages or more: two are launched, each with a split of its own (records a row: theirs, of up to
    64 rows two a split, and the own cache's)."""
    print("shared prefix", B, Hq, Hkv, D, P, T, flush=True)
    assert sa.slim_attn_decode_int8_shared_prefix_workspace_bytes(B, Hq, Hkv, P, T, D) == B * Hq * records * (D + 2) * 4
    gen = torch.Generator(device="cuda").manual_seed(P)

    def random_cache(*shape):
        return (torch.randint(-127, 128, shape, generator=gen, device="cuda", dtype=I8),
                0.02 * torch.rand(shape[:-1], generator=gen, device="cuda") + 0.005)

    prefix, own = [*random_cache(1, Hkv, P, D), *random_cache(1, Hkv, P, D)], [*random_cache(B, Hkv, T, D), *random_cache(B, Hkv, T, D)]
    q = torch.randn((B, Hq, 1, D), generator=gen, device="cuda").to(BF16)
    lens = torch.randint(0, T + 1, (B,), generator=gen, device="cuda", dtype=I32)
    scale = 1 / math.sqrt(D)
    got = sa.slim_attn_decode_int8_shared_prefix(q, *prefix, *own, lens, scale).double().view(B, Hkv, -1, D)
    past = (torch.arange(T, device="cuda") >= lens[:, None])[:, None]
    for g in range(Hkv):
        rows = q.double().view(B, Hkv, -1, D)[:, g]
        (pk, pv), (k, v) = (((x[0][i, g].double() * x[1][i, g].double()[..., None]), (x[2][i, g].double() * x[3][i, g].double()[..., None]))
                            for x, i in ((prefix, 0), (own, slice(None))))
        s = torch.cat([rows @ pk.T, (rows[:, :, None] * k[:, None]).sum(-1).masked_fill(past, -math.inf)], 2) * scale
        p = torch.softmax(s, 2)
        want, bound = (p[:, :, :P] @ f(pv) + (p[:, :, P:, None] * f(v)[:, None]).sum(2) for f in (lambda x: x, torch.abs))
        bound = (2.0 ** -8 + 2.0 ** -14) * bound + 2.0 ** -8 * (1 + 2.0 ** -8) * want.abs()
        assert ((got[:, g] - want).abs() <= bound).all(), g


@gpu
@pytest.mark.parametrize("B,Hq,Hkv", [(2, 8, 2), (8, 8, 2), (12, 8, 2), (40, 8, 2), (90, 8, 2)])
@pytest.mark.parametrize("D", [64, 128])
def test_shared_prefix_sharp_rows(sa, B, Hq, Hkv, D):
    """Rows that one token carries, of the prefix or of the own cache, the last of either among them; scores of up to some 60."""
    rng = np.random.default_rng(B)
    P, T, scale = 700, 90, 1 / math.sqrt(D)
    prefix, own = [*cache(rng, 1, Hkv, P, D), *cache(rng, 1, Hkv, P, D)], [*cache(rng, B, Hkv, T, D), *cache(rng, B, Hkv, T, D)]
    lens = torch.from_numpy(rng.integers(1, T + 1, B).astype(np.int32))
    q = queries(rng, B, Hq, D)
    for b in range(B):
        for h in range(Hq):
            g = h // (Hq // Hkv)
            where = rng.integers(4)
            t = int(rng.integers(P)) if where == 0 else P - 1 if where == 1 else int(rng.integers(lens[b])) if where == 2 else int(lens[b]) - 1
            k = prefix[0][0, g, t].float() * prefix[1][0, g, t] if where < 2 else own[0][b, g, t].float() * own[1][b, g, t]
            q[b, h, 0] = (k * float(rng.uniform(1.0, 5.0))).to(BF16)
    check(sa, q, prefix, own, lens, scale, "sharp")


@gpu
@pytest.mark.parametrize("B,Hq,Hkv", [(2, 8, 2), (5, 8, 2), (12, 8, 2), (40, 8, 2)])
def test_shared_prefix_all_zero_tokens_and_huge_scores(sa, B, Hq, Hkv):
    """A prefix of zeros leaves uniform weights on it; queries of 2^60 make scores that only the running maximum keeps finite: then
    the largest score alone counts (which of several near ones is largest is beyond fp32, so the values are all the same)."""
    rng = np.random.default_rng(3)
    D, P, T = 128, 333, 50
    prefix, own = [*cache(rng, 1, Hkv, P, D), *cache(rng, 1, Hkv, P, D)], [*cache(rng, B, Hkv, T, D), *cache(rng, B, Hkv, T, D)]
    prefix[0].zero_(), prefix[1].zero_()
    lens = torch.full((B,), T, dtype=I32)
    lens[0] = 0
    check(sa, queries(rng, B, Hq, D), prefix, own, lens, 1 / math.sqrt(D), "zero keys")
    prefix = [*cache(rng, 1, Hkv, P, D), *cache(rng, 1, Hkv, P, D)]
    for t in (prefix[2], own[2]):
        t[:] = t[:, :1, :1]
    prefix[2][:], own[2][:] = own[2][0, 0, 0], own[2][0, 0, 0]
    prefix[3].fill_(0.01), own[3].fill_(0.01)
    q = queries(rng, B, Hq, D, 2.0 ** 60)
    got = sa.slim_attn_decode_int8_shared_prefix(q.cuda(), *on_gpu(prefix), *on_gpu(own), lens.cuda(), 1 / math.sqrt(D))
    v = own[2][0, 0, 0].double() * float(np.float32(0.01))
    # (every product p v_scale is rounded, 2^-8, and the result, 2^-8)
    assert ((got.double().cpu() - v).abs() <= (2.0 ** -7 + 2.0 ** -13) * v.abs()).all()


@gpu
@pytest.mark.parametrize("B,Hq,Hkv", [(2, 8, 2), (6, 8, 2), (12, 8, 2), (40, 8, 2)])
@pytest.mark.parametrize("D", [64, 128])
def test_shared_prefix_of_extreme_queries(sa, B, Hq, Hkv, D):
    """Rows around 2^60 (the largest score alone counts) and 2^-50 (every token the same), the prefix ending inside a tile; and a row
    that is not finite, which no other row shows."""
    rng = np.random.default_rng(D + B)
    P, T, scale = 777, 90, 1 / math.sqrt(D)
    prefix, own = [*cache(rng, 1, Hkv, P, D), *cache(rng, 1, Hkv, P, D)], [*cache(rng, B, Hkv, T, D), *cache(rng, B, Hkv, T, D)]
    lens = torch.from_numpy(rng.integers(0, T + 1, B).astype(np.int32))
    q = queries(rng, B, Hq, D)
    for shift in (60, -50):
        qs = (q.float() * 2.0 ** shift).to(BF16)
        want, bound = reference(qs, prefix, own, lens, scale)
        got = sa.slim_attn_decode_int8_shared_prefix(qs.cuda(), *on_gpu(prefix), *on_gpu(past_the_end(own, lens)), lens.cuda(), scale)
        assert ((got.double().cpu() - want).abs() <= bound).all(), shift
    fine = sa.slim_attn_decode_int8_shared_prefix(q.cuda(), *on_gpu(prefix), *on_gpu(own), lens.cuda(), scale)
    for bad in (math.inf, -math.inf, math.nan):
        qn = q.clone()
        qn[1, 3, 0, 5] = bad
        got = sa.slim_attn_decode_int8_shared_prefix(qn.cuda(), *on_gpu(prefix), *on_gpu(own), lens.cuda(), scale)
        off = (got != fine).any(-1)
        assert torch.equal(off.nonzero().cpu(), torch.tensor([[1, 3, 0]])) and not torch.isfinite(got[1, 3]).any()


@gpu
@pytest.mark.parametrize("B,Hq,Hkv", [(2, 8, 2), (6, 8, 2), (12, 8, 2), (40, 8, 2)])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("low", [2.0 ** 8, 2.0 ** 14, 2.0 ** 60, 2.0 ** 127])
def test_shared_prefix_behind_tokens_of_far_lower_scores(sa, B, Hq, Hkv, D, low):
    """Every other 64 tokens of the prefix have scores `low` times the others' size, all negative: a running maximum that such tokens set
    leaves little of the others' scores in fp32, or nothing, if it is taken off them before they have moved it.  (Of 2^127 the scores are
    below what fp32 holds: -infinity, a weight of zero all the same.)"""
    rng = np.random.default_rng(B + D)
    P, T, scale = 1500, 40, 1 / math.sqrt(D)
    prefix, own = [*cache(rng, 1, Hkv, P, D), *cache(rng, 1, Hkv, P, D)], [*cache(rng, B, Hkv, T, D), *cache(rng, B, Hkv, T, D)]
    far = torch.arange(P) // 64 % 2 == 0
    prefix[0][:, :, far] = -prefix[0][:, :, far].abs().clamp(min=32)
    prefix[1][:, :, far] *= low
    q = queries(rng, B, Hq, D).abs()
    lens = torch.from_numpy(rng.integers(0, T + 1, B).astype(np.int32))
    check(sa, q, prefix, own, lens, scale, "%g below" % low)
    q[:, ::3] = 0.0     # (and beside them rows that have these tokens' scores at zero, like all others')
    check(sa, q, prefix, own, lens, scale, "%g below, but for some rows" % low)


@gpu
@pytest.mark.parametrize("B", [2, 6, 12, 40])
def test_shared_prefix_of_very_low_scores(sa, B):
    """All scores of a row around -2^100, where they are all the same in fp32: the mean of the values, without what lies past the end."""
    rng = np.random.default_rng(7)
    Hq, Hkv, D, P, T = 8, 2, 128, 333, 1
    prefix, own = [*cache(rng, 1, Hkv, P, D), *cache(rng, 1, Hkv, P, D)], [*cache(rng, B, Hkv, T, D), *cache(rng, B, Hkv, T, D)]
    prefix[0].fill_(64), prefix[1].fill_(1.0)
    q = torch.full((B, Hq, 1, D), -(2.0 ** 97), dtype=BF16)
    lens = torch.zeros(B, dtype=I32)
    want, bound = reference(q, prefix, own, lens, 0.125)
    got = sa.slim_attn_decode_int8_shared_prefix(q.cuda(), *on_gpu(prefix), *on_gpu(own), lens.cuda(), 0.125)
    assert ((got.double().cpu() - want).abs() <= bound).all()


@gpu
def test_shared_prefix_lengths_out_of_range_and_repeats(sa):
    """Lengths are taken as the nearest bound; ten calls give the same bits, on two streams at once with a workspace each."""
    rng = np.random.default_rng(4)
    B, Hq, Hkv, D, P, T = 40, 8, 2, 128, 2000, 600
    prefix = on_gpu([*cache(rng, 1, Hkv, P, D), *cache(rng, 1, Hkv, P, D)])
    own = on_gpu([*cache(rng, B, Hkv, T, D), *cache(rng, B, Hkv, T, D)])
    q = queries(rng, B, Hq, D).cuda()
    lens = torch.from_numpy(rng.integers(0, T + 1, B).astype(np.int32))
    lens[3], lens[4] = 0, T
    wild = lens.clone()
    wild[3], wild[4] = -(2 ** 31), 2 ** 31 - 1
    want = sa.slim_attn_decode_int8_shared_prefix(q, *prefix, *own, lens.cuda(), 0.1)
    assert torch.equal(want, sa.slim_attn_decode_int8_shared_prefix(q, *prefix, *own, wild.cuda(), 0.1))
    other = [x.flip(0).contiguous() for x in (q, *own)]
    lens_other = lens.flip(0).cuda()
    streams = [torch.cuda.Stream() for _ in range(2)]
    lens = lens.cuda()
    torch.cuda.synchronize()
    got = [[], []]
    for _ in range(10):
        for i, (s, qq, oo, ll) in enumerate(((streams[0], q, own, lens), (streams[1], other[0], other[1:], lens_other))):
            with torch.cuda.stream(s):
                got[i].append(sa.slim_attn_decode_int8_shared_prefix(qq, *prefix, *oo, ll, 0.1))
    torch.cuda.synchronize()
    for a, b in zip(*got):
        assert torch.equal(a, want) and torch.equal(b.flip(0), want)


@gpu
def test_shared_prefix_replays_from_a_graph(sa):
    rng = np.random.default_rng(5)
    B, Hq, Hkv, D, P, T = 20, 16, 2, 64, 900, 400
    prefix = on_gpu([*cache(rng, 1, Hkv, P, D), *cache(rng, 1, Hkv, P, D)])
    own = on_gpu([*cache(rng, B, Hkv, T, D), *cache(rng, B, Hkv, T, D)])
    q, lens = queries(rng, B, Hq, D).cuda(), torch.full((B,), 7, dtype=I32, device="cuda")
    out = torch.empty_like(q)
    ws = torch.empty(sa.slim_attn_decode_int8_shared_prefix_workspace_bytes(B, Hq, Hkv, P, T, D), dtype=torch.uint8, device="cuda")

    def step():
        return sa.slim_attn_decode_int8_shared_prefix(q, *prefix, *own, lens, 0.125, out=out, workspace=ws)

    assert step() is out
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for rep in range(4):
        lens.copy_(torch.from_numpy(rng.integers(0, T + 1, B).astype(np.int32)))
        q.copy_(queries(rng, B, Hq, D))
        want = sa.slim_attn_decode_int8_shared_prefix(q, *prefix, *own, lens, 0.125)
        ws.fill_(255)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want), "replay %d" % rep


@gpu
def test_a_conversation_behind_a_shared_prompt(sa):
    """The prompt once through the prefill, then steps of a batch: every step as if each sequence had the prompt in its own cache."""
    rng = np.random.default_rng(6)
    B, Hq, Hkv, D, P, steps = 6, 8, 2, 128, 210, 5
    scale, T = 1 / math.sqrt(D), 8
    table = sa.slim_rope_table(P + T, D)
    w = [(1 + 0.25 * torch.from_numpy(rng.standard_normal(D, dtype=np.float32))).to(BF16).cuda() for _ in range(2)]

    def split(x):
        return x[:, :, :Hq], x[:, :, Hq:Hq + Hkv], x[:, :, Hq + Hkv:]

    def rows(b, s):
        return torch.from_numpy(rng.standard_normal((b, s, Hq + 2 * Hkv, D), dtype=np.float32)).to(BF16).cuda()

    at = torch.arange(P, dtype=I32, device="cuda")[None]
    _, *prompt = sa.slim_attn_prefill_emit_int8(*sa.slim_qk_norm_rope(*split(rows(1, P)), table, at, *w), scale, True)
    own = [torch.zeros(s, dtype=t, device="cuda") for s, t in (((B, Hkv, T, D), I8), ((B, Hkv, T), F32)) * 2]
    whole = [torch.zeros(s, dtype=t, device="cuda") for s, t in (((B, Hkv, P + T, D), I8), ((B, Hkv, P + T), F32)) * 2]
    for a, p in zip(whole, prompt):
        a[:, :, :P] = p
    for i in range(steps):
        x, slot = rows(B, 1), torch.full((B,), i, dtype=I32, device="cuda")
        q = sa.slim_qk_norm_rope_append_int8(*split(x), table, (slot + P)[:, None], slot, *own, *w)
        q2 = sa.slim_qk_norm_rope_append_int8(*split(x), table, (slot + P)[:, None], slot + P, *whole, *w)
        assert torch.equal(q, q2)
        got = sa.slim_attn_decode_int8_shared_prefix(q, *prompt, *own, slot + 1, scale)
        want, bound = reference(q.cpu(), [t.cpu() for t in prompt], [t.cpu() for t in own], (slot + 1).cpu(), scale)
        assert ((got.double().cpu() - want).abs() <= bound).all()
        plain = sa.slim_attn_decode_int8_varlen(q, *whole, slot + P + 1, scale)
        assert ((plain.double().cpu() - want).abs() <= bound).all()


# ------------------------------------------------------------------ refusals (CPU)

P_, A = ctypes.c_void_p, 0x1000   # (an address that is never dereferenced)


def test_shared_prefix_refusals(sa):
    lib = sa.load()
    size = lib.slim_attn_decode_int8_shared_prefix_workspace_bytes
    assert size(2, 4, 2, 100, 50, 128) > 0
    assert size(2, 3, 2, 100, 50, 128) == 0 and size(2, 4, 2, 0, 50, 128) == 0 and size(2, 4, 2, 100, 0, 128) == 0
    assert size(2, 4, 2, 100, 50, 96) == 0 and size(40000, 512, 512, 10, 1, 64) == 0 and size(0, 4, 2, 100, 50, 64) == 0
    names = ("q", "pkc", "pks", "pvc", "pvs", "kc", "ks", "vc", "vs", "lens", "out", "ws")

    def call(wsb=1 << 30, B=2, Hq=4, Hkv=2, P=100, T=50, D=128, causal=0, scale=0.1, **other):
        return lib.slim_attn_decode_int8_shared_prefix(*(P_(other.get(n, A)) for n in names), wsb, B, Hq, Hkv, P, T, D, causal, scale, None)

    for n in names:
        assert call(**{n: None}) == 1, n
        assert call(**{n: A + 2}) == 4, n
    assert call(lens=A + 4, wsb=0) == 5       # (lengths need no more than their own alignment)
    assert call(P=0) == 2 and call(T=0) == 2 and call(B=-1) == 2 and call(Hq=5) == 2 and call(scale=0.0) == 2 and call(causal=2) == 2
    assert call(scale=math.inf) == 2 and call(D=80) == 3 and call(B=40000, Hq=512, Hkv=512, T=1) == 2
    assert call(wsb=size(2, 4, 2, 100, 50, 128) - 1) == 5


def test_shared_prefix_refuses_results_over_other_buffers(sa):
    """The merge writes `out` while other workgroups read the records in `ws`, and the sweep writes `ws` while others read the caches."""
    lib = sa.load()
    B, Hq, Hkv, P, T, D, far = 2, 4, 2, 100, 50, 128, 0x1000000
    need = lib.slim_attn_decode_int8_shared_prefix_workspace_bytes(B, Hq, Hkv, P, T, D)
    size = {"q": B * Hq * D * 2, "pkc": Hkv * P * D, "pks": Hkv * P * 4, "pvc": Hkv * P * D, "pvs": Hkv * P * 4, "kc": B * Hkv * T * D,
            "ks": B * Hkv * T * 4, "vc": B * Hkv * T * D, "vs": B * Hkv * T * 4, "lens": B * 4, "out": B * Hq * D * 2, "ws": need}
    home = {n: (i + 1) * far for i, n in enumerate(size)}

    def call(**other):
        at = dict(home, **other)
        return lib.slim_attn_decode_int8_shared_prefix(*(P_(at[n]) for n in size), need, B, Hq, Hkv, P, T, D, 0, 0.1, None)

    for result in ("out", "ws"):
        for n in size:
            if n != result:
                last = (size[n] - 1) // 16 * 16       # (the last 16 bytes of one, the first of the other)
                assert call(**{result: home[n]}) == 7 and call(**{result: home[n] + last}) == 7, (result, n)
                assert call(**{result: home[n] - (size[result] - 1) // 16 * 16}) == 7, (result, n)


def test_shared_prefix_binding_refusals(sa):
    B, Hq, Hkv, D, P, T = 2, 4, 2, 64, 7, 5

    def z(*shape, dtype=F32):
        return torch.zeros(shape, dtype=dtype)

    good = dict(q=z(B, Hq, 1, D, dtype=BF16), prefix_k_codes=z(1, Hkv, P, D, dtype=I8), prefix_k_scale=z(1, Hkv, P),
                prefix_v_codes=z(1, Hkv, P, D, dtype=I8), prefix_v_scale=z(1, Hkv, P), k_codes=z(B, Hkv, T, D, dtype=I8),
                k_scale=z(B, Hkv, T), v_codes=z(B, Hkv, T, D, dtype=I8), v_scale=z(B, Hkv, T), kv_lens=z(B, dtype=I32), softmax_scale=0.1)

    def refused(text, kind=AssertionError, **other):
        with pytest.raises(kind, match=text):
            sa.slim_attn_decode_int8_shared_prefix(**dict(good, **other))

    refused("device tensors")
    refused("one query token", q=z(B, Hq, 2, D, dtype=BF16))
    refused("prefix_k_codes", prefix_k_codes=z(B, Hkv, P, D, dtype=I8))
    refused("prefix_v_codes", prefix_v_codes=z(1, Hkv, P + 1, D, dtype=I8))
    refused("prefix_k_scale", prefix_k_scale=z(Hkv, P))
    refused("prefix_v_scale", prefix_v_scale=z(1, Hkv, P + 1))
    refused("shape of k_codes", k_codes=z(B + 1, Hkv, T, D, dtype=I8))
    refused("v_codes", v_codes=z(B, Hkv, T, D + 64, dtype=I8))
    refused("k_scale", k_scale=z(B, Hkv, T, 1))
    refused("v_scale", v_scale=z(B, Hkv, T + 1))
    refused("one length", kv_lens=z(B + 1, dtype=I32))
    refused("four dimensions", ValueError, k_codes=z(B, Hkv, T, dtype=I8))
