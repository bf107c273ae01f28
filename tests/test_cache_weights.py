"""Decode that gives the cached tokens' attention weights, and the eviction that goes by them.

Results of the decode are held to the bound of tests/test_decode_prefix.py, weights to this one.  A score is a sum of D products in fp32
(each exact), times two factors: off by at most (D + 4) 2^-24 A in units of the exponent to the base of two, A = log2(e) scale k_scale
sum_d |q_d code_d|.  The maximum that is taken off is a whole number; the difference is rounded once more (2^-24 of it, at most 2 A),
and exponential, sum, inverse and product add some 2^-21.  A probability is thus off by at most its (D + 8) 2^-24 ln 2 A + 2^-21, and
by as much again through the sum that it is divided by, where A is its row's largest.
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
    x = rng.standard_normal(shape, dtype=np.float32)
    scale = (np.abs(x).max(-1) / np.float32(127)).astype(np.float32)
    return torch.from_numpy(np.rint(x / scale[..., None]).astype(np.int8)), torch.from_numpy(scale)


def reference(q, own, lens, scale, w_in=None):
    """(o, its bound, weights, their bound) in 64 bits"""
    B, Hq, _, D = q.shape
    Hkv, T = own[0].shape[1:3]
    q = q.double().view(B, Hkv, Hq // Hkv, D)
    o, o_bound = torch.empty_like(q), torch.empty_like(q)
    w, w_bound = torch.zeros((B, Hkv, T), dtype=torch.float64), torch.zeros((B, Hkv, T), dtype=torch.float64)
    for b in range(B):
        n = int(lens[b])
        for g in range(Hkv):
            k, v = (own[i][b, g, :n].double() * own[i + 1][b, g, :n].double()[:, None] for i in (0, 2))
            p = torch.softmax((q[b, g] @ k.T) * scale, 1)
            a = ((q[b, g].abs() @ k.abs().T) * scale / math.log(2)).amax(1, keepdim=True)
            o[b, g] = p @ v
            o_bound[b, g] = (2.0 ** -8 + 2.0 ** -14) * (p @ v.abs()) + 2.0 ** -8 * (1 + 2.0 ** -8) * o[b, g].abs()
            w[b, g, :n] = p.sum(0)
            w_bound[b, g, :n] = (p * 2 * ((D + 8) * 2.0 ** -24 * math.log(2) * a + 2.0 ** -21)).sum(0)
            if w_in is not None:
                w[b, g, :n] += w_in[b, g, :n].double()
                w_bound[b, g, :n] += 2.0 ** -23 * w[b, g, :n].abs()
    return o.view(B, Hq, 1, D), o_bound.view(B, Hq, 1, D), w, w_bound


def on_gpu(ts):
    return [t.cuda() for t in ts]


def check(sa, q, own, lens, scale, what, w_in=None, dirty=True):
    B, Hq, _, D = q.shape
    Hkv, T = own[0].shape[1:3]
    want, o_bound, w, w_bound = reference(q, own, lens, scale, w_in)
    dirt = [t.clone() for t in own]
    for b, n in enumerate(lens.tolist()):   # past a length: numbers that would show in any result
        for t, x in zip(dirt, (127, math.nan, -127, math.inf)):
            t[b, :, n:] = x
    size = sa.slim_attn_decode_int8_weights_workspace_bytes(B, Hq, Hkv, T, D)
    ws = torch.full((size + 64,), 255, dtype=torch.uint8, device="cuda")    # (NaN in 32 bits)
    sums = None
    if w_in is not None:
        sums = w_in.clone()
        for b, n in enumerate(lens.tolist()):
            sums[b, :, n:] = math.nan
        sums = sums.cuda()
    out, got = sa.slim_attn_decode_int8_weights(q.cuda(), *on_gpu(dirt), lens.cuda(), scale, weights_in=sums, workspace=ws[:size])
    assert (ws[size:] == 255).all(), "written past the workspace"
    off = (out.double().cpu() - want).abs()
    assert (off <= o_bound).all(), "%s: %.3g of the result's bound" % (what, (off / o_bound).max())
    off = (got.double().cpu() - w).abs()
    assert (off <= w_bound).all(), "%s: %.3g of the weights' bound" % (what, (off / w_bound).nan_to_num(math.inf).max())
    return out, got


SHAPES = [(1, 1, 1), (1, 8, 8), (3, 10, 2), (4, 32, 1), (2, 40, 1), (2, 70, 1), (5, 16, 4), (16, 32, 8), (40, 9, 3), (130, 6, 2)]


@gpu
@pytest.mark.parametrize("B,Hq,Hkv", SHAPES)
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("T", [1, 31, 33, 300, 1025])
def test_weights_small_shapes(sa, B, Hq, Hkv, D, T):
    print("weights", B, Hq, Hkv, D, T, flush=True)
    rng = np.random.default_rng(B * Hq + T + D)
    own = [*cache(rng, B, Hkv, T, D), *cache(rng, B, Hkv, T, D)]
    lens = torch.from_numpy(rng.integers(1, T + 1, B).astype(np.int32))
    lens[0] = T
    q = torch.from_numpy(rng.standard_normal((B, Hq, 1, D), dtype=np.float32)).to(BF16)
    w_in = torch.from_numpy(rng.random((B, Hkv, T), dtype=np.float32)) if T != 33 else None
    check(sa, q, own, lens, 1 / math.sqrt(D), "B%d Hq%d Hkv%d D%d T%d" % (B, Hq, Hkv, D, T), w_in)


@gpu
@pytest.mark.parametrize("B,Hq,Hkv,D,T", [(1, 64, 8, 128, 20000), (1, 32, 32, 128, 3000), (8, 64, 8, 64, 8192), (48, 32, 8, 128, 2001),
                                          (2, 40, 1, 128, 9001), (3, 8, 8, 64, 5000)])
def test_weights_long_caches(sa, B, Hq, Hkv, D, T):
    print("weights", B, Hq, Hkv, D, T, flush=True)
    rng = np.random.default_rng(T)
    own = [*cache(rng, B, Hkv, T, D), *cache(rng, B, Hkv, T, D)]
    lens = torch.from_numpy(rng.integers(T // 8, T + 1, B).astype(np.int32))
    lens[-1] = T
    q = torch.from_numpy(rng.standard_normal((B, Hq, 1, D), dtype=np.float32)).to(BF16)
    check(sa, q, own, lens, 1 / math.sqrt(D), "T%d" % T, torch.from_numpy(rng.random((B, Hkv, T), dtype=np.float32)))


@gpu
@pytest.mark.parametrize("B,Hq,Hkv,T", [(1, 8, 8, 33), (3, 4, 4, 700), (1, 32, 32, 3000), (100, 4, 4, 300), (2, 40, 1, 300), (1, 70, 1, 2500)])
@pytest.mark.parametrize("D", [64, 128])
def test_results_have_the_bits_of_the_decode_without_weights(sa, B, Hq, Hkv, T, D):
    """One query head a KV head, or more than 32: the decode keeps its probabilities in fp32 there, and so does this one but for the last
    of two roundings to bf16, 2^-16 of a probability.  What is left of the file's bound is 2^-16 + 2^-14 of sum_t p_t |v^_t| and the result's
    own rounding."""
    print("bits of the result", B, Hq, Hkv, T, D, flush=True)
    rng = np.random.default_rng(B + Hq + T + D)
    own = [*cache(rng, B, Hkv, T, D), *cache(rng, B, Hkv, T, D)]
    lens = torch.from_numpy(rng.integers(1, T + 1, B).astype(np.int32))
    lens[0] = T
    q = torch.from_numpy(rng.standard_normal((B, Hq, 1, D), dtype=np.float32)).to(BF16)
    scale = 1 / math.sqrt(D)
    want, bound, _, _ = reference(q, own, lens, scale)
    last = 2.0 ** -8 * (1 + 2.0 ** -8) * want.abs()
    bound = last + (bound - last) * (2.0 ** -16 + 2.0 ** -14) / (2.0 ** -8 + 2.0 ** -14)
    dev = (q.cuda(), *on_gpu(own), lens.cuda(), scale)
    for out, what in ((sa.slim_attn_decode_int8_varlen(*dev), "without weights"), (sa.slim_attn_decode_int8_weights(*dev)[0], "with weights")):
        off = (out.double().cpu() - want).abs()
        assert (off <= bound).all(), "%s: %.3g of its bound" % (what, (off / bound).max())


@gpu
@pytest.mark.parametrize("B,Hq,Hkv,D,T", [(40, 280, 4, 64, 1100), (37, 320, 8, 128, 1030)])
@pytest.mark.parametrize("weights", [False, True])
def test_weights_of_rows_dealt_by_length(sa, B, Hq, Hkv, D, T, weights):
    """More than 32 query heads a KV head in as many rows (sequences x head groups) as are dealt by their lengths, which are spread: each
    row is a (KV head, head group), with a record of its own, and the second launch turns all groups' scores into weights."""
    print("rows dealt by length", B, Hq, Hkv, D, T, weights, flush=True)
    groups = Hkv * ((Hq // Hkv + 31) // 32)
    ranked, through = ctypes.c_int(), ctypes.c_int()
    assert sa.load().slim_attn_decode_int8_plan_options(B, 32 * groups, groups, T, D, 1, ctypes.byref(ranked), ctypes.byref(through)) == 0
    assert ranked.value == 1
    rng = np.random.default_rng(T)
    own = [*cache(rng, B, Hkv, T, D), *cache(rng, B, Hkv, T, D)]
    lens = torch.from_numpy(np.where(rng.random(B) < 0.25, T, rng.integers(T // 8, T + 1, B)).astype(np.int32))
    q = torch.from_numpy(rng.standard_normal((B, Hq, 1, D), dtype=np.float32)).to(BF16)
    check(sa, q, own, lens, 1 / math.sqrt(D), "dealt", torch.from_numpy(rng.random((B, Hkv, T), dtype=np.float32)) if weights else None)


@gpu
@pytest.mark.parametrize("B,Hq,Hkv,T", [(1, 8, 4, 33), (3, 32, 8, 700), (60, 16, 2, 300), (1, 64, 8, 5000), (2, 20, 1, 2500), (100, 32, 1, 200)])
@pytest.mark.parametrize("D", [64, 128])
def test_results_of_grouped_heads_have_the_bits_of_fp32(sa, B, Hq, Hkv, T, D):
    """2 to 32 query heads a KV head: the same bound, which the decode without weights, whose probabilities are one bf16 each there, does not
    hold."""
    print("bits of the result", B, Hq, Hkv, T, D, flush=True)
    rng = np.random.default_rng(B + Hq + T + D)
    own = [*cache(rng, B, Hkv, T, D), *cache(rng, B, Hkv, T, D)]
    lens = torch.from_numpy(rng.integers(1, T + 1, B).astype(np.int32))
    lens[0] = T
    q = torch.from_numpy(rng.standard_normal((B, Hq, 1, D), dtype=np.float32)).to(BF16)
    want, bound, _, _ = reference(q, own, lens, 1 / math.sqrt(D))
    last = 2.0 ** -8 * (1 + 2.0 ** -8) * want.abs()
    bound = last + (bound - last) * (2.0 ** -16 + 2.0 ** -14) / (2.0 ** -8 + 2.0 ** -14)
    off = (sa.slim_attn_decode_int8_weights(q.cuda(), *on_gpu(own), lens.cuda(), 1 / math.sqrt(D))[0].double().cpu() - want).abs()
    assert (off <= bound).all(), "%.3g of its bound" % (off / bound).max()


@gpu
@pytest.mark.parametrize("B,Hq,Hkv,T", [(2, 8, 2, 700), (40, 12, 3, 333), (1, 20, 1, 2500)])
def test_weights_of_sharp_rows_and_zero_tokens(sa, B, Hq, Hkv, T):
    """Rows that one token carries; a tenth of the tokens have a scale of zero, and so a score of zero and no value."""
    rng = np.random.default_rng(T)
    D = 128
    own = [*cache(rng, B, Hkv, T, D), *cache(rng, B, Hkv, T, D)]
    off = torch.from_numpy(rng.random((B, Hkv, T)) < 0.1)
    for i in (1, 3):
        own[i][off] = 0.0
    lens = torch.from_numpy(rng.integers(1, T + 1, B).astype(np.int32))
    q = torch.from_numpy(rng.standard_normal((B, Hq, 1, D), dtype=np.float32)).to(BF16)
    for b in range(B):
        for h in range(0, Hq, 2):
            g, t = h // (Hq // Hkv), int(rng.integers(lens[b]))
            q[b, h, 0] = (own[0][b, g, t].float() * own[1][b, g, t] * float(rng.uniform(1, 5))).to(BF16)
    check(sa, q, own, lens, 1 / math.sqrt(D), "sharp")


@gpu
@pytest.mark.parametrize("B,Hq,Hkv,T", [(2, 8, 2, 1500), (60, 8, 4, 200)])
def test_weights_of_extreme_queries(sa, B, Hq, Hkv, T):
    """Rows around 2^-50: every token the same weight.  Rows around 2^60: the largest score has all of it.  A row that is not finite shows
    in its own result and its KV head's weights alone."""
    rng = np.random.default_rng(T)
    D, scale = 64, 0.125
    own = [*cache(rng, B, Hkv, T, D), *cache(rng, B, Hkv, T, D)]
    lens = torch.from_numpy(rng.integers(1, T + 1, B).astype(np.int32))
    q = torch.from_numpy(rng.standard_normal((B, Hq, 1, D), dtype=np.float32)).to(BF16)
    check(sa, (q.float() * 2.0 ** -50).to(BF16), own, lens, scale, "2^-50")
    big = (q.float() * 2.0 ** 60).to(BF16)
    want, o_bound, w, _ = reference(big, own, lens, scale)
    out, got = sa.slim_attn_decode_int8_weights(big.cuda(), *on_gpu(own), lens.cuda(), scale)
    assert ((out.double().cpu() - want).abs() <= o_bound).all() and torch.equal(got.double().cpu(), w.round())
    out, fine = sa.slim_attn_decode_int8_weights(q.cuda(), *on_gpu(own), lens.cuda(), scale)
    q[1, 1, 0, 3] = math.nan
    bad, got = sa.slim_attn_decode_int8_weights(q.cuda(), *on_gpu(own), lens.cuda(), scale)
    assert torch.equal((bad != out).any(-1).nonzero().cpu(), torch.tensor([[1, 1, 0]]))
    same = (got == fine).all(-1)
    same[1, 1 // (Hq // Hkv)] = True
    assert same.all()


@gpu
def test_weights_in_place_over_steps_streams_and_replays(sa):
    """weights_out == weights_in adds up; lengths out of range are the nearest bound; two streams and a graph give the same bits."""
    rng = np.random.default_rng(2)
    for B, Hq, Hkv, T in ((3, 16, 2, 3000), (90, 8, 4, 200)):
        D, scale = 128, 0.08
        own = on_gpu([*cache(rng, B, Hkv, T, D), *cache(rng, B, Hkv, T, D)])
        q = torch.from_numpy(rng.standard_normal((B, Hq, 1, D), dtype=np.float32)).to(BF16).cuda()
        lens = torch.from_numpy(rng.integers(1, T + 1, B).astype(np.int32)).cuda()
        lens[0], lens[1] = 1, T
        wild = lens.clone()
        wild[0], wild[1] = -7, 2 ** 31 - 1
        out, once = sa.slim_attn_decode_int8_weights(q, *own, lens, scale)
        out2, again = sa.slim_attn_decode_int8_weights(q, *own, wild, scale)
        assert torch.equal(out, out2) and torch.equal(once, again)
        sums = torch.zeros_like(once)
        for i in range(3):
            r, s = sa.slim_attn_decode_int8_weights(q, *own, lens, scale, weights_in=sums, weights_out=sums, out=out2)
            assert r is out2 and s is sums and torch.equal(out, out2)
        assert torch.equal(sums, (once + once) + once)
        streams, got = [torch.cuda.Stream() for _ in range(2)], []
        torch.cuda.synchronize()
        for _ in range(10):
            for s in streams:
                with torch.cuda.stream(s):
                    got.append(sa.slim_attn_decode_int8_weights(q, *own, lens, scale))
        torch.cuda.synchronize()
        assert all(torch.equal(o, out) and torch.equal(w, once) for o, w in got)
        ws = torch.empty(sa.slim_attn_decode_int8_weights_workspace_bytes(B, Hq, Hkv, T, D), dtype=torch.uint8, device="cuda")
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            sa.slim_attn_decode_int8_weights(q, *own, lens, scale, weights_in=sums, weights_out=sums, out=out2, workspace=ws)
        sums.zero_()
        want = torch.zeros_like(sums)
        for rep in range(4):
            lens.copy_(torch.from_numpy(rng.integers(1, T + 1, B).astype(np.int32)))
            ref, _ = sa.slim_attn_decode_int8_weights(q, *own, lens, scale, weights_in=want, weights_out=want)
            ws.fill_(255)
            torch.cuda.synchronize()
            graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(out2, ref) and torch.equal(sums, want), "replay %d" % rep


# ------------------------------------------------------------------ eviction

def chosen(weights, n, keep, recent):
    """The former indices of what stays, in order: one row of weights."""
    if n <= keep:
        return np.arange(n)
    w = weights[:n - recent].astype(np.float64)
    w = np.where(np.isnan(w), -np.inf, w)
    first = np.where(np.isnan(weights[:n - recent]), 1, 0)          # (NaN behind every number, the least too)
    order = np.lexsort((np.arange(n - recent), first, -w))
    return np.concatenate([np.sort(order[:keep - recent]), np.arange(n - recent, n)])


def check_evict(sa, rng, B, Hkv, D, T, keep, recent, out_len, weights, lens, what):
    codes = [torch.from_numpy(rng.integers(-127, 128, (B, Hkv, T, D), dtype=np.int8)) for _ in range(2)]
    scales = [torch.from_numpy(rng.random((B, Hkv, T), dtype=np.float32)) for _ in range(2)]
    src = [codes[0], scales[0], codes[1], scales[1], torch.from_numpy(weights)]
    dst = [torch.full((B, Hkv, out_len, D), 5, dtype=I8), torch.full((B, Hkv, out_len), 6.0), torch.full((B, Hkv, out_len, D), 7, dtype=I8),
           torch.full((B, Hkv, out_len), 8.0), torch.full((B, Hkv, out_len), 9.0)]
    got = sa.slim_cache_evict_int8(*on_gpu(src), torch.from_numpy(lens).cuda(), keep, recent, *on_gpu(dst))
    kept, new_lens = got[5].cpu().numpy(), got[6].cpu().numpy()
    dst[4].zero_()
    for b in range(B):
        n = min(max(int(lens[b]), 0), T)
        assert new_lens[b] == min(n, keep), what
        for g in range(Hkv):
            at = chosen(weights[b, g], n, keep, recent)
            assert np.array_equal(kept[b, g, :len(at)], at) and (kept[b, g, len(at):] == -1).all(), (what, b, g)
            for s, d in zip(src, dst):
                d[b, g, :len(at)] = s[b, g, at]
    for d, x in zip(dst, got):
        assert d.numpy().tobytes() == x.cpu().numpy().tobytes(), what      # (bits: weights may be NaN)


@gpu
@pytest.mark.parametrize("T,keep,recent", [(1, 1, 0), (2, 1, 1), (2, 1, 0), (64, 63, 5), (100, 100, 3), (100, 150, 150), (1000, 1, 0),
                                           (1000, 500, 500), (1000, 500, 0), (4095, 77, 70), (4097, 2000, 9), (9000, 8999, 8998),
                                           (70001, 4000, 512)])
@pytest.mark.parametrize("D", [64, 128])
def test_eviction_keeps_the_largest_weights(sa, T, keep, recent, D):
    print("eviction", T, keep, recent, D, flush=True)
    rng = np.random.default_rng(T + keep + recent + D)
    B, Hkv = (2, 2) if T > 50000 else (5, 3)
    weights = np.exp(2 * rng.standard_normal((B, Hkv, T))).astype(np.float32)
    lens = rng.integers(0, T + 1, B).astype(np.int32)
    lens[0] = T
    if B > 2:
        lens[1], lens[2], lens[3] = 0, T + 5, -3
    check_evict(sa, rng, B, Hkv, D, T, keep, recent, keep + int(rng.integers(0, 9)), weights, lens, "T%d keep%d" % (T, keep))


@gpu
@pytest.mark.parametrize("kind", ["equal", "zeros", "few", "signs", "ends", "nan", "near", "rising", "falling"])
def test_eviction_of_difficult_weights(sa, kind):
    rng = np.random.default_rng(11)
    B, Hkv, T, D = 3, 2, 5000, 64
    w = rng.random((B, Hkv, T), dtype=np.float32)
    if kind == "equal":
        w[:] = np.float32(0.3)
    elif kind == "zeros":
        w[rng.random(w.shape) < 0.9] = 0.0
    elif kind == "few":
        w = (w * 4).round() / 4
    elif kind == "signs":
        w = np.where(rng.random(w.shape) < 0.5, np.float32(0.0), np.float32(-0.0)) * np.float32(1) + np.where(rng.random(w.shape) < 0.3, w - 0.5, 0)
        w = np.where(rng.random(w.shape) < 0.3, np.float32(-0.0), w)
    elif kind == "ends":
        w = rng.choice(np.array([np.inf, -np.inf, 3.4028235e38, -3.4028235e38, 1e-45, -1e-45, 0.0, -0.0, 1.0], np.float32), w.shape)
    elif kind == "nan":
        w = np.where(rng.random(w.shape) < 0.6, np.float32(np.nan), np.where(rng.random(w.shape) < 0.5, np.float32(-np.inf), w - 0.5))
        w[0] = np.nan
    elif kind == "near":
        w = (1 + rng.integers(0, 3000, w.shape) * 2.0 ** -23).astype(np.float32)
    else:
        w = np.sort(w, -1) if kind == "rising" else -np.sort(-w, -1)
    w = np.ascontiguousarray(w.astype(np.float32))
    lens = np.array([T, T - 1, 4000], np.int32)
    for keep, recent in ((1, 0), (700, 30), (2500, 0), (3999, 1000), (4900, 0)):
        check_evict(sa, rng, B, Hkv, D, T, keep, recent, keep, w, lens, "%s keep%d" % (kind, keep))


@gpu
@pytest.mark.parametrize("T", [20000, 40001])
@pytest.mark.parametrize("spread", [1, 1 << 8, 1 << 20, 1 << 21])
def test_eviction_of_many_near_weights(sa, T, spread):
    """Weights of one binade, as many steps apart as `spread`: the first digits of tens of thousands are the same."""
    rng = np.random.default_rng(T + spread)
    w = (1 + rng.integers(0, spread, (1, 2, T)) * 2.0 ** -23).astype(np.float32)
    for keep, recent in ((T // 2, 100), (T - 1, 0), (5, 0)):
        check_evict(sa, rng, 1, 2, 64, T, keep, recent, keep, w, np.array([T], np.int32), "T%d spread%d keep%d" % (T, spread, keep))


@gpu
@pytest.mark.parametrize("kind", ["ties", "nan"])
def test_eviction_of_lengths_about_a_chunk(sa, kind):
    """Lengths (without the recent tokens) one token either side of a wave's, a chunk's and a round's, in caches of more."""
    rng = np.random.default_rng(23)
    for T, edges in ((9000, (256, 4096, 4096 + 256, 8192)), (38000, (32768, 32768 + 4096))):
        lens = np.array([e + 7 + d for e in edges for d in (-1, 0, 1)], np.int32)
        w = (rng.random((len(lens), 1, T)) * 8).round().astype(np.float32)
        if kind == "nan":
            w[rng.random(w.shape) < 0.5] = np.nan
        for keep in (8, 100, 200):
            check_evict(sa, rng, len(lens), 1, 64, T, keep, 7, keep, w, lens, "%s T%d keep%d" % (kind, T, keep))


@gpu
def test_eviction_replays_from_a_graph(sa):
    rng = np.random.default_rng(12)
    B, Hkv, T, D, keep, recent = 4, 2, 3000, 128, 1000, 64
    src = on_gpu([*cache(rng, B, Hkv, T, D), *cache(rng, B, Hkv, T, D)])
    weights, lens = torch.rand(B, Hkv, T, device="cuda"), torch.full((B,), T, dtype=I32, device="cuda")
    dst = [torch.zeros_like(t) for t in (*src, weights)] + [torch.empty((B, Hkv, keep), dtype=I32, device="cuda"), torch.empty_like(lens)]
    got = sa.slim_cache_evict_int8(*src, weights, lens, keep, recent, *dst)
    assert all(a is b for a, b in zip(got, dst))
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        sa.slim_cache_evict_int8(*src, weights, lens, keep, recent, *dst)
    for rep in range(4):
        weights.uniform_()
        lens.copy_(torch.from_numpy(rng.integers(500, T + 1, B).astype(np.int32)))
        for t in dst:
            t.zero_()
        want = [torch.zeros_like(t) for t in dst]
        sa.slim_cache_evict_int8(*src, weights, lens, keep, recent, *want)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(dst, want)), "replay %d" % rep


@gpu
def test_a_bounded_cache_over_many_tokens(sa, oracle):
    """A serving loop whose cache holds 64 tokens a KV head and is cut down to 40 whenever it is full: appends, decodes with
    weights, evictions, against a model of the same in 64 bits that makes the same choices from the same weights."""
    rng = np.random.default_rng(13)
    B, Hq, Hkv, D, T, keep, recent, steps = 2, 8, 2, 128, 64, 40, 16, 150
    scale = 1 / math.sqrt(D)
    table = sa.slim_rope_table(steps, D)

    def empty():
        return [torch.zeros(s, dtype=t, device="cuda") for s, t in (((B, Hkv, T, D), I8), ((B, Hkv, T), F32)) * 2]

    live, spare = [*empty(), torch.zeros((B, Hkv, T), device="cuda")], [*empty(), torch.zeros((B, Hkv, T), device="cuda")]
    lens = torch.zeros(B, dtype=I32, device="cuda")
    evictions = 0
    for i in range(steps):
        if int(lens.max()) == T:
            before = [t.cpu() for t in live]
            *spare, kept, new_lens = sa.slim_cache_evict_int8(*live, lens, keep, recent, *spare)
            assert (new_lens == keep).all()
            for b in range(B):
                for g in range(Hkv):
                    at = chosen(before[4][b, g].numpy(), T, keep, recent)
                    assert np.array_equal(kept[b, g].cpu().numpy(), at)
                    for x, y in zip(before, spare):
                        assert torch.equal(x[b, g, at], y[b, g, :keep].cpu())
            live, spare, lens = spare, live, new_lens
            evictions += 1
        qkv = torch.from_numpy(rng.standard_normal((B, 1, Hq + 2 * Hkv, D), dtype=np.float32)).to(BF16).cuda()
        at = torch.full((B, 1), i, dtype=I32, device="cuda")
        q = sa.slim_qk_norm_rope_append_int8(qkv[:, :, :Hq], qkv[:, :, Hq:Hq + Hkv], qkv[:, :, Hq + Hkv:], table, at, lens, *live[:4])
        lens = lens + 1
        was = live[4].cpu()
        out, _ = sa.slim_attn_decode_int8_weights(q, *live[:4], lens, scale, weights_in=live[4], weights_out=live[4])
        want, o_bound, w, w_bound = reference(q.cpu(), [t.cpu() for t in live[:4]], lens.cpu(), scale, was)
        assert ((out.double().cpu() - want).abs() <= o_bound).all() and ((live[4].double().cpu() - w).abs() <= w_bound).all(), i
    assert evictions >= 3


# ------------------------------------------------------------------ refusals (CPU)

P_, A = ctypes.c_void_p, 0x1000000   # (an address that is never dereferenced)


def test_weights_refusals(sa):
    lib = sa.load()
    size = lib.slim_attn_decode_int8_weights_workspace_bytes
    assert size(2, 4, 2, 100, 128) >= 2 * 4 * (128 * 4 + 130 * 4)
    assert size(2, 3, 2, 100, 128) == 0 and size(2, 4, 2, 0, 128) == 0 and size(2, 4, 2, 100, 72) == 0 and size(60000, 200, 200, 10, 64) == 0
    names = ("q", "kc", "ks", "vc", "vs", "lens", "wi", "wo", "out", "ws")

    def call(wsb=1 << 30, B=2, Hq=4, Hkv=2, T=100, D=128, causal=0, scale=0.1, **other):
        at = {n: (i + 1) * A for i, n in enumerate(names)}
        at.update(other)
        return lib.slim_attn_decode_int8_weights(*(P_(at[n]) for n in names), wsb, B, Hq, Hkv, T, D, causal, scale, None)

    for n in names:
        if n != "wi":
            assert call(**{n: None}) == 1, n
        assert call(**{n: A + 2}) == 4, n
    assert call(T=0) == 2 and call(B=0) == 2 and call(Hq=3) == 2 and call(scale=-1.0) == 2 and call(causal=-1) == 2 and call(D=32) == 3
    assert call(B=60000, Hq=200, Hkv=200, T=10, D=64) == 2
    assert call(wsb=size(2, 4, 2, 100, 128) - 1) == 5
    for n in ("q", "kc", "ks", "vc", "vs", "lens", "out", "ws"):
        assert call(wo=(names.index(n) + 1) * A) == 7, n
    assert call(wo=7 * A + 16) == 7 and call(out=A) == 7 and call(ws=2 * A + 64) == 7     # (into weights_in, but not the same)
    assert call(wo=7 * A, D=96) == 3


def test_eviction_refusals(sa):
    lib = sa.load()
    names = ("kc", "ks", "vc", "vs", "w", "lens", "kc2", "ks2", "vc2", "vs2", "w2", "kept", "lens2")

    def call(B=2, Hkv=2, T=100, out=50, D=128, keep=50, recent=10, **other):
        at = {n: (i + 1) * A for i, n in enumerate(names)}
        at.update(other)
        return lib.slim_cache_evict_int8(*(P_(at[n]) for n in names), B, Hkv, T, out, D, keep, recent, None)

    for n in names:
        assert call(**{n: None}) == 1, n
        assert call(**{n: A + 2}) == 4, n
    assert call(B=0) == 2 and call(T=0) == 2 and call(out=0) == 2 and call(keep=0) == 2 and call(keep=51) == 2 and call(recent=-1) == 2
    assert call(recent=51) == 2 and call(D=100) == 3 and call(B=2048, Hkv=2048) == 2 and call(B=65535, Hkv=60, out=500) == 2
    for n in names[:6]:
        for m in names[6:]:
            assert call(**{m: (names.index(n) + 1) * A}) == 7, (n, m)
    assert call(kept=13 * A) == 7 and call(vc2=7 * A + 2 * 2 * 50 * 128 - 16) == 7


def test_binding_refusals(sa):
    B, Hq, Hkv, D, T = 2, 4, 2, 64, 9

    def z(*shape, dtype=F32):
        return torch.zeros(shape, dtype=dtype)

    own = dict(k_codes=z(B, Hkv, T, D, dtype=I8), k_scale=z(B, Hkv, T), v_codes=z(B, Hkv, T, D, dtype=I8), v_scale=z(B, Hkv, T),
               kv_lens=z(B, dtype=I32))
    decode = dict(own, q=z(B, Hq, 1, D, dtype=BF16), softmax_scale=0.1)
    evict = dict(own, weights=z(B, Hkv, T), keep=4, recent=2)

    def refused(f, args, text, kind=AssertionError, **other):
        with pytest.raises(kind, match=text):
            f(**dict(args, **other))

    for f, args in ((sa.slim_attn_decode_int8_weights, decode), (sa.slim_cache_evict_int8, evict)):
        refused(f, args, "device tensors")
        refused(f, args, "v_codes", v_codes=z(B, Hkv, T + 1, D, dtype=I8))
        refused(f, args, "k_scale", k_scale=z(B, Hkv, T + 1))
        refused(f, args, "v_scale", v_scale=z(B, T, Hkv))
        refused(f, args, "one length", kv_lens=z(B + 1, dtype=I32))
    f = sa.slim_attn_decode_int8_weights
    refused(f, decode, "one query token", q=z(B, Hq, 2, D, dtype=BF16))
    refused(f, decode, "weights_in", weights_in=z(B, Hkv, T + 1))
    f = sa.slim_cache_evict_int8
    refused(f, evict, "weights", weights=z(B, Hkv))
    refused(f, evict, "keep", ValueError, keep=0)
    refused(f, evict, "keep", ValueError, keep=1 << 31)
    refused(f, evict, "keep", ValueError, recent=5)
    refused(f, evict, "integer", TypeError, keep=2.5)
