"""Norm and rotation of queries and keys, with and without the append to the INT8 cache, against their definition in 64 bits.

The kernel computes in 64 bits as well, so results, codes and scales are held to the oracle's bits: two 64-bit evaluations
differ by some 2^-50 of a value, and a rounding to 24 bits can turn on that for one value in 2^26 at most, of which one in 2^16 lies
where the rounding to 8 bits turns on it too.
"""
import ctypes
import math
import os

import numpy as np
import pytest
import torch

from paper_2407_07304_amd.inputs import bf16_bits_to_f32, f32_to_bf16_bits, normal_bf16

BF16, F32, I8, I32 = torch.bfloat16, torch.float32, torch.int8, torch.int32
gpu = pytest.mark.gpu


@pytest.fixture(scope="module")
def sa():
    from paper_2407_07304_amd import build, slimattn
    if not (os.path.exists(slimattn.LIB_PATH) and os.path.exists(slimattn.BINDING_PATH)):
        build.build()
    slimattn.load()
    return slimattn


# ------------------------------------------------------------------ the definition

def table_of(length, D, base=10000.0):
    angle = np.arange(length)[:, None] * base ** (-np.arange(0, D, 2) / D)
    return np.concatenate([np.cos(angle), np.sin(angle)], 1).astype(np.float32)


def rotated(bits, weight, table, positions, eps, interleaved):
    """[B,S,H,D] bf16 bits -> [B,H,S,D] bf16 bits"""
    x = bf16_bits_to_f32(bits).astype(np.float64)
    D = x.shape[-1]
    if weight is not None:
        x = x / np.sqrt((x * x).mean(-1, keepdims=True) + eps) * bf16_bits_to_f32(weight).astype(np.float64)
    there = (positions >= 0) & (positions < len(table))
    t = table.astype(np.float64)[np.where(there, positions, 0)][:, :, None]
    c, s = t[..., :D // 2], t[..., D // 2:]
    i = np.arange(0, D, 2) if interleaved else np.arange(D // 2)
    j = i + (1 if interleaved else D // 2)
    y = np.empty_like(x)
    y[..., i] = x[..., i] * c - x[..., j] * s
    y[..., j] = x[..., j] * c + x[..., i] * s
    y = np.where(there[:, :, None, None], y, 0.0)
    with np.errstate(over="ignore"):
        return f32_to_bf16_bits(y.astype(np.float32)).transpose(0, 2, 1, 3)


def dev(bits):
    return torch.from_numpy(np.ascontiguousarray(bits).view(np.int16)).cuda().view(BF16)


def host(t):
    return t.contiguous().view(torch.int16).cpu().numpy().view(np.uint16)


def same_bits(got, want, what):
    g = host(got)
    bad = (g != want) & ~((g & 0x7fff == 0) & (want & 0x7fff == 0))   # (a zero's sign is nobody's)
    assert not bad.any(), "%s: %d of %d values differ, the first at %s" % (what, bad.sum(), bad.size, np.argwhere(bad)[0])


def case(rng, B, S, Hq, Hkv, D, length, norm=True):
    qkv = normal_bf16(rng, (B, S, Hq + 2 * Hkv, D))
    weights = [f32_to_bf16_bits((1 + 0.25 * rng.standard_normal(D)).astype(np.float32)) if norm else None for _ in range(2)]
    return qkv, weights, rng.integers(0, length, (B, S)).astype(np.int32)


def views(t, Hq, Hkv):
    return t[:, :, :Hq], t[:, :, Hq:Hq + Hkv], t[:, :, Hq + Hkv:]


def on_device(weights):
    return [None if w is None else dev(w) for w in weights]


SHAPES = [(1, 1, 1, 1, 128), (1, 1, 64, 8, 128), (3, 1, 6, 3, 64), (2, 5, 5, 5, 128), (1, 777, 8, 2, 64), (4, 100, 40, 8, 128),
          (2, 1000, 32, 8, 128), (3, 700, 9, 3, 64), (1, 2048, 32, 32, 128), (37, 1, 16, 2, 64)]


@gpu
@pytest.mark.parametrize("B,S,Hq,Hkv,D", SHAPES)
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("norm", [True, False])
def test_rows_are_the_definitions_bits(sa, B, S, Hq, Hkv, D, interleaved, norm):
    print("norm and rotation", B, S, Hq, Hkv, D, interleaved, norm, flush=True)
    rng = np.random.default_rng(B * S + Hq)
    length = 4096
    qkv, (qw, kw), positions = case(rng, B, S, Hq, Hkv, D, length, norm)
    table = table_of(length, D)
    q, k, v = views(dev(qkv), Hq, Hkv)
    out = sa.slim_qk_norm_rope(q, k, v, torch.from_numpy(table).cuda(), torch.from_numpy(positions).cuda(), *on_device((qw, kw)),
                               1e-6, interleaved)
    hq, hk, hv = views(qkv, Hq, Hkv)
    same_bits(out[0], rotated(hq, qw, table, positions, 1e-6, interleaved), "q")
    same_bits(out[1], rotated(hk, kw, table, positions, 1e-6, interleaved), "k")
    same_bits(out[2], hv.transpose(0, 2, 1, 3), "v")


@gpu
@pytest.mark.parametrize("B,S,Hq,Hkv,D", SHAPES)
@pytest.mark.parametrize("interleaved", [False, True])
def test_append_writes_the_quantisers_codes(sa, oracle, B, S, Hq, Hkv, D, interleaved):
    print("norm, rotation and append", B, S, Hq, Hkv, D, interleaved, flush=True)
    rng = np.random.default_rng(B + S * Hq)
    length, T = 5000, S + 13
    qkv, (qw, kw), positions = case(rng, B, S, Hq, Hkv, D, length)
    if S > 3:
        positions[0, S // 2:] = -1                # padding
        positions[-1, 1] = length                 # past the table
    slots = rng.integers(0, 14, B).astype(np.int32)
    if B > 2:
        slots[1], slots[2] = -1, T - 1            # before the cache; the last place, and past it
    table = table_of(length, D)
    q, k, v = views(dev(qkv), Hq, Hkv)
    cache = [torch.full((B, Hkv, T, D), 7, dtype=I8, device="cuda"), torch.full((B, Hkv, T), -3.0, device="cuda"),
             torch.full((B, Hkv, T, D), 9, dtype=I8, device="cuda"), torch.full((B, Hkv, T), -5.0, device="cuda")]
    out = sa.slim_qk_norm_rope_append_int8(q, k, v, torch.from_numpy(table).cuda(), torch.from_numpy(positions).cuda(),
                                           torch.from_numpy(slots).cuda(), *cache, *on_device((qw, kw)), 1e-6, interleaved)
    hq, hk, hv = views(qkv, Hq, Hkv)
    same_bits(out, rotated(hq, qw, table, positions, 1e-6, interleaved), "q")
    new = (*oracle.kv_quant_int8(np.ascontiguousarray(rotated(hk, kw, table, positions, 1e-6, interleaved))),
           *oracle.kv_quant_int8(np.ascontiguousarray(hv.transpose(0, 2, 1, 3))))
    want = [np.full((B, Hkv, T, D), 7, np.int8), np.full((B, Hkv, T), -3.0, np.float32), np.full((B, Hkv, T, D), 9, np.int8),
            np.full((B, Hkv, T), -5.0, np.float32)]
    for b in range(B):
        for s in range(S):
            if 0 <= positions[b, s] < length and 0 <= slots[b] + s < T:
                for w, n in zip(want, new):
                    w[b, :, slots[b] + s] = n[b, :, s]
    for got, w, what in zip(cache, want, ("k codes", "k scales", "v codes", "v scales")):
        assert np.array_equal(got.cpu().numpy(), w), what


@gpu
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("interleaved", [False, True])
def test_rows_of_extreme_values(sa, D, interleaved):
    """Zero rows, one value among zeros, the smallest and the largest numbers, a large eps, far positions."""
    rng = np.random.default_rng(5)
    B, S, H, length = 1, 24, 3, 70000
    qkv, (qw, kw), positions = case(rng, B, S, H, H, D, length)
    positions[0, :4] = (0, 1, length - 1, length - 2)
    x = bf16_bits_to_f32(qkv)
    x[0, 1] = 0.0
    x[0, 2] = 0.0
    x[0, 2, :, 5] = 3.0
    x[0, 3] *= np.float32(2.0 ** -120)
    x[0, 4] *= np.float32(2.0 ** -133)                        # subnormal in bf16
    x[0, 5] = np.where(x[0, 5] > 0, np.float32(3.38e38), np.float32(-3.38e38))
    x[0, 6] *= np.float32(2.0 ** 60)
    qkv = f32_to_bf16_bits(x)
    table = table_of(length, D)
    args = [torch.from_numpy(table).cuda(), torch.from_numpy(positions).cuda(), *on_device((qw, kw))]
    hq, hk, hv = views(qkv, H, H)
    for eps in (1e-6, 1e-300, 0.5, 1e30):
        out = sa.slim_qk_norm_rope(*views(dev(qkv), H, H), *args, eps, interleaved)
        same_bits(out[0], rotated(hq, qw, table, positions, eps, interleaved), "q, eps %g" % eps)
        same_bits(out[1], rotated(hk, kw, table, positions, eps, interleaved), "k, eps %g" % eps)


@gpu
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("norm", [True, False])
def test_rows_that_are_not_finite(sa, oracle, D, interleaved, norm):
    """A row with an infinity has the mean square infinity: its values become zeros, the pair that holds the infinity NaN; without a norm,
    and with a NaN, the formula's values too.  The other rows, and their codes, are as ever."""
    rng = np.random.default_rng(D)
    B, S, H, length, T = 2, 9, 5, 40, 12
    qkv, (qw, kw), positions = case(rng, B, S, H, H, D, length, norm)
    positions[0, 0] = 0                                       # (cosines of one, sines of zero)
    positions[1, 8] = -1                                      # padding, an infinity in it or not
    x = bf16_bits_to_f32(qkv)
    bad = np.zeros((B, S, 2 * H), bool)
    for b, s, h, d, v in ((0, 0, 1, 3, np.inf), (0, 1, 6, D - 1, -np.inf), (0, 2, 2, 0, np.nan), (1, 3, 9, D // 2, np.inf), (1, 8, 0, 1, np.inf),
                          (1, 4, 4, 7, np.inf), (1, 4, 4, 8, -np.inf), (1, 5, 7, 2, np.nan)):
        x[b, s, h, d] = v
        bad[b, s, h] = True
    qkv = f32_to_bf16_bits(x)
    qkv[np.isnan(x)] = 0x7fc0
    table, slots = table_of(length, D), np.array([0, 3], np.int32)
    args = [torch.from_numpy(table).cuda(), torch.from_numpy(positions).cuda()]
    out = sa.slim_qk_norm_rope(*views(dev(qkv), H, H), *args, *on_device((qw, kw)), 1e-6, interleaved)
    cache = [torch.zeros((B, H, T, D), dtype=I8, device="cuda"), torch.zeros((B, H, T), device="cuda"),
             torch.zeros((B, H, T, D), dtype=I8, device="cuda"), torch.zeros((B, H, T), device="cuda")]
    q2 = sa.slim_qk_norm_rope_append_int8(*views(dev(qkv), H, H), *args, torch.from_numpy(slots).cuda(), *cache, *on_device((qw, kw)), 1e-6,
                                          interleaved)
    with np.errstate(invalid="ignore"):
        want = [rotated(h, w, table, positions, 1e-6, interleaved) for h, w in zip(views(qkv, H, H)[:2], (qw, kw))]
    for got, w, what in ((out[0], want[0], "q"), (out[1], want[1], "k"), (q2, want[0], "q, with the append")):
        g, w = bf16_bits_to_f32(host(got)), bf16_bits_to_f32(w)
        assert np.array_equal(np.isnan(g), np.isnan(w)), what
        assert np.array_equal(g[~np.isnan(w)], w[~np.isnan(w)]), what
    codes, scales = oracle.kv_quant_int8(np.ascontiguousarray(np.where(bad[:, :, H:].transpose(0, 2, 1)[..., None], 0, want[1]).astype(np.uint16)))
    for b in range(B):
        for s in range(S):
            if positions[b, s] >= 0:
                fine = ~bad[b, s, H:]
                assert np.array_equal(cache[0][b, :, slots[b] + s].cpu().numpy()[fine], codes[b, :, s][fine])
                assert np.array_equal(cache[1][b, :, slots[b] + s].cpu().numpy()[fine], scales[b, :, s][fine])


@gpu
def test_one_of_the_norms_and_tensors_of_their_own(sa):
    """Keys normed and queries not, and the other way round; q, k and v as tensors of their own, and as every other row of one."""
    rng = np.random.default_rng(6)
    B, S, Hq, Hkv, D, length = 2, 33, 7, 1, 128, 100
    qkv, (qw, kw), positions = case(rng, B, S, Hq, Hkv, D, length)
    table = table_of(length, D)
    rest = [torch.from_numpy(table).cuda(), torch.from_numpy(positions).cuda()]
    hq, hk, hv = views(qkv, Hq, Hkv)
    own = [dev(x) for x in (hq, hk, hv)]
    wide = torch.zeros((B, S, 2, Hq, D), dtype=BF16, device="cuda")
    wide[:, :, 1] = own[0]
    for q in (own[0], wide[:, :, 1]):
        for w in ((qw, None), (None, kw)):
            out = sa.slim_qk_norm_rope(q, own[1], own[2], *rest, *on_device(w), 1e-5)
            same_bits(out[0], rotated(hq, w[0], table, positions, 1e-5, False), "q")
            same_bits(out[1], rotated(hk, w[1], table, positions, 1e-5, False), "k")
            same_bits(out[2], hv.transpose(0, 2, 1, 3), "v")


@gpu
@pytest.mark.parametrize("interleaved", [False, True])
def test_position_zero_without_norm_changes_nothing(sa, interleaved):
    """More tokens than one grid holds, rows beyond 2^32 bytes: every one is moved as it is, those without a position are zero."""
    S, D = 33_500_000, 64
    qkv = torch.randint(-30000, 30000, (1, S, 3, D), dtype=torch.int16, device="cuda").remainder_(0x3f80).view(BF16)   # (finite)
    positions = torch.zeros((1, S), dtype=I32, device="cuda")
    positions[0, 12_345_678] = positions[0, S - 2] = -1
    table = torch.from_numpy(table_of(2, D)).cuda()
    out = sa.slim_qk_norm_rope(*views(qkv, 1, 1), table, positions, interleaved=interleaved)
    torch.cuda.synchronize()
    qkv[0, 12_345_678] = 0
    qkv[0, S - 2] = 0
    for i in range(3):
        got, want = out[i].view(torch.int16)[0, 0], qkv.view(torch.int16)[0, :, i]
        for lo in range(0, S, 1 << 22):
            assert torch.equal(got[lo:lo + (1 << 22)], want[lo:lo + (1 << 22)]), (i, lo)


@gpu
def test_the_librarys_table(sa):
    for D in (64, 128):
        t = sa.slim_rope_table(3001, D, 500000.0)
        assert t.shape == (3001, D) and t.dtype == F32
        # (two 64-bit routes to one angle, rounded to fp32: half a step of a value of at most 1, and the 64-bit error of angles to 3001)
        assert np.abs(t.cpu().numpy() - table_of(3001, D, 500000.0)).max() <= 2.0 ** -24


@gpu
def test_captured_calls_on_a_stream_of_their_own(sa):
    """Both calls in a graph on another stream, replayed with new inputs in the same place, eager work between the replays."""
    rng = np.random.default_rng(8)
    B, S, Hq, Hkv, D, length, T = 3, 4, 8, 2, 128, 64, 20
    qkv, weights, positions = case(rng, B, S, Hq, Hkv, D, length)
    x, w = dev(qkv), on_device(weights)
    table, pos = torch.from_numpy(table_of(length, D)).cuda(), torch.from_numpy(positions).cuda()
    slots = torch.tensor([0, 5, T - 2], dtype=I32, device="cuda")

    def fresh():
        return [torch.zeros((B, Hkv, T, D), dtype=I8, device="cuda"), torch.zeros((B, Hkv, T), device="cuda"),
                torch.zeros((B, Hkv, T, D), dtype=I8, device="cuda"), torch.zeros((B, Hkv, T), device="cuda")]

    outs = [torch.empty((B, h, S, D), dtype=BF16, device="cuda") for h in (Hq, Hkv, Hkv)]
    q_out, cache = torch.empty_like(outs[0]), fresh()

    def step(outs, q_out, cache):
        sa.slim_qk_norm_rope(*views(x, Hq, Hkv), table, pos, *w, q_out=outs[0], k_out=outs[1], v_out=outs[2])
        sa.slim_qk_norm_rope_append_int8(*views(x, Hq, Hkv), table, pos, slots, *cache, *w, q_out=q_out)

    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(stream):
        step(outs, q_out, cache)
        stream.synchronize()
        with torch.cuda.graph(graph, stream=stream):
            step(outs, q_out, cache)
    for rep in range(4):
        x.copy_(dev(normal_bf16(rng, qkv.shape)))
        slots.copy_(torch.tensor([rep, 5 + rep, T - 2 - rep], dtype=I32))
        for c in cache:
            c.zero_()
        want = [torch.empty_like(t) for t in outs], torch.empty_like(q_out), fresh()
        step(*want)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for got, ref in zip((*outs, q_out, *cache), (*want[0], want[1], *want[2])):
            assert torch.equal(got, ref), "replay %d" % rep


@gpu
def test_a_prompt_through_the_cache_and_the_attention(sa, oracle):
    """Prompt: rows into the INT8 cache, prefill over it; the same by way of bf16 K and V and the emitting prefill; then steps."""
    rng = np.random.default_rng(9)
    B, S, steps, Hq, Hkv, D = 2, 150, 3, 8, 2, 128
    T, scale = S + steps, 1 / math.sqrt(D)
    qkv, (qw, kw), _ = case(rng, B, T, Hq, Hkv, D, 1)
    positions = np.broadcast_to(np.arange(T, dtype=np.int32), (B, T)).copy()
    table = table_of(T, D)
    x, w, pos = dev(qkv), on_device((qw, kw)), torch.from_numpy(positions).cuda()
    t = torch.from_numpy(table).cuda()
    zero = torch.zeros(B, dtype=I32, device="cuda")

    def cache(n):
        return [torch.zeros((B, Hkv, n, D), dtype=I8, device="cuda"), torch.zeros((B, Hkv, n), device="cuda"),
                torch.zeros((B, Hkv, n, D), dtype=I8, device="cuda"), torch.zeros((B, Hkv, n), device="cuda")]

    prompt = cache(S)
    p = views(x[:, :S].contiguous(), Hq, Hkv)
    q = sa.slim_qk_norm_rope_append_int8(*p, t, pos[:, :S].contiguous(), zero, *prompt, *w)
    out = sa.slim_attn_prefill(q, prompt[0], prompt[2], scale, True, k_scale=prompt[1], v_scale=prompt[3])
    rows = sa.slim_qk_norm_rope(*p, t, pos[:, :S].contiguous(), *w)
    emitted = sa.slim_attn_prefill_emit_int8(*rows, scale, True)
    for a, b in zip(prompt, emitted[1:]):
        assert torch.equal(a, b)
    hq, hk, hv = views(qkv, Hq, Hkv)
    wq = np.ascontiguousarray(rotated(hq, qw, table, positions, 1e-6, False))
    kc, ks = oracle.kv_quant_int8(np.ascontiguousarray(rotated(hk, kw, table, positions, 1e-6, False)))
    vc, vs = oracle.kv_quant_int8(np.ascontiguousarray(hv.transpose(0, 2, 1, 3)))
    want = oracle.attn(wq, kc, vc, scale, True, k_scale=ks, v_scale=vs)
    assert np.abs(out.double().cpu().numpy() - want[:, :, :S]).max() <= 2e-2
    grown = cache(T)
    for g, c in zip(grown, prompt):
        g[:, :, :S] = c
    for i in range(S, T):
        at = torch.full((B,), i, dtype=I32, device="cuda")
        q = sa.slim_qk_norm_rope_append_int8(*views(x[:, i:i + 1], Hq, Hkv), t, pos[:, i:i + 1].contiguous(), at, *grown, *w)
        got = sa.slim_attn_decode_int8_varlen(q, *grown, at + 1, scale)
        assert np.abs(got.double().cpu().numpy()[:, :, 0] - want[:, :, i]).max() <= 2e-2, i
    for g, c in zip(grown, (kc, ks, vc, vs)):
        assert np.array_equal(g.cpu().numpy(), c)


# ------------------------------------------------------------------ refusals (CPU)

P, A = ctypes.c_void_p, 0x100000   # (an address that is never dereferenced)


def rows_call(sa, q=A, k=2 * A, v=3 * A, sq=1024, sk=1024, sv=1024, qw=4 * A, kw=5 * A, table=6 * A, pos=7 * A, qo=8 * A, ko=9 * A,
              vo=10 * A, B=2, Hq=4, Hkv=2, S=10, D=128, L=64, pairs=0, eps=1e-6):
    return sa.load().slim_qk_norm_rope(P(q), P(k), P(v), sq, sk, sv, P(qw), P(kw), P(table), P(pos), P(qo), P(ko), P(vo), B, Hq, Hkv, S,
                                       D, L, pairs, eps, None)


def append_call(sa, slots=8 * A, qo=9 * A, kc=10 * A, ks=11 * A, vc=12 * A, vs=13 * A, T=50, S=10, eps=1e-6, pairs=0, L=64, pos=7 * A):
    return sa.load().slim_qk_norm_rope_append_int8(P(A), P(2 * A), P(3 * A), 1024, 1024, 1024, P(None), P(None), P(6 * A), P(pos),
                                                   P(slots), P(qo), P(kc), P(ks), P(vc), P(vs), 2, 4, 2, S, T, 128, L, pairs, eps, None)


def test_rows_refusals(sa):
    NULL, SHAPE, UNSUP, ALIGN, OVERLAP = 1, 2, 3, 4, 7
    for name in ("q", "k", "v", "table", "pos", "qo", "ko", "vo"):
        assert rows_call(sa, **{name: None}) == NULL, name
    assert rows_call(sa, S=0) == SHAPE and rows_call(sa, B=0) == SHAPE and rows_call(sa, Hq=3) == SHAPE and rows_call(sa, L=0) == SHAPE
    assert rows_call(sa, eps=0.0) == SHAPE and rows_call(sa, eps=math.nan) == SHAPE and rows_call(sa, eps=math.inf) == SHAPE
    assert rows_call(sa, pairs=2) == SHAPE and rows_call(sa, D=96) == UNSUP
    assert rows_call(sa, sq=504) == SHAPE and rows_call(sa, sk=248) == SHAPE and rows_call(sa, sv=1 << 31) == SHAPE
    assert rows_call(sa, sq=1028) == ALIGN and rows_call(sa, sv=1025) == ALIGN
    assert rows_call(sa, q=A + 8) == ALIGN and rows_call(sa, kw=5 * A + 2) == ALIGN and rows_call(sa, table=6 * A + 4) == ALIGN
    assert rows_call(sa, vo=10 * A + 8) == ALIGN and rows_call(sa, pos=7 * A + 2) == ALIGN
    assert rows_call(sa, qo=A) == OVERLAP and rows_call(sa, ko=8 * A + 2 * 4 * 10 * 128 * 2 - 16) == OVERLAP
    assert rows_call(sa, vo=7 * A) == OVERLAP and rows_call(sa, qo=6 * A + 64 * 128 * 4 - 16) == OVERLAP
    assert rows_call(sa, k=A + 1024, ko=A) == OVERLAP
    assert "overlap" in sa.status_string(OVERLAP)


def test_append_refusals(sa):
    NULL, SHAPE, ALIGN, OVERLAP = 1, 2, 4, 7
    for name in ("slots", "qo", "kc", "ks", "vc", "vs", "pos"):
        assert append_call(sa, **{name: None}) == NULL, name
    assert append_call(sa, T=0) == SHAPE and append_call(sa, S=-1) == SHAPE and append_call(sa, eps=-1.0) == SHAPE
    assert append_call(sa, L=-5) == SHAPE and append_call(sa, pairs=-1) == SHAPE
    assert append_call(sa, kc=10 * A + 8) == ALIGN and append_call(sa, vs=13 * A + 4) == ALIGN and append_call(sa, slots=8 * A + 1) == ALIGN
    assert append_call(sa, vc=10 * A) == OVERLAP and append_call(sa, ks=10 * A + 2 * 2 * 50 * 128 - 16) == OVERLAP
    assert append_call(sa, qo=2 * A) == OVERLAP and append_call(sa, vs=8 * A) == OVERLAP


def z(*shape, dtype=BF16):
    return torch.zeros(shape, dtype=dtype)


def test_binding_refusals(sa):
    B, S, Hq, Hkv, D, T = 2, 6, 4, 2, 64, 9
    good = dict(q=z(B, S, Hq, D), k=z(B, S, Hkv, D), v=z(B, S, Hkv, D), cos_sin=z(10, D, dtype=F32), positions=z(B, S, dtype=I32))
    cache = dict(slots=z(B, dtype=I32), k_codes=z(B, Hkv, T, D, dtype=I8), k_scale=z(B, Hkv, T, dtype=F32),
                 v_codes=z(B, Hkv, T, D, dtype=I8), v_scale=z(B, Hkv, T, dtype=F32))

    def refused(text, kind=AssertionError, **other):
        for f, args in ((sa.slim_qk_norm_rope, good), (sa.slim_qk_norm_rope_append_int8, dict(good, **cache))):
            if all(n in args or n in ("q_weight", "k_weight", "q_out") for n in other):
                with pytest.raises(kind, match=text):
                    f(**dict(args, **other))

    refused("device tensors")                                   # (all shapes are fine)
    refused("same tokens", k=z(B, S + 1, Hkv, D), v=z(B, S + 1, Hkv, D))
    refused("one shape", v=z(B, S, Hkv + 1, D))
    refused("four dimensions", ValueError, q=z(S, Hq, D))
    refused("cos_sin", cos_sin=z(10, D // 2, dtype=F32))
    refused("position", positions=z(B * S, dtype=I32))
    refused("weight", q_weight=z(D + 8))
    refused("weight", k_weight=z(1, D))
    refused("one stride", q=z(B, Hq, S, D).transpose(1, 2))
    refused("one stride", k=z(B, S, Hkv, 2 * D)[..., ::2])
    refused("one stride", q=z(B, S + 1, Hq, D)[:, :S])
    refused("slot", slots=z(B + 1, dtype=I32))
    refused("shape of k_codes", k_codes=z(B, Hkv + 1, T, D, dtype=I8))
    refused("v_codes", v_codes=z(B, Hkv, T + 1, D, dtype=I8))
    refused("k_scale", k_scale=z(B, Hkv, T + 1, dtype=F32))
    refused("v_scale", v_scale=z(B, Hkv, dtype=F32))
    refused("torch tensor", TypeError, q=None)
