"""Rows whose scores are all far below zero: -2^107 and so below -1e30, where each attention call still weighs what a row sees, and that only.

All scores of a row are the same here, and each product and sum of one is exact in fp32: -2^97 times 64, the sum over 64 or 128 values and a
scale of 1 are powers of two, and the softmax scale times log2(e) is then rounded once, for all of them alike.  (So it has to be: a score of
2^107 that is rounded is off by up to 2^83, in an exponent.  Codes of 127 with the scale 64 / 127, the quantiser's for rows of 64, make a
product of 31 bits, which a fused multiply-add and a product of its own give differently.)  A result is the mean of the values that the row
sees.  Tolerance, element by element, that of tests/test_decode_prefix.py: one rounding of the probabilities (times v_scale) to bf16
and one of the result, 2^-8 each, and 2^-14 of the sum for what is done in fp32.
"""
import os

import pytest
import torch

BF16, F32, I8, I32 = torch.bfloat16, torch.float32, torch.int8, torch.int32
pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def sa():
    from paper_2407_07304_amd import build, slimattn
    if not (os.path.exists(slimattn.LIB_PATH) and os.path.exists(slimattn.BINDING_PATH)):
        build.build()
    slimattn.load()
    return slimattn


def held(got, want, weighed, what):
    """weighed: sum_t p_t |v^_t|"""
    bound = (2.0 ** -8 + 2.0 ** -14) * weighed + 2.0 ** -8 * (1 + 2.0 ** -8) * want.abs()
    assert torch.isfinite(got).all() and ((got.double() - want).abs() <= bound).all(), what


def low_queries(*shape):
    return torch.full(shape, -(2.0 ** 97), dtype=BF16, device="cuda")


# one, 2 to 32 and more query heads a KV head; lengths inside a tile, waves without tokens, several splits
@pytest.mark.parametrize("B,Hq,Hkv,T", [(1, 8, 8, 333), (3, 4, 4, 40), (1, 2, 2, 9000), (2, 8, 2, 333), (2, 20, 1, 70), (1, 64, 8, 5000), (1, 40, 1, 5)])
@pytest.mark.parametrize("D", [64, 128])
def test_decodes_of_very_low_scores(sa, B, Hq, Hkv, T, D):
    print("low scores", B, Hq, Hkv, T, D, flush=True)
    gen = torch.Generator(device="cuda").manual_seed(T + D)
    kc, ks = torch.full((B, Hkv, T, D), 64, dtype=I8, device="cuda"), torch.ones((B, Hkv, T), device="cuda")
    vc = torch.randint(-127, 128, (B, Hkv, T, D), generator=gen, device="cuda", dtype=I8)
    vs = torch.full((B, Hkv, T), 0.01, device="cuda")
    q, v = low_queries(B, Hq, 1, D), vc.double() * float(vs[0, 0, 0])
    lens = torch.randint(1, T + 1, (B,), generator=gen, device="cuda", dtype=I32)
    lens[0] = T - 1

    def means(n):
        rows = [(v[b, :, :n[b]].mean(1), v[b, :, :n[b]].abs().mean(1)) for b in range(B)]
        return (torch.stack(x).repeat_interleave(Hq // Hkv, 1)[:, :, None] for x in zip(*rows))

    want, weighed = means([T] * B)
    held(sa.slim_attn_decode_int8(q, kc, ks, vc, vs, 0.125), want, weighed, "equal lengths")
    held(sa.slim_attn_decode_int8_static(q, kc, ks, vc, vs, 0.125, torch.empty_like(q)), want, weighed, "without a workspace")
    want, weighed = means(lens.tolist())
    held(sa.slim_attn_decode_int8_varlen(q, kc, ks, vc, vs, lens, 0.125), want, weighed, "lengths of their own")
    held(sa.slim_attn_decode_int8_weights(q, kc, ks, vc, vs, lens, 0.125)[0], want, weighed, "with weights")


# row blocks of 32, 128 and 256 rows
@pytest.mark.parametrize("B,Hq,Hkv,S,D", [(1, 4, 2, 50, 64), (2, 8, 8, 700, 128), (1, 32, 32, 2048, 128), (4, 32, 8, 2100, 64), (4, 32, 8, 2100, 128)])
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("codes", [False, True])
def test_prefills_of_very_low_scores(sa, B, Hq, Hkv, S, D, causal, codes):
    print("low scores", B, Hq, Hkv, S, D, causal, codes, flush=True)
    gen = torch.Generator(device="cuda").manual_seed(S + D)
    q, k = low_queries(B, Hq, S, D), torch.full((B, Hkv, S, D), 64.0, dtype=BF16, device="cuda")
    v = torch.randn((B, Hkv, S, D), generator=gen, device="cuda").to(BF16)
    scales = {}
    x = v.double()
    if codes:
        k, ks, (v, vs) = k.to(I8), torch.ones((B, Hkv, S), device="cuda"), sa.kv_quant_int8(v)
        scales, x = {"k_scale": ks, "v_scale": vs}, v.double() * vs.double()[..., None]
    seen = torch.arange(1, S + 1, device="cuda", dtype=torch.float64)[:, None]
    want, weighed = ((t.cumsum(2) / seen if causal else t.mean(2, keepdim=True).expand_as(t)).repeat_interleave(Hq // Hkv, 1) for t in (x, x.abs()))
    for dtype in (BF16, F32):
        held(sa.slim_attn_prefill(q, k, v, 0.125, causal, out_dtype=dtype, **scales), want, weighed, dtype)
    if not codes:
        held(sa.slim_attn_prefill_emit_int8(q, k, v, 0.125, causal)[0], want, weighed, "with the cache")
        held(sa.slim_attn_prefill_strip(q, k, v, 0.125, causal), want, weighed, "strip")
        held(sa.slim_attn_prefill_two_sweep(q, k, v, 0.125, causal), want, weighed, "two sweeps")
