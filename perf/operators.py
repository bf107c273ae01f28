"""What a serving loop does around the attention calls, as cases that can be timed and compared.

A case is one of five kinds:

  rotate   norms of queries and keys for each head and the rotation by position, from the projection's rows to the layout
           that the prefill reads (``slim_qk_norm_rope``)
  append   the same for new tokens whose K and V go into the INT8 cache (``slim_qk_norm_rope_append_int8``)
  prefix   one decode step of a batch whose sequences share a long prefix and have a cache each for what follows it
           (``slim_attn_decode_int8_shared_prefix``)
  weights  one decode step that also adds up the attention weight of every cached token (``slim_attn_decode_int8_weights``)
  evict    the tokens of largest weight and the most recent ones go to another cache, in order (``slim_cache_evict_int8``)

Where ``own`` is false, ``run`` computes them with elementary torch operations.  The codes of the cache are whole numbers
next to a border, so ``rotate`` and ``append`` are computed in 64 bits there, the attention in 32.
``exact`` is the operators' definition in 64 bits.
"""
import math

import torch

own = False

EPS = 1e-6
BASE = 10000.0


# ------------------------------------------------------------------ cases

def _rotate(name, batch, q_heads, kv_heads, seq_len, head_dim=128, interleaved=False):
    return {"name": name, "kind": "rotate", "batch": batch, "q_heads": q_heads, "kv_heads": kv_heads, "seq_len": seq_len,
            "head_dim": head_dim, "interleaved": interleaved}


def _append(name, batch, q_heads, kv_heads, seq_len, kv_len, head_dim=128, interleaved=False):
    return {"name": name, "kind": "append", "batch": batch, "q_heads": q_heads, "kv_heads": kv_heads, "seq_len": seq_len,
            "kv_len": kv_len, "head_dim": head_dim, "interleaved": interleaved}


def _prefix(name, batch, q_heads, kv_heads, prefix_len, kv_len, head_dim=128):
    return {"name": name, "kind": "prefix", "batch": batch, "q_heads": q_heads, "kv_heads": kv_heads,
            "prefix_len": prefix_len, "kv_len": kv_len, "head_dim": head_dim}


def _weights(name, batch, q_heads, kv_heads, kv_len, head_dim=128):
    return {"name": name, "kind": "weights", "batch": batch, "q_heads": q_heads, "kv_heads": kv_heads, "kv_len": kv_len,
            "head_dim": head_dim}


def _evict(name, batch, kv_heads, kv_len, keep, recent, head_dim=128):
    return {"name": name, "kind": "evict", "batch": batch, "kv_heads": kv_heads, "kv_len": kv_len, "keep": keep,
            "recent": recent, "head_dim": head_dim}


def listed():
    return [
        # a prompt of the headline configuration between its projection and its attention
        _rotate("rotate_2k", 1, 32, 32, 2048),
        # a batch of prompts of an odd length, grouped heads, pairs next to each other
        _rotate("rotate_batch_pairs", 4, 32, 8, 777, head_dim=64, interleaved=True),
        # one user's new token: the latency of a launch
        _append("append_one_user", 1, 64, 8, 1, 1000),
        # a serving batch's new tokens, each sequence at a place of its own
        _append("append_batch", 48, 32, 8, 1, 3001),
        # prompts of different lengths, padded, into the cache in one go
        _append("append_prompts", 8, 32, 8, 1000, 1200),
        # a few users behind a short instruction: little of anything
        _prefix("prefix_few_users", 4, 32, 8, 1000, 64),
        # a serving batch behind a long instruction, conversations of different lengths
        _prefix("prefix_batch", 48, 32, 8, 8192, 1000),
        # many questions about one long document: the largest
        _prefix("prefix_long_document", 64, 64, 8, 32768, 300),
        # one user, a head for each query head, short cache
        _weights("weights_one_user", 1, 32, 32, 1000),
        # the benchmark's grouped-query decode, lengths of their own
        _weights("weights_batch", 16, 64, 8, 8192),
        # one user's long document cut down to an eighth
        _evict("evict_long_document", 1, 8, 32768, 4096, 512),
        # a batch's caches cut down by a half
        _evict("evict_batch", 16, 8, 8192, 4096, 100),
    ]


_HEADS = ((8, 8), (32, 32), (32, 8), (64, 8), (16, 2), (4, 4))
_MOST_ROWS = 4 << 20          # rows of q, k and v of a drawn rotation or append
_MOST_CACHE = 128 << 20       # bytes of K codes of a drawn case's caches
_MOST_FLOPS = 6.0e10          # of a drawn prefix case: below the largest listed one


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(("rotate", "append", "append", "prefix", "prefix", "weights", "weights", "evict"))
    head_dim = rng.choice((64, 128, 128))
    q_heads, kv_heads = rng.choice(_HEADS)
    interleaved = rng.random() < 0.3
    while True:
        if kind == "rotate":
            c = _rotate("", _log_int(rng, 1, 16), q_heads, kv_heads, _log_int(rng, 1, 8192), head_dim, interleaved)
            if c["batch"] * c["seq_len"] * (q_heads + 2 * kv_heads) <= _MOST_ROWS // 8:
                break
        elif kind == "append":
            seq_len = 1 if rng.random() < 0.5 else _log_int(rng, 2, 2048)
            c = _append("", _log_int(rng, 1, 128), q_heads, kv_heads, seq_len, _log_int(rng, max(64, seq_len), 16384), head_dim,
                        interleaved)
            if (c["batch"] * seq_len * (q_heads + 2 * kv_heads) <= _MOST_ROWS // 8
                    and c["batch"] * kv_heads * c["kv_len"] * head_dim <= _MOST_CACHE):
                break
        elif kind == "prefix":
            c = _prefix("", _log_int(rng, 1, 128), q_heads, kv_heads, _log_int(rng, 64, 32768), _log_int(rng, 1, 4096), head_dim)
            if (work(c)["flops"] <= _MOST_FLOPS and c["batch"] * kv_heads * c["kv_len"] * head_dim <= _MOST_CACHE
                    and c["batch"] * q_heads * (c["prefix_len"] + c["kv_len"]) <= 150 << 20):
                break
        elif kind == "weights":
            c = _weights("", _log_int(rng, 1, 64), q_heads, kv_heads, _log_int(rng, 64, 32768), head_dim)
            if c["batch"] * kv_heads * c["kv_len"] * head_dim <= _MOST_CACHE:
                break
        else:
            kv_len = _log_int(rng, 64, 32768)
            keep = max(2, int(kv_len * rng.uniform(0.1, 0.9)))
            c = _evict("", _log_int(rng, 1, 64), kv_heads, kv_len, keep, int(keep * rng.uniform(0.0, 0.5)), head_dim)
            if c["batch"] * kv_heads * kv_len * head_dim <= _MOST_CACHE:
                break
    del c["name"]
    return c


def _mean_len(kv_len):
    """The mean of the lengths that _lengths() draws."""
    return (kv_len + max(1, kv_len // 8)) / 2


def work(case):
    kind, b, hkv, d = case["kind"], case["batch"], case["kv_heads"], case["head_dim"]
    row = 2 * (d + 4)                       # a token's K and V codes and scales
    if kind in ("rotate", "append"):
        n, hq, s = b * case["seq_len"], case["q_heads"], case["seq_len"]
        read = 2 * n * (hq + 2 * hkv) * d + 4 * s * d + 4 * n
        written = 2 * n * (hq + 2 * hkv) * d if kind == "rotate" else n * (2 * hq * d + hkv * row)
        return {"bytes": read + written, "flops": n * (hq + hkv) * d * 7 + (0 if kind == "rotate" else 6 * n * hkv * d)}
    if kind == "prefix":
        hq, p, t = case["q_heads"], case["prefix_len"], _mean_len(case["kv_len"])
        return {"bytes": hkv * (p + b * t) * row + 4 * b * hq * d, "flops": 4 * hq * d * b * (p + t)}
    if kind == "weights":
        hq, t = case["q_heads"], _mean_len(case["kv_len"])
        return {"bytes": b * hkv * (t * (row + 4) + 4 * case["kv_len"]) + 4 * b * hq * d, "flops": 4 * b * hq * t * d}
    return {"bytes": b * hkv * (4 * case["kv_len"] + case["keep"] * (2 * (row + 4) + 4)), "flops": 2 * b * hkv * case["kv_len"]}


# ------------------------------------------------------------------ inputs

def _generator(seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    return gen


def _normal(gen, *shape, dtype=torch.bfloat16):
    return torch.randn(shape, generator=gen, device="cuda", dtype=dtype)


def _cache(gen, *shape):
    """INT8 codes and fp32 scales of normally distributed rows."""
    codes = torch.empty(shape, device="cuda", dtype=torch.int8)
    scales = torch.empty(shape[:-1], device="cuda")
    for i in range(shape[0]):
        x = _normal(gen, *shape[1:], dtype=torch.float32)
        scales[i] = x.abs().amax(-1) / 127
        codes[i] = (x / scales[i][..., None]).round()
    return codes, scales


def _lengths(gen, batch, kv_len):
    """Sequences that have got somewhere between an eighth of their cache and all of it."""
    return torch.randint(max(1, kv_len // 8), kv_len + 1, (batch,), generator=gen, device="cuda", dtype=torch.int32)


def _table(length, head_dim):
    """cos, then sin, of position times the pairs' frequencies: fp32 [length, head_dim]."""
    inv = BASE ** (-torch.arange(0, head_dim, 2, device="cuda", dtype=torch.float64) / head_dim)
    angle = torch.arange(length, device="cuda", dtype=torch.float64)[:, None] * inv
    return torch.cat([angle.cos(), angle.sin()], 1).float()


def prepare(case, seed):
    gen = _generator(seed)
    kind, b, hkv, d = case["kind"], case["batch"], case["kv_heads"], case["head_dim"]
    st = {"case": dict(case), "scale": 1.0 / math.sqrt(d)}
    if own:
        from paper_2407_07304_amd import slimattn as sa
        st["sa"] = sa
    if kind in ("rotate", "append"):
        s, hq = case["seq_len"], case["q_heads"]
        # one projection's output: a token's queries, keys and values next to each other
        qkv = _normal(gen, b, s, hq + 2 * hkv, d)
        st["q"], st["k"], st["v"] = qkv[:, :, :hq], qkv[:, :, hq:hq + hkv], qkv[:, :, hq + hkv:]
        st["q_weight"], st["k_weight"] = 1 + 0.25 * _normal(gen, d), 1 + 0.25 * _normal(gen, d)
        if kind == "rotate":
            st["table"] = _table(s, d)
            st["positions"] = torch.arange(s, device="cuda", dtype=torch.int32).expand(b, s).contiguous()
        else:
            t = case["kv_len"]
            st["table"] = _table(t, d)
            # the new tokens follow what is cached; of prompts, each of a length of its own, the padding has no position
            first = torch.randint(0, t - s + 1, (b,), generator=gen, device="cuda", dtype=torch.int32)
            count = _lengths(gen, b, s)[:, None]
            i = torch.arange(s, device="cuda", dtype=torch.int32)
            st["positions"] = torch.where(i < count, first[:, None] + i, -1).contiguous()
            st["slots"] = first
            st["k_codes"], st["k_scale"] = _cache(gen, b, hkv, t, d)
            st["v_codes"], st["v_scale"] = _cache(gen, b, hkv, t, d)
    elif kind == "prefix":
        hq, p, t = case["q_heads"], case["prefix_len"], case["kv_len"]
        st["prefix"] = _cache(gen, 1, hkv, p, d) + _cache(gen, 1, hkv, p, d)
        st["cache"] = _cache(gen, b, hkv, t, d) + _cache(gen, b, hkv, t, d)
        st["q"], st["lens"] = _normal(gen, b, hq, 1, d), _lengths(gen, b, t)
        # what a serving loop keeps from step to step
        st["out"] = torch.empty_like(st["q"])
        if own:
            n = sa.slim_attn_decode_int8_shared_prefix_workspace_bytes(b, hq, hkv, p, t, d)
            st["workspace"] = torch.empty(n, dtype=torch.uint8, device="cuda")
    elif kind == "weights":
        hq, t = case["q_heads"], case["kv_len"]
        st["cache"] = _cache(gen, b, hkv, t, d) + _cache(gen, b, hkv, t, d)
        st["q"], st["lens"] = _normal(gen, b, hq, 1, d), _lengths(gen, b, t)
        # the sums of some hundred steps; a token that has none yet comes in with a zero
        seen = torch.arange(t, device="cuda") < st["lens"][:, None, None]
        st["sums"] = torch.where(seen, (2 * _normal(gen, b, hkv, t, dtype=torch.float32)).exp() * (100 * hq / hkv / t), 0.0)
        st["out"], st["new_sums"] = torch.empty_like(st["q"]), torch.zeros_like(st["sums"])
        if own:
            n = sa.slim_attn_decode_int8_weights_workspace_bytes(b, hq, hkv, t, d)
            st["workspace"] = torch.empty(n, dtype=torch.uint8, device="cuda")
    else:
        t = case["kv_len"]
        st["cache"] = _cache(gen, b, hkv, t, d) + _cache(gen, b, hkv, t, d)
        # most caches are full when they are cut down; a tenth of the tokens never got any weight
        st["lens"] = torch.where(torch.rand(b, generator=gen, device="cuda") < 0.75, t, _lengths(gen, b, t)).int()
        weights = (2 * _normal(gen, b, hkv, t, dtype=torch.float32)).exp()
        st["weights"] = torch.where(torch.rand(b, hkv, t, generator=gen, device="cuda") < 0.1, 0.0, weights)
        # the other cache, as it was left
        st["to"] = [torch.zeros_like(x) for x in st["cache"]] + [torch.zeros_like(st["weights"])]
        st["kept"] = torch.empty((b, hkv, case["keep"]), dtype=torch.int32, device="cuda")
        st["new_lens"] = torch.empty_like(st["lens"])
    return st


# ------------------------------------------------------------------ one pass

def run(state):
    return {"rotate": _run_rotate, "append": _run_append, "prefix": _run_prefix, "weights": _run_weights,
            "evict": _run_evict}[state["case"]["kind"]](state)


def _rotated(x, weight, table, positions, interleaved):
    """Rows [B,S,H,D] bf16 -> [B,H,S,D] bf16; a row without a position is zero."""
    x, half = x.double(), x.shape[-1] // 2
    if weight is not None:
        x = x * (x.square().mean(-1, keepdim=True) + EPS).rsqrt() * weight.double()
    good = (positions >= 0) & (positions < table.shape[0])
    rows = table.double()[positions.clamp(0, table.shape[0] - 1).long()][:, :, None]
    c, s = rows[..., :half], rows[..., half:]
    if interleaved:
        a, b = x[..., 0::2], x[..., 1::2]
        y = torch.stack([a * c - b * s, b * c + a * s], -1).flatten(-2)
    else:
        a, b = x[..., :half], x[..., half:]
        y = torch.cat([a * c - b * s, b * c + a * s], -1)
    y = y.float().bfloat16() * good[:, :, None, None]
    return y.transpose(1, 2).contiguous()


def _run_rotate(st):
    pairs = st["case"]["interleaved"]
    if own:
        q, k, v = st["sa"].slim_qk_norm_rope(st["q"], st["k"], st["v"], st["table"], st["positions"], st["q_weight"],
                                             st["k_weight"], EPS, pairs)
    else:
        q = _rotated(st["q"], st["q_weight"], st["table"], st["positions"], pairs)
        k = _rotated(st["k"], st["k_weight"], st["table"], st["positions"], pairs)
        v = st["v"].transpose(1, 2).contiguous()
    return {"q": q, "k": k, "v": v}


def _codes(x):
    """bf16 rows -> (codes, scales): each a quotient rounded to 32 bits once, then the code to a whole number."""
    x = x.float()
    scale = (x.abs().amax(-1).double() / 127).float()      # (in 32 bits torch multiplies by 1 / 127, which is rounded twice)
    return (x / torch.where(scale > 0, scale, 1.0)[..., None]).round().clamp(-127, 127).to(torch.int8), scale


def _run_append(st):
    pairs = st["case"]["interleaved"]
    kc, ks, vc, vs = st["k_codes"], st["k_scale"], st["v_codes"], st["v_scale"]
    if own:
        q = st["sa"].slim_qk_norm_rope_append_int8(st["q"], st["k"], st["v"], st["table"], st["positions"], st["slots"], kc, ks,
                                                   vc, vs, st["q_weight"], st["k_weight"], EPS, pairs)
    else:
        positions = st["positions"]
        q = _rotated(st["q"], st["q_weight"], st["table"], positions, pairs)
        new_k = _rotated(st["k"], st["k_weight"], st["table"], positions, pairs)
        new_v = st["v"].transpose(1, 2)
        at = (st["slots"][:, None] + torch.arange(positions.shape[1], device=positions.device))[:, None].expand(new_k.shape[:3])
        good = (positions >= 0)[:, None].expand(new_k.shape[:3])
        wide = at[..., None].expand(new_k.shape)
        for codes, scales, new in ((kc, ks, new_k), (vc, vs, new_v)):
            c, s = _codes(new)
            codes.scatter_(2, wide, torch.where(good[..., None], c, codes.gather(2, wide)))
            scales.scatter_(2, at, torch.where(good, s, scales.gather(2, at)))
    # (the codes are defined bit for bit: whole numbers that have to be equal)
    return {"q": q, "k_codes": kc, "k_scale": ks, "v_codes": vc, "v_scale": vs}


def _past(lens, kv_len):
    return torch.arange(kv_len, device=lens.device) >= lens[:, None, None, None]


def _grouped(q, kv_heads):
    """[B,Hq,1,D] bf16 -> [B,Hkv,G,D] fp32"""
    return q.float().view(q.shape[0], kv_heads, -1, q.shape[-1])


def _run_prefix(st):
    pkc, pks, pvc, pvs = st["prefix"]
    kc, ks, vc, vs = st["cache"]
    if own:
        return st["sa"].slim_attn_decode_int8_shared_prefix(st["q"], pkc, pks, pvc, pvs, kc, ks, vc, vs, st["lens"], st["scale"],
                                                            out=st["out"], workspace=st["workspace"])
    b, hkv, t, d = kc.shape
    q = _grouped(st["q"], hkv) * st["scale"]
    rows = q.transpose(0, 1).reshape(hkv, -1, d)                                          # of all sequences, by KV head
    far = rows @ (pkc[0].float() * pks[0][..., None]).transpose(1, 2)
    near = (q @ (kc.float() * ks[..., None]).transpose(2, 3)).masked_fill_(_past(st["lens"], t), -math.inf)
    far = far.view(hkv, b, -1, far.shape[-1])
    top = torch.maximum(far.amax(-1).transpose(0, 1), near.amax(-1))[..., None]
    far, near = (far - top.transpose(0, 1)).exp_(), (near - top).exp_()
    total = far.sum(-1).transpose(0, 1) + near.sum(-1)
    out = (far.reshape(hkv, -1, far.shape[-1]) @ (pvc[0].float() * pvs[0][..., None])).view(hkv, b, -1, d).transpose(0, 1)
    out = (out + near @ (vc.float() * vs[..., None])) / total[..., None]
    return out.reshape(st["q"].shape).bfloat16()


def _run_weights(st):
    kc, ks, vc, vs = st["cache"]
    if own:
        out, sums = st["sa"].slim_attn_decode_int8_weights(st["q"], kc, ks, vc, vs, st["lens"], st["scale"], weights_in=st["sums"],
                                                           weights_out=st["new_sums"], out=st["out"], workspace=st["workspace"])
        return {"out": out, "weights": sums}
    b, hkv, t, d = kc.shape
    scores = (_grouped(st["q"], hkv) * st["scale"]) @ (kc.float() * ks[..., None]).transpose(2, 3)
    p = scores.masked_fill_(_past(st["lens"], t), -math.inf)
    p = (p - p.amax(-1, keepdim=True)).exp_()
    p = p / p.sum(-1, keepdim=True)
    out = p @ (vc.float() * vs[..., None])
    sums = (st["sums"] + p.sum(2)) * ~_past(st["lens"], t)[:, :, 0]
    return {"out": out.view(st["q"].shape).bfloat16(), "weights": sums}


def _run_evict(st):
    c, lens, to = st["case"], st["lens"], st["to"]
    keep, recent, t = c["keep"], c["recent"], c["kv_len"]
    if own:
        st["sa"].slim_cache_evict_int8(*st["cache"], st["weights"], lens, keep, recent, *to, st["kept"], st["new_lens"])
        kept, new_lens = st["kept"], st["new_lens"]
    else:
        i = torch.arange(t, device=lens.device)
        ends = lens[:, None, None]
        rank = torch.where(i >= ends - recent, math.inf, st["weights"]).masked_fill_(i >= ends, -math.inf)
        order = torch.sort(rank, dim=-1, descending=True, stable=True).indices[..., :keep]
        new_lens = lens.clamp(max=keep)
        there = torch.arange(keep, device=lens.device) < new_lens[:, None, None]
        order = torch.where(there, order, t).sort(-1).values
        at = order.clamp(max=t - 1)
        for x, y in zip(st["cache"] + (st["weights"],), to):
            wide, good = (at[..., None].expand(*at.shape, x.shape[-1]), there[..., None]) if x.dim() == 4 else (at, there)
            y[:, :, :keep] = torch.where(good, x.gather(2, wide), y[:, :, :keep])
        to[4].masked_fill_(i >= new_lens[:, None, None], 0.0)
        kept = torch.where(there, order, -1).int()
    return {"k_codes": to[0], "k_scale": to[1], "v_codes": to[2], "v_scale": to[3], "weights": to[4], "kept": kept,
            "lens": new_lens.int()}


# ------------------------------------------------------------------ the definitions in 64 bits

def exact(case, seed):
    st = prepare(case, seed)
    kind = case["kind"]
    if kind in ("rotate", "append"):
        return _exact_rows(st)
    if kind in ("prefix", "weights"):
        return _exact_attention(st)
    return None         # (an eviction computes nothing: its outputs are chosen inputs)


def _exact_rows(st):
    case = st["case"]
    d, table = case["head_dim"], st["table"].double()
    there = st["positions"] >= 0
    angle = torch.complex(table[:, :d // 2], table[:, d // 2:])[torch.where(there, st["positions"], 0).long()]

    def turned(x, weight):
        x = x.double()
        x = x / torch.linalg.vector_norm(x, dim=-1, keepdim=True).square().div(d).add(EPS).sqrt() * weight.double()
        pairs = x.unflatten(-1, (d // 2, 2)) if case["interleaved"] else x.unflatten(-1, (2, d // 2)).transpose(-1, -2)
        z = torch.complex(pairs[..., 0], pairs[..., 1]) * angle[:, :, None]
        y = torch.stack([z.real, z.imag], -1 if case["interleaved"] else -2).flatten(-2)
        return torch.where(there[:, :, None, None], y, 0.0).movedim(2, 1)

    q, k = turned(st["q"], st["q_weight"]), turned(st["k"], st["k_weight"])
    if case["kind"] == "rotate":
        return {"q": q, "k": k, "v": st["v"].double().movedim(2, 1)}
    # a scale is the largest of its row's values, as the cache gets them (in 16 bits), over 127
    scales = []
    for old, new in ((st["k_scale"], k.float().bfloat16()), (st["v_scale"], st["v"].movedim(2, 1))):
        scales.append(old.double())
        largest = new.double().abs().amax(-1) / 127
        for b, (first, n) in enumerate(zip(st["slots"].tolist(), there.sum(1).tolist())):
            scales[-1][b, :, first:first + n] = largest[b, :, :n]
    return {"q": q, "k_codes": None, "k_scale": scales[0], "v_codes": None, "v_scale": scales[1]}


def _exact_attention(st):
    kc, ks, vc, vs = st["cache"]
    b, hkv, t, d = kc.shape
    q = st["q"].double().reshape(b, hkv, -1, d)
    out = torch.empty_like(q)
    weights = torch.zeros((b, hkv, t), device=q.device, dtype=torch.float64)
    for g in range(hkv):
        if "prefix" in st:
            pkc, pks, pvc, pvs = (x[0, g].double() for x in st["prefix"])
            far_s = torch.einsum("nd,td->nt", q[:, g].reshape(-1, d), pkc * pks[:, None]).view(b, -1, pkc.shape[0]) * st["scale"]
        for i, n in enumerate(st["lens"].tolist()):
            k, v = kc[i, g, :n].double() * ks[i, g, :n, None].double(), vc[i, g, :n].double() * vs[i, g, :n, None].double()
            s = torch.einsum("hd,td->ht", q[i, g], k) * st["scale"]
            if "prefix" in st:
                p = torch.softmax(torch.cat([far_s[i], s], 1), 1)
                out[i, g] = p[:, :-n] @ (pvc * pvs[:, None]) + p[:, -n:] @ v
            else:
                p = torch.softmax(s, 1)
                out[i, g] = p @ v
                weights[i, g, :n] = st["sums"][i, g, :n].double() + p.sum(0)
    out = out.reshape(st["q"].shape)
    return out if "prefix" in st else {"out": out, "weights": weights}
