"""Python face of the C-ABI library (``include/slimattn.h``): signatures and defaults.

Tensors are torch tensors on the GPU (PyTorch supplies device memory and the HIP stream);
every step of the path runs in the library's kernels.  The tensors are checked, the results a
caller leaves out allocated and the library called by the native binding ``_slimbind``
(``csrc/binding.cpp``); ``load()`` gives the plain C ABI through ctypes.  There is no CPU
fallback: if a built library is missing, the first call raises.
"""
import ctypes
import importlib
import os

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libslimattn.so")
BINDING_PATH = os.path.join(_HERE, "_slimbind.so")

SLIM_OK = 0
SLIM_BF16, SLIM_F32, SLIM_I8 = 0, 1, 2

_lib = None
_native = None


class SlimError(RuntimeError):
    def __init__(self, status, text):
        super().__init__("slimattn status %d: %s" % (status, text))
        self.status = status


def load():
    """Loads ``libslimattn.so`` and returns its C ABI; raises if it has not been built (``build.build()``)."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise ImportError("%s is missing: run `python -m paper_2407_07304_amd.build` (hipcc, gfx950) first; "
                              "there is no fallback path" % LIB_PATH)
        lib = ctypes.CDLL(LIB_PATH)
        p, i, f = ctypes.c_void_p, ctypes.c_int, ctypes.c_float
        lib.kv_quant_int8.argtypes = [p, p, p, i, i, i, i, i, i, f, p]
        lib.kv_quant_int8.restype = i
        lib.kv_quant_int8_pair.argtypes = [p, p, p, p, p, p, i, i, i, i, i, i, f, p]
        lib.kv_quant_int8_pair.restype = i
        lib.kv_quant_int8_append.argtypes = [p, p, p, p, i, i, i, i, i, i, f, p]
        lib.kv_quant_int8_append.restype = i
        lib.slim_attn_prefill.argtypes = [p, p, p, p, p, p, i, i, i, i, i, i, f, i, i, p]
        lib.slim_attn_prefill.restype = i
        lib.slim_attn_prefill_block_rows.argtypes = [i, i, i, i, i, i, i, i]
        lib.slim_attn_prefill_block_rows.restype = i
        lib.slim_attn_prefill_emit_int8.argtypes = [p, p, p, p, p, p, p, p, i, i, i, i, i, i, f, i, p]
        lib.slim_attn_prefill_emit_int8.restype = i
        lib.slim_attn_prefill_two_sweep_workspace_bytes.argtypes = [i, i, i, i, i]
        lib.slim_attn_prefill_two_sweep_workspace_bytes.restype = ctypes.c_size_t
        lib.slim_attn_prefill_two_sweep.argtypes = [p, p, p, p, p, ctypes.c_size_t, i, i, i, i, i, i, f, i, p]
        lib.slim_attn_prefill_two_sweep.restype = i
        lib.slim_attn_prefill_strip_max_seq_len.argtypes = []
        lib.slim_attn_prefill_strip_max_seq_len.restype = i
        lib.slim_attn_prefill_strip.argtypes = [p, p, p, p, i, i, i, i, i, i, f, i, p]
        lib.slim_attn_prefill_strip.restype = i
        lib.slim_attn_decode_int8_workspace_bytes.argtypes = [i, i, i, i, i]
        lib.slim_attn_decode_int8_workspace_bytes.restype = ctypes.c_size_t
        lib.slim_attn_decode_int8.argtypes = [p, p, p, p, p, p, p, ctypes.c_size_t, i, i, i, i, i, i, f, p]
        lib.slim_attn_decode_int8.restype = i
        lib.slim_attn_decode_int8_static_max_bytes.argtypes = []
        lib.slim_attn_decode_int8_static_max_bytes.restype = ctypes.c_size_t
        lib.slim_attn_decode_int8_static.argtypes = [p, p, p, p, p, p, i, i, i, i, i, i, f, p]
        lib.slim_attn_decode_int8_static.restype = i
        lib.slim_attn_decode_int8_varlen.argtypes = [p, p, p, p, p, p, p, p, ctypes.c_size_t, i, i, i, i, i, i, f, p]
        lib.slim_attn_decode_int8_varlen.restype = i
        lib.slim_attn_decode_int8_plan.argtypes = [i, i, i, i, i, i, ctypes.POINTER(i), ctypes.POINTER(i)]
        lib.slim_attn_decode_int8_plan.restype = i
        lib.slim_attn_decode_int8_plan_options.argtypes = [i, i, i, i, i, i, ctypes.POINTER(i), ctypes.POINTER(i)]
        lib.slim_attn_decode_int8_plan_options.restype = i
        d, n = ctypes.c_double, ctypes.c_int64
        lib.slim_qk_norm_rope.argtypes = [p, p, p, n, n, n, p, p, p, p, p, p, p] + [i] * 7 + [d, p]
        lib.slim_qk_norm_rope.restype = i
        lib.slim_qk_norm_rope_append_int8.argtypes = [p, p, p, n, n, n, p, p, p, p, p, p, p, p, p, p] + [i] * 8 + [d, p]
        lib.slim_qk_norm_rope_append_int8.restype = i
        lib.slim_attn_decode_int8_shared_prefix_workspace_bytes.argtypes = [i] * 6
        lib.slim_attn_decode_int8_shared_prefix_workspace_bytes.restype = ctypes.c_size_t
        lib.slim_attn_decode_int8_shared_prefix.argtypes = [p] * 12 + [ctypes.c_size_t] + [i] * 7 + [f, p]
        lib.slim_attn_decode_int8_shared_prefix.restype = i
        lib.slim_attn_decode_int8_weights_workspace_bytes.argtypes = [i] * 5
        lib.slim_attn_decode_int8_weights_workspace_bytes.restype = ctypes.c_size_t
        lib.slim_attn_decode_int8_weights.argtypes = [p] * 10 + [ctypes.c_size_t] + [i] * 6 + [f, p]
        lib.slim_attn_decode_int8_weights.restype = i
        lib.slim_cache_evict_int8.argtypes = [p] * 13 + [i] * 7 + [p]
        lib.slim_cache_evict_int8.restype = i
        lib.slim_status_string.argtypes = [i]
        lib.slim_status_string.restype = ctypes.c_char_p
        _lib = lib
    return _lib


def status_string(status: int) -> str:
    return load().slim_status_string(int(status)).decode()


def _check(status):
    if status != SLIM_OK:
        raise SlimError(status, status_string(status))


def _load_native():
    """The native binding; raises like ``load()`` if it has not been built."""
    global _native
    if _native is None:
        load()
        if not os.path.exists(BINDING_PATH):
            raise ImportError("%s is missing: run `python -m paper_2407_07304_amd.build` (hipcc, gfx950) first; "
                              "there is no fallback path" % BINDING_PATH)
        native = importlib.import_module(__package__ + "._slimbind")
        native.set_raise_status(_check)
        _native = native
    return _native


def kv_quant_int8(x, codes=None, scales=None):
    """x [B,Hkv,S,D] bf16 -> (codes int8 [B,Hkv,S,D], scales fp32 [B,Hkv,S])."""
    return (_native or _load_native()).kv_quant(x, codes, scales)


def kv_quant_int8_pair(k, v, k_codes=None, k_scale=None, v_codes=None, v_scale=None):
    """kv_quant_int8 on k and v [B,Hkv,S,D] bf16 in one launch -> (k_codes, k_scale, v_codes, v_scale)."""
    return (_native or _load_native()).kv_quant_pair(k, v, k_codes, k_scale, v_codes, v_scale)


def slim_attn_prefill(q, k, v, softmax_scale, causal=True, k_scale=None, v_scale=None, out=None,
                      out_dtype=torch.bfloat16):
    """q [B,Hq,S,D] bf16; k, v [B,Hkv,S,D] bf16, or int8 with k_scale/v_scale [B,Hkv,S] fp32."""
    return (_native or _load_native()).prefill(q, k, v, softmax_scale, causal, k_scale, v_scale, out, out_dtype)


def slim_attn_decode_int8_workspace_bytes(batch, q_heads, kv_heads, kv_len, head_dim) -> int:
    return int(load().slim_attn_decode_int8_workspace_bytes(batch, q_heads, kv_heads, kv_len, head_dim))


def slim_attn_decode_int8(q, k_codes, k_scale, v_codes, v_scale, softmax_scale, causal=False, out=None,
                          workspace=None):
    """q [B,Hq,1,D] bf16; codes [B,Hkv,T,D] int8; scales [B,Hkv,T] fp32 -> out [B,Hq,1,D] bf16."""
    return (_native or _load_native()).decode(q, k_codes, k_scale, v_codes, v_scale, softmax_scale, causal, out, workspace)


def slim_attn_decode_int8_static_max_bytes() -> int:
    return int(load().slim_attn_decode_int8_static_max_bytes())


def slim_attn_decode_int8_static(q, k_codes, k_scale, v_codes, v_scale, softmax_scale, out, causal=False):
    """slim_attn_decode_int8 with the library's own static scratch array: no workspace argument, and nothing is
    allocated here either, so the caller passes ``out`` [B,Hq,1,D] bf16."""
    return (_native or _load_native()).decode_static(q, k_codes, k_scale, v_codes, v_scale, softmax_scale, out, causal)


def slim_attn_decode_int8_varlen(q, k_codes, k_scale, v_codes, v_scale, kv_lens, softmax_scale, causal=False, out=None,
                                 workspace=None):
    """As slim_attn_decode_int8, sequence b attending to its first kv_lens[b] cached tokens (kv_lens [B] int32,
    on the device)."""
    return (_native or _load_native()).decode_varlen(q, k_codes, k_scale, v_codes, v_scale, softmax_scale, causal, out,
                                                     workspace, kv_lens)


def kv_quant_int8_append(x_new, codes, scales, positions):
    """Quantises x_new [B,Hkv,1,D] bf16 into token positions[b] of the cache (codes [B,Hkv,T,D] int8, scales
    [B,Hkv,T] fp32, both updated in place); positions [B] int32 on the device."""
    return (_native or _load_native()).kv_quant_append(x_new, codes, scales, positions)


def slim_attn_prefill_emit_int8(q, k, v, softmax_scale, causal=True, out=None, out_dtype=torch.bfloat16):
    """Prefill on bf16 K/V that also writes their INT8 cache: returns (out, k_codes, k_scale, v_codes, v_scale)."""
    return (_native or _load_native()).prefill_emit(q, k, v, softmax_scale, causal, out, out_dtype)


def slim_attn_prefill_two_sweep(q, k, v, softmax_scale, causal=True, out=None, out_dtype=torch.bfloat16, workspace=None):
    """The two-sweep comparison variant of the bf16 prefill (row maxima first, then everything else)."""
    return (_native or _load_native()).prefill_two_sweep(q, k, v, softmax_scale, causal, out, out_dtype, workspace)


def slim_attn_prefill_strip_max_seq_len() -> int:
    return int(load().slim_attn_prefill_strip_max_seq_len())


def slim_attn_prefill_strip(q, k, v, softmax_scale, causal=True, out=None, out_dtype=torch.bfloat16):
    """The comparison variant of the bf16 prefill that keeps a row block's whole score strip on chip."""
    return (_native or _load_native()).prefill_strip(q, k, v, softmax_scale, causal, out, out_dtype)


def slim_rope_table(length, head_dim, base=10000.0, device="cuda"):
    """The cosines, then the sines, of position x base^(-2i / head_dim): fp32 [length, head_dim], the angles in 64 bits.
    (Any other table of this layout will do for the two calls below: scaled frequencies are the caller's affair.)"""
    inverse = float(base) ** (-torch.arange(0, head_dim, 2, dtype=torch.float64) / head_dim)
    angle = torch.arange(length, dtype=torch.float64)[:, None] * inverse
    return torch.cat([angle.cos(), angle.sin()], 1).float().to(device)


def slim_qk_norm_rope(q, k, v, cos_sin, positions, q_weight=None, k_weight=None, eps=1e-6, interleaved=False, q_out=None,
                      k_out=None, v_out=None):
    """q [B,S,Hq,D], k, v [B,S,Hkv,D] bf16, tokens at any stride (slices of one projection's output) -> normed and rotated
    q [B,Hq,S,D], k [B,Hkv,S,D] and v [B,Hkv,S,D] bf16; cos_sin fp32 [table length, D], positions int32 [B,S] (-1: padding,
    rows of zeros), weights bf16 [D] or None (no norm)."""
    return (_native or _load_native()).qk_norm_rope(q, k, v, cos_sin, positions, q_weight, k_weight, eps, interleaved, q_out,
                                                    k_out, v_out)


def slim_qk_norm_rope_append_int8(q, k, v, cos_sin, positions, slots, k_codes, k_scale, v_codes, v_scale, q_weight=None,
                                  k_weight=None, eps=1e-6, interleaved=False, q_out=None):
    """slim_qk_norm_rope with K and V quantised into tokens slots[b] + s of the cache (codes [B,Hkv,T,D] int8, scales
    [B,Hkv,T] fp32, updated in place; slots int32 [B] on the device) -> q [B,Hq,S,D] bf16."""
    return (_native or _load_native()).qk_norm_rope_append(q, k, v, cos_sin, positions, slots, k_codes, k_scale, v_codes, v_scale,
                                                           q_weight, k_weight, eps, interleaved, q_out)


def slim_attn_decode_int8_shared_prefix_workspace_bytes(batch, q_heads, kv_heads, prefix_len, kv_len, head_dim) -> int:
    return int(load().slim_attn_decode_int8_shared_prefix_workspace_bytes(batch, q_heads, kv_heads, prefix_len, kv_len, head_dim))


def slim_attn_decode_int8_shared_prefix(q, prefix_k_codes, prefix_k_scale, prefix_v_codes, prefix_v_scale, k_codes, k_scale,
                                        v_codes, v_scale, kv_lens, softmax_scale, causal=False, out=None, workspace=None):
    """slim_attn_decode_int8_varlen behind a prefix that all sequences share: its cache has codes [1,Hkv,P,D] int8 and scales
    [1,Hkv,P] fp32, the sequences' own follows as in slim_attn_decode_int8_varlen; kv_lens [B] int32 may be 0."""
    return (_native or _load_native()).decode_shared_prefix(q, prefix_k_codes, prefix_k_scale, prefix_v_codes, prefix_v_scale, k_codes,
                                                            k_scale, v_codes, v_scale, kv_lens, softmax_scale, causal, out, workspace)


def slim_attn_decode_int8_weights_workspace_bytes(batch, q_heads, kv_heads, kv_len, head_dim) -> int:
    return int(load().slim_attn_decode_int8_weights_workspace_bytes(batch, q_heads, kv_heads, kv_len, head_dim))


def slim_attn_decode_int8_weights(q, k_codes, k_scale, v_codes, v_scale, kv_lens, softmax_scale, weights_in=None, weights_out=None,
                                  causal=False, out=None, workspace=None):
    """slim_attn_decode_int8_varlen that also gives the cached tokens' attention weights -> (out, weights_out): weights_out fp32
    [B,Hkv,T] is weights_in (or zero) plus the sum of the token's probabilities over the query heads of its KV head, and zero past
    a sequence's length; weights_out may be weights_in."""
    return (_native or _load_native()).decode_weights(q, k_codes, k_scale, v_codes, v_scale, kv_lens, softmax_scale, weights_in,
                                                      weights_out, causal, out, workspace)


def slim_cache_evict_int8(k_codes, k_scale, v_codes, v_scale, weights, kv_lens, keep, recent=0, k_codes_out=None, k_scale_out=None,
                          v_codes_out=None, v_scale_out=None, weights_out=None, kept=None, kv_lens_out=None):
    """Of every (sequence, KV head)'s first kv_lens[b] tokens the `recent` last and, of the others, those of largest weight, `keep` in
    all, copied in their order to another cache (of `keep` tokens where none is passed) -> (k_codes_out, k_scale_out, v_codes_out,
    v_scale_out, weights_out, kept int32 [B,Hkv,keep] with -1 past what stays, kv_lens_out)."""
    return (_native or _load_native()).cache_evict(k_codes, k_scale, v_codes, v_scale, weights, kv_lens, keep, recent, k_codes_out,
                                                   k_scale_out, v_codes_out, v_scale_out, weights_out, kept, kv_lens_out)
