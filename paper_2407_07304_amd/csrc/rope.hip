// Norms of queries and keys for each head and their rotation by position, in one pass over the rows that a projection
// gives, into the layout that the attention reads: bf16 [batch, heads, tokens, D], or (K and V) straight into the INT8
// cache (paper section 2.2 keeps it in INT8 from the first token on).
//
// A row x of D values: r = 1 / sqrt(mean(x^2) + eps), y = x r w, and each of its D/2 pairs (a, b) turned by the angle of
// the token's position, a' = a c - b s, b' = b c + a s.  The result is rounded to fp32 and that to bf16; the cache takes
// the codes of the bf16 row.
//
// All of it is computed in 64 bits: a code is a whole number, and which one it is hangs on the last bit of the row's
// values and of its largest one.  With 53 bits the order of the sum and the way to the root no longer decide any of them,
// so that codes, scales and queries are the same on every IEEE machine, as the quantiser's are.  A 64-bit multiply-add
// takes a vector unit here as long as a 32-bit one; what it costs is registers and the conversions.
//
// A row is held by D/8 adjacent lanes, and both values of a pair by one lane (pairs i and i + D/2: two loads of 8 bytes;
// pairs 2i and 2i + 1: one of 16), so that a rotation needs no other lane.  A wave serves one token, 64 / (D/8) heads at a
// time: position, angles and weights are fetched once for all its heads.  Bound by memory where there are many tokens and
// by the latency of position, then angles, where there are few.
#include <algorithm>
#include <type_traits>

#include "slim_common.h"
#include "slim_kernels.h"

namespace slim {

// sum over the LPR (8 or 16) adjacent lanes that hold a row, in every one of them
template <int CTRL>
__device__ __forceinline__ double dpp_mov_f64(double v) {
    const u32x2 b = __builtin_bit_cast(u32x2, v);
    u32x2 r;
    r[0] = (unsigned)__builtin_amdgcn_update_dpp(0, (int)b[0], CTRL, 0xf, 0xf, false);
    r[1] = (unsigned)__builtin_amdgcn_update_dpp(0, (int)b[1], CTRL, 0xf, 0xf, false);
    return __builtin_bit_cast(double, r);
}
template <int LPR>
__device__ __forceinline__ double row_group_sum(double v) {
    static_assert(LPR == 8 || LPR == 16, "a row is held by 8 or 16 adjacent lanes");
    v += dpp_mov_f64<0xB1>(v);                    // quad_perm [1,0,3,2]
    v += dpp_mov_f64<0x4E>(v);                    // quad_perm [2,3,0,1]
    v += dpp_mov_f64<0x141>(v);                   // row_half_mirror
    if (LPR == 16) v += dpp_mov_f64<0x140>(v);    // row_mirror
    return v;
}

// 1 / sqrt(a), a > 0: the hardware's estimate (some 24 bits) and two steps of Newton's method.  The estimate of an infinity is 0, which
// no step takes further (infinity times 0 is not a number).
__device__ __forceinline__ double inverse_root(double a) {
    const double estimate = __builtin_amdgcn_rsq(a);
    double y = estimate;
#pragma unroll
    for (int i = 0; i < 2; ++i) y = fma(y, fma(-a * y, 0.5 * y, 0.5), y);
    return estimate == 0.0 ? estimate : y;
}

// The first of a result's two roundings, to fp32 and from there to bf16.  (Contracted, the compiler makes one of the two, which is
// another result where fp32 lies on a tie of bf16 and the 64-bit value beside it: one value in 2^16.)
__device__ __forceinline__ float round_to_f32(double v) {
#pragma clang fp contract(off)
    return (float)v;
}

// This lane's 8 values of a row: bf16 pairs, both values of a rotated pair among them.  PAIRS: values 8 c to 8 c + 7, else
// 4 c to 4 c + 3 and those D/2 further.
template <int D, bool PAIRS>
__device__ __forceinline__ u32x4 load_piece(const uint16_t* row, int c) {
    if (PAIRS) return *reinterpret_cast<const u32x4*>(row + 8 * c);
    const u32x2 lo = *reinterpret_cast<const u32x2*>(row + 4 * c), hi = *reinterpret_cast<const u32x2*>(row + D / 2 + 4 * c);
    return u32x4{lo[0], lo[1], hi[0], hi[1]};
}
template <int D, bool PAIRS>
__device__ __forceinline__ void store_piece(uint16_t* row, int c, u32x4 v) {
    if (PAIRS) {
        *reinterpret_cast<u32x4*>(row + 8 * c) = v;
    } else {
        *reinterpret_cast<u32x2*>(row + 4 * c) = u32x2{v[0], v[1]};
        *reinterpret_cast<u32x2*>(row + D / 2 + 4 * c) = u32x2{v[2], v[3]};
    }
}
__device__ __forceinline__ void widen_piece(u32x4 raw, double (&x)[8]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        x[2 * i] = (double)bf16_bits_to_f32(raw[i] & 0xffffu);
        x[2 * i + 1] = (double)__uint_as_float(raw[i] & 0xffff0000u);
    }
}

template <int D, bool PAIRS, bool APPEND>
__global__ __launch_bounds__(256) void slim_qk_norm_rope_kernel(const RopeArgs p, int parts, int per_part) {
    constexpr int LPR = D / 8, RW = 64 / LPR;   // lanes a row, rows (heads) a wave
    const int lane = threadIdx.x & 63, c = lane % LPR, sub = lane / LPR;
    // units of RW heads of one kind: queries, then keys, then values
    const int uq = (p.q_heads + RW - 1) / RW, uk = (p.kv_heads + RW - 1) / RW;
    const long n_items = (long)p.batch * p.seq_len * parts;
    for (long item = (long)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6)); item < n_items; item += (long)gridDim.x * 4) {
        const long token = item / parts;
        const int part = (int)(item - token * parts);
        const int b = (int)(token / p.seq_len), s = (int)(token - (long)b * p.seq_len);
        const int u_end = min((part + 1) * per_part, uq + 2 * uk);

        // unit u's kind (uniform), and this lane's head of it: past the last one that head's again, which is not stored
        auto unit = [&](int u, int& kind, int& heads, int& h) {
            kind = u < uq ? 0 : u < uq + uk ? 1 : 2;
            heads = kind == 0 ? p.q_heads : p.kv_heads;
            h = (u - (kind == 0 ? 0 : kind == 1 ? uq : uq + uk)) * RW + sub;
        };
        auto load = [&](int u) {
            int kind, heads, h;
            unit(u, kind, heads, h);
            return load_piece<D, PAIRS>((const uint16_t*)(kind == 0 ? p.q : kind == 1 ? p.k : p.v) +
                                            token * (kind == 0 ? p.q_stride : kind == 1 ? p.k_stride : p.v_stride) + (long)min(h, heads - 1) * D, c);
        };
        u32x4 raw_next = load(part * per_part);   // (ahead of the position, which the angles wait for)
        __builtin_amdgcn_sched_barrier(0);
        const int pos = p.positions[token];
        const bool there = pos >= 0 && pos < p.table_len;
        const long slot = APPEND ? (long)p.slots[b] + s : s;
        const bool room = slot >= 0 && slot < p.kv_len;
        double cs[4], sn[4];
        {
            const float* t = p.cos_sin + (long)(there ? pos : 0) * D + 4 * c;
            const f32x4 tc = *reinterpret_cast<const f32x4*>(t), ts = *reinterpret_cast<const f32x4*>(t + D / 2);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                cs[i] = (double)tc[i];
                sn[i] = (double)ts[i];
            }
        }
        if (!there) {   // (uniform) padding: rows of zeros, nothing into the cache, no more of its rows read
            for (int u = part * per_part; u < (APPEND ? min(u_end, uq) : u_end); ++u) {
                int kind, heads, h;
                unit(u, kind, heads, h);
                uint16_t* dst = (uint16_t*)(kind == 0 ? p.q_out : kind == 1 ? p.k_out : p.v_out) +
                                (((long)b * heads + min(h, heads - 1)) * p.seq_len + s) * D;
                if (h < heads) store_piece<D, PAIRS>(dst, c, u32x4{0u, 0u, 0u, 0u});
            }
            continue;
        }
        for (int u = part * per_part; u < u_end; ++u) {
            int kind, heads, h;
            unit(u, kind, heads, h);
            const int hc = min(h, heads - 1);
            u32x4 raw = raw_next;
            raw_next = load(min(u + 1, u_end - 1));
            if (kind < 2) {
                const uint16_t* wt = (const uint16_t*)(kind == 0 ? p.q_weight : p.k_weight);
                double x[8];
                widen_piece(raw, x);
                double r = 1.0;
                if (wt != nullptr) {   // (uniform)
                    double sum = 0.0, w[8];
#pragma unroll
                    for (int i = 0; i < 8; ++i) sum = fma(x[i], x[i], sum);
                    r = inverse_root(row_group_sum<LPR>(sum) * (1.0 / D) + p.eps);
                    widen_piece(load_piece<D, PAIRS>(wt, c), w);
#pragma unroll
                    for (int i = 0; i < 8; ++i) x[i] *= w[i];
                }
                float y[8];
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    constexpr int A = PAIRS ? 2 : 1, B = PAIRS ? 1 : 4;
                    const double a = x[A * i], o = x[A * i + B];
                    y[A * i] = round_to_f32(r * fma(a, cs[i], -(o * sn[i])));
                    y[A * i + B] = round_to_f32(r * fma(o, cs[i], a * sn[i]));
                }
#pragma unroll
                for (int i = 0; i < 4; ++i) raw[i] = pack_bf16x2(y[2 * i], y[2 * i + 1]);
            }
            if (!APPEND || kind == 0) {
                uint16_t* dst = (uint16_t*)(kind == 0 ? p.q_out : kind == 1 ? p.k_out : p.v_out) +
                                (((long)b * heads + hc) * p.seq_len + s) * D;
                if (h < heads) store_piece<D, PAIRS>(dst, c, raw);
            } else {
                u32x2 codes;
                float scale;
                quant_row_piece<LPR>(raw, codes, scale);
                if (h < heads && room) {
                    const long row = ((long)b * heads + hc) * p.kv_len + slot;
                    int8_t* dst = (kind == 1 ? p.k_codes : p.v_codes) + row * D;
                    if (PAIRS) {
                        *reinterpret_cast<u32x2*>(dst + 8 * c) = codes;
                    } else {
                        *reinterpret_cast<unsigned*>(dst + 4 * c) = codes[0];
                        *reinterpret_cast<unsigned*>(dst + D / 2 + 4 * c) = codes[1];
                    }
                    if (c == 0) (kind == 1 ? p.k_scale : p.v_scale)[row] = scale;
                }
            }
        }
    }
}

hipError_t launch_qk_norm_rope(const RopeArgs& a, bool append, hipStream_t stream) {
    const int rw = 512 / a.head_dim, units = (a.q_heads + rw - 1) / rw + 2 * ((a.kv_heads + rw - 1) / rw);
    const long tokens = (long)a.batch * a.seq_len;
    // a wave for each unit of heads where tokens are few, up to six units a wave (its position, angles and weights once) where
    // that leaves 8192 waves: 32 heads, 2048 tokens 29.9 us with one unit a wave, 25.2 with two, 23.6 with six, 28.7 with twelve; 8192
    // tokens, 64 on 8 heads 94.4, 75.0, 72.1, 72.3 (three sets of inputs and of results in turn, so that neither stays in the caches)
    long per = tokens * units / 8192;
    per = per < 1 ? 1 : per > 6 ? 6 : per;
    const int parts = (units + (int)per - 1) / (int)per;
    per = (units + parts - 1) / parts;
    // (the loop over items is for more tokens than this many workgroups)
    const dim3 grid((unsigned)std::min((tokens * parts + 3) / 4, 1L << 22)), block(256);
    auto launch = [&](auto d_c, auto pairs_c, auto append_c) {
        hipLaunchKernelGGL((slim_qk_norm_rope_kernel<decltype(d_c)::value, decltype(pairs_c)::value, decltype(append_c)::value>), grid,
                           block, 0, stream, a, parts, (int)per);
        return hipGetLastError();
    };
    auto pick = [&](auto d_c) {
        if (append) return a.interleaved ? launch(d_c, std::true_type{}, std::true_type{}) : launch(d_c, std::false_type{}, std::true_type{});
        return a.interleaved ? launch(d_c, std::true_type{}, std::false_type{}) : launch(d_c, std::false_type{}, std::false_type{});
    };
    return a.head_dim == 128 ? pick(std::integral_constant<int, 128>{}) : pick(std::integral_constant<int, 64>{});
}

}  // namespace slim
