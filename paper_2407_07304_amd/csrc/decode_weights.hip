// Decode attention over the INT8 KV cache that also gives the attention weight of every cached token: what a cache of bounded
// length goes by when it drops tokens (cache_evict.hip).
//
//     w_t = w_in,t + sum over the query heads h of the KV head of softmax_t(s_h)
//
// The softmax's maximum and sum are known at the end of the sweep only, so the sweep of the grouped decode (decode_sweep.h)
// leaves its scores, fp32, in the workspace: 4 bytes a query head and token beside the 2 (D + 4) of the cache, written once and read
// once.  The writes are what the sweep takes longer for than a plain decode's: 16 sequences, 64 on 8 heads, T=8192 all full 42 and 56 us
// of kernel (with one bf16 a probability 54, and 43.4 with the same stores into one small piece of memory); past the L2 or through it they cost as
// much or more.  (K again
// in the place of the scores would be D bytes and the first product again.)  Where one workgroup has a
// whole (sequence, KV head), it turns its own scores into weights as soon as its waves are merged; where several have a part
// each, a second launch does, beside the merge of their records.  A lone query head a KV head takes this kernel too: 15 of the 16 columns of
// its products are empty, but the cache's bytes are the same.
//
// Results have the bits of fp32 probabilities: the second product takes a probability (times its v_scale) as two bf16, 16 bits of it.  (Rounded
// to one, as in the decode of 2 to 32 query heads a KV head without weights, a result is 1.4 times as far from the 64-bit one; the decode of
// one head, or more than 32, has them in fp32.)  It costs 0 to 4 %: one bf16 and two, 32 heads, T=1000 7.7 and 7.9 us, 8 sequences, T=4000
// 33.2 and 34.2, on another card 37.2 and 38.9; 16 sequences, 64 on 8 heads, T=8192 45.9 and 46.5, 64 codes 31.1 and 30.9, 40 on 1 heads, T=9000 29.8 and 30.8.
#include <algorithm>
#include <type_traits>

#include "decode_sweep.h"
#include "slim_common.h"
#include "slim_kernels.h"

namespace slim {

struct WeightsParams {
    const uint16_t* q;
    const int8_t *kc, *vc;
    const float *ks, *vs;
    const int* kv_lens;
    const float* w_in;   // null, or [batch, Hkv, T_alloc]; may be w_out
    float* w_out;
    uint16_t* out;
    // scores in log2 units, by tile, so that a wave's 16 rows are one piece: [batch, Hkv, tiles, G, 32].  (A row of T each, of T = 8192
    // tokens, all 16 would go to one memory channel.)
    float *scores, *ws_acc, *ws_ml;
    int batch, Hkv, G, T_alloc, tiles, head_groups, n_split, mode;
    unsigned split_rate;
    float scale_log2e;
};

typedef float f32x4u __attribute__((ext_vector_type(4), aligned(4)));

// Weights of tokens t to t + 3 by `heads` rows of scores, each by its maximum and the inverse of its sum; G rows a tile
__device__ __forceinline__ f32x4 weights_of(const float* scores, int t, int G, int heads, const float* top, const float* inverse) {
    f32x4 w = {0.0f, 0.0f, 0.0f, 0.0f};
    scores += ((long)(t / kGqaTile) * G) * kGqaTile + t % kGqaTile;
    for (int h = 0; h < heads; ++h) {
        const f32x4 s = *reinterpret_cast<const f32x4*>(scores + h * kGqaTile);
        const float m = top[h], f = inverse[h];
#pragma unroll
        for (int e = 0; e < 4; ++e) w[e] = fmaf(fast_exp2(s[e] - m), f, w[e]);
    }
    return w;
}
// ... and where they go: tokens t to t + 3 of a row of T_alloc, T of which count (the others' weights are zero)
__device__ __forceinline__ void store_weights(const float* w_in, float* w_out, int t, int T, int T_alloc, f32x4 w) {
    if (t + 3 < T) {
        if (w_in) w += *reinterpret_cast<const f32x4u*>(w_in + t);
        *reinterpret_cast<f32x4u*>(w_out + t) = w;
    } else {
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (t + e < T_alloc) w_out[t + e] = t + e < T ? w[e] + (w_in ? w_in[t + e] : 0.0f) : 0.0f;
    }
}

// D head dimension, W waves, NC groups of 16 heads; WHOLE: a workgroup has all of a (sequence, KV head)'s tokens and heads
template <int D, int W, int NC, bool WHOLE>
__global__ __launch_bounds__(64 * W) void slim_decode_weights_kernel(const WeightsParams p) {
    constexpr int WAVE_BYTES = GqaLds<D, NC>::WAVE_BYTES;
    __shared__ __attribute__((aligned(16))) char smem[W * WAVE_BYTES];
    __shared__ float topS[16 * NC], inverseS[16 * NC];

    const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
    const int Hq = p.G * p.Hkv;
    int y = blockIdx.y, b = blockIdx.z, T;
    const int sp = blockIdx.x;
    if (p.mode > 0) {   // (dealt by length; one split)
        const SequenceHead row = ranked_row(p.kv_lens, p.mode, p.Hkv * p.head_groups, p.T_alloc, b, y);
        y = row.h;
        b = row.b;
        T = row.T;
    } else {
        T = min(max(p.kv_lens[b], 1), p.T_alloc);
    }
    const int g = WHOLE ? y : y / p.head_groups, h0 = WHOLE ? 0 : (y - g * p.head_groups) * 32, heads = min(p.G - h0, 32);
    char* const kS = smem + w * WAVE_BYTES;
    const int n_used = WHOLE ? 1 : splits_of(T, p.n_split, p.split_rate);
    if (sp >= n_used) return;   // (nobody reads this split's record)
    const long kvrow0 = ((long)b * p.Hkv + g) * (long)p.T_alloc, row0 = (long)b * Hq + (long)g * p.G + h0;
    int first, end;
    split_span((T + kGqaTile - 1) / kGqaTile, n_used, sp, first, end);
    first += w;
    float* const scores = p.scores + (((long)b * p.Hkv + g) * p.tiles * p.G + h0) * kGqaTile;
    const int l16 = lane & 15, lq = lane >> 4;

    f32x4 o[NC][D / 16];
    float M[NC], lsum[NC];
    gqa_sweep<D, W, NC, true>(kS, lane, [&](int i) { return p.q + (row0 + min(i, heads - 1)) * D; }, p.kc + kvrow0 * D, p.ks + kvrow0,
                               p.vc + kvrow0 * D, p.vs + kvrow0, T, first, first < end ? (end - first + W - 1) / W : 0, p.scale_log2e,
                               [&](int nc, int t0, const float (&u)[8]) {
                                   // (through a descriptor over the tile's rows: the columns past the last head store nothing, and the store is the
                                   // same instructions for all, so that the waits for the loads around it are still counted exactly)
                                   const __amdgpu_buffer_rsrc_t to =
                                       __builtin_amdgcn_make_buffer_rsrc((void*)(scores + (long)t0 * p.G), 0, heads * (kGqaTile * 4), 0x00020000);
                                   const int off = (16 * nc + l16) * (kGqaTile * 4) + 16 * lq;
                                   __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u32x4, f32x4{u[0], u[1], u[2], u[3]}), to, off, 0, 0);
                                   __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u32x4, f32x4{u[4], u[5], u[6], u[7]}), to, off + 64, 0, 0);
                               },
                               o, M, lsum);
    gqa_record<D, NC>(kS, lane, o, M, lsum);
    __syncthreads();
    for (int x = threadIdx.x; x < heads * D; x += 64 * W) {
        const int h = x / D, d = x % D;
        float acc, top, L;
        gqa_merged<D, W, NC>(smem, h, d, acc, top, L);
        if (WHOLE) {
            p.out[(row0 + h) * D + d] = (uint16_t)(pack_bf16x2(acc / L, 0.0f) & 0xffffu);
            if (d == 0) {
                topS[h] = top;
                inverseS[h] = 1.0f / L;
            }
        } else {
            store_record<D>(p.ws_acc, p.ws_ml, (row0 + h) * p.n_split + sp, d, acc, top, L, p.mode < 0);
        }
    }
    if (WHOLE) {
        __syncthreads();   // (the workgroup's scores as well)
        const float* const w_in = p.w_in ? p.w_in + kvrow0 : nullptr;
        for (int t = 4 * threadIdx.x; t < p.T_alloc; t += 256 * W)
            store_weights(w_in, p.w_out + kvrow0, t, T, p.T_alloc,
                          t < T ? weights_of(scores, t, p.G, heads, topS, inverseS) : f32x4{0.0f, 0.0f, 0.0f, 0.0f});
    }
}

// The second launch: workgroups below n_combine merge records into result rows, the others turn 1024 tokens' scores into weights.
constexpr int kWeightsChunk = 1024, kWeightsHeads = 64;
template <int D, int WAVES, int U>
__global__ __launch_bounds__(256) void slim_decode_weights_finish_kernel(const WeightsParams p, int n_combine, int chunks) {
    __shared__ float topS[kWeightsHeads], inverseS[kWeightsHeads];
    const int tid = threadIdx.x, lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int Hq = p.G * p.Hkv;
    const f32x2* const ml = reinterpret_cast<const f32x2*>(p.ws_ml);
    if ((int)blockIdx.x < n_combine) {
        const long row = (long)blockIdx.x * (4 / WAVES) + (WAVES == 1 ? w : 0);
        if (row >= (long)p.batch * Hq) return;
        const int n_used = splits_of(min(max(p.kv_lens[(unsigned)row / (unsigned)Hq], 1), p.T_alloc), p.n_split, p.split_rate);
        combine_row<D, WAVES, U>(ml + row * p.n_split, reinterpret_cast<const f32x4*>(p.ws_acc) + row * p.n_split * (D / 4), p.out + row * D, n_used,
                                 lane, w);
        return;
    }
    const int x = (int)blockIdx.x - n_combine, chunk = x % chunks, bg = x / chunks, b = bg / p.Hkv, g = bg - b * p.Hkv;
    const int T = min(max(p.kv_lens[b], 1), p.T_alloc), n_used = splits_of(T, p.n_split, p.split_rate);
    const int t = chunk * kWeightsChunk + 4 * tid;
    const long row0 = (long)b * Hq + (long)g * p.G, kvrow0 = (long)bg * p.T_alloc;
    f32x4 sum = {0.0f, 0.0f, 0.0f, 0.0f};
    if (chunk * kWeightsChunk < T) {   // (uniform)
        for (int h0 = 0; h0 < p.G; h0 += kWeightsHeads) {
            const int heads = min(p.G - h0, kWeightsHeads);
            if (h0 > 0) __syncthreads();
            // a head's maximum and sum over its records: 16 lanes a head
            for (int h = tid >> 4; h < heads; h += 16) {
                const f32x2* const r = ml + (row0 + h0 + h) * p.n_split;
                float m = kMasked, l = 0.0f;
                for (int i = tid & 15; i < n_used; i += 16) {
                    const f32x2 v = r[i];
                    const float m_new = fmaxf(m, v[0]);
                    l = fmaf(l, fast_exp2(m - m_new), v[1] * fast_exp2(v[0] - m_new));
                    m = m_new;
                }
                const float top = row_group_max<16>(m);
                l *= fast_exp2(m - top);
                l += dpp_mov_f32<0xB1>(l);
                l += dpp_mov_f32<0x4E>(l);
                l += dpp_mov_f32<0x141>(l);
                l += dpp_mov_f32<0x140>(l);
                if ((tid & 15) == 0) {
                    topS[h] = top;
                    inverseS[h] = 1.0f / l;
                }
            }
            __syncthreads();
            if (t < T) sum += weights_of(p.scores + ((long)bg * p.tiles * p.G + h0) * kGqaTile, t, p.G, heads, topS, inverseS);
        }
    }
    if (t < p.T_alloc) store_weights(p.w_in ? p.w_in + kvrow0 : nullptr, p.w_out + kvrow0, t, T, p.T_alloc, sum);
}

static int weights_head_groups(int q_heads, int kv_heads) { return (q_heads / kv_heads + 31) / 32; }
static DecodePlan weights_plan(int batch, int q_heads, int kv_heads, int kv_len, int head_dim) {
    const int hg = weights_head_groups(q_heads, kv_heads), group = std::min(q_heads / kv_heads, 32);
    return decode_grouped_plan(batch, kv_heads * hg * group, kv_heads * hg, kv_len, head_dim);
}
static long weights_tiles(int kv_len) { return ((long)kv_len + kGqaTile - 1) / kGqaTile; }

size_t decode_weights_workspace_bytes(int batch, int q_heads, int kv_heads, int kv_len, int head_dim) {
    const long rows = (long)batch * q_heads;
    return decode_records_bytes(rows, weights_plan(batch, q_heads, kv_heads, kv_len, head_dim).n_split, head_dim) +
           (size_t)rows * weights_tiles(kv_len) * kGqaTile * sizeof(float);
}

bool decode_weights_fits(int batch, int q_heads, int kv_heads, int kv_len, int head_dim) {
    const DecodePlan plan = weights_plan(batch, q_heads, kv_heads, kv_len, head_dim);
    const long rows = (long)batch * kv_heads, hg = weights_head_groups(q_heads, kv_heads);
    // (a launch has less than 2^32 threads, a grid's second and third index less than 2^16)
    return rows * hg * plan.n_split < (1L << 23) && kv_heads * hg < 65536 &&
           rows * ((kv_len + kWeightsChunk - 1) / kWeightsChunk) + (long)batch * q_heads < (1L << 24);
}

hipError_t launch_decode_weights(const DecodeArgs& a, const float* w_in, float* w_out, hipStream_t stream) {
    const DecodePlan plan = weights_plan(a.batch, a.q_heads, a.kv_heads, a.kv_len, a.head_dim);
    const long rows = (long)a.batch * a.q_heads;
    WeightsParams p;
    p.q = (const uint16_t*)a.q;
    p.kc = a.k_codes, p.ks = a.k_scale, p.vc = a.v_codes, p.vs = a.v_scale;
    p.kv_lens = a.kv_lens, p.w_in = w_in, p.w_out = w_out, p.out = (uint16_t*)a.out;
    p.batch = a.batch, p.Hkv = a.kv_heads, p.G = a.q_heads / a.kv_heads, p.T_alloc = a.kv_len;
    p.tiles = (int)weights_tiles(a.kv_len);
    p.head_groups = weights_head_groups(a.q_heads, a.kv_heads);
    p.n_split = plan.n_split, p.split_rate = plan.split_rate, p.mode = decode_mode(plan, a.batch);
    p.scores = a.workspace;
    p.ws_acc = p.scores + rows * p.tiles * kGqaTile;
    p.ws_ml = p.ws_acc + rows * plan.n_split * a.head_dim;
    p.scale_log2e = a.softmax_scale * kLog2e;
    const bool whole = plan.n_split == 1 && p.head_groups == 1;
    const dim3 grid((unsigned)plan.n_split, (unsigned)(a.kv_heads * p.head_groups), (unsigned)a.batch);
    using std::integral_constant;
    auto with_d = [&](auto d_c) {
        constexpr int D = decltype(d_c)::value, RPW = 256 / D;
        auto sweep = [&](auto w_c, auto nc_c) {
            constexpr int W = decltype(w_c)::value, NC = decltype(nc_c)::value;
            if (whole) hipLaunchKernelGGL((slim_decode_weights_kernel<D, W, NC, true>), grid, dim3(64 * W), 0, stream, p);
            else hipLaunchKernelGGL((slim_decode_weights_kernel<D, W, NC, false>), grid, dim3(64 * W), 0, stream, p);
            return hipGetLastError();
        };
        const integral_constant<int, 1> one{};
        const integral_constant<int, 4> four{};
        const integral_constant<int, 8> eight{};
        const hipError_t e = p.G > 16 ? sweep(eight, integral_constant<int, 2>{}) : plan.waves == 8 ? sweep(eight, one) : sweep(four, one);
        if (e != hipSuccess || whole) return e;
        const int chunks = (a.kv_len + kWeightsChunk - 1) / kWeightsChunk;
        auto finish = [&](auto waves_c, auto u_c) {
            constexpr int WAVES = decltype(waves_c)::value, U = decltype(u_c)::value;
            const long n_combine = (rows * WAVES + 3) / 4;
            hipLaunchKernelGGL((slim_decode_weights_finish_kernel<D, WAVES, U>), dim3((unsigned)(n_combine + (long)a.batch * a.kv_heads * chunks)),
                               dim3(256), 0, stream, p, (int)n_combine, chunks);
            return hipGetLastError();
        };
        if (plan.n_split <= 2 * RPW) return finish(one, integral_constant<int, 2>{});
        if (plan.n_split <= 4 * RPW) return finish(one, four);
        return finish(four, four);
    };
    return a.head_dim == 128 ? with_d(integral_constant<int, 128>{}) : with_d(integral_constant<int, 64>{});
}

}  // namespace slim
