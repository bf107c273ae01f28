// Eviction from the INT8 KV cache by accumulated attention weight: of a (sequence, KV head)'s tokens the `recent` last ones stay, and
// of the others those of largest weight, `keep` in all, in their order, which go to another cache.
//
// Two launches.  The first chooses: a workgroup for each (sequence, KV head) finds the weight of the last token that stays by
// its bits, 11, 11 and 10 of them (a histogram in LDS, then the bin that the count runs out in), and numbers the tokens that stay
// with prefix sums.  Whole numbers only: no order of atomics changes a result.  The second copies: 16 bytes a lane, a row
// of codes by D/16 adjacent lanes, and is bound by memory: (2 (D + 4) + 4) bytes a token, read and written.
#include "slim_common.h"
#include "slim_kernels.h"

namespace slim {

typedef float f32x4u __attribute__((ext_vector_type(4), aligned(4)));

constexpr int kSelectThreads = 1024, kSelectChunk = 4 * kSelectThreads;

// A weight as a whole number of the same order: NaN below everything, the two zeros equal
__device__ __forceinline__ unsigned weight_key(float w) {
    const unsigned b = __float_as_uint(w);
    if ((b & 0x7fffffffu) > 0x7f800000u) return 0u;
    if ((b & 0x7fffffffu) == 0u) return 0x80000000u;
    return (b >> 31) ? ~b : b | 0x80000000u;
}

// Inclusive prefix sum over a wave
__device__ __forceinline__ int wave_prefix(int v, int lane) {
#pragma unroll
    for (int x = 1; x < 64; x *= 2) {
        const int o = __shfl_up(v, x);
        if (lane >= x) v += o;
    }
    return v;
}

__global__ __launch_bounds__(kSelectThreads) void slim_cache_select_kernel(const float* __restrict__ weights, const int* __restrict__ kv_lens,
                                                                           int* __restrict__ kept, int* __restrict__ kv_lens_out, int Hkv, int T_alloc,
                                                                           int keep, int recent) {
    constexpr int BINS = 2048, WAVES = kSelectThreads / 64;
    __shared__ int hist[BINS];
    __shared__ int sumS[WAVES][2];
    __shared__ int foundS[2];
    const int tid = threadIdx.x, lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int g = blockIdx.x, b = blockIdx.y;
    const long row = (long)b * Hkv + g;
    const float* const wt = weights + row * T_alloc;
    int* const to = kept + row * keep;
    const int n = min(max(kv_lens[b], 0), T_alloc), stay = min(n, keep);
    if (g == 0 && tid == 0) kv_lens_out[b] = stay;
    for (int i = stay + tid; i < keep; i += kSelectThreads) to[i] = -1;
    if (n <= keep) {
        for (int i = tid; i < n; i += kSelectThreads) to[i] = i;
        return;
    }
    // of the first n - recent tokens the keep - recent largest
    const int among = n - recent;
    int need = keep - recent;
    unsigned prefix = 0u, known = 0u;   // bits of the smallest weight that stays, and which of them are known
    for (int pass = 0; pass < 3 && need > 0; ++pass) {
        const int shift = pass == 0 ? 21 : pass == 1 ? 10 : 0, bins = pass == 2 ? 1024 : 2048;
        for (int i = tid; i < BINS; i += kSelectThreads) hist[i] = 0;
        __syncthreads();
        for (int t = tid; t < among; t += kSelectThreads) {
            const unsigned key = weight_key(wt[t]);
            const bool in = (key & known) == prefix;
            const int bin = (int)((key >> shift) & (unsigned)(bins - 1));
            // (the lanes that have the first lane's bin count together: equal weights, zeros above all, would queue up)
            const unsigned long long all = __builtin_amdgcn_ballot_w64(in);
            if (all != 0) {
                const int first = __builtin_amdgcn_readlane(bin, __builtin_ctzll(all));
                const unsigned long long same = __builtin_amdgcn_ballot_w64(in && bin == first);
                if (in && bin != first) atomicAdd(&hist[bin], 1);
                if (lane == __builtin_ctzll(same)) atomicAdd(&hist[first], __builtin_popcountll(same));
            }
        }
        __syncthreads();
        // the bin, from the top, in which the count reaches `need`: thread i has bins from the top 2 i and 2 i + 1
        const int b0 = bins - 1 - 2 * tid, c0 = b0 >= 0 ? hist[b0] : 0, c1 = b0 >= 1 ? hist[b0 - 1] : 0;
        const int incl = wave_prefix(c0 + c1, lane);
        if (lane == 63) sumS[w][0] = incl;
        __syncthreads();
        int before = incl - c0 - c1;
        for (int i = 0; i < w; ++i) before += sumS[i][0];
        if (before < need && before + c0 >= need) foundS[0] = b0, foundS[1] = before;
        else if (before + c0 < need && before + c0 + c1 >= need) foundS[0] = b0 - 1, foundS[1] = before + c0;
        __syncthreads();
        prefix |= (unsigned)foundS[0] << shift;
        known |= (unsigned)(bins - 1) << shift;
        need -= foundS[1];
        __syncthreads();
    }
    // tokens above `prefix` stay, and the first `need` of those that have it (none stay where recent == keep)
    const bool any = keep > recent;
    int above = 0, equal = 0;   // so far
    for (int t0 = 0; t0 < among; t0 += kSelectChunk) {
        const int t = t0 + 4 * tid;
        bool up[4], eq[4];
        int a = 0, e = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const unsigned key = t + i < among ? weight_key(wt[t + i]) : 0u;
            up[i] = any && t + i < among && key > prefix;
            eq[i] = any && t + i < among && key == prefix;
            a += up[i];
            e += eq[i];
        }
        const int ia = wave_prefix(a, lane), ie = wave_prefix(e, lane);
        if (lane == 63) {
            sumS[w][0] = ia;
            sumS[w][1] = ie;
        }
        __syncthreads();
        int na = above + ia - a, ne = equal + ie - e;
        for (int i = 0; i < WAVES; ++i) {
            if (i < w) {
                na += sumS[i][0];
                ne += sumS[i][1];
            }
            above += sumS[i][0];
            equal += sumS[i][1];
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if (up[i] || (eq[i] && ne < need)) to[na + min(ne, need)] = t + i;
            na += up[i];
            ne += eq[i];
        }
        __syncthreads();
    }
    for (int i = tid; i < recent; i += kSelectThreads) to[keep - recent + i] = among + i;
}

struct EvictParams {
    const int8_t* codes[2];
    const float* scale[2];
    const float* weights;
    const int *kept, *kv_lens;
    int8_t* codes_out[2];
    float* scale_out[2];
    float* weights_out;
    int Hkv, T_alloc, keep, out_len;
};

// U rows a lane in flight
template <int D, int U>
__global__ __launch_bounds__(256) void slim_cache_copy_kernel(const EvictParams p) {
    constexpr int LPR = D / 16, ROWS = 256 / LPR;
    const int tid = threadIdx.x, c = tid % LPR, r = tid / LPR;
    const int g = blockIdx.y, b = blockIdx.z;
    const long row = (long)b * p.Hkv + g;
    const int stay = min(min(max(p.kv_lens[b], 0), p.T_alloc), p.keep);
    const int first = (int)blockIdx.x * (ROWS * U);
    for (int i = first + tid; i < min(first + ROWS * U, p.out_len); i += 256)
        if (i >= stay) p.weights_out[row * p.out_len + i] = 0.0f;
    if (first >= stay) return;
    const int* const from = p.kept + row * p.keep;
    int at[U];
#pragma unroll
    for (int u = 0; u < U; ++u) at[u] = from[min(first + u * ROWS + r, stay - 1)];
#pragma unroll
    for (int x = 0; x < 2; ++x) {
        u32x4 v[U];
#pragma unroll
        for (int u = 0; u < U; ++u) v[u] = *reinterpret_cast<const u32x4*>(p.codes[x] + (row * p.T_alloc + at[u]) * D + 16 * c);
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int i = first + u * ROWS + r;
            if (i < stay) *reinterpret_cast<u32x4*>(p.codes_out[x] + (row * p.out_len + i) * D + 16 * c) = v[u];
        }
    }
    for (int i = first + tid; i < min(first + ROWS * U, stay); i += 256) {
        const int t = from[i];
        p.scale_out[0][row * p.out_len + i] = p.scale[0][row * p.T_alloc + t];
        p.scale_out[1][row * p.out_len + i] = p.scale[1][row * p.T_alloc + t];
        p.weights_out[row * p.out_len + i] = p.weights[row * p.T_alloc + t];
    }
}

hipError_t launch_cache_evict(const EvictArgs& a, hipStream_t stream) {
    hipLaunchKernelGGL(slim_cache_select_kernel, dim3((unsigned)a.kv_heads, (unsigned)a.batch), dim3(kSelectThreads), 0, stream, a.weights,
                       a.kv_lens, a.kept, a.kv_lens_out, a.kv_heads, a.kv_len, a.keep, a.recent);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    EvictParams p;
    p.codes[0] = a.k_codes, p.codes[1] = a.v_codes;
    p.scale[0] = a.k_scale, p.scale[1] = a.v_scale;
    p.weights = a.weights, p.kept = a.kept, p.kv_lens = a.kv_lens;
    p.codes_out[0] = a.k_codes_out, p.codes_out[1] = a.v_codes_out;
    p.scale_out[0] = a.k_scale_out, p.scale_out[1] = a.v_scale_out;
    p.weights_out = a.weights_out;
    p.Hkv = a.kv_heads, p.T_alloc = a.kv_len, p.keep = a.keep, p.out_len = a.out_len;
    constexpr int U = 4;
    const int rows = 256 / (a.head_dim / 16) * U;
    const dim3 grid((unsigned)((a.out_len + rows - 1) / rows), (unsigned)a.kv_heads, (unsigned)a.batch);
    if (a.head_dim == 128) hipLaunchKernelGGL((slim_cache_copy_kernel<128, U>), grid, dim3(256), 0, stream, p);
    else hipLaunchKernelGGL((slim_cache_copy_kernel<64, U>), grid, dim3(256), 0, stream, p);
    return hipGetLastError();
}

}  // namespace slim
