// Eviction from the INT8 KV cache by accumulated attention weight: of a (sequence, KV head)'s tokens the `recent` last ones stay, and
// of the others those of largest weight, `keep` in all, in their order, which go to another cache.
//
// Two launches.  The first chooses: a workgroup for each (sequence, KV head) holds the weights in registers, as whole numbers of
// the same order, finds the smallest one that stays by its bits, 11, 11 and 10 of them (a histogram in LDS, then the bin that the
// count runs out in; no further where a whole bin stays), and numbers the tokens that stay with prefix sums.  Whole numbers only:
// no order of atomics changes a result.  It is bound by its steps' latencies, and on long rows by the unit's instructions (8 rows of 32768
// tokens: load 2.3 us, the histograms 4.2, 3.2 and 1, a bin 0.7 each, numbers 3.4).  The second copies: 16 bytes a lane, a row of codes by
// D/16 adjacent lanes, and is bound by memory: 2 (D + 4) + 4 bytes a token, read and written.
#include <type_traits>

#include "slim_common.h"
#include "slim_kernels.h"

namespace slim {

typedef float f32x4u __attribute__((ext_vector_type(4), aligned(4)));

constexpr int kSelectThreads = 1024, kSelectWaves = kSelectThreads / 64, kSelectChunk = 4 * kSelectThreads;

// A weight as a whole number of the same order: NaN below everything, the two zeros equal, none 0 (a token that has none to be chosen by)
__device__ __forceinline__ unsigned weight_key(float w) {
    const unsigned b = __float_as_uint(w), size = b & 0x7fffffffu;
    const unsigned key = (b >> 31) ? ~b : b | 0x80000000u;
    return size > 0x7f800000u ? 1u : size == 0u ? 0x80000000u : key;
}

// Inclusive prefix sum over a wave (within rows of 16 lanes, then the rows' last lanes to those behind them)
__device__ __forceinline__ int wave_prefix(int v) {
    v += __builtin_amdgcn_update_dpp(0, v, 0x111, 0xf, 0xf, false);   // row_shr:1
    v += __builtin_amdgcn_update_dpp(0, v, 0x112, 0xf, 0xf, false);   // row_shr:2
    v += __builtin_amdgcn_update_dpp(0, v, 0x114, 0xf, 0xf, false);   // row_shr:4
    v += __builtin_amdgcn_update_dpp(0, v, 0x118, 0xf, 0xf, false);   // row_shr:8
    v += __builtin_amdgcn_update_dpp(0, v, 0x142, 0xa, 0xf, false);   // row_bcast:15 to rows 1 and 3
    v += __builtin_amdgcn_update_dpp(0, v, 0x143, 0xc, 0xf, false);   // row_bcast:31 to rows 2 and 3
    return v;
}

// C chunks of 4096 weights in registers, four adjacent ones a thread and chunk.  Caches of more are gone through that many at a time, in
// every pass again.
template <int C>
__global__ __launch_bounds__(kSelectThreads) void slim_cache_select_kernel(const float* __restrict__ weights, const int* __restrict__ kv_lens,
                                                                           int* __restrict__ kept, int* __restrict__ kv_lens_out, int Hkv, int T_alloc,
                                                                           int keep, int recent) {
    constexpr int BINS = 2048, COPIES = 4, ROOM = 16384, GROUPS = C * kSelectWaves;
    static_assert(GROUPS <= 256, "four groups a lane");
    __shared__ __attribute__((aligned(16))) int hist[BINS][COPIES];   // (lanes that meet in a bin, four ways apart)
    __shared__ unsigned listS[ROOM];                                  // the weights in the first pass's bin
    __shared__ int sumS[kSelectWaves];
    __shared__ int foundS[3];
    __shared__ int listed;
    __shared__ int groupS[GROUPS];
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
    const int among = n - recent, rounds = (among + C * kSelectChunk - 1) / (C * kSelectChunk);
    u32x4 key[C];
    auto load = [&](int t0) __attribute__((always_inline)) {
        f32x4 v[C];
#pragma unroll
        for (int c = 0; c < C; ++c) {
            const int t = t0 + c * kSelectChunk + 4 * tid;
            v[c] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
            if (t + 4 <= T_alloc) v[c] = *reinterpret_cast<const f32x4u*>(wt + t);
            else
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    if (t + e < T_alloc) v[c][e] = wt[t + e];
        }
#pragma unroll
        for (int c = 0; c < C; ++c) {
#pragma unroll
            for (int e = 0; e < 4; ++e) key[c][e] = t0 + c * kSelectChunk + 4 * tid + e < among ? weight_key(v[c][e]) : 0u;
        }
    };
    // f(key) for all of them, and for 0s that fill up a wave's last 256 (for all 4096 of a chunk's, the first histogram of 2000 tokens took
    // 2.4 us and not 1.1: the 0s meet in one bin)
    auto each = [&](auto f) __attribute__((always_inline)) {
        for (int r = 0; r < rounds; ++r) {
            if (rounds > 1) load(r * C * kSelectChunk);
#pragma unroll
            for (int c = 0; c < C; ++c) {
                if ((r * C + c) * kSelectChunk + 256 * w < among) {
#pragma unroll
                    for (int e = 0; e < 4; ++e) f(key[c][e]);
                }
            }
        }
    };
    auto clear = [&]() __attribute__((always_inline)) {
        for (int i = tid; i < BINS; i += kSelectThreads) *reinterpret_cast<u32x4*>(hist[i]) = u32x4{0u, 0u, 0u, 0u};
    };
    clear();
    if (tid == 0) listed = 0;
    load(0);

    int need = keep - recent, count = -1;   // tokens that stay of those that have the known bits, and how many have them
    bool in_list = false;
    unsigned prefix = 0u, known = 0u;       // bits of the smallest weight that stays, and which of them are known
    for (int pass = 0; pass < 3 && need > 0 && count != need; ++pass) {
        const int shift = pass == 0 ? 21 : pass == 1 ? 10 : 0, bins = pass == 2 ? 1024 : BINS;
        if (pass > 0) clear();
        __syncthreads();
        int* const mine = &hist[0][lane % COPIES];
        if (pass == 0) {
            // (0 counts as well, behind all that may stay)
            each([&](unsigned k) __attribute__((always_inline)) { atomicAdd(mine + (k >> 21) * COPIES, 1); });
        } else if (in_list || (pass == 1 && count <= ROOM)) {
            if (pass == 1) {
                in_list = true;
                int have = 0;
                each([&](unsigned k) __attribute__((always_inline)) { have += (k & known) == prefix; });
                const int incl = wave_prefix(have);
                int base = 0;
                if (lane == 63) base = atomicAdd(&listed, incl);
                int at = __builtin_amdgcn_readlane(base, 63) + incl - have;
                each([&](unsigned k) __attribute__((always_inline)) {
                    if ((k & known) == prefix) listS[at++] = k;
                });
                __syncthreads();
            }
            const int m = listed;
            for (int i = tid; i < m; i += kSelectThreads) {
                const unsigned k = listS[i];
                if ((k & known) == prefix) atomicAdd(mine + ((k >> shift) & (unsigned)(bins - 1)) * COPIES, 1);
            }
        } else {   // (a bin of more: equal weights for the most part)
            each([&](unsigned k) __attribute__((always_inline)) {
                if ((k & known) == prefix) atomicAdd(mine + ((k >> shift) & (unsigned)(bins - 1)) * COPIES, 1);
            });
        }
        __syncthreads();
        // the bin, from the top, in which the count reaches `need`: thread i has bins from the top 2 i and 2 i + 1
        const int b0 = bins - 1 - 2 * tid;
        int c0 = 0, c1 = 0;
        if (b0 > 0) {
            const u32x4 x = *reinterpret_cast<const u32x4*>(hist[b0]), y = *reinterpret_cast<const u32x4*>(hist[b0 - 1]);
            c0 = (int)(x[0] + x[1] + x[2] + x[3]);
            c1 = (int)(y[0] + y[1] + y[2] + y[3]);
        }
        const int incl = wave_prefix(c0 + c1);
        if (lane == 63) sumS[w] = incl;
        __syncthreads();
        int before = incl - c0 - c1;
#pragma unroll
        for (int i = 0; i < kSelectWaves; ++i) before += i < w ? sumS[i] : 0;
        if (before < need && before + c0 >= need) foundS[0] = b0, foundS[1] = before, foundS[2] = c0;
        else if (before + c0 < need && before + c0 + c1 >= need) foundS[0] = b0 - 1, foundS[1] = before + c0, foundS[2] = c1;
        __syncthreads();
        prefix |= (unsigned)foundS[0] << shift;
        known |= (unsigned)(bins - 1) << shift;
        need -= foundS[1];
        count = foundS[2];
    }
    if (keep == recent) prefix = known = 0xffffffffu;   // (none of them; no weight has these bits)
    // Tokens from `prefix` on stay, where all of those that have its bits do (bits that are not known are 0 in it); else those above it and the
    // first `need` of those that have them, counted together: those above in the low half (a round has at most 2^16 - 2^12 tokens),
    // the others in the high one.  (One comparison a token, not two and their counts: of 8 rows of 32768 tokens' choice 3.4 us in the place of
    // 6.1.)
    static_assert(C * kSelectChunk < 65536, "a round's counts fit 16 bits");
    auto number = [&](auto ties_c) __attribute__((always_inline)) {
        constexpr bool TIES = decltype(ties_c)::value;
        int above = 0, equal = 0;   // so far
        for (int r = 0; r < rounds; ++r) {
            if (rounds > 1) load(r * C * kSelectChunk);
            int mine[C], before[C];
#pragma unroll
            for (int c = 0; c < C; ++c) {
                mine[c] = 0;
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    mine[c] += TIES ? (key[c][e] > prefix ? 1 : key[c][e] == prefix ? 65536 : 0) : key[c][e] >= prefix;
                before[c] = wave_prefix(mine[c]);
                if (lane == 63) groupS[c * kSelectWaves + w] = before[c];
                before[c] -= mine[c];
            }
            __syncthreads();
            // every wave: lane l has groups 4 l to 4 l + 3 (in the order of their tokens)
            int of[4], sum = 0;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                of[i] = 4 * lane + i < GROUPS ? groupS[4 * lane + i] : 0;
                sum += of[i];
            }
            const int incl = wave_prefix(sum);
            int base = incl - sum;   // before this lane's group of this wave's number: those of the lanes before, and of its own
#pragma unroll
            for (int i = 0; i < 3; ++i) base += i < (w & 3) ? of[i] : 0;
#pragma unroll
            for (int c = 0; c < C; ++c) {
                before[c] += __builtin_amdgcn_readlane(base, (c * kSelectWaves + w) >> 2);
                const int t = (r * C + c) * kSelectChunk + 4 * tid;
                if constexpr (TIES) {
                    int na = above + (before[c] & 0xffff), ne = equal + (int)((unsigned)before[c] >> 16);
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const bool up = key[c][e] > prefix, eq = key[c][e] == prefix;
                        if (up || (eq && ne < need)) to[na + min(ne, need)] = t + e;
                        na += up;
                        ne += eq;
                    }
                } else {
                    unsigned at = (unsigned)(above + before[c]);
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        if (key[c][e] >= prefix) to[at++] = t + e;
                }
            }
            const int total = __builtin_amdgcn_readlane(incl, 63);
            above += total & 0xffff;
            equal += (int)((unsigned)total >> 16);
            __syncthreads();
        }
    };
    if (count != need && keep != recent) number(std::true_type{});   // (then all the bits are known)
    else number(std::false_type{});
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
    int Hkv, T_alloc, keep, out_len, n_copy;
};

// Workgroups below n_copy copy U rows a lane, all of their loads in flight; the others clear 4096 weights past what stays.
constexpr int kClear = 4096;
template <int D, int U>
__global__ __launch_bounds__(256) void slim_cache_copy_kernel(const EvictParams p) {
    constexpr int LPR = D / 16, ROWS = 256 / LPR;
    const int tid = threadIdx.x, c = tid % LPR, r = tid / LPR;
    const int g = blockIdx.y, b = blockIdx.z;
    const long row = (long)b * p.Hkv + g;
    const int stay = min(min(max(p.kv_lens[b], 0), p.T_alloc), p.keep);
    if ((int)blockIdx.x >= p.n_copy) {
        const int first = ((int)blockIdx.x - p.n_copy) * kClear, end = min(first + kClear, p.out_len);
        for (int i = max(first, stay) + tid; i < end; i += 256) p.weights_out[row * p.out_len + i] = 0.0f;
        return;
    }
    const int first = (int)blockIdx.x * (ROWS * U);
    if (first >= stay) return;
    const int* const from = p.kept + row * p.keep;
    int at[U];
#pragma unroll
    for (int u = 0; u < U; ++u) at[u] = from[min(first + u * ROWS + r, stay - 1)];
    static_assert(ROWS * U <= 256, "a thread has at most one token's scales");
    const bool scalar = tid < ROWS * U && first + tid < stay;
    const long mine = row * p.T_alloc + from[scalar ? first + tid : first];
    u32x4 v[2][U];
#pragma unroll
    for (int x = 0; x < 2; ++x)
#pragma unroll
        for (int u = 0; u < U; ++u)
            v[x][u] = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(p.codes[x] + (row * p.T_alloc + at[u]) * D + 16 * c));
    const float s0 = p.scale[0][mine], s1 = p.scale[1][mine], wt = p.weights[mine];
#pragma unroll
    for (int x = 0; x < 2; ++x)
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int i = first + u * ROWS + r;
            if (i < stay) __builtin_nontemporal_store(v[x][u], reinterpret_cast<u32x4*>(p.codes_out[x] + (row * p.out_len + i) * D + 16 * c));
        }
    if (scalar) {
        const long i = row * p.out_len + first + tid;
        p.scale_out[0][i] = s0;
        p.scale_out[1][i] = s1;
        p.weights_out[i] = wt;
    }
}

hipError_t launch_cache_evict(const EvictArgs& a, hipStream_t stream) {
    auto select = [&](auto c_c) {
        hipLaunchKernelGGL(slim_cache_select_kernel<decltype(c_c)::value>, dim3((unsigned)a.kv_heads, (unsigned)a.batch), dim3(kSelectThreads), 0,
                           stream, a.weights, a.kv_lens, a.kept, a.kv_lens_out, a.kv_heads, a.kv_len, a.keep, a.recent);
        return hipGetLastError();
    };
    using std::integral_constant;
    const hipError_t e = a.kv_len <= 2 * kSelectChunk ? select(integral_constant<int, 2>{}) : select(integral_constant<int, 8>{});
    if (e != hipSuccess) return e;
    EvictParams p;
    p.codes[0] = a.k_codes, p.codes[1] = a.v_codes;
    p.scale[0] = a.k_scale, p.scale[1] = a.v_scale;
    p.weights = a.weights, p.kept = a.kept, p.kv_lens = a.kv_lens;
    p.codes_out[0] = a.k_codes_out, p.codes_out[1] = a.v_codes_out;
    p.scale_out[0] = a.k_scale_out, p.scale_out[1] = a.v_scale_out;
    p.weights_out = a.weights_out;
    p.Hkv = a.kv_heads, p.T_alloc = a.kv_len, p.keep = a.keep, p.out_len = a.out_len;
    constexpr int U = 2;
    const int rows = 256 / (a.head_dim / 16) * U;
    p.n_copy = (a.keep + rows - 1) / rows;
    const dim3 grid((unsigned)(p.n_copy + (a.out_len + kClear - 1) / kClear), (unsigned)a.kv_heads, (unsigned)a.batch);
    if (a.head_dim == 128) hipLaunchKernelGGL((slim_cache_copy_kernel<128, U>), grid, dim3(256), 0, stream, p);
    else hipLaunchKernelGGL((slim_cache_copy_kernel<64, U>), grid, dim3(256), 0, stream, p);
    return hipGetLastError();
}

}  // namespace slim
