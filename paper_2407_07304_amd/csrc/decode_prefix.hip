// Decode attention of a batch whose sequences share a long prefix: one query token a sequence attends to the prefix's tokens,
// cached once for all of them, and to its sequence's own.
//
//     o = (sum over the prefix + sum over the own tokens) / (the same of the probabilities),
//
// a softmax over both parts, which only the merge of the records joins.  The prefix's part is, for each KV head, a product of
// (batch x query heads of the KV head) rows: the cache is read once for 128 of them in the place of once a sequence, and from
// some 200 rows on the matrix cores bound it.  The own part is what it is in any decode: bound by memory.  Both are one
// launch, the prefix's workgroups first, so that the one's arithmetic runs beside the other's loads.
//
// A workgroup (four waves) of the prefix has a run of its tokens for
//   - up to 32 rows: the sweep of the grouped decode (decode_sweep.h), the waves' tiles merged in LDS;
//   - up to 128 rows, 32 a wave: a stage of tokens, widened to bf16 on its way into LDS by all waves and used by all, two
//     stages in turn, one barrier each; S^T = K Q^T and O^T += V^T P^T with v_mfma_f32_32x32x16_bf16, V^T through the LDS
//     transpose read.  Up to 64 rows, two waves have the rows and two the same rows over every other tile, with records
//     of their own.
// One of the own caches has a run of a (sequence, KV head)'s tokens for its query heads, up to 32.
#include <algorithm>
#include <type_traits>

#include "decode_sweep.h"
#include "slim_common.h"
#include "slim_kernels.h"

namespace slim {

// LDS of the form with shared tiles: two stages of K and V rows (padded so that row reads and transpose reads spread over the
// banks) and of their scales
template <int D, int RG>
struct PrefixLds {
    static constexpr int PHASES = 4 / RG;                                            // tiles of 32 tokens at a time
    static constexpr int STAGE = 32 * PHASES > 4096 / D ? 32 * PHASES : 4096 / D;    // tokens: a 128-bit load of K or V a thread, or two
    static constexpr int PITCHK = 2 * D + 16, PITCHV = 2 * D + 64;
    static constexpr int STAGE_BYTES = STAGE * (PITCHK + PITCHV) + 8 * STAGE;
    static constexpr int BYTES = 2 * STAGE_BYTES;
};

// RG groups of 32 rows (2 or 4), q_row(i) row i's queries, record(i, phase) the index of its record; tokens [t_begin, t_end) of the T
template <int D, int RG, class QRow, class Record>
__device__ __forceinline__ void prefix_sweep(char* const smem, const QRow q_row, const int n_rows, const int8_t* kc, const float* ks,
                                             const int8_t* vc, const float* vs, const int T, const int t_begin, const int t_end,
                                             const float scale_log2e, const Record record, float* ws_acc, float* ws_ml) {
    using Lds = PrefixLds<D, RG>;
    constexpr int KS = D / 16, DT = D / 32;            // k-steps of the score MFMA, 32-row tiles of O^T
    constexpr int STAGE = Lds::STAGE, PHASES = Lds::PHASES, PITCHK = Lds::PITCHK, PITCHV = Lds::PITCHV;
    constexpr int NP = STAGE * D / 4096;               // 128-bit loads a thread, stage and tensor
    constexpr int SUB = STAGE / (32 * PHASES);         // tiles a wave and stage
    const int tid = threadIdx.x, lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int l32 = lane & 31, hh = lane >> 5;
    const int rg = w % RG, phase = w / RG;
    const bool busy = 32 * rg < n_rows;                // (uniform)

    // Q^T B operands: lane holds row l32, d = 16 s + 8 hh + [0,8)
    bf16x8 qB[KS];
    {
        const uint16_t* qp = q_row(min(32 * rg + l32, n_rows - 1)) + 8 * hh;
#pragma unroll
        for (int s = 0; s < KS; ++s) qB[s] = *reinterpret_cast<const bf16x8*>(qp + 16 * s);
    }
    const __amdgpu_buffer_rsrc_t krs = __builtin_amdgcn_make_buffer_rsrc((void*)kc, 0, (int)((unsigned)T * D), 0x00020000);
    const __amdgpu_buffer_rsrc_t vrs = __builtin_amdgcn_make_buffer_rsrc((void*)vc, 0, (int)((unsigned)T * D), 0x00020000);
    const __amdgpu_buffer_rsrc_t ksr = __builtin_amdgcn_make_buffer_rsrc((void*)ks, 0, (int)((unsigned)T * 4u), 0x00020000);
    const __amdgpu_buffer_rsrc_t vsr = __builtin_amdgcn_make_buffer_rsrc((void*)vs, 0, (int)((unsigned)T * 4u), 0x00020000);
    u32x4 kbuf[NP], vbuf[NP];
    uint32_t sc = 0u;
    // (rows past the end of the prefix read as zeros and are masked; threads without a scale ask past the end)
    const int off_ks = tid < STAGE ? tid * 4 : (int)0x7ffffff0, off_vs = tid >= 64 && tid < 64 + STAGE ? (tid - 64) * 4 : (int)0x7ffffff0;
    auto issue = [&](int t0) {
        const int base = t0 < t_end ? t0 : T;          // (a stage that is not wanted: nothing is read)
#pragma unroll
        for (int n = 0; n < NP; ++n) {
            kbuf[n] = __builtin_amdgcn_raw_buffer_load_b128(krs, (int)((unsigned)base * D + (unsigned)(tid * 16 + n * 4096)), 0, 0);
            vbuf[n] = __builtin_amdgcn_raw_buffer_load_b128(vrs, (int)((unsigned)base * D + (unsigned)(tid * 16 + n * 4096)), 0, 0);
        }
        sc = __builtin_amdgcn_raw_buffer_load_b32(ksr, off_ks + base * 4, 0, 0) | __builtin_amdgcn_raw_buffer_load_b32(vsr, off_vs + base * 4, 0, 0);
    };
    auto widen16 = [&](const u32x4 c, char* to) {      // 16 codes -> 16 bf16, exact
        *reinterpret_cast<bf16x8*>(to) = widen8(i32x2{(int)c[0], (int)c[1]});
        *reinterpret_cast<bf16x8*>(to + 16) = widen8(i32x2{(int)c[2], (int)c[3]});
    };
    auto stage = [&](char* buf) {
        char* const vS = buf + STAGE * PITCHK;
#pragma unroll
        for (int n = 0; n < NP; ++n) {
            const int at = tid * 16 + n * 4096, row = at / D, col = at % D;
            widen16(kbuf[n], buf + row * PITCHK + col * 2);
            widen16(vbuf[n], vS + row * PITCHV + col * 2);
        }
        float* const scS = reinterpret_cast<float*>(vS + STAGE * PITCHV);   // [0, STAGE) k_scale * c, then v_scale
        const float s = __uint_as_float(sc);
        if (tid < STAGE) scS[tid] = s * scale_log2e;
        else if (tid >= 64 && tid < 64 + STAGE) scS[STAGE + tid - 64] = s;
    };
    static_assert(STAGE <= 64, "a wave has the K scales, the next one the V scales");

    const int k_addr = l32 * PITCHK + 16 * hh;   // K fragment of k-step s: row l32, bytes 32 s + 16 hh + [0,16)
    // V transpose reads: 16 lanes fetch rows k..k+3, lane i receives column i of them
    const int v_addr = (4 * hh + ((lane & 15) >> 2)) * PITCHV + (2 * ((lane >> 4) & 1) + ((lane & 3) >> 1)) * 16 + 8 * (lane & 1);
    f32x16 o[DT];
#pragma unroll
    for (int dt = 0; dt < DT; ++dt)
#pragma unroll
        for (int r = 0; r < 16; ++r) o[dt][r] = 0.0f;
    float M = kMasked, lsum = 0.0f;   // running max of this lane's row (log2 units), this lane's part of the row sum

    issue(t_begin);
    stage(smem);
    issue(t_begin + STAGE);
    __syncthreads();
    int turn = 0;
    for (int t0 = t_begin; t0 < t_end; t0 += STAGE, turn ^= 1) {
        const char* const kS = smem + turn * Lds::STAGE_BYTES;
        const char* const vS = kS + STAGE * PITCHK;
        const float* const scS = reinterpret_cast<const float*>(vS + STAGE * PITCHV);
        stage(smem + (turn ^ 1) * Lds::STAGE_BYTES);   // (the other stage: every wave is done with it since the last barrier)
        issue(t0 + 2 * STAGE);
#pragma unroll
        for (int x = 0; x < SUB; ++x) {
            const int tile = (phase + x * PHASES) * 32, tt = t0 + tile;
            if (!busy || tt >= t_end) continue;        // (uniform)
            const char* const kT = kS + tile * PITCHK;
            const char* const vT = vS + tile * PITCHV;
            f32x16 acc;
#pragma unroll
            for (int r = 0; r < 16; ++r) acc[r] = 0.0f;
#pragma unroll
            for (int s = 0; s < KS; ++s)
                acc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(*reinterpret_cast<const bf16x8*>(kT + k_addr + 32 * s), qB[s], acc, 0, 0, 0);
            // register r of this lane is token tt + 8 (r/4) + 4 hh + r%4
            float u[16];
#pragma unroll
            for (int r4 = 0; r4 < 4; ++r4) {
                const f32x4 f = *reinterpret_cast<const f32x4*>(&scS[tile + 8 * r4 + 4 * hh]);
#pragma unroll
                for (int e = 0; e < 4; ++e) u[4 * r4 + e] = acc[4 * r4 + e] * f[e];
            }
            if (tt + 32 > T) {
#pragma unroll
                for (int r = 0; r < 16; ++r) u[r] = tt + 8 * (r / 4) + 4 * hh + r % 4 < T ? u[r] : kMasked;
            }
            float umax = fmaxf(u[0], u[1]);
#pragma unroll
            for (int r = 2; r < 16; r += 2) umax = fmaxf(umax, fmaxf(u[r], u[r + 1]));
            // the running max, a whole number (decode_gqa.hip says why), moves only when a score has passed it by 2^8
            if (__builtin_amdgcn_ballot_w64(umax - M > 8.0f) != 0) {
                const float m_new = ceilf(fmaxf(M, half_max(umax)));
                const float alpha = fast_exp2(M - m_new);
#pragma unroll
                for (int dt = 0; dt < DT; ++dt)
#pragma unroll
                    for (int r = 0; r < 16; ++r) o[dt][r] *= alpha;
                lsum *= alpha;
                M = m_new;
            }
            float ps0 = 0.0f, ps1 = 0.0f;
#pragma unroll
            for (int r = 0; r < 16; r += 2) {
                u[r] = fast_exp2(u[r] - M);
                u[r + 1] = fast_exp2(u[r + 1] - M);
                ps0 += u[r];
                ps1 += u[r + 1];
            }
            lsum += ps0 + ps1;
            // the probabilities take their token's v_scale before they are rounded to bf16, operands of the second product
            u32x4 pw[2];
#pragma unroll
            for (int r4 = 0; r4 < 4; ++r4) {
                const f32x4 f = *reinterpret_cast<const f32x4*>(&scS[STAGE + tile + 8 * r4 + 4 * hh]);
                pw[r4 >> 1][2 * (r4 & 1)] = pack_bf16x2(u[4 * r4] * f[0], u[4 * r4 + 1] * f[1]);
                pw[r4 >> 1][2 * (r4 & 1) + 1] = pack_bf16x2(u[4 * r4 + 2] * f[2], u[4 * r4 + 3] * f[3]);
            }
            // O^T += V^T P^T: k-step u2 covers tokens 16 u2 + {4 hh .. 4 hh + 3} and 16 u2 + 8 + {4 hh .. 4 hh + 3} of the tile
#pragma unroll
            for (int u2 = 0; u2 < 2; ++u2)
#pragma unroll
                for (int dt = 0; dt < DT; ++dt) {
                    const char* va = vT + v_addr + 64 * dt + 16 * u2 * PITCHV;
                    const s16x4 lo = lds_read_tr16(reinterpret_cast<const uint16_t*>(va));
                    const s16x4 hi = lds_read_tr16(reinterpret_cast<const uint16_t*>(va + 8 * PITCHV));
                    const s16x8 av = {lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]};
                    o[dt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, av), __builtin_bit_cast(bf16x8, pw[u2]), o[dt], 0, 0, 0);
                }
        }
        __syncthreads();
    }
    const float L = half_sum(lsum);
    const int row = 32 * rg + l32;
    if (row < n_rows) {
        const long idx = record(row, phase);
#pragma unroll
        for (int dt = 0; dt < DT; ++dt)
#pragma unroll
            for (int r4 = 0; r4 < 4; ++r4)
                *reinterpret_cast<f32x4*>(ws_acc + idx * D + 32 * dt + 8 * r4 + 4 * hh) =
                    f32x4{o[dt][4 * r4], o[dt][4 * r4 + 1], o[dt][4 * r4 + 2], o[dt][4 * r4 + 3]};
        if (hh == 0) reinterpret_cast<f32x2*>(ws_ml)[idx] = f32x2{M, L};
    }
}

// Own tokens a split takes (2^32 / 256 of splits_of's units a token); an own cache has no more splits than its tokens make
constexpr unsigned kOwnSplitRate = 1u << 24;

struct PrefixParams {
    const uint16_t* q;
    const int8_t *pkc, *pvc, *kc, *vc;   // the prefix's cache, the sequences' own
    const float *pks, *pvs, *ks, *vs;
    const int* kv_lens;
    uint16_t* out;
    float *ws_acc, *ws_ml;
    int batch, Hkv, G, P, T_alloc;
    int n_blocks, n_prefix, row_blocks, head_groups, n_own, n_records;   // workgroups of the prefix; its splits; ...
    float scale_log2e;
};

// FORM: rows of the prefix's workgroups: 1, 2: 16 or 32, waves of their own; 3, 4: 64 or 128, shared tiles.  NC: groups of 16 query
// heads of the own caches' workgroups.
template <int D, int FORM, int NC>
__global__ __launch_bounds__(256) void slim_decode_prefix_kernel(const PrefixParams p) {
    constexpr int RG = FORM == 4 ? 4 : 2;
    constexpr int OWN_LDS = 4 * GqaLds<D, NC>::WAVE_BYTES;
    constexpr int SHARED_LDS = FORM >= 3 ? PrefixLds<D, RG>::BYTES : 4 * GqaLds<D, (FORM < 3 ? FORM : 1)>::WAVE_BYTES;
    __shared__ __attribute__((aligned(16))) char smem[OWN_LDS > SHARED_LDS ? OWN_LDS : SHARED_LDS];
    const int tid = threadIdx.x, lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int Hq = p.G * p.Hkv;
    const int id = (int)blockIdx.x;
    auto nothing = [](int, int, const float (&)[8]) {};

    if (id < p.n_blocks) {   // the prefix: heads in turn (XCDs take workgroups in turn), then row blocks, then splits
        const int g = id % p.Hkv, x = id / p.Hkv, rb = x % p.row_blocks, sp = x / p.row_blocks;
        const int row0 = rb * 128, n_rows = min(p.batch * p.G - row0, 128);
        const long kv0 = (long)g * p.P;
        auto row_of = [&](int i) {   // the query row that row i of this block is: sequence by sequence
            const int r = row0 + i, b = r / p.G;
            return (long)b * Hq + g * p.G + (r - b * p.G);
        };
        if constexpr (FORM >= 3) {
            constexpr int STAGE = PrefixLds<D, RG>::STAGE, PHASES = PrefixLds<D, RG>::PHASES;
            int first, end;
            split_span((p.P + STAGE - 1) / STAGE, p.n_prefix / PHASES, sp, first, end);
            prefix_sweep<D, RG>(smem, [&](int i) { return p.q + row_of(i) * D; }, n_rows, p.pkc + kv0 * D, p.pks + kv0, p.pvc + kv0 * D,
                                p.pvs + kv0, p.P, first * STAGE, min(end * STAGE, p.P), p.scale_log2e,
                                [&](int i, int phase) { return row_of(i) * p.n_records + sp * PHASES + phase; }, p.ws_acc, p.ws_ml);
        } else {
            int first, end;
            split_span((p.P + kGqaTile - 1) / kGqaTile, p.n_prefix, sp, first, end);
            first += w;
            f32x4 o[FORM][D / 16];
            float M[FORM], lsum[FORM];
            char* const kS = smem + w * GqaLds<D, FORM>::WAVE_BYTES;
            gqa_sweep<D, 4, FORM, false>(kS, lane, [&](int i) { return p.q + row_of(min(i, n_rows - 1)) * D; }, p.pkc + kv0 * D, p.pks + kv0,
                                         p.pvc + kv0 * D, p.pvs + kv0, p.P, first, first < end ? (end - first + 3) / 4 : 0, p.scale_log2e,
                                         nothing, o, M, lsum);
            gqa_record<D, FORM>(kS, lane, o, M, lsum);
            __syncthreads();
            for (int i = tid; i < n_rows * D; i += 256) {
                float acc, top, L;
                gqa_merged<D, 4, FORM>(smem, i / D, i % D, acc, top, L);
                store_record<D>(p.ws_acc, p.ws_ml, row_of(i / D) * p.n_records + sp, i % D, acc, top, L, false);
            }
        }
        return;
    }
    const int x = id - p.n_blocks, so = x % p.n_own, y = x / p.n_own;
    const int hg = y % p.head_groups, bg = y / p.head_groups, g = bg % p.Hkv, b = bg / p.Hkv;
    const int T = min(max(p.kv_lens[b], 0), p.T_alloc);
    if (T == 0) return;
    const int n_used = splits_of(T, p.n_own, kOwnSplitRate);
    if (so >= n_used) return;
    const int h0 = hg * 32, heads = min(p.G - h0, 32);
    const long row0 = (long)b * Hq + g * p.G + h0, kv0 = ((long)b * p.Hkv + g) * (long)p.T_alloc;
    int first, end;
    split_span((T + kGqaTile - 1) / kGqaTile, n_used, so, first, end);
    first += w;
    f32x4 o[NC][D / 16];
    float M[NC], lsum[NC];
    char* const kS = smem + w * GqaLds<D, NC>::WAVE_BYTES;
    gqa_sweep<D, 4, NC, false>(kS, lane, [&](int i) { return p.q + (row0 + min(i, heads - 1)) * D; }, p.kc + kv0 * D, p.ks + kv0, p.vc + kv0 * D,
                               p.vs + kv0, T, first, first < end ? (end - first + 3) / 4 : 0, p.scale_log2e, nothing, o, M, lsum);
    gqa_record<D, NC>(kS, lane, o, M, lsum);
    __syncthreads();
    for (int i = tid; i < heads * D; i += 256) {
        float acc, top, L;
        gqa_merged<D, 4, NC>(smem, i / D, i % D, acc, top, L);
        store_record<D>(p.ws_acc, p.ws_ml, (row0 + i / D) * p.n_records + p.n_prefix + so, i % D, acc, top, L, false);
    }
}

template <int D, int WAVES, int U>
__global__ __launch_bounds__(256) void slim_decode_prefix_combine_kernel(const PrefixParams p) {
    const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
    const int Hq = p.G * p.Hkv;
    const long row = (long)blockIdx.x * (4 / WAVES) + (WAVES == 1 ? w : 0);
    if (row >= (long)p.batch * Hq) return;
    const int T = min(max(p.kv_lens[(unsigned)row / (unsigned)Hq], 0), p.T_alloc);
    const int n_used = p.n_prefix + (T == 0 ? 0 : splits_of(T, p.n_own, kOwnSplitRate));
    combine_row<D, WAVES, U>(reinterpret_cast<const f32x2*>(p.ws_ml) + row * p.n_records, reinterpret_cast<const f32x4*>(p.ws_acc) + row * p.n_records * (D / 4),
                             p.out + row * D, n_used, lane, w);
}

struct PrefixPlan {
    int form, row_blocks, n_prefix, n_own, head_groups;
};

static PrefixPlan prefix_plan(int batch, int q_heads, int kv_heads, int prefix_len, int kv_len, int head_dim) {
    const int G = q_heads / kv_heads;
    const long rows = (long)batch * G;
    PrefixPlan plan;
    plan.form = rows <= 16 ? 1 : rows <= 32 ? 2 : rows <= 64 ? 3 : 4;
    plan.row_blocks = (int)((rows + 127) / 128);
    plan.head_groups = (G + 31) / 32;
    const int phases = plan.form == 3 ? 2 : 1;
    const long items = (long)kv_heads * plan.row_blocks, stage = plan.form < 3 ? 128 : plan.form == 3 ? 64 : 4096 / head_dim;
    const long most = (prefix_len + stage * 4 - 1) / (stage * 4);
    long n = (512 + items - 1) / items;
    n = n < most ? n : most;
    plan.n_prefix = (int)(n < 1 ? 1 : n) * phases;
    const long own = (long)batch * kv_heads * plan.head_groups;
    n = (512 + own - 1) / own;
    const long most_own = ((long)kv_len + 255) / 256;
    n = n < most_own ? n : most_own;
    plan.n_own = (int)(n < 1 ? 1 : n);
    return plan;
}

bool decode_prefix_fits(int batch, int q_heads, int kv_heads, int prefix_len, int kv_len, int head_dim) {
    const PrefixPlan plan = prefix_plan(batch, q_heads, kv_heads, prefix_len, kv_len, head_dim);
    // (a launch has less than 2^32 threads)
    return (long)kv_heads * plan.row_blocks * plan.n_prefix + (long)batch * kv_heads * plan.head_groups * plan.n_own < (1L << 24) &&
           (long)batch * q_heads < (1L << 24);
}

size_t decode_prefix_workspace_bytes(int batch, int q_heads, int kv_heads, int prefix_len, int kv_len, int head_dim) {
    const PrefixPlan plan = prefix_plan(batch, q_heads, kv_heads, prefix_len, kv_len, head_dim);
    return decode_records_bytes((long)batch * q_heads, plan.n_prefix + plan.n_own, head_dim);
}

hipError_t launch_decode_prefix(const PrefixArgs& a, hipStream_t stream) {
    const PrefixPlan plan = prefix_plan(a.batch, a.q_heads, a.kv_heads, a.prefix_len, a.kv_len, a.head_dim);
    PrefixParams p;
    p.q = (const uint16_t*)a.q;
    p.pkc = a.prefix_k_codes, p.pks = a.prefix_k_scale, p.pvc = a.prefix_v_codes, p.pvs = a.prefix_v_scale;
    p.kc = a.k_codes, p.ks = a.k_scale, p.vc = a.v_codes, p.vs = a.v_scale;
    p.kv_lens = a.kv_lens;
    p.out = (uint16_t*)a.out;
    p.batch = a.batch, p.Hkv = a.kv_heads, p.G = a.q_heads / a.kv_heads, p.P = a.prefix_len, p.T_alloc = a.kv_len;
    p.row_blocks = plan.row_blocks, p.head_groups = plan.head_groups, p.n_prefix = plan.n_prefix, p.n_own = plan.n_own;
    p.n_records = plan.n_prefix + plan.n_own;
    p.ws_acc = a.workspace;
    p.ws_ml = a.workspace + (size_t)a.batch * a.q_heads * p.n_records * a.head_dim;
    p.scale_log2e = a.softmax_scale * kLog2e;
    p.n_blocks = a.kv_heads * plan.row_blocks * (plan.form == 3 ? plan.n_prefix / 2 : plan.n_prefix);
    const unsigned grid = (unsigned)(p.n_blocks + (long)a.batch * a.kv_heads * plan.head_groups * plan.n_own);
    const long rows = (long)a.batch * a.q_heads;
    using std::integral_constant;
    auto with_d = [&](auto d_c) {
        constexpr int D = decltype(d_c)::value, RPW = 256 / D;
        auto sweep = [&](auto form_c, auto nc_c) {
            hipLaunchKernelGGL((slim_decode_prefix_kernel<D, decltype(form_c)::value, decltype(nc_c)::value>), dim3(grid), dim3(256), 0, stream, p);
            return hipGetLastError();
        };
        auto with_form = [&](auto form_c) {
            return p.G > 16 ? sweep(form_c, integral_constant<int, 2>{}) : sweep(form_c, integral_constant<int, 1>{});
        };
        const hipError_t e = plan.form == 1   ? with_form(integral_constant<int, 1>{})
                             : plan.form == 2 ? with_form(integral_constant<int, 2>{})
                             : plan.form == 3 ? with_form(integral_constant<int, 3>{})
                                              : with_form(integral_constant<int, 4>{});
        if (e != hipSuccess) return e;
        auto combine = [&](auto waves_c, auto u_c) {
            constexpr int WAVES = decltype(waves_c)::value, U = decltype(u_c)::value;
            hipLaunchKernelGGL((slim_decode_prefix_combine_kernel<D, WAVES, U>), dim3((unsigned)((rows * WAVES + 3) / 4)), dim3(256), 0, stream, p);
            return hipGetLastError();
        };
        const integral_constant<int, 1> one{};
        const integral_constant<int, 4> four{};
        if (p.n_records <= 2 * RPW) return combine(one, integral_constant<int, 2>{});
        if (p.n_records <= 4 * RPW) return combine(one, four);
        return combine(four, four);
    };
    return a.head_dim == 128 ? with_d(integral_constant<int, 128>{}) : with_d(integral_constant<int, 64>{});
}

}  // namespace slim
