// Decode attention of a batch whose sequences share a long prefix: one query token a sequence attends to the prefix's tokens,
// cached once for all of them, and to its sequence's own.
//
//     o = (sum over the prefix + sum over the own tokens) / (the same of the probabilities),
//
// a softmax over both parts, which only the merge of the records joins.  The prefix's part is, for each KV head, a product of
// (batch x query heads of the KV head) rows: the cache is read once for 128 of them in the place of once a sequence, and from
// some 200 rows on vector issue bounds it, beside the matrix cores.  The own part is what it is in any decode: bound by memory.  Both are one
// launch, the prefix's workgroups first, so that the one's arithmetic runs beside the other's loads.
//
// A workgroup (four waves) of the prefix has a run of its tokens for
//   - up to 32 rows: the sweep of the grouped decode (decode_sweep.h), the waves' tiles merged in LDS;
//   - up to 128 rows, 32 a wave: a stage of tokens, widened to bf16 on its way into LDS by all waves and used by all, two
//     stages in turn, one barrier each; S^T = K Q^T and O^T += V^T P^T with v_mfma_f32_32x32x16_bf16, V^T through the LDS
//     transpose read.  Up to 64 rows, two waves have the rows and two the same rows over every other tile, with records
//     of their own.
// One of the own caches has a run of a (sequence, KV head)'s tokens for its query heads, up to 32.
// Probabilities times v_scale are operands of the second product.  Up to 16 rows, where memory and latency bound the call, they are two bf16
// each and results have the bits of fp32 probabilities; 14 shapes took 4 % less to 2 % more than with one (4 sequences, 32 on 8 heads, P=1000
// 9.4 and 9.5 us, P=30000 19.0 both; 16, 32 heads, P=4000, T=2000 38.2 and 39.0).  Above, they are rounded to one, as in the prefill and the
// grouped decode: each is off by up to 2^-8 of itself, a result by 1.4 times what its own rounding to bf16 makes.  Two would cost up to 9 % with
// 32 rows (8 sequences, 32 on 8 heads, P=30000 22.5 -> 24.2) and a fifth with more (64, 64 on 8, P=32768 98 -> 118; 48, 32 on 8, P=8192, T=1000
// 34.0 -> 37.2).
#include <algorithm>
#include <type_traits>

#include "decode_sweep.h"
#include "slim_common.h"
#include "slim_kernels.h"

namespace slim {

// LDS of the form with shared tiles: two stages of 64 tokens' K and V rows (padded so that row reads and transpose reads spread over
// the banks) and of their scales
template <int D>
struct PrefixLds {
    static constexpr int STAGE = 64;
    static constexpr int PITCHK = 2 * D + 16, PITCHV = 2 * D + 64;
    static constexpr int STAGE_BYTES = STAGE * (PITCHK + PITCHV) + 16 * STAGE;   // (64 floats a wave, of which two have something to say)
    static constexpr int BYTES = 2 * STAGE_BYTES;
};

// RG groups of 32 rows: 4, a wave has a stage's two tiles, or 2, and a wave has one of them (phase 0 or 1).  q_row(i): row i's queries,
// record(i, phase): the index of its record; tokens [t_begin, t_end) of the T.
// What a tile costs a wave: 16 matrix instructions (512 cycles of D = 128) and some 150 vector ones, 16 exponentials among them (and 48 of
// the codes' conversion, of which a workgroup's waves have a fourth each).  In the order of the formulas the one waits for the other and
// both for LDS, and two waves a SIMD do not fill that; so the steps of both products carry, one for one, a piece of something else: the
// first's the conversion of the next stage, the second's the exponentials of the tokens behind.  64 sequences, 64 on 8 heads, P=32768, T=1: 96 us;
// without the matrix instructions 74, without the conversion 86, the exponentials 91, the scales' reads 92, the stages' loads 95.
template <int D, int RG, class QRow, class Record>
__device__ __forceinline__ void prefix_sweep(char* const smem, const QRow q_row, const int n_rows, const int8_t* kc, const float* ks,
                                             const int8_t* vc, const float* vs, const int T, const int t_begin, const int t_end,
                                             const float scale_log2e, const Record record, float* ws_acc, float* ws_ml) {
    using Lds = PrefixLds<D>;
    constexpr int KS = D / 16, DT = D / 32;            // k-steps of the score MFMA, 32-row tiles of O^T
    constexpr int STAGE = Lds::STAGE, PITCHK = Lds::PITCHK, PITCHV = Lds::PITCHV;
    constexpr int NT = RG / 2;                         // tiles a wave and stage
    constexpr int NP = STAGE * D / 4096;               // 128-bit loads a thread, stage and tensor
    static_assert(4 * NP == KS, "a piece of the next stage for each k-step");
    const int tid = threadIdx.x, lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int l32 = lane & 31, hh = lane >> 5;
    const int rg = w % RG, phase = w / RG;

    // Q^T B operands: lane holds row l32, d = 16 s + 8 hh + [0,8)
    bf16x8 qB[KS];
    {
        const uint16_t* qp = q_row(min(32 * rg + l32, n_rows - 1)) + 8 * hh;
#pragma unroll
        for (int s = 0; s < KS; ++s) qB[s] = *reinterpret_cast<const bf16x8*>(qp + 16 * s);
    }
    const __amdgpu_buffer_rsrc_t krs = __builtin_amdgcn_make_buffer_rsrc((void*)kc, 0, (int)((unsigned)T * D), 0x00020000);
    const __amdgpu_buffer_rsrc_t vrs = __builtin_amdgcn_make_buffer_rsrc((void*)vc, 0, (int)((unsigned)T * D), 0x00020000);
    // (rows past the end of the prefix read as zeros and are masked.  Wave 0 has the stage's K scales, wave 1 its V scales, the
    // others ask past the end: a load is the same instructions for all)
    const __amdgpu_buffer_rsrc_t srs = __builtin_amdgcn_make_buffer_rsrc((void*)(w == 1 ? vs : ks), 0, w < 2 ? (int)((unsigned)T * 4u) : 0, 0x00020000);
    u32x4 buf[2][2][NP];                               // two stages in flight
    uint32_t sc[2];
    auto issue = [&](auto set_c, int t0) __attribute__((always_inline)) {
        constexpr int set = decltype(set_c)::value;
        const int base = t0 < t_end ? t0 : T;          // (a stage that is not wanted: nothing is read)
        sc[set] = __builtin_amdgcn_raw_buffer_load_b32(srs, (base + lane) * 4, 0, 0);
        const int off = (int)((unsigned)base * D + (unsigned)(tid * 16));
#pragma unroll
        for (int n = 0; n < NP; ++n) buf[set][0][n] = __builtin_amdgcn_raw_buffer_load_b128(krs, off + n * 4096, 0, 0);
#pragma unroll
        for (int n = 0; n < NP; ++n) buf[set][1][n] = __builtin_amdgcn_raw_buffer_load_b128(vrs, off + n * 4096, 0, 0);
    };
    const int tile0 = NT == 1 ? 32 * phase : 0;  // of the stage
    // Addresses in a buffer, K's, V's and the scales' (the compiler sees no constant in them: it would add it to a buffer's offset, more than
    // the 16 bits of an instruction, and keep a register for every sum, when there is none to spare)
    int k_addr = (tile0 + l32) * PITCHK + 16 * hh;   // K fragment of k-step s: row l32, bytes 32 s + 16 hh + [0,16)
    // V transpose reads: 16 lanes fetch rows k..k+3, lane i receives column i of them
    int v_addr = STAGE * PITCHK + (tile0 + 4 * hh + ((lane & 15) >> 2)) * PITCHV + (2 * ((lane >> 4) & 1) + ((lane & 3) >> 1)) * 16 + 8 * (lane & 1);
    int s_addr = STAGE * (PITCHK + PITCHV) + 4 * (tile0 + 4 * hh);
    int k_to = tid * 16 / D * PITCHK + tid * 16 % D * 2, v_to = STAGE * PITCHK + tid * 16 / D * PITCHV + tid * 16 % D * 2;
    int s_to = STAGE * (PITCHK + PITCHV) + 4 * tid;
    asm("" : "+v"(k_addr), "+v"(v_addr), "+v"(s_addr), "+v"(k_to), "+v"(v_to), "+v"(s_to));
    // piece i of a stage on its way into LDS: 8 codes of K (the first half) or V -> 8 bf16, exact
    auto piece = [&](int set, char* to, int i) __attribute__((always_inline)) {
        const int x = i / (2 * NP), n = i / 2 % NP, half = i % 2;
        char* const dst = to + (x == 0 ? k_to : v_to) + 4096 / D * n * (x == 0 ? PITCHK : PITCHV) + 16 * half;
        *reinterpret_cast<bf16x8*>(dst) = widen8(i32x2{(int)buf[set][x][n][2 * half], (int)buf[set][x][n][2 * half + 1]});
    };
    const float scale_by = w == 0 ? scale_log2e : 1.0f;
    auto scales = [&](int set, char* to) __attribute__((always_inline)) {   // [0, STAGE) k_scale * c, then v_scale
        *reinterpret_cast<float*>(to + s_to) = __uint_as_float(sc[set]) * scale_by;
    };

    f32x16 o[DT];
#pragma unroll
    for (int dt = 0; dt < DT; ++dt)
#pragma unroll
        for (int r = 0; r < 16; ++r) o[dt][r] = 0.0f;
    float M = 0.0f, lsum = 0.0f;   // running max of this lane's row (log2 units), this lane's part of the row sum
    bool first = true;             // (uniform)
    float move_above = -INFINITY;  // what a score relative to the running max passes where that moves (uniform; 8 behind the first stage)

    const std::integral_constant<int, 0> set0{};
    const std::integral_constant<int, 1> set1{};
    // (The compiler waits for a load by counting those issued behind it, on the path that has fewest: here they come in the order in which the
    // loop issues them, none is under a branch, and the loop, which has two stages, is not left between them; an odd number's last one is
    // all mask.  Where one of the three was not so, every other stage waited for its successor's loads: 64 on 8 heads, 20 sequences,
    // P=32768 57.8 us and 52.2, 32 on 8, 64 sequences, P=2048 21.6 and 20.0.)
    __builtin_amdgcn_sched_barrier(0);
    issue(set0, t_begin);
    __builtin_amdgcn_sched_barrier(0);
    issue(set1, t_begin + STAGE);
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int i = 0; i < KS; ++i) piece(0, smem, i);
    scales(0, smem);
    __builtin_amdgcn_sched_barrier(0);
    issue(set0, t_begin + 2 * STAGE);
    __builtin_amdgcn_sched_barrier(0);
    __syncthreads();
    // the stage from token t0 on, in LDS buffer `turn`; the one behind it goes into the other, which every wave is done with since the
    // last barrier
    auto work = [&](auto turn_c, int t0) __attribute__((always_inline)) {
        constexpr int turn = decltype(turn_c)::value;
        const char* const kS = smem + turn * Lds::STAGE_BYTES;
        char* const next = smem + (turn ^ 1) * Lds::STAGE_BYTES;
        const float* const scS = reinterpret_cast<const float*>(kS + s_addr);
        scales(turn ^ 1, next);
        f32x16 u[NT];
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
            for (int r = 0; r < 16; ++r) u[t][r] = 0.0f;
        bf16x8 kf[2][NT];
#pragma unroll
        for (int t = 0; t < NT; ++t) kf[0][t] = *reinterpret_cast<const bf16x8*>(kS + k_addr + t * 32 * PITCHK);
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int s = 0; s < KS; ++s) {
            if (s + 1 < KS) {
#pragma unroll
                for (int t = 0; t < NT; ++t) kf[(s + 1) & 1][t] = *reinterpret_cast<const bf16x8*>(kS + k_addr + t * 32 * PITCHK + 32 * (s + 1));
            }
#pragma unroll
            for (int t = 0; t < NT; ++t) u[t] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf[s & 1][t], qB[s], u[t], 0, 0, 0);
            piece(turn ^ 1, next, s);
            __builtin_amdgcn_sched_barrier(0);
        }
        f32x4 kscale[NT][4];
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
            for (int r4 = 0; r4 < 4; ++r4) kscale[t][r4] = *reinterpret_cast<const f32x4*>(scS + 32 * t + 8 * r4);
        // V fragments of k-step x of the second product (tokens 16 x + ...): two ahead of their use
        s16x4 vf[2][DT][2];
        auto fetch_v = [&](int x) __attribute__((always_inline)) {
#pragma unroll
            for (int dt = 0; dt < DT; ++dt) {
                const char* va = kS + v_addr + 64 * dt + 16 * x * PITCHV;
                vf[x & 1][dt][0] = lds_read_tr16(reinterpret_cast<const uint16_t*>(va));
                vf[x & 1][dt][1] = lds_read_tr16(reinterpret_cast<const uint16_t*>(va + 8 * PITCHV));
            }
        };
        f32x4 vscale[2][2];
        auto fetch_scales = [&](int x) __attribute__((always_inline)) {
#pragma unroll
            for (int i = 0; i < 2; ++i) vscale[x & 1][i] = *reinterpret_cast<const f32x4*>(scS + STAGE + 16 * x + 8 * i);
        };
        // register r of u[t] is token t0 + tile0 + 32 t + 8 (r/4) + 4 hh + r%4; scores relative to the running max
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
            for (int r = 0; r < 16; ++r) u[t][r] = fmaf(u[t][r], kscale[t][r / 4][r % 4], -M);
        __builtin_amdgcn_sched_barrier(0);
        fetch_scales(0);
        fetch_scales(1);
        fetch_v(0);
        issue(std::integral_constant<int, turn ^ 1>{}, t0 + 3 * STAGE);   // (here, where registers are free again)
        __builtin_amdgcn_sched_barrier(0);
        auto masked_max = [&]() __attribute__((always_inline)) {   // (masks what lies past the end)
            if (t0 + STAGE > T) {
#pragma unroll
                for (int t = 0; t < NT; ++t)
#pragma unroll
                    for (int r = 0; r < 16; ++r) u[t][r] = t0 + tile0 + 32 * t + 8 * (r / 4) + 4 * hh + r % 4 < T ? u[t][r] : -INFINITY;
            }
            float top = u[0][0];
#pragma unroll
            for (int t = 0; t < NT; ++t)
#pragma unroll
                for (int r = 0; r < 16; r += 2) top = fmaxf(top, fmaxf(u[t][r], u[t][r + 1]));
            return top;
        };
        const float umax = masked_max();
        // the running max, a whole number (decode_gqa.hip says why), moves only when a score has passed it by 2^8, but for the first
        // stage, which sets it (not if the wave's tile of it is past the end, all -infinity: it has no other)
        if (__builtin_expect(__builtin_amdgcn_ballot_w64(umax > move_above) != 0, 0)) {
            const float up = fmaxf(ceilf(half_max(umax)), kMasked);   // (-infinity, of scores below what fp32 holds, cannot be taken off one)
            float by = first ? up : fmaxf(up, 0.0f), m_new = M + by;
            float alpha = first ? 0.0f : fast_exp2(-by);   // (nothing to rescale yet)
            if (__builtin_expect(!first && __builtin_amdgcn_ballot_w64(umax > 256.0f) != 0, 0)) {
                // Scores so far above it have lost their last bits to the running max (all of them where that is below -2^24): once more,
                // without it
                __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                for (int t = 0; t < NT; ++t) {
#pragma unroll
                    for (int r = 0; r < 16; ++r) u[t][r] = 0.0f;
#pragma unroll
                    for (int s = 0; s < KS; ++s) {
                        u[t] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(*reinterpret_cast<const bf16x8*>(kS + k_addr + t * 32 * PITCHK + 32 * s), qB[s],
                                                                       u[t], 0, 0, 0);
                        __builtin_amdgcn_sched_barrier(0);
                    }
#pragma unroll
                    for (int r4 = 0; r4 < 4; ++r4) {
                        const f32x4 f = *reinterpret_cast<const f32x4*>(scS + 32 * t + 8 * r4);
#pragma unroll
                        for (int e = 0; e < 4; ++e) u[t][4 * r4 + e] *= f[e];
                        __builtin_amdgcn_sched_barrier(0);
                    }
                }
                by = m_new = fmaxf(ceilf(half_max(masked_max())), M);
                alpha = fast_exp2(M - m_new);
            }
#pragma unroll
            for (int dt = 0; dt < DT; ++dt)
#pragma unroll
                for (int r = 0; r < 16; ++r) o[dt][r] *= alpha;
            lsum *= alpha;
            M = m_new;
#pragma unroll
            for (int t = 0; t < NT; ++t)
#pragma unroll
                for (int r = 0; r < 16; ++r) u[t][r] -= by;
            first = false;
            move_above = 8.0f;
        }
        // O^T += V^T P^T: k-step x covers tokens 16 x + {4 hh .. 4 hh + 3} and 16 x + 8 + {4 hh .. 4 hh + 3}, registers 8 x to 8 x + 7; the
        // probabilities take their token's v_scale before they are rounded to bf16, operands of the product
        u32x4 pw[2];
        float ps = 0.0f;
        auto probabilities = [&](int x, int e) __attribute__((always_inline)) {   // registers 8 x + 2 e and the next
            const int t = x / 2, r = 8 * (x % 2) + 2 * e;
            const f32x4 f = vscale[x & 1][e / 2];
            const float a = fast_exp2(u[t][r]), b = fast_exp2(u[t][r + 1]);
            ps += a + b;
            pw[x & 1][e] = pack_bf16x2(a * f[2 * (e % 2)], b * f[2 * (e % 2) + 1]);
        };
#pragma unroll
        for (int e = 0; e < 4; ++e) probabilities(0, e);
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int x = 0; x < 2 * NT; ++x) {
            if (x + 1 < 2 * NT) fetch_v(x + 1);
#pragma unroll
            for (int dt = 0; dt < DT; ++dt) {
                const s16x4 lo = vf[x & 1][dt][0], hi = vf[x & 1][dt][1];
                const s16x8 av = {lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]};
                o[dt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, av), __builtin_bit_cast(bf16x8, pw[x & 1]), o[dt], 0, 0, 0);
                if (x + 1 < 2 * NT)
#pragma unroll
                    for (int e = 0; e < 4 / DT; ++e) probabilities(x + 1, dt * (4 / DT) + e);
                __builtin_amdgcn_sched_barrier(0);
            }
            if (x + 2 < 2 * NT) fetch_scales(x + 2);
        }
        lsum += ps;
        __syncthreads();
    };
    for (int t0 = t_begin; t0 < t_end; t0 += 2 * STAGE) {
        work(set0, t0);
        work(set1, t0 + STAGE);
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
        if (hh == 0) reinterpret_cast<f32x2*>(ws_ml)[idx] = f32x2{first ? kMasked : M, L};   // (nothing: behind everything)
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
__global__ __launch_bounds__(256, 2) void slim_decode_prefix_kernel(const PrefixParams p) {
    constexpr int RG = FORM == 4 ? 4 : 2;
    constexpr int OWN_LDS = 4 * GqaLds<D, NC>::WAVE_BYTES;
    constexpr int SHARED_LDS = FORM >= 3 ? PrefixLds<D>::BYTES : 4 * GqaLds<D, (FORM < 3 ? FORM : 1)>::WAVE_BYTES;
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
            constexpr int STAGE = PrefixLds<D>::STAGE, PHASES = 4 / RG;
            int first, end;
            split_span((p.P + 2 * STAGE - 1) / (2 * STAGE), p.n_prefix / PHASES, sp, first, end);
            prefix_sweep<D, RG>(smem, [&](int i) { return p.q + row_of(i) * D; }, n_rows, p.pkc + kv0 * D, p.pks + kv0, p.pvc + kv0 * D,
                                p.pvs + kv0, p.P, first * 2 * STAGE, min(end * 2 * STAGE, p.P), p.scale_log2e,
                                [&](int i, int phase) { return row_of(i) * p.n_records + sp * PHASES + phase; }, p.ws_acc, p.ws_ml);
        } else {
            int first, end;
            split_span((p.P + kGqaTile - 1) / kGqaTile, p.n_prefix, sp, first, end);
            first += w;
            f32x4 o[FORM][D / 16];
            float M[FORM], lsum[FORM];
            char* const kS = smem + w * GqaLds<D, FORM>::WAVE_BYTES;
            gqa_sweep<D, 4, FORM, FORM == 1>(kS, lane, [&](int i) { return p.q + row_of(min(i, n_rows - 1)) * D; }, p.pkc + kv0 * D, p.pks + kv0,
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
    gqa_sweep<D, 4, NC, FORM == 1>(kS, lane, [&](int i) { return p.q + (row0 + min(i, heads - 1)) * D; }, p.kc + kv0 * D, p.ks + kv0, p.vc + kv0 * D,
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
    // The prefix: a workgroup a compute unit, beside which there is room for one of an own cache, or two where each still has 32 stages
    // (64 on 8 heads, 64 sequences, P=32768 107 and 93 us); and none with less than 4 stages, 8 from 2048 query rows on, as every one
    // costs a record of its rows besides (with 4, 8 and 16 stages 32 on 8 heads, 48 sequences, P=1024, T=100 14.3, 18.6 and 27.9 us; 128
    // sequences, P=2000 27.8, 21.2 and 29.3; 32 heads, 128 sequences, P=2000 43.7, 38.3 and 36.6).  Up to 32 rows a record is little: two
    // tiles a wave (32 on 8 heads, 2 sequences, P=4000, T=100 14.0 us with 8, 11.0 with 4, 9.5).  (All of 128 codes a token; calls of 64
    // follow the same rule.)
    const int phases = plan.form == 3 ? 2 : 1;
    const long items = (long)kv_heads * plan.row_blocks, stages = ((long)prefix_len + (plan.form < 3 ? 127 : 63)) / (plan.form < 3 ? 128 : 64);
    long n = (256 + items - 1) / items;
    if (plan.form >= 3 && stages / (2 * n) >= 32) n *= 2;
    const long least = plan.form < 3 ? 2 : (long)batch * q_heads < 2048 ? 4 : 8;
    n = std::min(n, (stages + least - 1) / least);
    plan.n_prefix = (int)n * phases;
    const long own = (long)batch * kv_heads * plan.head_groups;
    plan.n_own = (int)std::min((512 + own - 1) / own, ((long)kv_len + 255) / 256);
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
        const hipError_t e = plan.form == 1   ? sweep(integral_constant<int, 1>{}, integral_constant<int, 1>{})   // (16 rows: no more heads)
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
        // (a wave a row up to three passes, four beyond.  Four and one wave, us: 32 on 8 heads, 36 sequences, P=4096, 18 records 24.9 and 21.9; 48, P=2500,
        // 12 23.5 and 20.2; 4 sequences, P=16000, 33 13.8 and 13.9; 2, P=16000, 33 12.5 and 13.0; 64 on 8, 5 sequences, 66 19.8 and 21.6:
        // all of 128 codes, where a pass of four loads is 8 records)
        if (p.n_records <= 12 * RPW) return combine(one, four);
        return combine(four, four);
    };
    return a.head_dim == 128 ? with_d(integral_constant<int, 128>{}) : with_d(integral_constant<int, 64>{});
}

}  // namespace slim
