// What decode kernels over the INT8 cache share: the sweep of a run of a KV head's tokens for several rows of queries on the matrix
// cores and the merge of a workgroup's waves (the grouped decode's; decode_gqa.hip, which explains them, has them written out: inlined from
// here, the same steps take that kernel 4 % less to 4 % more, shape by shape), and the merge of the records that workgroups leave.
#pragma once
#include "slim_common.h"

namespace slim {

constexpr int kGqaTile = 32;    // tokens per tile
typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef int i32x2 __attribute__((ext_vector_type(2)));
typedef __attribute__((address_space(3))) i32x2 lds_i32x2;

// Two fp32 values as two bf16 each: the value rounded, and what that leaves (off by at most 2^-16 of the value together)
__device__ __forceinline__ void pack_bf16x2_twice(float lo, float hi, unsigned& rounded, unsigned& rest) {
    rounded = pack_bf16x2(lo, hi);
    rest = pack_bf16x2(lo - bf16_bits_to_f32(rounded & 0xffffu), hi - __uint_as_float(rounded & 0xffff0000u));
}

// 8 INT8 codes -> 8 bf16, exact
__device__ __forceinline__ bf16x8 widen8(const i32x2 cw) {
    u32x4 r;
#pragma unroll
    for (int e = 0; e < 2; ++e) {
        r[2 * e] = pack_bf16x2(i8_to_f32<0>(cw[e]), i8_to_f32<1>(cw[e]));
        r[2 * e + 1] = pack_bf16x2(i8_to_f32<2>(cw[e]), i8_to_f32<3>(cw[e]));
    }
    return __builtin_bit_cast(bf16x8, r);
}

// LDS of a wave: its K tile, its V tile, the tile's 32 + 32 scales; over them, once they are dead, its record for the merge
template <int D, int NC>
struct GqaLds {
    static constexpr int PITCH = D + 16;         // LDS row pitch: 16 rows' pieces of a read fall on 16 different groups of four banks
    static constexpr int TILE = kGqaTile * PITCH;
    static constexpr int WAVE_LDS = 2 * TILE + 256;
    static constexpr int OPITCH = D + 4;         // floats per column in a wave's merge record (behind its maxima and sums)
    static constexpr int MERGE_LDS = 16 * NC * (OPITCH + 2) * 4;
    static constexpr int WAVE_BYTES = WAVE_LDS > MERGE_LDS ? WAVE_LDS : MERGE_LDS;
};

// One wave's sweep: tiles first, first + W, ... (n_tiles of them) of the T tokens at kc, ks, vc, vs, for 16 NC columns.  q_row(i) is
// column i's row of D query values.  Out: running max of this lane's column (log2 units), this lane's part of its sum, the
// accumulators.  keep(nc, t0, u): sees the scores (log2 units; register 4 tt + r is token t0 + 16 tt + 4 lq + r) of every tile.
// FINE: the second product takes a probability (times v_scale) as two bf16 and not as one: twice the matrix instructions.
// kS: the wave's own LDS.
template <int D, int W, int NC, bool FINE, class QRow, class Keep>
__device__ __forceinline__ void gqa_sweep(char* const kS, const int lane, const QRow q_row, const int8_t* kc, const float* ks, const int8_t* vc,
                                          const float* vs, const int T, const int first, const int n_tiles, const float scale_log2e,
                                          const Keep keep, f32x4 (&o)[NC][D / 16], float (&M)[NC], float (&lsum)[NC]) {
    constexpr int KS = D / 64;            // 16-byte pieces of a K row per lane (two k-steps of the score MFMA each)
    constexpr int DT = D / 16;            // 16-row tiles of O^T
    constexpr int CPR = D / 16;           // 16-byte pieces per row
    constexpr int NP = kGqaTile * CPR / 64;   // 128-bit loads per lane, tile and tensor
    constexpr int PITCH = GqaLds<D, NC>::PITCH, TILE = GqaLds<D, NC>::TILE;
    const int l16 = lane & 15, lq = lane >> 4;
    char* const vS = kS + TILE;
    float* const scS = reinterpret_cast<float*>(kS + 2 * TILE);   // [0,32) k_scale * c, [32,64) v_scale

    // Q^T B operands: lane holds column l16 of its group of 16,
    // d = 64 s + 16 lq + 8 e + [0,8)
    bf16x8 qB[NC][KS][2];
#pragma unroll
    for (int nc = 0; nc < NC; ++nc) {
        const uint16_t* qp = q_row(16 * nc + l16) + 16 * lq;
#pragma unroll
        for (int s = 0; s < KS; ++s)
#pragma unroll
            for (int e = 0; e < 2; ++e) qB[nc][s][e] = *reinterpret_cast<const bf16x8*>(qp + 64 * s + 8 * e);
    }

    // Piece lane + 64 n of a tile (row-major, 16 codes each), through buffer descriptors that cover exactly this
    // (batch, KV head)'s slab: rows past the end of the cache read as zero (and are masked) and a load costs one
    // vector add.  The codes are used once: non-temporal.
    const __amdgpu_buffer_rsrc_t krs = __builtin_amdgcn_make_buffer_rsrc((void*)kc, 0, (int)((unsigned)T * D), 0x00020000);
    const __amdgpu_buffer_rsrc_t vrs = __builtin_amdgcn_make_buffer_rsrc((void*)vc, 0, (int)((unsigned)T * D), 0x00020000);
    // (the scales through descriptors as well: lanes 0-31 want the K scale of token lane, lanes 32-63 the V scale; each
    // load asks the other half's lanes for an offset past the end, which reads nothing, so a tile's loads are the
    // same instructions whether the tile is wanted or not)
    const __amdgpu_buffer_rsrc_t ksr = __builtin_amdgcn_make_buffer_rsrc((void*)ks, 0, (int)((unsigned)T * 4u), 0x00020000);
    const __amdgpu_buffer_rsrc_t vsr = __builtin_amdgcn_make_buffer_rsrc((void*)vs, 0, (int)((unsigned)T * 4u), 0x00020000);
    const bool k_half = lane < 32;
    const int s_off_k = k_half ? lane * 4 : (int)0x7ffffff0, s_off_v = k_half ? (int)0x7ffffff0 : (lane - 32) * 4;
    u32x4 kbuf[NP], vbuf[NP];
    float sc = 0.0f;
    auto issue = [&](const __amdgpu_buffer_rsrc_t rs, u32x4 (&buf)[NP], int t0) {
#pragma unroll
        for (int n = 0; n < NP; ++n) buf[n] = __builtin_amdgcn_raw_buffer_load_b128(rs, lane * 16 + n * 1024 + t0 * D, 0, 2 /* nt */);
    };
    auto issue_k = [&](int t0) {
        issue(krs, kbuf, t0);
        const uint32_t a = __builtin_amdgcn_raw_buffer_load_b32(ksr, s_off_k + t0 * 4, 0, 0);
        const uint32_t c = __builtin_amdgcn_raw_buffer_load_b32(vsr, s_off_v + t0 * 4, 0, 0);
        sc = __builtin_bit_cast(float, a | c);   // (the lanes a load left out received zero)
    };
    auto issue_v = [&](int t0) { issue(vrs, vbuf, t0); };
    auto stage = [&](const u32x4 (&buf)[NP], char* tile) {   // a tile's codes into LDS
#pragma unroll
        for (int n = 0; n < NP; ++n)
            *reinterpret_cast<u32x4*>(tile + ((lane + 64 * n) / CPR) * PITCH + (lane % CPR) * 16) = buf[n];
    };

    // Every load of the kernel is issued unconditionally: a tile that is not wanted (past the end of this wave's
    // run) is asked for at token T, past the end of the descriptor, so zeros arrive and no memory is read.  The
    // compiler places a wait by counting the loads issued after the one it needs, along the worst path that leads
    // there; loads under a branch are not outstanding on the path that skips them, and at the loop's head the
    // worst path may be the one from the prologue.  So the prologue's four groups keep the order the loop issues
    // them in (K, V of a tile, then the next tile's).
    auto t_of = [&](int i) { return i < n_tiles ? (first + i * W) * kGqaTile : T; };
    __builtin_amdgcn_sched_barrier(0);
    issue_k(t_of(0));
    __builtin_amdgcn_sched_barrier(0);
    issue_v(t_of(0));
    __builtin_amdgcn_sched_barrier(0);

    // K fragments of token tile tt, k-steps 2 s and 2 s + 1: row 16 tt + l16, bytes 64 s + 16 lq + [0,16).  V^T fragment of tile dt: the
    // 16 lanes of a group fetch 8 rows (2 lanes a row, 8 columns each) and lane j of the group receives column j of
    // them; the rows of group lq are the tokens its probabilities belong to: 4 lq + [0,4) and 16 + 4 lq + [0,4).
    const int k_addr = l16 * PITCH + 16 * lq;
    const int v_row = l16 >> 1;
    const int v_addr = (4 * lq + (v_row & 3) + 16 * (v_row >> 2)) * PITCH + 8 * (l16 & 1);

#pragma unroll
    for (int nc = 0; nc < NC; ++nc) {
        M[nc] = kMasked;
        lsum[nc] = 0.0f;
#pragma unroll
        for (int dt = 0; dt < DT; ++dt) o[nc][dt] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    }

    for (int i = 0; i < n_tiles; ++i) {
        const int t0 = t_of(i);
        const int t_next = t_of(i + 1);

        stage(kbuf, kS);
        scS[lane] = k_half ? sc * scale_log2e : sc;
        issue_k(t_next);
        i32x4 kw[2][KS];
#pragma unroll
        for (int tt = 0; tt < 2; ++tt)
#pragma unroll
            for (int s = 0; s < KS; ++s) kw[tt][s] = *reinterpret_cast<const i32x4*>(kS + k_addr + 16 * tt * PITCH + 64 * s);
        __builtin_amdgcn_sched_barrier(0);
        stage(vbuf, vS);
        issue_v(t_next);
        __builtin_amdgcn_sched_barrier(0);

        // scores: register r of token tile tt is token 16 tt + 4 lq + r, column = head l16 of the group
        bf16x8 kf[2][KS][2];
#pragma unroll
        for (int tt = 0; tt < 2; ++tt)
#pragma unroll
            for (int s = 0; s < KS; ++s) {
                kf[tt][s][0] = widen8(i32x2{kw[tt][s][0], kw[tt][s][1]});
                kf[tt][s][1] = widen8(i32x2{kw[tt][s][2], kw[tt][s][3]});
            }
        u32x4 pw[NC], rest[FINE ? NC : 1];
#pragma unroll
        for (int nc = 0; nc < NC; ++nc) {
            f32x4 acc[2] = {{0.0f, 0.0f, 0.0f, 0.0f}, {0.0f, 0.0f, 0.0f, 0.0f}};
#pragma unroll
            for (int s = 0; s < KS; ++s)
#pragma unroll
                for (int e = 0; e < 2; ++e)
#pragma unroll
                    for (int tt = 0; tt < 2; ++tt)
                        acc[tt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf[tt][s][e], qB[nc][s][e], acc[tt], 0, 0, 0);
            float u[8];
#pragma unroll
            for (int tt = 0; tt < 2; ++tt) {
                const f32x4 kf4 = *reinterpret_cast<const f32x4*>(&scS[16 * tt + 4 * lq]);
#pragma unroll
                for (int r = 0; r < 4; ++r) u[4 * tt + r] = acc[tt][r] * kf4[r];
            }
            if (t0 + kGqaTile > T) {   // the sequence ends inside this tile (or before it)
#pragma unroll
                for (int r = 0; r < 8; ++r) u[r] = (t0 + 16 * (r / 4) + 4 * lq + r % 4 < T) ? u[r] : kMasked;
            }
            keep(nc, t0, u);
            float umax = fmaxf(u[0], u[1]);
#pragma unroll
            for (int r = 2; r < 8; r += 2) umax = fmaxf(umax, fmaxf(u[r], u[r + 1]));
            // the running max moves only when a score has passed it by 2^8 (always on a wave's first tile)
            if (__builtin_amdgcn_ballot_w64(umax - M[nc] > 8.0f) != 0) {
                float m_new = fmaxf(M[nc], umax);
                m_new = fmaxf(m_new, __shfl_xor(m_new, 16));
                m_new = ceilf(fmaxf(m_new, __shfl_xor(m_new, 32)));
                const float alpha = fast_exp2(M[nc] - m_new);
#pragma unroll
                for (int dt = 0; dt < DT; ++dt) o[nc][dt] *= alpha;
                lsum[nc] *= alpha;
                M[nc] = m_new;
            }
            float ps0 = 0.0f, ps1 = 0.0f;
#pragma unroll
            for (int r = 0; r < 8; r += 2) {
                u[r] = fast_exp2(u[r] - M[nc]);
                u[r + 1] = fast_exp2(u[r + 1] - M[nc]);
                ps0 += u[r];
                ps1 += u[r + 1];
            }
            lsum[nc] += ps0 + ps1;
            // the probabilities take their token's v_scale before they are rounded to bf16
#pragma unroll
            for (int tt = 0; tt < 2; ++tt) {
                const f32x4 vf = *reinterpret_cast<const f32x4*>(&scS[32 + 16 * tt + 4 * lq]);
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    const float a = u[4 * tt + 2 * i] * vf[2 * i], b = u[4 * tt + 2 * i + 1] * vf[2 * i + 1];
                    if constexpr (FINE) {
                        unsigned more, less;
                        pack_bf16x2_twice(a, b, more, less);
                        pw[nc][2 * tt + i] = more;
                        rest[nc][2 * tt + i] = less;
                    } else {
                        pw[nc][2 * tt + i] = pack_bf16x2(a, b);
                    }
                }
            }
        }

        // O^T += V^T P^T over the tile's 32 tokens: element j of lane group lq is token 4 lq + j (j < 4) or 16 + 4 lq + j - 4
#pragma unroll
        for (int dt = 0; dt < DT; ++dt) {
            const i32x2 vw = __builtin_amdgcn_ds_read_tr8_b64_v2i32((lds_i32x2*)(vS + v_addr + 16 * dt));
            const bf16x8 va = widen8(vw);
#pragma unroll
            for (int nc = 0; nc < NC; ++nc) {
                o[nc][dt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(va, __builtin_bit_cast(bf16x8, pw[nc]), o[nc][dt], 0, 0, 0);
                if constexpr (FINE) o[nc][dt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(va, __builtin_bit_cast(bf16x8, rest[nc]), o[nc][dt], 0, 0, 0);
            }
        }
    }
}

// A wave's record for the merge of its workgroup
template <int D, int NC>
__device__ __forceinline__ void gqa_record(char* const kS, const int lane, const f32x4 (&o)[NC][D / 16], const float (&M)[NC], const float (&lsum)[NC]) {
    constexpr int DT = D / 16, OPITCH = GqaLds<D, NC>::OPITCH;
    const int l16 = lane & 15, lq = lane >> 4;
    // Register r of tile dt is d = 16 dt + 4 lq + r of head l16.  A wave's record: 16 NC maxima (log2
    // units), as many sums, then the accumulators, a row of OPITCH floats per head (over its own tiles, which are dead).
    float* const rec = reinterpret_cast<float*>(kS);
#pragma unroll
    for (int nc = 0; nc < NC; ++nc) {
        float L = lsum[nc];
        L += __shfl_xor(L, 16);
        L += __shfl_xor(L, 32);
        if (lq == 0) {
            rec[16 * nc + l16] = M[nc];
            rec[16 * NC + 16 * nc + l16] = L;
        }
#pragma unroll
        for (int dt = 0; dt < DT; ++dt)
            *reinterpret_cast<f32x4*>(rec + 32 * NC + (16 * nc + l16) * OPITCH + 16 * dt + 4 * lq) = o[nc][dt];
    }
}
// ... and, behind a barrier, the merged value d of column h: accumulator, max and sum
template <int D, int W, int NC>
__device__ __forceinline__ void gqa_merged(const char* const smem, const int h, const int d, float& acc, float& top, float& L) {
    constexpr int OPITCH = GqaLds<D, NC>::OPITCH, WAVE_BYTES = GqaLds<D, NC>::WAVE_BYTES;
    float m[W];
    top = kMasked;
#pragma unroll
    for (int ww = 0; ww < W; ++ww) {
        m[ww] = reinterpret_cast<const float*>(smem + ww * WAVE_BYTES)[h];
        top = ww == 0 ? m[ww] : fmaxf(top, m[ww]);
    }
    L = 0.0f;
    acc = 0.0f;
#pragma unroll
    for (int ww = 0; ww < W; ++ww) {
        const float* r = reinterpret_cast<const float*>(smem + ww * WAVE_BYTES);
        const float f = fast_exp2(m[ww] - top);   // a wave without tiles has L = 0 and an accumulator of zeros
        L = fmaf(f, r[16 * NC + h], L);
        acc = fmaf(f, r[32 * NC + h * OPITCH + d], acc);
    }
}

// Merges the partial (max, sum, accumulator) triples of one (batch, head), n_used records at ml and acc, in a fixed order (records dealt to lane
// groups and waves, each group's in turn, then the groups by halves, then the waves) and writes the bf16 output row.  The launch is latency-bound (a few kilobytes per row, just written by the split kernel), so a row's records
// come in with few, wide loads that are all issued before anything is computed: D/4 lanes read a record with one 128-bit
// load each, a wave RPW = 256/D records at a time.  Up to U RPW records a row one wave does it, and a workgroup has four
// rows; more are shared by the four waves of a workgroup and merged through LDS.  Slots past the last split re-read the last
// one and count as empty (max = kMasked, sum = 0); runs longer than the slots take another pass with a running (max, sum,
// accumulator).  With a thread for every output value and sixteen records a thread (32-bit loads, 512 threads a row beyond sixteen
// splits) the wide form's decode took, before -> now: 64 on 8 heads, T=32768, 32 splits 18.6 -> 16.1 us, D=64 14.7 -> 12.6; 8
// heads, T=16000, 32 splits 11.8 -> 9.5; 32 heads, T=4000, 8 splits 9.5 -> 9.2; 16 sequences, 64 on 8 heads, T=8192, 2 splits 45.2 ->
// 44.6.
// w: the wave in its workgroup; with WAVES > 1 all four of them come here.
template <int D, int WAVES, int U>
__device__ __forceinline__ void combine_row(const f32x2* const ml, const f32x4* acc, uint16_t* const out, const int n_used, const int lane, const int w) {
    constexpr int LPR = D / 4, RPW = 64 / LPR;
    const int c = lane % LPR, sub = lane / LPR, part = WAVES == 1 ? 0 : w;
    acc += c;
    float M = kMasked, L = 0.0f;
    f32x4 o = {0.0f, 0.0f, 0.0f, 0.0f};
    for (int s0 = 0; s0 < n_used; s0 += WAVES * RPW * U) {
        float m[U], l[U];
        f32x4 a[U];
#pragma unroll
        for (int i = 0; i < U; ++i) {
            const int s = s0 + (i * WAVES + part) * RPW + sub, sp = min(s, n_used - 1);
            const f32x2 t = ml[sp];
            const f32x4 av = acc[(long)sp * LPR];
            m[i] = s < n_used ? t[0] : kMasked;
            l[i] = s < n_used ? t[1] : 0.0f;
            a[i] = s < n_used ? av : f32x4{0.0f, 0.0f, 0.0f, 0.0f};
        }
        float m_new = M;
#pragma unroll
        for (int i = 0; i < U; ++i) m_new = fmaxf(m_new, m[i]);
        const float keep = fast_exp2(M - m_new);   // first pass: L = o = 0, whatever this is
        L *= keep;
        o *= keep;
#pragma unroll
        for (int i = 0; i < U; ++i) {
            const float f = fast_exp2(m[i] - m_new);   // an empty split has sum = 0 and accumulator = 0
            L = fmaf(f, l[i], L);
#pragma unroll
            for (int e = 0; e < 4; ++e) o[e] = fmaf(f, a[i][e], o[e]);
        }
        M = m_new;
    }
    // the wave's groups of lanes, by halves
#pragma unroll
    for (int x = LPR; x < 64; x *= 2) {
        const float m_other = __shfl_xor(M, x), l_other = __shfl_xor(L, x), m_new = fmaxf(M, m_other);
        const float f = fast_exp2(M - m_new), g = fast_exp2(m_other - m_new);
        L = fmaf(L, f, l_other * g);
#pragma unroll
        for (int e = 0; e < 4; ++e) o[e] = fmaf(o[e], f, __shfl_xor(o[e], x) * g);
        M = m_new;
    }
    if constexpr (WAVES > 1) {
        __shared__ __attribute__((aligned(16))) f32x4 oS[WAVES][LPR];
        __shared__ float mS[WAVES], lS[WAVES];
        if (sub == 0) oS[w][c] = o;
        if (lane == 0) {
            mS[w] = M;
            lS[w] = L;
        }
        __syncthreads();
        if (w != 0) return;
        M = kMasked;
#pragma unroll
        for (int i = 0; i < WAVES; ++i) M = fmaxf(M, mS[i]);
        L = 0.0f;
        o = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
        for (int i = 0; i < WAVES; ++i) {
            const float f = fast_exp2(mS[i] - M);
            L = fmaf(f, lS[i], L);
#pragma unroll
            for (int e = 0; e < 4; ++e) o[e] = fmaf(f, oS[i][c][e], o[e]);
        }
    }
    if (sub == 0) {
        u32x2 ov;
        ov[0] = pack_bf16x2(o[0] / L, o[1] / L);
        ov[1] = pack_bf16x2(o[2] / L, o[3] / L);
        *reinterpret_cast<u32x2*>(out + 4 * c) = ov;
    }
}

}  // namespace slim
