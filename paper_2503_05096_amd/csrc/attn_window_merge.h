// Windowed verification attention: how the states of a unit's wavefronts become its result.  Shared by the matrix-core kernels.
#pragma once
#include "attn_mfma_common.h"
#include "attn_window.h"

namespace adaspec {

// State of one row over the entries [v0, v1) of its unit's list, by one wavefront: lane <-> token for the scores, lane <-> two
// channels side by side for the values.  A token that the row does not see is left out, whatever it holds.
template <class T, int D>
__device__ __forceinline__ void row_by_selection(const WindowUnit &u, const WindowDims &dims, const int32_t *block_table, const char *q,
                                                 const char *k_pages, const char *v_pages, int row, int v0, int v1, float scale_log2, float &m, float &l, float2 &acc)
{
    const int lane = threadIdx.x & 63, G = dims.Hq / dims.Hkv, pos = u.first_pos + row / G;
    const int64_t qbase = ((u.qrow0 + row / G) * dims.Hq + u.gkv * G + row % G) * (int64_t)D;
    m = -INFINITY; l = 0.f;
    acc = make_float2(0.f, 0.f);
    for (int vb = v0; vb < v1; vb += 4) {
        const int v = vb + (lane >> 4), pg = u.page_of(min(v, v1 - 1)), t = pg * 16 + (lane & 15);
        const bool vis = v < v1 && window_sees(u, pos, t);
        float s = -INFINITY;
        if (vis) {
            const int64_t at = (((int64_t)block_table[u.bt_off + pg] * dims.Hkv + u.gkv) * 16 + (lane & 15)) * D;
            s = 0.f;
            for (int c = 0; c < D; ++c) s = fmaf(load_as_float<T>(q, qbase + c), load_as_float<T>(k_pages, at + c), s);
            s *= scale_log2;
        }
        const float mn = fmaxf(m, wave_max(s));
        float p = 0.f, alpha = 1.f;
        if (mn > -INFINITY) {
            alpha = __builtin_amdgcn_exp2f(m - mn);
            p = vis ? __builtin_amdgcn_exp2f(s - mn) : 0.f;
        } else if (vis) {
            p = s == s ? 0.f : s;
        }
        l = l * alpha + wave_sum(p);
        m = mn;
        acc.x *= alpha; acc.y *= alpha;
        const unsigned long long seen = __ballot(vis);
        for (int tt = 0; tt < 64; ++tt) {
            if (!((seen >> tt) & 1)) continue;
            const float w = __shfl(p, tt, kWave);
            const int64_t at = (((int64_t)block_table[u.bt_off + u.page_of(vb + (tt >> 4))] * dims.Hkv + u.gkv) * 16 + (tt & 15)) * D;
            const int c = 2 * (lane & (D / 2 - 1));
            acc.x = fmaf(w, load_as_float<T>(v_pages, at + c), acc.x);
            acc.y = fmaf(w, load_as_float<T>(v_pages, at + c + 1), acc.y);
        }
    }
}

// A wavefront's state of one row tile in LDS: 16 rows of D fp32 values, whose 16-byte pieces are exchanged by the row's number so
// that neither who writes a piece per row nor who reads a row meets bank conflicts.
template <int D> __device__ __forceinline__ int window_piece(int row, int piece) { return row * (4 * D) + 16 * (piece ^ (row & (D / 4 - 1))); }

// Row tile nt of a unit, by its 256 threads: every wavefront has left its state of the tile at slabs + w * stride, and (m, l) of
// its rows in s_m, s_l [wavefront][kRows].
//   O = sum_w 2^(m_w - m*) O_w, m* = max over wavefronts.
// Thread: row tid / 16 of the tile, D / 16 channels.  The pages [v0, v1) of the unit's list are what the states cover; ns > 1: of
// several parts, whose states go to the rows of part_ml, part_o from `part` on.
template <class T, int D>
__device__ __forceinline__ void finish_window_tile(const WindowUnit &u, const WindowDims &dims, const int32_t *block_table, const char *q,
                                                   const char *k_pages, const char *v_pages, void *out, float *part_ml, float *part_o,
                                                   const char *slabs, int stride, const float *s_m, const float *s_l, int kRows, int nt, int ns,
                                                   int v0, int v1, float scale_log2, float shift_log2, int out_dtype, int64_t part)
{
    constexpr int kPieces = D / 64;
    const int tid = threadIdx.x, lane = tid & 63, wv = tid >> 6, G = dims.Hq / dims.Hkv;
    const int rt = tid >> 4, rl = 16 * nt + rt, row = u.r0 + rl;
    float ms = s_m[rl], ltot = 0.f;
#pragma unroll
    for (int w = 1; w < kWaves; ++w) ms = fmaxf(ms, s_m[w * kRows + rl]);
    f32x4 acc[kPieces];
#pragma unroll
    for (int p = 0; p < kPieces; ++p) acc[p] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
        const float sc = __builtin_amdgcn_exp2f(s_m[w * kRows + rl] - ms);
        ltot += sc * s_l[w * kRows + rl];
#pragma unroll
        for (int p = 0; p < kPieces; ++p)
            acc[p] += sc * *reinterpret_cast<const f32x4 *>(slabs + w * stride + window_piece<D>(rt, kPieces * (tid & 15) + p));
    }
    // a NaN or an infinity: the row's own, or that of a token which it does not see
    float total = ltot;
#pragma unroll
    for (int p = 0; p < kPieces; ++p) total += (acc[p][0] + acc[p][1]) + (acc[p][2] + acc[p][3]);
    unsigned long long odd = __ballot(row < u.rows && !(fabsf(total) < INFINITY));
    while (__builtin_expect(odd != 0, 0)) {
        const int of = (int)__builtin_ctzll(odd) >> 4;              // row of this wavefront, 0 .. 3
        float rm, rsum;
        float2 ra;
        row_by_selection<T, D>(u, dims, block_table, q, k_pages, v_pages, u.r0 + 16 * nt + 4 * wv + of, v0, v1, scale_log2, rm, rsum, ra);
#pragma unroll
        for (int p = 0; p < kPieces; ++p) {
            const int from = 2 * (kPieces * (lane & 15) + p);
            const f32x4 val = {__shfl(ra.x, from, kWave), __shfl(ra.y, from, kWave), __shfl(ra.x, from + 1, kWave), __shfl(ra.y, from + 1, kWave)};
            if (lane >> 4 == of) acc[p] = val;
        }
        if (lane >> 4 == of) { ms = rm + shift_log2; ltot = rsum; }         // (the stream's weights are that much larger)
        odd &= ~(0xffffull << (16 * of));
    }
    if (row >= u.rows) return;
    if (ns == 1) {
        const float inv = 1.0f / ltot;
        const int64_t obase = ((u.qrow0 + row / G) * dims.Hq + u.gkv * G + row % G) * (int64_t)D + 4 * kPieces * (tid & 15);
        if (sizeof(typename T::storage) == 4 || out_dtype == ADASPEC_F32) {
#pragma unroll
            for (int p = 0; p < kPieces; ++p) *reinterpret_cast<f32x4 *>(reinterpret_cast<float *>(out) + obase + 4 * p) = acc[p] * inv;
        } else if constexpr (sizeof(typename T::storage) == 2) {
            uint32_t w[2 * kPieces];
#pragma unroll
            for (int p = 0; p < kPieces; ++p) {
                w[2 * p] = Mma<T>::pack2(acc[p][0] * inv, acc[p][1] * inv);
                w[2 * p + 1] = Mma<T>::pack2(acc[p][2] * inv, acc[p][3] * inv);
            }
            uint16_t *to = reinterpret_cast<uint16_t *>(out) + obase;
            if constexpr (kPieces == 2) *reinterpret_cast<uint4 *>(to) = make_uint4(w[0], w[1], w[2], w[3]);
            else *reinterpret_cast<uint2 *>(to) = make_uint2(w[0], w[1]);
        }
    } else {
        const int64_t at = part + rl;
#pragma unroll
        for (int p = 0; p < kPieces; ++p) *reinterpret_cast<f32x4 *>(part_o + at * D + 4 * (kPieces * (tid & 15) + p)) = acc[p];
        if ((tid & 15) == 0) *reinterpret_cast<float2 *>(part_ml + at * 2) = make_float2(ms, ltot);
    }
}

}  // namespace adaspec
