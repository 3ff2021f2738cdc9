// Windowed verification attention for fp32 K/V/Q, head_dim 64 or 128 (v_mfma_f32_16x16x4: fp32 products and sums).
//
// The unit, its list of pages, the masks and the merge are those of attn_window_mfma.hip; the operands those of attn_f32.hip, which
// need neither LDS nor a transposition: wavefront w streams the pages w, w + 4, ... of the list through registers,
//   S^T[token][row] = K Q^T      lane (g, m) loads 4 channels of token m at channel 16 j + 4 g; element e is the A operand of step
//                                (j, e), whose four k-slots are the channels 16 j + 4 g + e;
//   O^T[d][row]    += V^T P^T    the accumulator lane (g, n) holds S^T[4 g + r][n]: step r takes it as B operand; lane (g, m) loads
//                                channels 64 h + 4 m .. + 3 of token 4 g + r, element e is the A operand of output tile (h, e).
//
// Up to 32 rows the reads bound it: 128 requests, 32 query on 8 kv heads, 3 drafts, window 1024: 182 us for 1095 MB at head_dim
// 128, 89 us for 547 MB at 64 (6.0-6.2 TB/s).  Beyond that the fp32 matrix products do (138 TFLOP/s in a large product): 64
// requests, 64 query heads, 48 rows 139 us, 93 of them products at that rate; 64 rows 178 and 124.  Two workgroups per compute
// unit wherever the registers last: at head_dim 64 always (64 rows: 88 us, one workgroup 105), at 128 up to 32 rows (48 rows:
// 139 us with one; two spill, 190; groups of 32 rows, which read the window twice, 196).
#include "attn_window_merge.h"

namespace adaspec {

__device__ __forceinline__ f32x4 window_mfma_f32(float a, float b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x4f32(a, b, c, 0, 0, 0); }

template <int D, int RT>
__global__ __launch_bounds__(256, (D == 64 || RT <= 2 ? 2 : 1)) void attn_window_f32_kernel(WindowDims dims, const int32_t *__restrict__ block_table,
                                                                                 const char *__restrict__ q, const char *__restrict__ k_pages,
                                                                                 const char *__restrict__ v_pages, void *__restrict__ out,
                                                                                 float *__restrict__ part_ml, float *__restrict__ part_o, int splits,
                                                                                 float scale_log2)
{
    constexpr int kRows = 16 * RT, kJ = D / 16, kH = D / 64, kSlab = 16 * D * 4, kQLoads = RT * kJ * 64 / 256;
    __shared__ __attribute__((aligned(16))) char slabs[kWaves * kSlab];
    __shared__ __attribute__((aligned(16))) f32x4 q_lds[RT * kJ * 64];     // Q^T operands, MFMA lane order
    __shared__ float s_m[kWaves * kRows], s_l[kWaves * kRows];
    const int tid = threadIdx.x, lane = tid & 63;
    const int wv = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int g = lane >> 4, n16 = lane & 15;
    const int G = dims.Hq / dims.Hkv;

    const int sp = blockIdx.z;
    int i, rg;
    window_place(dims, blockIdx.x, i, rg);
    const RowsBefore before(dims, i, lane);
    WindowUnit u;
    if (!window_unit(u, dims, i, rg, blockIdx.y)) return;
    const int per = (u.pages + splits - 1) / splits, ns = per > 0 ? (u.pages + per - 1) / per : 1;
    const int b0 = sp * per, b1 = min(u.pages, b0 + per);
    if (sp >= ns) return;

    constexpr int64_t head_bytes = (int64_t)16 * D * 4;
    const uint32_t k_lane_off = n16 * (D * 4) + 16 * g, v_lane_off = 4 * g * (D * 4) + 16 * n16;
    f32x4 kreg[kJ], vreg[4][kH];
    auto page_base = [&](int v) { return ((int64_t)block_table[u.bt_off + u.page_of(v)] * dims.Hkv + u.gkv) * head_bytes; };
    auto load_k = [&](int64_t at) {
#pragma unroll
        for (int j = 0; j < kJ; ++j) kreg[j] = __builtin_nontemporal_load(reinterpret_cast<const f32x4 *>(k_pages + at + k_lane_off + 64 * j));
    };
    auto load_v = [&](int64_t at) {
#pragma unroll
        for (int r = 0; r < 4; ++r)
#pragma unroll
            for (int h = 0; h < kH; ++h)
                vreg[r][h] = __builtin_nontemporal_load(reinterpret_cast<const f32x4 *>(v_pages + at + v_lane_off + r * (D * 4) + 256 * h));
    };
    if (b0 + wv < b1) {
        const int64_t at = page_base(b0 + wv);
        load_k(at);
        load_v(at);
    }
    u.qrow0 = before.sum(dims, i, lane);
    if (u.qrow0 + u.n > dims.total_q) return;                       // inconsistent lengths
    f32x4 qv[kQLoads];
#pragma unroll
    for (int k = 0; k < kQLoads; ++k) {                             // entry (row tile, j, lane)
        const int e = (tid >> 6) + 4 * k, row = min(u.r0 + 16 * (e / kJ) + n16, u.rows - 1);
        qv[k] = *reinterpret_cast<const f32x4 *>(q + (((u.qrow0 + row / G) * dims.Hq + u.gkv * G + row % G) * (int64_t)D + 16 * (e % kJ) + 4 * g) * 4);
    }
#pragma unroll
    for (int k = 0; k < kQLoads; ++k) q_lds[tid + 256 * k] = qv[k];
    lds_barrier();

    int pos[RT];
#pragma unroll
    for (int nt = 0; nt < RT; ++nt) {
        const int row = u.r0 + 16 * nt + n16;
        pos[nt] = row < u.rows ? u.first_pos + row / G : -1;
    }
    const int oldest = u.first_pos + u.r0 / G, newest = u.first_pos + (min(u.r0 + kRows, u.rows) - 1) / G;
    float m[RT], lsum[RT];
    f32x4 o[RT][kH][4];
#pragma unroll
    for (int nt = 0; nt < RT; ++nt) {
        m[nt] = kLowestRef; lsum[nt] = 0.f;
#pragma unroll
        for (int h = 0; h < kH; ++h)
#pragma unroll
            for (int e = 0; e < 4; ++e) o[nt][h][e] = f32x4{0.f, 0.f, 0.f, 0.f};
    }

    auto block = [&](int v, auto next_tag) {
        constexpr bool kNext = decltype(next_tag)::value;
        const int tb = u.page_of(v) * 16;
        const bool need_mask = tb + 15 > oldest || !(newest - tb < u.window || tb + 15 < u.sinks);
        int64_t nb = 0;
        if constexpr (kNext) nb = page_base(v + kWaves);

        // ---- S^T = K Q^T: two chains, so that one product's latency hides under the other's ----------
        f32x4 p[RT];
#pragma unroll
        for (int nt = 0; nt < RT; ++nt) {
            f32x4 acc0 = {0.f, 0.f, 0.f, 0.f}, acc1 = acc0;
#pragma unroll
            for (int j = 0; j < kJ; j += 2) {
                const f32x4 q0 = q_lds[(nt * kJ + j) * 64 + lane], q1 = q_lds[(nt * kJ + j + 1) * 64 + lane];
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    acc0 = window_mfma_f32(kreg[j][e], q0[e], acc0);
                    acc1 = window_mfma_f32(kreg[j + 1][e], q1[e], acc1);
                }
            }
            p[nt] = acc0 + acc1;
        }
        if constexpr (kNext) load_k(nb);

        // ---- online softmax (per lane: row n16 of each row tile, 4 of the 16 tokens) ----
#pragma unroll
        for (int nt = 0; nt < RT; ++nt) {
            if (need_mask) {
#pragma unroll
                for (int e = 0; e < 4; ++e) p[nt][e] = window_sees(u, pos[nt], tb + 4 * g + e) ? p[nt][e] : -INFINITY;
            }
            const float mx = max_over_row_groups(fmaxf(fmaxf(p[nt][0], p[nt][1]), fmaxf(p[nt][2], p[nt][3])));
            const float mxs = mx * scale_log2;
            const bool grow = mxs > m[nt] + kLazyLog2;
            if (__builtin_expect(__builtin_amdgcn_ballot_w64(grow) != 0, 0)) {
                const float m_new = grow ? mxs : m[nt];
                const float alpha = __builtin_amdgcn_exp2f(m[nt] - m_new);
                m[nt] = m_new;
                lsum[nt] *= alpha;
#pragma unroll
                for (int h = 0; h < kH; ++h)
#pragma unroll
                    for (int e = 0; e < 4; ++e) o[nt][h][e] *= alpha;
            }
            softmax_weights<4>(p[nt], scale_log2, m[nt], 0.f);
            lsum[nt] += (p[nt][0] + p[nt][1]) + (p[nt][2] + p[nt][3]);
        }

        // ---- O^T += V^T P^T; tokens that no row sees count as zero -----------------------------------
        if (need_mask) {
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const int t = tb + 4 * g + r;
                if (t > newest || (oldest - t >= u.window && t >= u.sinks)) {
#pragma unroll
                    for (int h = 0; h < kH; ++h) vreg[r][h] = f32x4{0.f, 0.f, 0.f, 0.f};
                }
            }
        }
#pragma unroll
        for (int r = 0; r < 4; ++r)
#pragma unroll
            for (int h = 0; h < kH; ++h)
#pragma unroll
                for (int e = 0; e < 4; ++e)
#pragma unroll
                    for (int nt = 0; nt < RT; ++nt) o[nt][h][e] = window_mfma_f32(vreg[r][h][e], p[nt][r], o[nt][h][e]);
        if constexpr (kNext) load_v(nb);
    };
    if (b0 + wv < b1) {
        int v = b0 + wv;
        for (; v + kWaves < b1; v += kWaves) block(v, std::true_type{});
        block(v, std::false_type{});
    }

    // ---- merge the four wavefronts' states through LDS, one row tile at a time.  Lane (g, n16) holds the channels
    // 64 h + 16 g + 4 r + e of row n16.
#pragma unroll
    for (int nt = 0; nt < RT; ++nt) {
        lsum[nt] += __shfl_xor(lsum[nt], 16, kWave);
        lsum[nt] += __shfl_xor(lsum[nt], 32, kWave);
        if (g == 0) { s_m[wv * kRows + 16 * nt + n16] = m[nt]; s_l[wv * kRows + 16 * nt + n16] = lsum[nt]; }
    }
#pragma unroll
    for (int nt = 0; nt < RT; ++nt) {
        if (u.r0 + 16 * nt >= u.rows) break;
#pragma unroll
        for (int h = 0; h < kH; ++h)
#pragma unroll
            for (int r = 0; r < 4; ++r)
                *reinterpret_cast<f32x4 *>(slabs + wv * kSlab + window_piece<D>(n16, 16 * h + 4 * g + r)) =
                    f32x4{o[nt][h][0][r], o[nt][h][1][r], o[nt][h][2][r], o[nt][h][3][r]};
        lds_barrier();
        finish_window_tile<F32, D>(u, dims, block_table, q, k_pages, v_pages, out, part_ml, part_o, slabs, kSlab, s_m, s_l, kRows, nt, ns, b0, b1, scale_log2,
                                   0.f, ADASPEC_F32, (((int64_t)blockIdx.x * dims.Hkv + blockIdx.y) * splits + sp) * kRows);
        if (nt + 1 < RT) lds_barrier();                             // the next tile overwrites the slabs
    }
}

hipError_t launch_attn_window_f32(const WindowArgs &a, const WindowDims &w)
{
    const WindowPlan &p = a.plan;
    auto launch = [&](auto dim, auto rt) {
        hipLaunchKernelGGL((attn_window_f32_kernel<decltype(dim)::value, decltype(rt)::value>), 
                           dim3((unsigned)(a.dims.batch * p.groups), a.dims.n_kv_heads, p.splits), dim3(256), 0, a.stream, w, a.block_table, (const char *)a.q, (const char *)a.k_pages, (const char *)a.v_pages, a.out,
                           (float *)(a.ws + p.off_part_ml), (float *)(a.ws + p.off_part_o), p.splits, a.scale_log2);
    };
    auto with_rt = [&](auto dim) {
        switch (p.rows_per_group / 16) {
        case 1: launch(dim, std::integral_constant<int, 1>{}); break;
        case 2: launch(dim, std::integral_constant<int, 2>{}); break;
        case 3: launch(dim, std::integral_constant<int, 3>{}); break;
        default: launch(dim, std::integral_constant<int, 4>{}); break;
        }
    };
    if (a.dims.head_dim == 128) with_rt(std::integral_constant<int, 128>{});
    else with_rt(std::integral_constant<int, 64>{});
    return hipGetLastError();
}

}  // namespace adaspec
