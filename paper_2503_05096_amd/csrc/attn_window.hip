// Windowed verification attention: the plan of a call, the merge of a unit's parts, and the portable form: any of the three storage types, any head_dim that is a multiple of 8 up
// to 256.  One wavefront per (request, kv head, chunk of 8 query rows).
//
// Per 64 tokens: lane <-> token for the scores (each lane walks its key row, the query rows are broadcast from LDS),
// wavefront reductions for the online softmax, then lane <-> channel for P.V.  A token that a row does not see has a weight
// below zero in LDS and is left out of that row's sum, not multiplied by zero: whatever it holds cannot reach the row.
#include <type_traits>

#include "attn_window.h"

namespace adaspec {

constexpr int kWinRows = 8;
constexpr int kWinMaxD = 256;
constexpr int kWindowMaxSplits = 64;        // a lane of the combine kernel each

template <class T>
__global__ __launch_bounds__(64) void attn_window_vector_kernel(WindowDims dims, const void *__restrict__ q,
                                                                const void *__restrict__ k_pages, const void *__restrict__ v_pages,
                                                                void *__restrict__ out, int d, float scale_log2, int out_dtype)
{
    __shared__ float qs[kWinRows][kWinMaxD];
    __shared__ float ps[kWinRows][64];
    const int lane = threadIdx.x;
    const int G = dims.Hq / dims.Hkv;
    const int gkv = blockIdx.y, i = blockIdx.x / dims.groups;
    const RowsBefore before(dims, i, lane);
    WindowUnit u;
    if (!window_unit(u, dims, i, blockIdx.x % dims.groups, gkv)) return;
    u.qrow0 = before.sum(dims, i, lane);
    if (u.qrow0 + u.n > dims.total_q) return;                       // inconsistent lengths

    for (int idx = lane; idx < kWinRows * d; idx += 64) {
        const int r = u.r0 + idx / d, c = idx % d;
        qs[idx / d][c] = r < u.rows ? load_as_float<T>(q, ((u.qrow0 + r / G) * dims.Hq + gkv * G + r % G) * d + c) : 0.f;
    }
    __syncthreads();

    float m[kWinRows], l[kWinRows], acc[kWinRows][4];
#pragma unroll
    for (int r = 0; r < kWinRows; ++r) {
        m[r] = -INFINITY; l[r] = 0.f;
#pragma unroll
        for (int e = 0; e < 4; ++e) acc[r][e] = 0.f;
    }
    for (int v0 = 0; v0 < u.pages; v0 += 4) {
        const int v = v0 + (lane >> 4);
        const int pg = u.page_of(min(v, u.pages - 1)), t = pg * 16 + (lane & 15);
        const bool valid = v < u.pages && t < u.L;
        float sc[kWinRows];
#pragma unroll
        for (int r = 0; r < kWinRows; ++r) sc[r] = 0.f;
        if (valid) {
            const int64_t page = dims.block_table[u.bt_off + pg];
            const int64_t koff = ((page * dims.Hkv + gkv) * 16 + (lane & 15)) * (int64_t)d;
            for (int c = 0; c < d; c += 8) {
                float kv[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) kv[e] = load_as_float<T>(k_pages, koff + c + e);
#pragma unroll
                for (int r = 0; r < kWinRows; ++r)
#pragma unroll
                    for (int e = 0; e < 8; ++e) sc[r] = fmaf(qs[r][c + e], kv[e], sc[r]);
            }
        }
        __syncthreads();                                            // the last 64 tokens' weights have been read
#pragma unroll
        for (int r = 0; r < kWinRows; ++r) {
            const int row = u.r0 + r;
            const bool vis = valid && row < u.rows && window_sees(u, u.first_pos + row / G, t);
            const float sv = vis ? sc[r] * scale_log2 : -INFINITY;
            const float mn = fmaxf(m[r], wave_max(sv));
            float p = 0.f, alpha = 1.f;
            if (mn > -INFINITY) {
                alpha = __builtin_amdgcn_exp2f(m[r] - mn);
                p = vis ? __builtin_amdgcn_exp2f(sv - mn) : 0.f;
            } else if (vis) {
                p = sv == sv ? 0.f : sv;                            // (every score so far is -inf or NaN)
            }
            l[r] = l[r] * alpha + wave_sum(p);
            m[r] = mn;
#pragma unroll
            for (int e = 0; e < 4; ++e) acc[r][e] *= alpha;
            ps[r][lane] = vis ? p : -1.f;
        }
        __syncthreads();
        const int most = min(4, u.pages - v0) * 16;
        for (int tt = 0; tt < most; ++tt) {
            const int pv = u.page_of(v0 + (tt >> 4));
            if (pv * 16 + (tt & 15) >= u.L) break;                  // (the last page of the list is the newest)
            const int64_t page = dims.block_table[u.bt_off + pv];
            const int64_t voff = ((page * dims.Hkv + gkv) * 16 + (tt & 15)) * (int64_t)d;
            float vv[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int c = lane + 64 * e;
                vv[e] = c < d ? load_as_float<T>(v_pages, voff + c) : 0.f;
            }
#pragma unroll
            for (int r = 0; r < kWinRows; ++r) {
                const float p = ps[r][tt];
#pragma unroll
                for (int e = 0; e < 4; ++e) acc[r][e] = p < 0.f ? acc[r][e] : fmaf(p, vv[e], acc[r][e]);
            }
        }
    }
#pragma unroll
    for (int r = 0; r < kWinRows; ++r) {
        const int row = u.r0 + r;
        if (row >= u.rows) continue;
        const float inv = 1.0f / l[r];
        const int64_t obase = ((u.qrow0 + row / G) * dims.Hq + gkv * G + row % G) * (int64_t)d;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const int c = lane + 64 * e;
            if (c < d) store_out(out, obase + c, acc[r][e] * inv, out_dtype);
        }
    }
}

// Rows of a unit whose pages were cut: out = sum_s 2^(m_s - m*) O_s / sum_s 2^(m_s - m*) l_s.  One wavefront per row, four
// rows of a unit per workgroup; lane s looks at (m_s, l_s).  Latency is all there is to it: the states of the first parts are
// requested before it is known how many parts there are (the places are there in any case).
template <int D>
__global__ __launch_bounds__(256) void attn_window_combine_kernel(WindowDims dims, const float *__restrict__ part_ml,
                                                                  const float *__restrict__ part_o, void *__restrict__ out, int splits,
                                                                  int block_pages, int out_dtype)
{
    constexpr int kE = D / 64, kAhead = 16;
    const int lane = threadIdx.x & 63, wv = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int i = blockIdx.x / dims.groups, rl = 4 * blockIdx.z + wv;
    const RowsBefore before(dims, i, lane);
    const int64_t first = ((int64_t)blockIdx.x * dims.Hkv + blockIdx.y) * splits * dims.rows_per_group + rl;
    float2 ml = make_float2(-INFINITY, 0.f);
    if (lane < splits) ml = *reinterpret_cast<const float2 *>(part_ml + (first + (int64_t)lane * dims.rows_per_group) * 2);
    const float *o = part_o + first * D + kE * lane;
    float x[kAhead][kE];
#pragma unroll
    for (int s = 0; s < kAhead; ++s)
#pragma unroll
        for (int e = 0; e < kE; ++e) x[s][e] = s < splits ? o[(int64_t)s * dims.rows_per_group * D + e] : 0.f;
    WindowUnit u;
    if (!window_unit(u, dims, i, blockIdx.x % dims.groups, blockIdx.y)) return;
    const int row = u.r0 + rl;
    const int all_blocks = (u.pages + block_pages - 1) / block_pages, per = (all_blocks + splits - 1) / splits;
    const int ns = per > 0 ? (all_blocks + per - 1) / per : 1;      // (at most kWindowMaxSplits)
    u.qrow0 = before.sum(dims, i, lane);
    if (ns == 1 || row >= u.rows || u.qrow0 + u.n > dims.total_q) return;
    if (lane >= ns) ml = make_float2(-INFINITY, 0.f);
    const float m = wave_max(ml.x);
    const float w = lane < ns ? (m > -INFINITY ? __builtin_amdgcn_exp2f(ml.x - m) : 1.f) : 0.f;
    const float inv = 1.0f / wave_sum(w * ml.y);
    float acc[kE] = {};
#pragma unroll
    for (int s = 0; s < kAhead; ++s) {
        const float ws = __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, w), s));
        if (s < ns) {
#pragma unroll
            for (int e = 0; e < kE; ++e) acc[e] += ws * x[s][e];
        }
    }
    for (int s = kAhead; s < ns; ++s) {
        const float ws = __shfl(w, s, kWave);
#pragma unroll
        for (int e = 0; e < kE; ++e) acc[e] += ws * o[(int64_t)s * dims.rows_per_group * D + e];
    }
    const int G = dims.Hq / dims.Hkv;
    const int64_t obase = ((u.qrow0 + row / G) * dims.Hq + u.gkv * G + row % G) * (int64_t)D + kE * lane;
#pragma unroll
    for (int e = 0; e < kE; ++e) store_out(out, obase + e, acc[e] * inv, out_dtype);
}

bool window_fast_supported(const adaspec_attn_dims &d)
{
    return d.head_dim == 64 || d.head_dim == 128;
}

WindowPlan make_window_plan(const adaspec_attn_dims &d, int window, int sinks)
{
    WindowPlan p;
    const int G = d.n_q_heads / d.n_kv_heads;
    const int64_t rows = (int64_t)(d.max_spec_len + 1) * G;
    p.kind = d.path != ADASPEC_PATH_VECTOR && window_fast_supported(d) ? WindowKind::kMfma : WindowKind::kVector;
    p.rows_per_group = p.kind == WindowKind::kVector ? kWinRows : 16 * (int)(rows < 64 ? (rows + 15) / 16 : 4);
    p.groups = (int)((rows + p.rows_per_group - 1) / p.rows_per_group);
    p.units = (int64_t)d.batch * d.n_kv_heads * p.groups;
    p.splits = 1;
    p.alone = false;
    p.block_pages = d.dtype == ADASPEC_F32 ? 1 : d.head_dim == 64 ? 4 : 2;
    if (p.kind == WindowKind::kMfma) {
        // entries of a unit's list of pages at most: a row group spans this many positions
        const int64_t span = (p.rows_per_group - 1) / G + 2 < d.max_spec_len + 1 ? (p.rows_per_group - 1) / G + 2 : d.max_spec_len + 1;
        int64_t pages = ((int64_t)sinks + 15) / 16 + ((int64_t)window + span + 14) / 16 + 1;
        if (pages > d.max_pages_per_req) pages = d.max_pages_per_req;
        const int64_t blocks = (pages + p.block_pages - 1) / p.block_pages, turns = (blocks + 3) / 4;   // turns of four wavefronts
        // One wavefront per unit where units are many and short.  A workgroup of four costs its look-ups, its merging and its
        // quarter-filled last turn whatever the length: 512 of them fill the chip, a thousand lone wavefronts take their place.
        // Measured, alone / four (us, 16 bits, 8 kv heads, 1-3 drafts; window 16, 128, 256, 512, 1024):
        //   head_dim 128, 320 units   7.5/7.3   11.6/9.9    17.0/12.7  27.8/19.7   48.8/33.9
        //   head_dim 128, 528 units   8.0/10.3  13.2/15.4   20.0/20.4  33.1/31.3   59.6/53.5
        //   head_dim 128, 1152 units  10.4/15.6 19.8/25.1   32.0/33.6  56.7/55.2  105.7/101.7
        //   head_dim 64, 1152 units   7.7/14.6  13.4/16.9   19.6/25.2  31.9/32.7   56.3/53.8
        p.alone = d.dtype != ADASPEC_F32 && p.rows_per_group <= 48 && p.units > 512 && blocks <= 10;
        // Parts of a unit where units are few: one workgroup per compute unit in all, at least two blocks in a part, and only
        // where that saves the joining launch's 3-4 us: four turns, or eight with less than four parts, whose workgroups
        // still wait for each other's memory.  Measured, parts / whole (us, head_dim 128, 16 bits):
        //   window 1024: 8 units, 16 parts 10.7/17.6; 64 units, 4 parts 15.7/18.6; 128 units, 2 parts 21.0/19.5; 256 units, 2 parts 33/26.5
        //   window 4096: 8 units, 16 parts 13.5/47.7; 64 units, 4 parts 29.9/49.0; 128 units, 2 parts 50.0/53.5
        if (!p.alone && p.units > 0) {
            int64_t want = 256 / p.units;
            if (want > blocks / 2) want = blocks / 2;
            if (want > kWindowMaxSplits) want = kWindowMaxSplits;
            if (want > 1 && turns - (blocks + 4 * want - 1) / (4 * want) >= (want >= 4 ? 4 : 8)) p.splits = (int)want;
        }
    }
    size_t off = 0;
    p.off_part_ml = off;
    if (p.splits > 1) off = align_up(off + (size_t)p.units * p.splits * p.rows_per_group * 2 * sizeof(float), 256);
    p.off_part_o = off;
    if (p.splits > 1) off = align_up(off + (size_t)p.units * p.splits * p.rows_per_group * d.head_dim * sizeof(float), 256);
    p.total_bytes = off > 0 ? off : 256;
    return p;
}

hipError_t launch_attn_window(const WindowArgs &a)
{
    const adaspec_attn_dims &d = a.dims;
    const WindowDims w{a.block_table, a.ctx_lens, a.spec_lens, d.batch, d.total_q, d.max_spec_len, d.max_pages_per_req, d.n_q_heads,
                       d.n_kv_heads, a.window, a.sinks, a.plan.groups, a.plan.rows_per_group};
    const WindowPlan &p = a.plan;
    if (p.kind == WindowKind::kMfma) {
        const hipError_t e = d.dtype == ADASPEC_F32 ? launch_attn_window_f32(a, w) : launch_attn_window_mfma(a, w);
        if (e != hipSuccess || p.splits == 1) return e;
        auto combine = [&](auto dim) {
            hipLaunchKernelGGL((attn_window_combine_kernel<decltype(dim)::value>), dim3((unsigned)(d.batch * p.groups), d.n_kv_heads, p.rows_per_group / 4), dim3(256), 0,
                               a.stream, w, (const float *)(a.ws + p.off_part_ml), (const float *)(a.ws + p.off_part_o), a.out, p.splits,
                               p.block_pages, d.out_dtype);
        };
        if (d.head_dim == 128) combine(std::integral_constant<int, 128>{});
        else combine(std::integral_constant<int, 64>{});
        return hipGetLastError();
    }
    auto launch = [&](auto tag) {
        hipLaunchKernelGGL(attn_window_vector_kernel<decltype(tag)>, dim3((unsigned)(d.batch * a.plan.groups), d.n_kv_heads), dim3(64), 0, a.stream, w, a.q,
                           a.k_pages, a.v_pages, a.out, d.head_dim, a.scale_log2, d.out_dtype);
    };
    if (d.dtype == ADASPEC_F32) launch(F32{});
    else if (d.dtype == ADASPEC_F16) launch(F16{});
    else launch(BF16{});
    return hipGetLastError();
}

}  // namespace adaspec
