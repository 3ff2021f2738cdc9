// Windowed verification attention: the plan of a call, the merge of a unit's parts, and the portable form: any of the three
// storage types, any head_dim that is a multiple of 8 up to 256.  A workgroup of four wavefronts per (request, kv head, chunk of
// 8 or 4 query rows); wavefront w takes the 64 tokens w, w + 4, ... of the unit's list of pages.
//
// Per 64 tokens: lane <-> token for the scores (each lane walks its key row in pieces of 8 channels, the query rows are broadcast
// from LDS), wavefront reductions for the online softmax, then lane <-> two channels side by side for P.V, 16 value rows (8 above 128
// channels) under way at a time.  In pages that some row does not see whole, a token that a row does not see has a weight below zero in LDS
// and is left out of that row's sum, not multiplied by zero: whatever it holds cannot reach the row.
//
// Its vector units bound it: 16 multiply-adds per value of K and of V that arrives, twice as many instructions with unpacking
// and LDS; with few units the latency of a wavefront's turns does.  Window 1024, 32 requests of 16 rows at 8 kv heads: 81 us for
// 102 MB (bf16, head_dim 96; one wavefront per unit, a value row at a time: 1125), 172 us for 273 MB (head_dim 256; 2236), 92 us
// for 204 MB (fp32, 96; 855).
#include <type_traits>

#include "attn_window.h"

namespace adaspec {

constexpr int kWinWaves = 4;
constexpr int kWindowMaxSplits = 64;        // a lane of the combine kernel each

// 8 values side by side, from a multiple of 8 on
template <class T> __device__ __forceinline__ void load8(const void *base, int64_t at, float (&v)[8])
{
    if constexpr (sizeof(typename T::storage) == 4) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const float4 x = reinterpret_cast<const float4 *>(base)[at / 4 + h];
            v[4 * h] = x.x; v[4 * h + 1] = x.y; v[4 * h + 2] = x.z; v[4 * h + 3] = x.w;
        }
    } else {
        const uint4 x = reinterpret_cast<const uint4 *>(base)[at / 8];
        const uint32_t w[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            v[2 * e] = load_as_float<T>(&w[e], 0);
            v[2 * e + 1] = load_as_float<T>(&w[e], 1);
        }
    }
}
template <class T> struct Pair { typedef uint32_t type; };
template <> struct Pair<F32> { typedef float2 type; };
template <class T> __device__ __forceinline__ float2 pair_values(typename Pair<T>::type x)
{
    return make_float2(load_as_float<T>(&x, 0), load_as_float<T>(&x, 1));
}

// kP: pairs of channels that a lane has, head_dim at most 128 kP; kWinRows: 8, or 4 where no request has more
template <class T, int kP, int kWinRows>
__global__ __launch_bounds__(64 * kWinWaves, kP == 1 ? 4 : 3) void attn_window_vector_kernel(WindowDims dims, const void *__restrict__ q,
                                                                            const void *__restrict__ k_pages,
                                                                            const void *__restrict__ v_pages, void *__restrict__ out, int d,
                                                                            float scale_log2, int out_dtype)
{
    constexpr int kD = 128 * kP, kAhead = 16 / kP;                  // value rows under way
    typedef typename Pair<T>::type pair;
    // Q rows and weights of every wavefront; then its state.  (12 or 16 KB; 16 or 32)
    __shared__ __attribute__((aligned(16))) float smem[kWinWaves * kWinRows * kD];
    static_assert(kD + kWinWaves * 64 <= kWinWaves * kD, "Q and weights fit where the states go");
    __shared__ float s_m[kWinWaves][kWinRows], s_l[kWinWaves][kWinRows];
    const int tid = threadIdx.x, lane = tid & 63, wv = __builtin_amdgcn_readfirstlane(tid >> 6);
    float *qs = smem, *ps = smem + kWinRows * kD + wv * 64 * kWinRows;      // [row][channel]; [token][row]
    const int G = dims.Hq / dims.Hkv;
    const int gkv = blockIdx.y;
    int i, rg;
    window_place(dims, blockIdx.x, i, rg);
    const RowsBefore before(dims, i, lane);
    WindowUnit u;
    if (!window_unit(u, dims, i, rg, gkv)) return;
    u.qrow0 = before.sum(dims, i, lane);
    if (u.qrow0 + u.n > dims.total_q) return;                       // inconsistent lengths

    for (int idx = tid; idx < kWinRows * (d / 8); idx += 64 * kWinWaves) {
        const int r = idx / (d / 8), row = min(u.r0 + r, u.rows - 1), c = 8 * (idx % (d / 8));
        float v[8];
        load8<T>(q, ((u.qrow0 + row / G) * dims.Hq + gkv * G + row % G) * d + c, v);
#pragma unroll
        for (int e = 0; e < 8; ++e) qs[r * kD + c + e] = v[e];
    }
    __syncthreads();

    int pos[kWinRows];
#pragma unroll
    for (int r = 0; r < kWinRows; ++r) pos[r] = u.r0 + r < u.rows ? u.first_pos + (u.r0 + r) / G : -1;
    const int oldest = u.first_pos + u.r0 / G, newest = u.first_pos + (min(u.r0 + kWinRows, u.rows) - 1) / G;
    float m[kWinRows], l[kWinRows], acc[kWinRows][2 * kP];          // l: this lane's tokens only
#pragma unroll
    for (int r = 0; r < kWinRows; ++r) {
        m[r] = -INFINITY; l[r] = 0.f;
#pragma unroll
        for (int e = 0; e < 2 * kP; ++e) acc[r][e] = 0.f;
    }
    for (int v0 = 4 * wv; v0 < u.pages; v0 += 4 * kWinWaves) {
        const int v = v0 + (lane >> 4), pg = u.page_of(min(v, u.pages - 1)), t = pg * 16 + (lane & 15);
        const bool there = v < u.pages;
        const int page = dims.block_table[u.bt_off + pg];
        const int64_t koff = (((int64_t)page * dims.Hkv + gkv) * 16 + (lane & 15)) * d;
        float sc[kWinRows];
#pragma unroll
        for (int r = 0; r < kWinRows; ++r) sc[r] = 0.f;
#pragma unroll 4
        for (int c = 0; c < d; c += 8) {
            float kv[8];
            load8<T>(k_pages, koff + c, kv);
#pragma unroll
            for (int r = 0; r < kWinRows; ++r) {
                const float4 a = *reinterpret_cast<const float4 *>(qs + r * kD + c), b = *reinterpret_cast<const float4 *>(qs + r * kD + c + 4);
                sc[r] = fmaf(a.x, kv[0], sc[r]); sc[r] = fmaf(a.y, kv[1], sc[r]); sc[r] = fmaf(a.z, kv[2], sc[r]); sc[r] = fmaf(a.w, kv[3], sc[r]);
                sc[r] = fmaf(b.x, kv[4], sc[r]); sc[r] = fmaf(b.y, kv[5], sc[r]); sc[r] = fmaf(b.z, kv[6], sc[r]); sc[r] = fmaf(b.w, kv[7], sc[r]);
            }
        }
        float p[kWinRows];
#pragma unroll
        for (int r = 0; r < kWinRows; ++r) {
            const bool vis = there && window_sees(u, pos[r], t);
            const float sv = vis ? sc[r] * scale_log2 : -INFINITY;
            const float mn = fmaxf(m[r], wave_max(sv));
            float alpha = 1.f;
            p[r] = 0.f;
            if (mn > -INFINITY) {
                alpha = __builtin_amdgcn_exp2f(m[r] - mn);
                p[r] = vis ? __builtin_amdgcn_exp2f(sv - mn) : 0.f;
            } else if (vis) {
                p[r] = sv == sv ? 0.f : sv;                         // (every score so far is -inf or NaN)
            }
            l[r] = l[r] * alpha + p[r];
            m[r] = mn;
#pragma unroll
            for (int e = 0; e < 2 * kP; ++e) acc[r][e] *= alpha;
            if (!vis) p[r] = -1.f;
        }
        // (the wavefront's own part of LDS, whose accesses keep their order)
#pragma unroll
        for (int r = 0; r < kWinRows; r += 4)
            *reinterpret_cast<float4 *>(ps + lane * kWinRows + r) = make_float4(p[r], p[r + 1], p[r + 2], p[r + 3]);
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
        for (int j = 0; j < 4 && v0 + j < u.pages; ++j) {
            const int tb = u.page_of(v0 + j) * 16;
            const int64_t voff = ((int64_t)__builtin_amdgcn_readlane(page, 16 * j) * dims.Hkv + gkv) * 16 * d;
            const bool whole = tb + 15 <= oldest && (newest - tb < u.window || tb + 15 < u.sinks);
            pair x[kAhead][kP];
            auto request = [&](int t0) {
#pragma unroll
                for (int tt = 0; tt < kAhead; ++tt)
#pragma unroll
                    for (int k = 0; k < kP; ++k) {
                        const int c = min(2 * lane + 128 * k, d - 2);       // (lanes behind the last channel repeat it)
                        x[tt][k] = *reinterpret_cast<const pair *>(reinterpret_cast<const typename T::storage *>(v_pages) + voff + (t0 + tt) * d + c);
                    }
            };
            auto add = [&](int t0, auto all) {                      // all: every row sees every token of the page
#pragma unroll
                for (int tt = 0; tt < kAhead; ++tt) {
                    const float *at = ps + (16 * j + t0 + tt) * kWinRows;
                    float w[kWinRows];
#pragma unroll
                    for (int r = 0; r < kWinRows; r += 4) {
                        const float4 a = *reinterpret_cast<const float4 *>(at + r);
                        w[r] = a.x; w[r + 1] = a.y; w[r + 2] = a.z; w[r + 3] = a.w;
                    }
#pragma unroll
                    for (int k = 0; k < kP; ++k) {
                        const float2 val = pair_values<T>(x[tt][k]);
#pragma unroll
                        for (int r = 0; r < kWinRows; ++r) {
                            const float y0 = fmaf(w[r], val.x, acc[r][2 * k]), y1 = fmaf(w[r], val.y, acc[r][2 * k + 1]);
                            const bool in = decltype(all)::value || !(w[r] < 0.f);
                            acc[r][2 * k] = in ? y0 : acc[r][2 * k];
                            acc[r][2 * k + 1] = in ? y1 : acc[r][2 * k + 1];
                        }
                    }
                }
            };
            for (int t0 = 0; t0 < 16; t0 += kAhead) {
                request(t0);
                if (whole) add(t0, std::true_type{});
                else add(t0, std::false_type{});
            }
        }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
    }
    // O = sum_w 2^(m_w - m*) O_w, m* = max over wavefronts
    __syncthreads();
#pragma unroll
    for (int r = 0; r < kWinRows; ++r) {
        const float all = wave_sum(l[r]);
        if (lane == 0) { s_m[wv][r] = m[r]; s_l[wv][r] = all; }
#pragma unroll
        for (int k = 0; k < kP; ++k)
            *reinterpret_cast<float2 *>(smem + (wv * kWinRows + r) * kD + 2 * lane + 128 * k) = make_float2(acc[r][2 * k], acc[r][2 * k + 1]);
    }
    __syncthreads();
    constexpr int kAcross = 64 * kWinWaves / kWinRows;              // threads of a row
    const int r = tid / kAcross, row = u.r0 + r;
    if (row >= u.rows) return;
    float ms = s_m[0][r], ltot = 0.f, sc[kWinWaves];
#pragma unroll
    for (int w = 1; w < kWinWaves; ++w) ms = fmaxf(ms, s_m[w][r]);
#pragma unroll
    for (int w = 0; w < kWinWaves; ++w) {
        sc[w] = ms > -INFINITY ? __builtin_amdgcn_exp2f(s_m[w][r] - ms) : 1.f;
        ltot += sc[w] * s_l[w][r];
    }
    const float inv = 1.0f / ltot;
    const int64_t obase = ((u.qrow0 + row / G) * dims.Hq + gkv * G + row % G) * (int64_t)d;
    for (int c = tid % kAcross; c < d; c += kAcross) {
        float o = 0.f;
#pragma unroll
        for (int w = 0; w < kWinWaves; ++w) o += sc[w] * smem[(w * kWinRows + r) * kD + c];
        store_out(out, obase + c, o * inv, out_dtype);
    }
}

// Rows of a unit whose pages were cut: out = sum_s 2^(m_s - m*) O_s / sum_s 2^(m_s - m*) l_s.  One wavefront per row, four
// rows of a unit per workgroup; lane s looks at (m_s, l_s).  Latency is all there is to it: the states of the first parts are
// requested before it is known how many parts there are (the places are there in any case).  4.9 us for 8 units of 24 rows in 16
// parts, of which a call sees 3.7 behind the main kernel.
template <int D>
__global__ __launch_bounds__(256) void attn_window_combine_kernel(WindowDims dims, const float *__restrict__ part_ml,
                                                                  const float *__restrict__ part_o, void *__restrict__ out, int splits,
                                                                  int block_pages, int out_dtype)
{
    constexpr int kE = D / 64, kAhead = 16;
    const int lane = threadIdx.x & 63, wv = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int rl = 4 * blockIdx.z + wv;
    int i, rg;
    window_place(dims, blockIdx.x, i, rg);
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
    if (!window_unit(u, dims, i, rg, blockIdx.y)) return;
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
    const int64_t rows = (int64_t)(d.max_spec_len + 1) * G, tiles = (rows + 15) / 16;
    p.kind = d.path != ADASPEC_PATH_VECTOR && window_fast_supported(d) ? WindowKind::kMfma : WindowKind::kVector;
    p.block_pages = d.dtype == ADASPEC_F32 ? 1 : d.head_dim == 64 ? 4 : 2;
    // as few groups of up to `most` 16-row tiles as there can be, of equal numbers of tiles (portable form: of 4 `most` rows)
    auto group = [&](int most) {
        const int64_t least = (tiles + most - 1) / most;
        p.rows_per_group = p.kind == WindowKind::kVector ? 4 * most : 16 * (int)((tiles + least - 1) / least);
        p.groups = (int)((rows + p.rows_per_group - 1) / p.rows_per_group);
        p.units = (int64_t)d.batch * d.n_kv_heads * p.groups;
    };
    // blocks of a unit's list of pages at most: a row group spans this many positions
    auto most_blocks = [&]() {
        const int64_t across = (p.rows_per_group - 1) / G + 2, span = across < d.max_spec_len + 1 ? across : d.max_spec_len + 1;
        const int64_t pages = ((int64_t)sinks + 15) / 16 + ((int64_t)window + span + 14) / 16 + 1;
        return ((pages < d.max_pages_per_req ? pages : d.max_pages_per_req) + p.block_pages - 1) / p.block_pages;
    };
    p.splits = 1;
    p.alone = false;
    if (p.kind == WindowKind::kVector) {
        // Units of four rows where there are no more, and where they leave room: a unit of eight takes up to twice as long, two of
        // four read K and V twice.  Four / eight (us; window 512, head_dim 96 bf16, 256 fp32):
        //   32 units of four rows 20/38, 55/80;  512 units 26/43, 99/100;  2048 units 85/95, 400/338;  4096 units 132/129, 610/424
        // and one row per kv head, 2048 units of which there are as many either way: 64/104, 300/299 (window 256).
        group(1);
        if (rows > 4 && p.units > 512) group(2);
    } else {
        group(4);
    }
    if (p.kind == WindowKind::kMfma) {
        int64_t blocks = most_blocks();
        // One wavefront per unit where units are many and short.  A workgroup of four costs its look-ups, its merging and its
        // quarter-filled last turn whatever the length: 512 of them fill the chip, a thousand lone wavefronts take their place.
        // Measured, alone / four (us, 16 bits, 8 kv heads, 1-3 drafts; window 16, 128, 256, 512, 1024):
        //   head_dim 128, 320 units   7.5/7.3   11.6/9.9    17.0/12.7  27.8/19.7   48.8/33.9
        //   head_dim 128, 528 units   8.0/10.3  13.2/15.4   20.0/20.4  33.1/31.3   59.6/53.5
        //   head_dim 128, 1152 units  10.4/15.6 19.8/25.1   32.0/33.6  56.7/55.2  105.7/101.7
        //   head_dim 64, 1152 units   7.7/14.6  13.4/16.9   19.6/25.2  31.9/32.7   56.3/53.8
        // A lone wavefront has registers for 48 rows; larger groups are cut into more, which read the window again.  8 kv heads, 64
        // rows, window 16, 128, 256:  head_dim 128, 128 requests 20/27, 33/39, 51/48; 200 requests 31/43, 55/61, 89/74;
        //                             head_dim 64, 200 requests 18/39, 34/43, 51/62.
        p.alone = d.dtype != ADASPEC_F32 && p.units > 512 && blocks <= (p.rows_per_group > 48 ? 7 : 10);
        if (p.alone && p.rows_per_group > 48) {
            group(3);
            blocks = most_blocks();
        }
        // Parts of a unit where units are few: one workgroup per compute unit in all, at least two blocks in a part, and only
        // where that saves the joining launch's 3-4 us: four turns, or eight with less than four parts, whose workgroups
        // still wait for each other's memory.  Measured, parts / whole (us, head_dim 128, 16 bits):
        //   window 1024: 8 units, 16 parts 10.7/17.6; 64 units, 4 parts 15.7/18.6; 128 units, 2 parts 21.0/19.5; 256 units, 2 parts 33/26.5
        //   window 4096: 8 units, 16 parts 13.5/47.7; 64 units, 4 parts 29.9/49.0; 128 units, 2 parts 50.0/53.5
        const int64_t turns = (blocks + 3) / 4;                     // of four wavefronts
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

static WindowDims window_dims(const WindowArgs &a)
{
    const adaspec_attn_dims &d = a.dims;
    return {a.block_table, a.ctx_lens, a.spec_lens, d.batch, d.total_q, d.max_spec_len, d.max_pages_per_req, d.n_q_heads, d.n_kv_heads, a.window,
            a.sinks, a.plan.groups, a.plan.rows_per_group};
}

hipError_t launch_attn_window_combine(const WindowArgs &a)
{
    const adaspec_attn_dims &d = a.dims;
    const WindowPlan &p = a.plan;
    auto combine = [&](auto dim) {
        hipLaunchKernelGGL((attn_window_combine_kernel<decltype(dim)::value>),
                           dim3((unsigned)(d.batch * p.groups), d.n_kv_heads, p.rows_per_group / 4), dim3(256), 0, a.stream, window_dims(a), (const float *)(a.ws + p.off_part_ml), (const float *)(a.ws + p.off_part_o), a.out, p.splits,
                           p.block_pages, d.out_dtype);
    };
    if (d.head_dim == 128) combine(std::integral_constant<int, 128>{});
    else combine(std::integral_constant<int, 64>{});
    return hipGetLastError();
}

hipError_t launch_attn_window(const WindowArgs &a)
{
    const adaspec_attn_dims &d = a.dims;
    const WindowDims w = window_dims(a);
    const WindowPlan &p = a.plan;
    if (p.kind == WindowKind::kMfma) return d.dtype == ADASPEC_F32 ? launch_attn_window_f32(a, w) : launch_attn_window_mfma(a, w);
    auto launch = [&](auto tag, auto pairs, auto rows) {
        hipLaunchKernelGGL((attn_window_vector_kernel<decltype(tag), decltype(pairs)::value, decltype(rows)::value>),
                           dim3((unsigned)(d.batch * a.plan.groups), d.n_kv_heads), dim3(64 * kWinWaves), 0, a.stream, w, a.q, a.k_pages, a.v_pages, a.out,
                           d.head_dim, a.scale_log2, d.out_dtype);
    };
    auto with_pairs = [&](auto tag) {
        auto with_rows = [&](auto pairs) {
            if (p.rows_per_group == 4) launch(tag, pairs, std::integral_constant<int, 4>{});
            else launch(tag, pairs, std::integral_constant<int, 8>{});
        };
        if (d.head_dim <= 128) with_rows(std::integral_constant<int, 1>{});
        else with_rows(std::integral_constant<int, 2>{});
    };
    if (d.dtype == ADASPEC_F32) with_pairs(F32{});
    else if (d.dtype == ADASPEC_F16) with_pairs(F16{});
    else with_pairs(BF16{});
    return hipGetLastError();
}

}  // namespace adaspec
