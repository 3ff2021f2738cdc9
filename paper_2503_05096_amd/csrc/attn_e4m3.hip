// Matrix-core verification attention over a cache of 8 bits (e4m3 with a scale per page and kv head): 16-bit Q, head_dim 64 or
// 128, any number of query rows per kv head.
//
// The scheme of attn_mfma.hip (units, schedule, direct calls, lazily moved softmax reference, merge of four wavefronts):
//   S^T = K Q^T,  O^T += V^T P^T,  in accumulator layouts that need no shuffle.
// What 8 bits change:
//   * An e4m3 value is exact in bf16 and in f16.  K becomes Q's type in registers, two elements an instruction; its scale is
//     one factor per page, applied to the scores.  V becomes f16; its scale is applied to the softmax weights, relative to the
//     largest so far, which the accumulators are kept in units of.
//   * Both products contract in any order of their k-slots, as long as their two operands agree.  So a lane takes 16
//     consecutive bytes of a key at a time, and Q is laid out to match.
//   * No LDS tile for V^T: a lane loads D / 16 neighbouring channels of the four tokens 4g .. 4g + 3 of a page, and byte
//     permutes put equal channels of two tokens side by side, which is what the conversion takes (two bytes in, two bf16
//     out).  The lane then holds D / 16 whole operand columns: tile t of O^T has channel (D / 16) m + t in row m.
// A block is 32 tokens of 128 channels or 64 of 64: 8 KB of K and V per wavefront, 32 registers.
//
// Bound: HBM where requests are many and rows few: 128 requests of 128-4096 tokens, 32/8 heads of 128, 562 MB, 102 us a call, 96 of them this
// kernel, 5.8 TB/s; 64 of 8192-32768, 64/8 heads, 2.7 GB in 452 us with one row tile, 6.0 TB/s, 517 with three (which spill 47 registers).  The
// vector ALU where rows are many: a score costs about 12 instructions whatever it weighs, and with four row tiles (trees of 13 nodes, G = 4:
// 156 us for those 562 MB) there are 64 of them per token.
#include <type_traits>

#include "adaspec_internal.h"
#include "attn_mfma_common.h"
#include "device_utils.h"
#include "e4m3.h"

namespace adaspec {

// two e4m3 (bytes 0, 1 or 2, 3 of w) as two values of T
template <class T, bool kHigh> __device__ __forceinline__ uint32_t e4m3_pair(uint32_t w)
{
    if constexpr (T::id == ADASPEC_BF16) return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, 1.0f, kHigh));
    else return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w, 1.0f, kHigh));
}
template <class T> __device__ __forceinline__ uint4 e4m3_operand(uint32_t lo, uint32_t hi)
{
    return make_uint4(e4m3_pair<T, false>(lo), e4m3_pair<T, true>(lo), e4m3_pair<T, false>(hi), e4m3_pair<T, true>(hi));
}
// What hi, the two f16 next to a and b, leaves of them, as two f16 more: 22 bits together.
__device__ __forceinline__ uint32_t f16_rest2(uint32_t hi, float a, float b)
{
    float one = 1.0f;
    asm("" : "+s"(one));                    // (a multiply-add takes f16 as they are, the subtraction that the compiler would make of it does not)
    const f16x2 h = __builtin_bit_cast(f16x2, hi);
    return Mma<F16>::pack2(fmaf(a, one, -(float)h.x), fmaf(b, one, -(float)h.y));
}
// the bytes of w that are NaN, as 0x80
__device__ __forceinline__ uint32_t e4m3_nans(uint32_t w) { return ((w & 0x7f7f7f7fu) + 0x01010101u) & 0x80808080u; }

// Softmax weights reach the matrix core as two f16, the nearest one and what it leaves: 22 bits, 2^kWeightShift larger: at most 2^15, as
// they trail 1 by 2^kLazyLog2 at most.  Off by 2^-22 of themselves, or by 2^-25 (half a subnormal) where that is more, as little as the
// fp32 sums they go into.  The first piece alone is off by up to 2^-11 and leaves that in the output wherever weights round alike.  MI355X, output in
// fp32 against 64 bits, relative, one piece / two: 128 requests of 128-4096 tokens, 32/8 heads of 128, 1.8e-4 / 2.7e-7 (100.9 / 101.7
// us), 64 trees of up to 13 nodes, 256-4096, 32/8 of 64, 1.8e-4 / 3.4e-7 (52.7 / 56.1); 64 of 8192-32768, 64/8 of 128, 495 / 517 us,
// of 8 rows each, four full row tiles, 624 / 724.
// They are multiplied by their value's scale before that, relative to the largest scale so far, which O is kept in units of: a factor
// per page.  That is sound where all scales are within kScalesApart of each other: 2^-25 of a unit, what a subnormal may be off by, is
// then at most 2^-26 of the row's largest weighted scale.  A wavefront that has met scales further apart, which it knows at the end of its
// blocks, takes them once more with a unit for every row, the largest weight times scale that this row has seen, so that neither a page
// that is far louder (and perhaps hidden from the row) nor one that is far quieter costs the others their bits.  (To leave the inner
// loop at the first such page instead, its keys kept or requested again, cost the usual case 3 % and 8 %.  128 requests of 128-4096 tokens,
// 32/8 heads: 106 us, 170 with a page a thousand times as loud in each.)
constexpr int kWeightShift = 7;
constexpr float kScalesApart = 64.f;
// (Units are powers of two: what is kept in them changes exactly.)  Units of rows times kUnitShift: the product of a scale and a weight up to
// 2^kLazyLog2 stays finite.
constexpr float kUnitShift = 0x1p-16f, kLeastUnit = 0x1p-110f, kMostUnit = 0x1p126f;

__device__ __forceinline__ float power_of_two_below(float x) { return __uint_as_float(__float_as_uint(x) & 0x7f800000u); }
// 2^kShift over a power of two
template <int kShift> __device__ __forceinline__ float one_over(float x) { return __uint_as_float(((254u + kShift) << 23) - __float_as_uint(x)); }

template <class T, int D, int RT, bool kTree, bool kDirect>
__global__ __launch_bounds__(256, (RT == 1 ? 3 : 2)) void attn_e4m3_kernel(
    const char *__restrict__ q, const char *__restrict__ k_pages, const char *__restrict__ v_pages,
    const float *__restrict__ k_scales, const float *__restrict__ v_scales,
    const int32_t *__restrict__ block_table, void *__restrict__ out, const int32_t *__restrict__ header,
    const int32_t *__restrict__ unit_meta, const int32_t *__restrict__ sched,
    const unsigned long long *__restrict__ anc, float *__restrict__ part_ml, float *__restrict__ part_o,
    int Hq, int Hkv, int max_pages_per_req, int max_rows, int n_row_groups, float scale_log2, int out_dtype, int cus, DirectArgs direct)
{
    constexpr int kRows = 16 * RT;
    constexpr int kTokens = attn_e4m3_block(D), kPages = kTokens / 16;
    constexpr int kKLoads = D / 64;                                 // 16-byte pieces of a key per lane
    constexpr int kSteps = D / 32;                                  // products per 16 x 16 tile of scores
    constexpr int kWords = D / 64;                                  // of a lane's channels of a token of V
    constexpr int kTiles = D / 16;                                  // of O^T
    constexpr int kHalves = kTokens / 32;
    constexpr int kORow = D + 4;                                    // floats per row of the merge buffer (padded: conflict-free b128)
    constexpr int kSlab = 16 * kORow * 4;                           // a row tile's state of one wavefront
    constexpr int kQEntries = RT * kSteps * 64, kQLoads = (kQEntries + 255) / 256;
    __shared__ __attribute__((aligned(16))) char smem[kWaves * kSlab];
    __shared__ __attribute__((aligned(16))) uint4 q_lds[kQEntries];   // Q^T operands, MFMA lane order
    __shared__ float s_m[kWaves][16], s_l[kWaves][16];
    __shared__ float s_unit[kWaves][kRows];                         // (rows' units, where one does not do for all)
    __shared__ unsigned long long s_anc[kTree ? kRows : 1];         // ancestor mask of each row of the unit

    const int tid = threadIdx.x, lane = tid & 63;
    const int wv = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int g = lane >> 4, n16 = lane & 15;
    const int G = Hq / Hkv;
    const int total_units = kDirect ? 0 : header[0] * Hkv * n_row_groups;
    float *my_state = reinterpret_cast<float *>(smem + wv * kSlab), *my_units = &s_unit[wv][n16];

    // Row m of a tile of K is token (m >> 2) + 4 (m & 3) of its page: lane (g, n) then holds scores of tokens g, g + 4, g + 8, g + 12, and of V
    // it takes the same, D / 16 channels from (D / 16) n on.  (Four neighbouring rows of V per load.)
    uint4 kreg[kPages][kKLoads];
    uint32_t vreg[kPages][4][kWords];
    float ks[kPages], vs[kPages];                                   // scales of the block in registers
    const uint32_t k_lane_off = ((n16 >> 2) + 4 * (n16 & 3)) * D + 16 * g;
    const uint32_t v_lane_off = g * D + kTiles * n16;

    const int W = gridDim.x, wg = blockIdx.x;
    const int n_rounds = kDirect ? 0 : header[2];
    int round = 0;
    int idx_ahead = kDirect ? 0 : sched_position(0, wg, W, cus, header[1]);     // round 0 needs no table
    auto next_unit = [&](Unit &u) -> bool {
        for (; round < n_rounds; ++round) {
            const int idx = idx_ahead;
            idx_ahead = round + 1 < n_rounds ? sched[(int64_t)(round + 1) * W + wg] : -1;
            if (idx < 0 || idx >= total_units) continue;
            const int rg = idx % n_row_groups;
            u.gkv = (idx / n_row_groups) % Hkv;
            const int32_t *mt = unit_meta + 8 * (int64_t)(idx / (n_row_groups * Hkv));
            u.i = mt[0];
            const int sp = mt[1];
            u.ns = mt[2]; u.L = mt[3]; u.n = mt[4]; u.qrow0 = mt[5]; u.item = mt[6];
            u.rows = u.n * G; u.r0 = rg * kRows;
            if (u.r0 >= u.rows) continue;
            const int slen = split_len_of(u.L, u.ns, kTokens);
            u.t0 = sp * slen; u.t1 = min(u.L, u.t0 + slen);
            u.nblk = (u.t1 - u.t0 + kTokens - 1) / kTokens;
            u.bt_off = (int64_t)u.i * max_pages_per_req;
            ++round;
            return true;
        }
        return false;
    };

    // Page ids and scales by scalar loads; pages past the split's end are replaced by the block's first (masks and the tail code
    // keep what they hold out of the result), so that every block issues the same loads.
    auto page_blocks = [&](const Unit &u, int bi, int64_t (&b)[kPages]) {
        const int tb = u.t0 + bi * kTokens;
        const int64_t at = u.bt_off + (tb >> 4);
#pragma unroll
        for (int p = 0; p < kPages; ++p) b[p] = (int64_t)block_table[tb + 16 * p < u.t1 ? at + p : at] * Hkv + u.gkv;
    };
    auto load_k = [&](const int64_t (&b)[kPages]) {
#pragma unroll
        for (int p = 0; p < kPages; ++p)
#pragma unroll
            for (int c = 0; c < kKLoads; ++c) kreg[p][c] = ld16_stream(k_pages + b[p] * (16 * D) + k_lane_off + 64 * c);
    };
    auto load_v = [&](const int64_t (&b)[kPages]) {
#pragma unroll
        for (int p = 0; p < kPages; ++p)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const char *at = v_pages + b[p] * (16 * D) + v_lane_off + 4 * i * D;
                if constexpr (kWords == 2) {
                    const u32x2v w = __builtin_nontemporal_load(reinterpret_cast<const u32x2v *>(at));
                    vreg[p][i][0] = w.x;
                    vreg[p][i][1] = w.y;
                } else {
                    vreg[p][i][0] = __builtin_nontemporal_load(reinterpret_cast<const uint32_t *>(at));
                }
            }
    };
    auto load_scales = [&](const int64_t (&b)[kPages]) {
#pragma unroll
        for (int p = 0; p < kPages; ++p) {
            ks[p] = k_scales[b[p]];
            vs[p] = v_scales[b[p]];
        }
    };
    auto first_loads = [&](const Unit &u) {
        if (wv < u.nblk) {
            int64_t b[kPages];
            page_blocks(u, wv, b);
            load_k(b);
            load_v(b);
            load_scales(b);
        }
    };
    // this thread's share of the unit's Q^T operands: entry (row tile, s, lane)
    auto load_q = [&](const Unit &u, uint4 (&qv)[kQLoads]) {
#pragma unroll
        for (int k = 0; k < kQLoads; ++k) {
            const int e = tid + 256 * k, s = (e >> 6) % kSteps;
            const int row = u.r0 + 16 * (e / (64 * kSteps)) + n16;
            qv[k] = make_uint4(0, 0, 0, 0);
            if (e < kQEntries && row < u.rows)
                qv[k] = ld16(q + (((u.qrow0 + row / G) * Hq + u.gkv * G + row % G) * D + 64 * (s >> 1) + 16 * g + 8 * (s & 1)) * 2);
        }
    };
    auto load_anc = [&](const Unit &u) -> unsigned long long {
        const int row = u.r0 + tid;
        return (tid < kRows && row < u.rows) ? anc[u.qrow0 + row / G] : 0ull;
    };

    Unit cur, nxt;
    bool have;
    uint4 qv[kQLoads];
    unsigned long long av = 0ull;
    if constexpr (kDirect) have = direct_unit(cur, direct, block_table, G, Hkv, n_row_groups, kRows, kTokens, max_pages_per_req, wv, lane);
    else have = next_unit(cur);
    if (have) {
        load_q(cur, qv);
        if constexpr (kTree) av = load_anc(cur);
        first_loads(cur);
    }

    while (have) {
        const Unit u = cur;
        const bool have_next = kDirect ? false : next_unit(nxt);
        const int first_masked = u.L - u.n + 1;                    // tokens >= this are hidden from some row
#pragma unroll
        for (int k = 0; k < kQLoads; ++k)
            if (kQEntries % 256 == 0 || tid + 256 * k < kQEntries) q_lds[tid + 256 * k] = qv[k];
        if constexpr (kTree) { if (tid < kRows) s_anc[tid] = av; }
        lds_barrier();

        float m[RT], lsum[RT];
        float vref = kLeastUnit / kUnitShift, vref_inv = one_over<kWeightShift>(vref);    // O is kept in units of vref 2^-kWeightShift
        float least_scale = kMostUnit;                              // of all so far
        bool wide = false;                                          // again, with a unit for every row
        f32x4 o[RT][kTiles];
#pragma unroll
        for (int nt = 0; nt < RT; ++nt) {
            m[nt] = kLowestRef; lsum[nt] = 0.f;
#pragma unroll
            for (int t = 0; t < kTiles; ++t) o[nt][t] = f32x4{0.f, 0.f, 0.f, 0.f};
        }

        const int tiles = min((u.rows - u.r0 + 15) / 16, RT);       // row tiles of the unit that have rows (others cost nothing)
        // One block.  kInner: every row sees all of it, and another one follows, whose K and V are requested as soon as their
        // registers are free (without a branch around the loads, so that the compiler's waits count exactly).
        // kNT: its row tiles that have rows, where that is known, else RT.
        // kWide: O in units of every row's own, 2^-kWeightShift / kUnitShift of it.
        auto block = [&](int bi, auto inner_tag, auto tiles_tag, auto wide_tag) {
            constexpr bool kInner = decltype(inner_tag)::value;
            constexpr int kNT = decltype(tiles_tag)::value;
            constexpr bool kWide = decltype(wide_tag)::value;
            constexpr int kE = 4 * kPages;                          // scores per lane and row tile
            constexpr bool kByTile = D == 64;
            const int tb = u.t0 + bi * kTokens;
            int64_t nb[kPages];
            const bool next = kInner || bi + kWaves < u.nblk;
            const bool masked = !kInner && (tb + kTokens > first_masked || tb + kTokens > u.t1);
            if (next) page_blocks(u, bi + kWaves, nb);

            // Two orders of the same work.  head_dim 64: row tile by row tile, with all keys in Q's type (32 registers) and P packed at once, so
            // that Q is read once per block, not once per page, and the scores of one tile are live, not of all: 64 requests of 256-4096
            // tokens, trees of up to 13 nodes, 32/8 heads: 56.1 us against 61.1.  head_dim 128, whose O leaves no registers for that: page by
            // page (the other way costs 64 requests of 8192-32768 tokens, 64/8 heads, 539 us against 517, trees of up to 13 nodes 160 against 156).
            float p[kByTile ? 1 : kNT][kE];
            uint4 packed[kByTile ? kNT : 1][kHalves][2];            // P as an operand, in two pieces
            uint32_t seen[kNT];                                     // masked: bit e = the row sees token e
            float weight[kPages];                                   // of a value: its scale in units of O
            auto find_weights = [&] {
                if constexpr (!kWide) {
                    // the values' scales relative to the largest so far, which O is kept in units of
                    float most_vs = vs[0];
                    least_scale = fminf(least_scale, vs[0]);
#pragma unroll
                    for (int mt = 1; mt < kPages; ++mt) {
                        most_vs = fmaxf(most_vs, vs[mt]);
                        least_scale = fminf(least_scale, vs[mt]);
                    }
                    if (__builtin_expect(most_vs > vref, 0)) {
                        const float up = __uint_as_float((__float_as_uint(most_vs) + 0x7fffffu) & 0x7f800000u), down = vref * one_over<0>(up);
                        vref = up;
                        vref_inv = one_over<kWeightShift>(up);
#pragma unroll
                        for (int nt = 0; nt < kNT; ++nt)
#pragma unroll
                            for (int t = 0; t < kTiles; ++t) o[nt][t] *= down;
                    }
                }
#pragma unroll
                for (int mt = 0; mt < kPages; ++mt) weight[mt] = vs[mt] * (kWide ? kUnitShift : vref_inv);
            };
            // Online softmax of row tile nt (per lane: row n16 of the tile, kE of the tokens), in log2 units: scores to weights.
            auto weigh = [&](int nt, float (&x)[kE]) {
                if (masked) {
                    seen[nt] = 0;
                    const unsigned long long am = kTree ? s_anc[16 * nt + n16] : 0ull;
                    const int row = u.r0 + 16 * nt + n16, base = u.L - u.n;
                    const int pos = row < u.rows ? base + row / G : -1, lim = min(pos, u.t1 - 1);
#pragma unroll
                    for (int e = 0; e < kE; ++e) {
                        const int t = tb + 16 * (e >> 2) + g + 4 * (e & 3), rel = t - base;
                        bool vis;
                        if constexpr (kTree) vis = t < u.t1 && (rel < 0 ? pos >= 0 : ((am >> (rel & 63)) & 1ull) != 0);
                        else vis = t <= lim;
                        x[e] = vis ? x[e] : -INFINITY;
                        seen[nt] |= vis ? 1u << e : 0u;
                    }
                }
                if constexpr (!kByTile && RT > 2) __builtin_amdgcn_sched_barrier(0);
                float mx = x[0];
#pragma unroll
                for (int e = 1; e < kE; ++e) mx = fmaxf(mx, x[e]);
                mx = max_over_row_groups(mx);
                // lazy reference: moves only when the block's maximum exceeds it by more than kLazyLog2
                const bool grow = mx > m[nt] + kLazyLog2;
                if (__builtin_expect(__builtin_amdgcn_ballot_w64(grow) != 0, 0)) {
                    const float m_new = grow ? mx : m[nt];
                    const float alpha = __builtin_amdgcn_exp2f(m[nt] - m_new);
                    m[nt] = m_new;
                    lsum[nt] *= alpha;
                    if constexpr (kWide) {
                        my_units[16 * nt] *= alpha;
                    } else {
#pragma unroll
                        for (int t = 0; t < kTiles; ++t) o[nt][t] *= alpha;
                    }
                }
                float psum = 0.f;
#pragma unroll
                for (int e = 0; e < kE; ++e) {
                    x[e] = __builtin_amdgcn_exp2f(x[e] - m[nt]);
                    psum += x[e];
                    x[e] *= weight[e >> 2];
                    // what hidden tokens hold stays out: no weight, whatever their scale
                    if (masked) x[e] = (seen[nt] >> e) & 1 ? x[e] : 0.f;
                }
                lsum[nt] += psum;
                if constexpr (kWide) {
                    // the row's unit follows the largest weight times scale that it has seen, as m the largest score
                    float most = x[0];
#pragma unroll
                    for (int e = 1; e < kE; ++e) most = fmaxf(most, x[e]);
                    most = max_over_row_groups(most);
                    const float was = my_units[16 * nt];
                    const bool move = was != power_of_two_below(was) || was < kLeastUnit || most > was * (float)(1 << (int)kLazyLog2);
                    const float to = move ? power_of_two_below(fmaxf(fmaxf(most, was), kLeastUnit)) : was;
                    if (__builtin_amdgcn_ballot_w64(move) != 0) {
                        const float ratio = was * one_over<0>(to);
#pragma unroll
                        for (int t = 0; t < kTiles; ++t) o[nt][t] *= ratio;
                        my_units[16 * nt] = to;
                    }
                    const float inv = one_over<kWeightShift>(to);
#pragma unroll
                    for (int e = 0; e < kE; ++e) x[e] *= inv;
                }
            };
            if constexpr (kByTile) {
                // ---- S^T = K Q^T, row tile by row tile: the keys once in Q's type, P packed as soon as it is known -------
                uint4 kop[kPages][kSteps];
#pragma unroll
                for (int mt = 0; mt < kPages; ++mt)
#pragma unroll
                    for (int s = 0; s < kSteps; ++s) {
                        const uint4 raw = kreg[mt][s >> 1];
                        kop[mt][s] = (s & 1) ? e4m3_operand<T>(raw.z, raw.w) : e4m3_operand<T>(raw.x, raw.y);
                    }
                float factor[kPages];
#pragma unroll
                for (int mt = 0; mt < kPages; ++mt) factor[mt] = ks[mt] * scale_log2;
                __builtin_amdgcn_sched_barrier(0);
                if (next) load_k(nb);
                __builtin_amdgcn_sched_barrier(0);
                find_weights();
#pragma unroll
                for (int nt = 0; nt < kNT; ++nt) {
                    if (!kInner && nt > 0 && nt >= tiles) break;
                    f32x4 acc[kPages];
#pragma unroll
                    for (int s = 0; s < kSteps; ++s) {
                        const uint4 qop = q_lds[(nt * kSteps + s) * 64 + lane];
#pragma unroll
                        for (int mt = 0; mt < kPages; ++mt) acc[mt] = Mma<T>::run(kop[mt][s], qop, s == 0 ? f32x4{0.f, 0.f, 0.f, 0.f} : acc[mt]);
                    }
#pragma unroll
                    for (int e = 0; e < kE; ++e) p[0][e] = acc[e >> 2][e & 3] * factor[e >> 2];
                    weigh(nt, p[0]);
#pragma unroll
                    for (int hf = 0; hf < kHalves; ++hf)
#pragma unroll
                        for (int j = 0; j < 4; ++j) {
                            const float a = p[0][8 * hf + 2 * j], b = p[0][8 * hf + 2 * j + 1];
                            const uint32_t hi = Mma<F16>::pack2(a, b);
                            (&packed[nt][hf][0].x)[j] = hi;
                            (&packed[nt][hf][1].x)[j] = f16_rest2(hi, a, b);
                        }
                }
            } else {
                // ---- S^T = K Q^T ------------------------------------------------------------
#pragma unroll
                for (int mt = 0; mt < kPages; ++mt) {
                    uint4 kop[kSteps];
#pragma unroll
                    for (int s = 0; s < kSteps; ++s) {
                        const uint4 raw = kreg[mt][s >> 1];
                        kop[s] = (s & 1) ? e4m3_operand<T>(raw.z, raw.w) : e4m3_operand<T>(raw.x, raw.y);
                    }
                    const float factor = ks[mt] * scale_log2;
                    if constexpr (RT > 2) __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                    for (int nt = 0; nt < kNT; ++nt) {
                        if (!kInner && nt > 0 && nt >= tiles) break;
                        f32x4 acc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                        for (int s = 0; s < kSteps; ++s) acc = Mma<T>::run(kop[s], q_lds[(nt * kSteps + s) * 64 + lane], acc);
#pragma unroll
                        for (int r = 0; r < 4; ++r) p[nt][4 * mt + r] = acc[r] * factor;
                        if constexpr (RT > 3) __builtin_amdgcn_sched_barrier(0);
                    }
                }
                __builtin_amdgcn_sched_barrier(0);
                if (next) load_k(nb);
                __builtin_amdgcn_sched_barrier(0);

                find_weights();
#pragma unroll
                for (int nt = 0; nt < kNT; ++nt) {
                    if (!kInner && nt > 0 && nt >= tiles) break;
                    weigh(nt, p[nt]);
                }
            }

            // ---- no value behind the request's end, and NaN values only in rows that see them ----
            if (masked) {
                uint32_t nans = 0;
#pragma unroll
                for (int pg = 0; pg < kPages; ++pg)
#pragma unroll
                    for (int i = 0; i < 4; ++i)
#pragma unroll
                        for (int w = 0; w < kWords; ++w) {
                            if (tb + 16 * pg + g + 4 * i >= u.t1) vreg[pg][i][w] = 0;
                            nans |= e4m3_nans(vreg[pg][i][w]);
                        }
                if (__builtin_expect(__builtin_amdgcn_ballot_w64(nans != 0) != 0, 0)) {
                    // rows that see a NaN, channel by channel: a product of what is NaN with what is seen
#pragma unroll
                    for (int hf = 0; hf < kHalves; ++hf)
#pragma unroll
                        for (int t = 0; t < kTiles; ++t) {
                            __builtin_amdgcn_sched_barrier(0);
                            uint32_t bad[8];
#pragma unroll
                            for (int e = 0; e < 8; ++e)
                                bad[e] = (e4m3_nans(vreg[2 * hf + (e >> 2)][e & 3][t >> 2]) >> (8 * (t & 3))) & 0x80u ? 0x3f80u : 0u;
                            const uint4 a = make_uint4(bad[0] | bad[1] << 16, bad[2] | bad[3] << 16, bad[4] | bad[5] << 16, bad[6] | bad[7] << 16);
#pragma unroll
                            for (int nt = 0; nt < kNT; ++nt) {
                                if (!kInner && nt > 0 && nt >= tiles) break;
                                uint32_t see[8];
#pragma unroll
                                for (int e = 0; e < 8; ++e) see[e] = (seen[nt] >> (8 * hf + e)) & 1 ? 0x3f80u : 0u;
                                const uint4 x = make_uint4(see[0] | see[1] << 16, see[2] | see[3] << 16, see[4] | see[5] << 16, see[6] | see[7] << 16);
                                const f32x4 hit = Mma<BF16>::run(a, x, f32x4{0.f, 0.f, 0.f, 0.f});
#pragma unroll
                                for (int r = 0; r < 4; ++r)
                                    if (hit[r] > 0.f) o[nt][t][r] = __uint_as_float(0x7fc00000u);
                            }
                        }
#pragma unroll
                    for (int pg = 0; pg < kPages; ++pg)
#pragma unroll
                        for (int i = 0; i < 4; ++i)
#pragma unroll
                            for (int w = 0; w < kWords; ++w) {
                                const uint32_t x = e4m3_nans(vreg[pg][i][w]);
                                vreg[pg][i][w] &= ~(x | (x - (x >> 7)));        // NaN bytes become 0
                            }
                }
            }

            __builtin_amdgcn_sched_barrier(0);
            // ---- O^T += V^T P^T, 32 tokens at a time ------------------------------
#pragma unroll
            for (int hf = 0; hf < kHalves; ++hf) {
                uint4 pop[kNT][2];
#pragma unroll
                for (int nt = 0; nt < kNT; ++nt) {
                    if (!kInner && nt > 0 && nt >= tiles) break;
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        if constexpr (kByTile) {
                            (&pop[nt][0].x)[j] = (&packed[nt][hf][0].x)[j];
                            (&pop[nt][1].x)[j] = (&packed[nt][hf][1].x)[j];
                        } else {
                            const float a = p[nt][8 * hf + 2 * j], b = p[nt][8 * hf + 2 * j + 1];
                            const uint32_t hi = Mma<F16>::pack2(a, b);
                            (&pop[nt][0].x)[j] = hi;
                            (&pop[nt][1].x)[j] = f16_rest2(hi, a, b);
                        }
                    }
                }
#pragma unroll
                for (int w = 0; w < kWords; ++w)
#pragma unroll
                    for (int up = 0; up < 2; ++up) {                // channels 0, 1 and 2, 3 of the word
                        uint32_t pair[4];                           // two tokens, two channels: (t0 c0, t1 c0, t0 c1, t1 c1)
#pragma unroll
                        for (int j = 0; j < 4; ++j) {
                            const uint32_t(&v)[4][kWords] = vreg[2 * hf + (j >> 1)];
                            pair[j] = __builtin_amdgcn_perm(v[2 * (j & 1) + 1][w], v[2 * (j & 1)][w], up ? 0x07030602u : 0x05010400u);
                        }
                        if constexpr (RT > 2) __builtin_amdgcn_sched_barrier(0);
                        const uint4 even = make_uint4(e4m3_pair<F16, false>(pair[0]), e4m3_pair<F16, false>(pair[1]),
                                                      e4m3_pair<F16, false>(pair[2]), e4m3_pair<F16, false>(pair[3]));
                        const uint4 odd = make_uint4(e4m3_pair<F16, true>(pair[0]), e4m3_pair<F16, true>(pair[1]),
                                                     e4m3_pair<F16, true>(pair[2]), e4m3_pair<F16, true>(pair[3]));
                        const int t = 4 * w + 2 * up;
#pragma unroll
                        for (int nt = 0; nt < kNT; ++nt) {
                            if (!kInner && nt > 0 && nt >= tiles) break;
#pragma unroll
                            for (int piece = 1; piece >= 0; --piece) {
                                o[nt][t] = Mma<F16>::run(even, pop[nt][piece], o[nt][t]);
                                o[nt][t + 1] = Mma<F16>::run(odd, pop[nt][piece], o[nt][t + 1]);
                            }
                        }
                    }
            }
            if (next) {
                load_v(nb);
                load_scales(nb);
            }
        };

        if (wv < u.nblk) {
            const int full = max(min(first_masked, u.t1) - u.t0, 0) / kTokens;         // blocks that every row sees all of
            int bi = wv;
            auto inner = [&](auto tiles_tag) {
                for (; bi + kWaves < u.nblk && bi < full; bi += kWaves) block(bi, std::true_type{}, tiles_tag, std::false_type{});
            };
            // (A copy of the loop for every number of tiles, so that none is looked at in it.  MI355X, us, with copies / one loop that skips tiles without
            // rows: 128 requests of 128-4096 tokens, 32/8 heads of 128, 102.0 / 104.4, in trees of up to 13 nodes 156 / 187, 64 of 8192-32768, 64/8
            // 517 / 529, of up to 8 rows 621 / 679; 64-channel trees 56.1 / 57.1.  Four tiles first: with that copy behind the others the
            // compiler spills twice as many registers, and those trees take 192 and 73 us.)
            if (RT == 4 && tiles > 3) inner(std::integral_constant<int, RT>{});
            else if (RT == 1 || tiles <= 1) inner(std::integral_constant<int, 1>{});
            else if (RT == 2 || tiles == 2) inner(std::integral_constant<int, RT < 2 ? 1 : 2>{});
            else inner(std::integral_constant<int, RT < 3 ? 1 : 3>{});
            for (; bi < u.nblk; bi += kWaves) block(bi, std::false_type{}, std::integral_constant<int, RT>{}, std::false_type{});
            wide = !(least_scale * kScalesApart >= vref && vref < kMostUnit);
            if (__builtin_expect(wide, 0)) {
                first_loads(u);
#pragma unroll
                for (int nt = 0; nt < RT; ++nt) {
                    m[nt] = kLowestRef; lsum[nt] = 0.f;
                    my_units[16 * nt] = kLeastUnit;
#pragma unroll
                    for (int t = 0; t < kTiles; ++t) o[nt][t] = f32x4{0.f, 0.f, 0.f, 0.f};
                }
                for (bi = wv; bi < u.nblk; bi += kWaves) block(bi, std::false_type{}, std::integral_constant<int, RT>{}, std::true_type{});
            }
        }

        // ---- next unit: its first block and its Q rows travel while this unit's states are merged
        if (have_next) {
            load_q(nxt, qv);
            if constexpr (kTree) av = load_anc(nxt);
            first_loads(nxt);
        }
        // ---- merge the four wavefronts' states through LDS (as in attn_mfma.hip), one row tile after the other ----------
#pragma unroll
        for (int nt = 0; nt < RT; ++nt) {
            if (nt > 0 && nt >= tiles) break;
            if (nt > 0) lds_barrier();                              // (the tile before has been read)
            const float o_unit = (wide ? my_units[16 * nt] * (1.f / kUnitShift) : vref) * (1.f / (1 << kWeightShift));
            lsum[nt] += __shfl_xor(lsum[nt], 16, kWave);
            lsum[nt] += __shfl_xor(lsum[nt], 32, kWave);
            if (g == 0) { s_m[wv][n16] = m[nt]; s_l[wv][n16] = lsum[nt]; }
#pragma unroll
            for (int r = 0; r < 4; ++r)
#pragma unroll
                for (int t = 0; t < kTiles; t += 4)
                    *reinterpret_cast<f32x4 *>(my_state + n16 * kORow + kTiles * (4 * g + r) + t) =
                        f32x4{o[nt][t][r], o[nt][t + 1][r], o[nt][t + 2][r], o[nt][t + 3][r]} * o_unit;
            lds_barrier();
            // 256 threads: 16 rows x D / 4 float4 columns
            constexpr int kCols = D / 4;
#pragma unroll
            for (int it = 0; it < 16 * kCols / 256; ++it) {
                const int idx = tid + 256 * it;
                const int rl = idx / kCols, c4 = idx % kCols;
                const int row = u.r0 + 16 * nt + rl;
                if (row >= u.rows) continue;
                float ms = s_m[0][rl], ltot = 0.f;
#pragma unroll
                for (int w = 1; w < kWaves; ++w) ms = fmaxf(ms, s_m[w][rl]);
                f32x4 acc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int w = 0; w < kWaves; ++w) {
                    const float sc = __builtin_amdgcn_exp2f(s_m[w][rl] - ms);
                    ltot += sc * s_l[w][rl];
                    acc += sc * *reinterpret_cast<const f32x4 *>(smem + w * kSlab + 4 * (rl * kORow + 4 * c4));
                }
                if (u.ns == 1) {
                    const float inv = 1.0f / ltot;
                    const int64_t obase = ((u.qrow0 + row / G) * Hq + u.gkv * G + row % G) * (int64_t)D + 4 * c4;
                    if (out_dtype == ADASPEC_F32) {
                        *reinterpret_cast<f32x4 *>(reinterpret_cast<float *>(out) + obase) = acc * inv;
                    } else {
                        uint2 pk = make_uint2(Mma<T>::pack2(acc[0] * inv, acc[1] * inv), Mma<T>::pack2(acc[2] * inv, acc[3] * inv));
                        *reinterpret_cast<uint2 *>(reinterpret_cast<uint16_t *>(out) + obase) = pk;
                    }
                } else {
                    const int64_t idx_row = ((int64_t)u.item * Hkv + u.gkv) * max_rows + row;
                    if (kDirect && attn_merge_fits(D, RT) && direct.flags) {
                        store_state(part_o + idx_row * D + 4 * c4, acc);
                        if (c4 == 0) store_ml(part_ml + idx_row * 2, ms, ltot);
                    } else {
                        *reinterpret_cast<f32x4 *>(part_o + idx_row * D + 4 * c4) = acc;
                        if (c4 == 0) {
                            part_ml[idx_row * 2] = ms;
                            part_ml[idx_row * 2 + 1] = ltot;
                        }
                    }
                }
            }
        }
        if constexpr (kDirect) {
            if constexpr (attn_merge_fits(D, RT)) {
                if (u.ns > 1 && direct.flags)
                    merge_splits<T, D, kRows>(direct, u, part_ml, part_o, out, out_dtype, Hq, Hkv, G, max_rows, tid);
            }
            break;
        }
        // the next loop iteration overwrites q_lds, the states and s_m: everyone must be done reading them
        lds_barrier();
        cur = nxt;
        have = have_next;
    }
}

// ---- host side -----------------------------------------------------------------------------------------------
bool attn_e4m3_supported(const adaspec_attn_dims &d)
{
    return (d.head_dim == 64 || d.head_dim == 128) && (d.dtype == ADASPEC_F16 || d.dtype == ADASPEC_BF16);
}

template <typename F>
static void with_e4m3_instance(const AttnArgs &a, F &&f)
{
    const int rt = attn_row_tiles(a.plan.max_rows);
    auto with_mode = [&](auto tag, auto d, auto rt_tag) {
        if (a.direct) f(tag, d, rt_tag, std::false_type{}, std::true_type{});
        else if (a.parents) f(tag, d, rt_tag, std::true_type{}, std::false_type{});
        else f(tag, d, rt_tag, std::false_type{}, std::false_type{});
    };
    auto with_rt = [&](auto tag, auto d) {
        if (rt == 1) with_mode(tag, d, std::integral_constant<int, 1>{});
        else if (rt == 2) with_mode(tag, d, std::integral_constant<int, 2>{});
        else if (rt == 3) with_mode(tag, d, std::integral_constant<int, 3>{});
        else with_mode(tag, d, std::integral_constant<int, 4>{});
    };
    auto with_d = [&](auto tag) {
        if (a.dims.head_dim == 64) with_rt(tag, std::integral_constant<int, 64>{});
        else with_rt(tag, std::integral_constant<int, 128>{});
    };
    if (a.dims.dtype == ADASPEC_F16) with_d(F16{});
    else with_d(BF16{});
}

template <typename T, int D, int RT, bool kTree, bool kDirect>
static int attn_e4m3_slots(int cus)
{
    static int slots = 0;
    if (slots == 0) {
        int per_cu = 1;
        if (hipOccupancyMaxActiveBlocksPerMultiprocessor(&per_cu, attn_e4m3_kernel<T, D, RT, kTree, kDirect>, 256, 0) != hipSuccess)
            per_cu = 1;
        const int n = cus * (per_cu > 0 ? per_cu : 1);
        slots = n < kMaxSchedW ? n : kMaxSchedW;
    }
    return slots;
}

int attn_e4m3_grid_slots(const AttnArgs &a, int cus)
{
    int slots = 1;
    with_e4m3_instance(a, [&](auto tag, auto d, auto rt, auto tree, auto direct) {
        slots = attn_e4m3_slots<decltype(tag), decltype(d)::value, decltype(rt)::value, decltype(tree)::value, decltype(direct)::value>(cus);
    });
    return slots;
}

hipError_t launch_attn_e4m3(const AttnArgs &a)
{
    const AttnPlan &p = a.plan;
    const adaspec_attn_dims &d = a.dims;
    if (a.sched_w <= 0) return hipSuccess;                          // no work item can exist
    with_e4m3_instance(a, [&](auto tag, auto dim, auto rt, auto tree, auto direct) {
        hipLaunchKernelGGL((attn_e4m3_kernel<decltype(tag), decltype(dim)::value, decltype(rt)::value, decltype(tree)::value, decltype(direct)::value>),
                           dim3(a.sched_w), dim3(256), 0, a.stream, (const char *)a.q, (const char *)a.k_pages,
                           (const char *)a.v_pages, a.k_scales, a.v_scales, a.block_table, a.out, (const int32_t *)(a.ws + p.off_header),
                           (const int32_t *)(a.ws + p.off_unit_meta), (const int32_t *)(a.ws + p.off_sched),
                           (const unsigned long long *)(a.ws + p.off_anc), (float *)(a.ws + p.off_part_ml),
                           (float *)(a.ws + p.off_part_o), d.n_q_heads, d.n_kv_heads, d.max_pages_per_req, p.max_rows,
                           a.n_row_groups, a.scale_log2, d.out_dtype, a.sched_cus, direct_args(a));
    });
    return hipGetLastError();
}

}  // namespace adaspec
