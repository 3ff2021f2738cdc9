// Windowed verification attention on the matrix cores: 16-bit K/V/Q, head_dim 64 or 128.
//
// Work unit = (request, kv head, group of up to 16 RT query rows, part of the pages they see).  A workgroup of 4 wavefronts
// takes one unit; wavefront w streams the blocks w, w + 4, ... of its list of pages (32 tokens at head_dim 128, 64 at 64:
// 8 KB of K and of V either way) and keeps the online-softmax state of all rows of the unit in registers.  As in
// attn_ring.hip K and V travel from memory straight into LDS, into a slot each that belongs to the wavefront, so that the
// block loop has no barrier; products are computed transposed (S^T = K Q^T, O^T += V^T P^T), so that the scores a lane
// holds are the operand it has to supply next; V^T comes out of the row-major slot through transposing reads.
//
// Rows and tokens: only the blocks at the ends of the two runs of pages hold tokens that some row does not see; their scores
// are replaced by -inf, and V of tokens that no row sees by zero.  A token that one row sees and another does not may hold
// anything: a NaN or an infinity there makes 0 * V a NaN in rows that must not notice.  Whoever finds a result that is not
// finite works the row out again with a selection per token (row_by_selection): nothing of this is in the stream's way.
//
// Softmax weights reach the matrix core as two 16-bit pieces, which hold 16 (bf16) or 22 (f16) bits of the fp32 weight; the
// sum of weights is taken before that.  One bf16 piece would be off by 2^-9 of the weight, the size of the output's own
// rounding; the second product costs nothing that the memory does not hide.
//
// Memory bounds it, and around that the start of a generation of workgroups (7-8 us: launch, lengths, page ids, first block,
// merge, store, one after the other).  128 requests of 128-4096 tokens, 32 query on 8 kv heads, up to 6 drafts, window 1024,
// head_dim 128: 84 us for 495 MB (5.9 TB/s); 64 requests, 64 query heads, window 4096: 172 us, 6.3 TB/s, the rate of a large
// read (in a stream that has been busy for some hundred calls; up to 187 us before that).  64 rows: 5.7 TB/s at window 4096, 4.8 at
// 1024 (matrix products and softmax of four row tiles by 8 wavefronts).  More rows: groups of equal numbers of tiles, of which a unit does
// all, whether it has rows for them or not (72 rows are 48 and 24, both with three tiles).
#include "attn_window_merge.h"

namespace adaspec {

constexpr int kSlotBytes = 8192;                // K, or V, of a block

template <class T> struct WindowWeights;
template <> struct WindowWeights<BF16> {
    static constexpr float kShiftLog2 = 0.f;
    static __device__ __forceinline__ float lo(uint32_t w) { return __uint_as_float(w << 16); }
    static __device__ __forceinline__ float hi(uint32_t w) { return __uint_as_float(w & 0xffff0000u); }
};
template <> struct WindowWeights<F16> {         // kept 2^7 larger: at most 2^15, and the second piece is not subnormal
    static constexpr float kShiftLog2 = 7.f;
    static __device__ __forceinline__ float lo(uint32_t w) { return f16_bits_to_float((uint16_t)w); }
    static __device__ __forceinline__ float hi(uint32_t w) { return f16_bits_to_float((uint16_t)(w >> 16)); }
};

// Two forms (make_window_plan chooses):
//   four wavefronts per unit: K and V through slots of the wavefronts, two workgroups per compute unit;
//   kAlone, one: nothing to merge, for many short units.  K goes to the registers that its operands are read into anyway, only V
//   has a slot, so that twelve to sixteen (of one row tile; eight of three) of these workgroups fit a compute unit.
// LDS: the slots; Q^T operands in MFMA lane order; (m, l) of every wavefront's rows, which take the place of Q where two
// workgroups would not fit otherwise.
template <int D, int RT, bool kAlone> struct WindowLds {
    static constexpr int kWavesHere = kAlone ? 1 : kWaves, kRows = 16 * RT;
    static constexpr int kV = kAlone ? 0 : kSlotBytes, kWaveBytes = kV + kSlotBytes;
    static constexpr bool kFull = RT == 4 && D == 128;
    static constexpr int kQ = kWavesHere * kWaveBytes, kQBytes = RT * (D / 32) * 1024;
    static constexpr int kMl = kFull ? kQ : kQ + kQBytes, kMlBytes = kAlone ? 0 : kWaves * kRows * 2 * 4;
    static constexpr int kBytes = kFull ? kQ + kQBytes : kMl + kMlBytes;
    static_assert(kBytes <= 81920, "two workgroups per compute unit");
};

__device__ __forceinline__ void load_lds_2(const v4i32 &rsrc, uint32_t off0, uint32_t off1, uint32_t lds)
{
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %3, 0 offen nt lds\n\t"
                 "buffer_load_dwordx4 %2, %3, 0 offen offset:1024 nt lds"
                 :: "s"(lds), "v"(off0), "v"(off1), "s"(rsrc) : "memory", "m0");
}

// a page of 4 KB that another row group reads at about the same time: it may stay in the L2
__device__ __forceinline__ void load_shared_page(const v4i32 &rsrc, uint32_t off0, uint32_t off1, uint32_t off2, uint32_t off3, uint32_t lds)
{
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %5, 0 offen lds\n\t"
                 "buffer_load_dwordx4 %2, %5, 0 offen offset:%6 lds\n\t"
                 "buffer_load_dwordx4 %3, %5, 0 offen offset:%7 lds\n\t"
                 "buffer_load_dwordx4 %4, %5, 0 offen offset:%8 lds"
                 :: "s"(lds), "v"(off0), "v"(off1), "v"(off2), "v"(off3), "s"(rsrc), "n"(1 << 10), "n"(2 << 10), "n"(3 << 10) : "memory", "m0");
}

template <class T, int D, int RT, bool kAlone, bool kShared>
__global__ __launch_bounds__(kAlone ? 64 : 256, kAlone ? (RT == 1 ? 4 : RT == 2 && D == 64 ? 3 : 2) : 2)
void attn_window_kernel(WindowDims dims, const int32_t *__restrict__ block_table, const char *__restrict__ q,
                        const char *__restrict__ k_pages, const char *__restrict__ v_pages, void *__restrict__ out,
                        float *__restrict__ part_ml, float *__restrict__ part_o, int splits, float scale_log2, int out_dtype)
{
    using Lds = WindowLds<D, RT, kAlone>;
    constexpr int kStep = Lds::kWavesHere;                          // wavefronts that share a unit's blocks
    using Weights = WindowWeights<T>;
    constexpr int kRows = 16 * RT, kS = D / 32, kDt = D / 16, kPages = 256 / D, kPageBytes = 32 * D, kRowBytes = 2 * D;
    __shared__ __attribute__((aligned(1024))) char smem[Lds::kBytes];
    const uint32_t lds_base = lds_address(smem);
    float *s_m = reinterpret_cast<float *>(smem + Lds::kMl), *s_l = s_m + kWaves * kRows;    // [wavefront][row]
    const int tid = threadIdx.x, lane = tid & 63;
    const int wv = kAlone ? 0 : __builtin_amdgcn_readfirstlane(tid >> 6);
    const int g = lane >> 4, n16 = lane & 15;
    const int G = dims.Hq / dims.Hkv;

    const int sp = blockIdx.z;
    int i, rg;
    window_place(dims, blockIdx.x, i, rg);
    const RowsBefore before(dims, i, lane);
    WindowUnit u;
    if (!window_unit(u, dims, i, rg, blockIdx.y)) return;
    const int all_blocks = (u.pages + kPages - 1) / kPages, per = (all_blocks + splits - 1) / splits;
    const int ns = per > 0 ? (all_blocks + per - 1) / per : 1;
    const int b0 = sp * per, b1 = min(all_blocks, b0 + per);
    if (sp >= ns) return;

    // ---- this wavefront's two slots ------------------------------------------------------------------------
    // Token rows of 256 (128) bytes.  In K's the 16-byte chunk c of token t stands at place c ^ key of its row (key: t % 16 at
    // head_dim 128, t / 2 % 8 at 64), in V's the 32-byte chunk cc at place cc ^ key (t % 8, t / 2 % 4): operand reads, of one chunk
    // of 16 tokens in a row, meet no bank twice, while the loader fetches whole rows.
    char *k_slot = smem + wv * Lds::kWaveBytes, *v_slot = k_slot + Lds::kV;
    const uint32_t k_lds = lds_base + wv * Lds::kWaveBytes, v_lds = k_lds + Lds::kV;
    constexpr int kLoads = kPageBytes / 1024;                       // load instructions per page
    uint32_t k_voff[kLoads], v_voff[kLoads], k_rd[kS], v_rd;
#pragma unroll
    for (int j = 0; j < kLoads; ++j) {
        if constexpr (D == 128) {
            k_voff[j] = g * 256 + 16 * (n16 ^ g ^ (4 * j));
            v_voff[j] = g * 256 + 16 * (n16 ^ (2 * g) ^ (8 * (j & 1)));
        } else {
            k_voff[j] = (lane >> 3) * 128 + 16 * ((lane & 7) ^ ((4 * j + g) & 7));
            v_voff[j] = (lane >> 3) * 128 + 32 * (((lane >> 1) & 3) ^ g) + 16 * (lane & 1);
        }
    }
#pragma unroll
    for (int s = 0; s < kS; ++s) k_rd[s] = n16 * kRowBytes + 16 * ((4 * s + g) ^ (D == 128 ? n16 : n16 >> 1));
    {
        const int t = 4 * g + (n16 >> 2);
        v_rd = v_lds + t * kRowBytes + 32 * (D == 128 ? t & 7 : (t >> 1) & 3) + 8 * (n16 & 3);
    }
    auto read_vt = [&](int half, int dt) -> uint4 {
        const uint32_t at = (v_rd ^ (32 * dt)) + half * 2 * kPageBytes;
        const uint2 lo = read_transposed(at), hi = read_transposed(at + kPageBytes);
        return make_uint4(lo.x, lo.y, hi.x, hi.y);
    };

    // Page ids are wave-uniform.  Places past the end of the list repeat the block's first page, so that every block issues the
    // same loads.
    const int64_t head_bytes = kPageBytes;
    int64_t base[kPages];
    auto look_up = [&](int bi) {
#pragma unroll
        for (int j = 0; j < kPages; ++j) {
            const int v = bi * kPages + j;
            const int64_t p = block_table[u.bt_off + u.page_of(v < u.pages ? v : bi * kPages)];
            base[j] = (p * dims.Hkv + u.gkv) * head_bytes;
        }
    };
    auto issue = [&](const char *pages, const uint32_t (&voff)[kLoads], uint32_t lds) {
#pragma unroll
        for (int j = 0; j < kPages; ++j) {
            const v4i32 rs = buffer_rsrc(pages + base[j], kPageBytes);
            if constexpr (kShared) load_shared_page(rs, voff[0], voff[1], voff[2], voff[3], lds + j * kPageBytes);
            else if constexpr (D == 128) load_page_to_lds(rs, voff[0], voff[1], voff[2], voff[3], lds + j * kPageBytes);
            else load_lds_2(rs, voff[0], voff[1], lds + j * kPageBytes);
        }
    };

    // K as A operand of (mt, s): lane (g, m) <- token m of page mt, channels 32 s + 8 g .. + 7
    uint4 ka[kPages][kS];
    auto request_k = [&]() {
        if constexpr (kAlone) {
#pragma unroll
            for (int mt = 0; mt < kPages; ++mt)
#pragma unroll
                for (int s = 0; s < kS; ++s) ka[mt][s] = ld16_stream(k_pages + base[mt] + n16 * kRowBytes + 64 * s + 16 * g);
        } else {
            issue(k_pages, k_voff, k_lds);
        }
    };

    const bool works = b0 + wv < b1;
    if (works) {
        look_up(b0 + wv);
        request_k();
    }
    u.qrow0 = __builtin_amdgcn_readfirstlane(before.sum(dims, i, lane));
    if (u.qrow0 + u.n > dims.total_q) {                             // inconsistent lengths
        wait_loads<0>();
        return;
    }
    // Q^T operands: entry (row tile, s) of 1 KB, shared out to the wavefronts.  Rows past the last one repeat it (their results
    // are never stored).
#pragma unroll
    for (int e0 = 0; e0 < RT * kS; e0 += kStep) {
        const int e = e0 + wv;
        if (RT * kS % kStep == 0 || e < RT * kS) {
            const int row = min(u.r0 + 16 * (e / kS) + n16, u.rows - 1), n0 = u.r0 / G;
            const v4i32 rs = buffer_rsrc(q + (u.qrow0 + n0) * dims.Hq * (int64_t)kRowBytes, (uint32_t)(min(u.n - n0, kRows + 1) * dims.Hq) * kRowBytes);
            load16_to_lds(rs, (uint32_t)(((row / G - n0) * dims.Hq + u.gkv * G + row % G) * kRowBytes + 64 * (e % kS) + 16 * g), lds_base + Lds::kQ + e * 1024);
        }
    }
    if (works) issue(v_pages, v_voff, v_lds);
    if (!works) wait_loads<0>();
    if constexpr (!kAlone) {
        if (works) wait_loads<8>();                                 // all but the first block's V
        lds_barrier();
    }

    int pos[RT];
#pragma unroll
    for (int nt = 0; nt < RT; ++nt) {
        const int row = u.r0 + 16 * nt + n16;
        pos[nt] = row < u.rows ? u.first_pos + row / G : -1;
    }
    const int oldest = u.first_pos + u.r0 / G, newest = u.first_pos + (min(u.r0 + kRows, u.rows) - 1) / G;      // rows' positions
    float m[RT], lsum[RT];
    f32x4 o[RT][kDt];
#pragma unroll
    for (int nt = 0; nt < RT; ++nt) {
        m[nt] = kLowestRef; lsum[nt] = 0.f;
#pragma unroll
        for (int dt = 0; dt < kDt; ++dt) o[nt][dt] = f32x4{0.f, 0.f, 0.f, 0.f};
    }

#pragma unroll 1
    for (int bi = b0 + wv; bi < b1; bi += kStep) {
        // first token of every page of the block; a place past the list's end is behind every row
        int tb[kPages];
        bool need_mask = false;
#pragma unroll
        for (int j = 0; j < kPages; ++j) {
            const int v = bi * kPages + j;
            tb[j] = v < u.pages ? u.page_of(v) * 16 : 1 << 30;
            need_mask |= tb[j] + 15 > oldest || !(newest - tb[j] < u.window || tb[j] + 15 < u.sinks);
        }
        const bool more = bi + kStep < b1;
        if (more) look_up(bi + kStep);
        if constexpr (kAlone) {
            wait_loads<0>();                                        // K and V of this block (and Q)
        } else {
            if (bi != b0 + wv) wait_loads<8>();                     // K of this block (its V is 8 loads younger)
            // ---- K operands out of the slot, the next block's K into it ----------------------------------------
#pragma unroll
            for (int mt = 0; mt < kPages; ++mt)
#pragma unroll
                for (int s = 0; s < kS; ++s) ka[mt][s] = *reinterpret_cast<const uint4 *>(k_slot + mt * kPageBytes + k_rd[s]);
            if (more) {
                wait_lds();
                request_k();
            }
        }

        // ---- S^T = K Q^T, online softmax (per lane: row n16 of each row tile, 4 tokens of every page) -----------
        uint4 pop[RT][kPages / 2], pop_lo[RT][kPages / 2];
#pragma unroll
        for (int nt = 0; nt < RT; ++nt) {
            uint4 qop[kS];
#pragma unroll
            for (int s = 0; s < kS; ++s) qop[s] = *reinterpret_cast<const uint4 *>(smem + Lds::kQ + (nt * kS + s) * 1024 + lane * 16);
            float p[4 * kPages];
#pragma unroll
            for (int mt = 0; mt < kPages; ++mt) {
                f32x4 acc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int s = 0; s < kS; ++s) acc = Mma<T>::run(ka[mt][s], qop[s], acc);
#pragma unroll
                for (int r = 0; r < 4; ++r) p[4 * mt + r] = acc[r];
            }
            if constexpr (kAlone) {
                if (nt == RT - 1 && more) request_k();              // (all row tiles have had their products)
            }
            if (need_mask) {
#pragma unroll
                for (int e = 0; e < 4 * kPages; ++e) p[e] = window_sees(u, pos[nt], tb[e >> 2] + 4 * g + (e & 3)) ? p[e] : -INFINITY;
            }
            float mx = p[0];
#pragma unroll
            for (int e = 1; e < 4 * kPages; ++e) mx = fmaxf(mx, p[e]);
            mx = max_over_row_groups(mx);
            // lazy reference: moves only when the block's maximum exceeds it by more than kLazyLog2
            const float mxs = mx * scale_log2;
            const bool grow = mxs > m[nt] + kLazyLog2;
            if (__builtin_expect(__builtin_amdgcn_ballot_w64(grow) != 0, 0)) {
                const float m_new = grow ? mxs : m[nt];
                const float alpha = __builtin_amdgcn_exp2f(m[nt] - m_new);
                m[nt] = m_new;
                lsum[nt] *= alpha;
#pragma unroll
                for (int dt = 0; dt < kDt; ++dt) o[nt][dt] *= alpha;
            }
            softmax_weights<4 * kPages>(p, scale_log2, m[nt], Weights::kShiftLog2);
            float psum = 0.f;
#pragma unroll
            for (int e = 0; e < 4 * kPages; ++e) psum += p[e];
            lsum[nt] += psum;
#pragma unroll
            for (int h = 0; h < kPages / 2; ++h) {
                uint32_t hi[4], lo[4];
#pragma unroll
                for (int w = 0; w < 4; ++w) {
                    const float x = p[8 * h + 2 * w], y = p[8 * h + 2 * w + 1];
                    hi[w] = Mma<T>::pack2(x, y);
                    lo[w] = Mma<T>::pack2(x - Weights::lo(hi[w]), y - Weights::hi(hi[w]));
                }
                pop[nt][h] = make_uint4(hi[0], hi[1], hi[2], hi[3]);
                pop_lo[nt][h] = make_uint4(lo[0], lo[1], lo[2], lo[3]);
            }
        }

        // ---- V of this block: zero for tokens that no row sees -----------------------------------------
        if constexpr (!kAlone) {
            if (more) wait_loads<8>();
            else wait_loads<0>();
        }
        if (need_mask) {
            constexpr int kLanesPerRow = kRowBytes / 16, kRowsPerStep = 64 / kLanesPerRow;
#pragma unroll
            for (int j = 0; j < kPages; ++j)
#pragma unroll
                for (int r0 = 0; r0 < 16; r0 += kRowsPerStep) {
                    const int r = r0 + lane / kLanesPerRow, t = tb[j] + r;
                    if (t > newest || (oldest - t >= u.window && t >= u.sinks))
                        *reinterpret_cast<uint4 *>(v_slot + j * kPageBytes + r0 * kRowBytes + lane * 16) = make_uint4(0, 0, 0, 0);
                }
        }
        // ---- O^T += V^T P^T, then the next block's V into the slot --------------------------------------------
#pragma unroll
        for (int h = 0; h < kPages / 2; ++h) {
            uint4 vt = read_vt(h, 0);
#pragma unroll
            for (int dt = 0; dt < kDt; ++dt) {
                uint4 vt_next = vt;
                if (dt + 1 < kDt) vt_next = read_vt(h, dt + 1);
#pragma unroll
                for (int nt = 0; nt < RT; ++nt) {
                    o[nt][dt] = Mma<T>::run(vt, pop[nt][h], o[nt][dt]);
                    o[nt][dt] = Mma<T>::run(vt, pop_lo[nt][h], o[nt][dt]);
                }
                vt = vt_next;
            }
        }
        if (more) {
            wait_lds();
            issue(v_pages, v_voff, v_lds);
        }
    }

    if constexpr (kAlone) {
        // the state is the result: lane (g, n16) holds the channels 16 dt + 4 g .. + 3 of row n16
#pragma unroll
        for (int nt = 0; nt < RT; ++nt) {
            lsum[nt] += __shfl_xor(lsum[nt], 16, kWave);
            lsum[nt] += __shfl_xor(lsum[nt], 32, kWave);
            const int row = u.r0 + 16 * nt + n16;
            float total = lsum[nt];
#pragma unroll
            for (int dt = 0; dt < kDt; ++dt) total += (o[nt][dt][0] + o[nt][dt][1]) + (o[nt][dt][2] + o[nt][dt][3]);
            unsigned long long odd = __ballot(row < u.rows && !(fabsf(total) < INFINITY));
            while (__builtin_expect(odd != 0, 0)) {
                const int of = (int)__builtin_ctzll(odd) & 15;
                float rm, rsum;
                float2 ra;
                row_by_selection<T, D>(u, dims, block_table, q, k_pages, v_pages, u.r0 + 16 * nt + of, 0, u.pages, scale_log2, rm, rsum, ra);
#pragma unroll
                for (int dt = 0; dt < kDt; ++dt) {
                    const int from = 8 * dt + 2 * g;
                    const f32x4 val = {__shfl(ra.x, from, kWave), __shfl(ra.y, from, kWave), __shfl(ra.x, from + 1, kWave), __shfl(ra.y, from + 1, kWave)};
                    if (n16 == of) o[nt][dt] = val;
                }
                if (n16 == of) lsum[nt] = rsum;
                odd &= ~(0x0001000100010001ull << of);
            }
            if (row >= u.rows) continue;
            const float inv = 1.0f / lsum[nt];
            const int64_t obase = ((u.qrow0 + row / G) * dims.Hq + u.gkv * G + row % G) * (int64_t)D + 4 * g;
#pragma unroll
            for (int dt = 0; dt < kDt; ++dt) {
                const f32x4 val = o[nt][dt] * inv;
                if (out_dtype == ADASPEC_F32)
                    *reinterpret_cast<f32x4 *>(reinterpret_cast<float *>(out) + obase + 16 * dt) = val;
                else
                    *reinterpret_cast<uint2 *>(reinterpret_cast<uint16_t *>(out) + obase + 16 * dt) =
                        make_uint2(Mma<T>::pack2(val[0], val[1]), Mma<T>::pack2(val[2], val[3]));
            }
        }
        return;
    }
    // ---- merge the four wavefronts' states through LDS, one row tile at a time, each wavefront's in its V slot
    if constexpr (Lds::kFull) lds_barrier();                        // (m, l) go where Q stands: all are done with it
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
        for (int dt = 0; dt < kDt; ++dt)
            *reinterpret_cast<f32x4 *>(v_slot + window_piece<D>(n16, 4 * dt + g)) = o[nt][dt];
        lds_barrier();
        finish_window_tile<T, D>(u, dims, block_table, q, k_pages, v_pages, out, part_ml, part_o, smem + Lds::kV, Lds::kWaveBytes, s_m, s_l,
                                 kRows, nt, ns, b0 * kPages, min(b1 * kPages, u.pages), scale_log2, Weights::kShiftLog2, out_dtype,
                                 (((int64_t)blockIdx.x * dims.Hkv + blockIdx.y) * splits + sp) * kRows);
        if (nt + 1 < RT) lds_barrier();                             // the next tile overwrites the slots
    }
}

hipError_t launch_attn_window_mfma(const WindowArgs &a, const WindowDims &w)
{
    const adaspec_attn_dims &d = a.dims;
    const WindowPlan &p = a.plan;
    float *ml = reinterpret_cast<float *>(a.ws + p.off_part_ml), *o = reinterpret_cast<float *>(a.ws + p.off_part_o);
    auto launch = [&](auto tag, auto dim, auto rt, auto alone, auto shared) {
        hipLaunchKernelGGL((attn_window_kernel<decltype(tag), decltype(dim)::value, decltype(rt)::value, decltype(alone)::value, decltype(shared)::value>),
                           dim3((unsigned)(d.batch * p.groups), d.n_kv_heads, p.splits), dim3(decltype(alone)::value ? 64 : 256), 0, a.stream, w,
                           a.block_table, (const char *)a.q, (const char *)a.k_pages, (const char *)a.v_pages, a.out, ml, o, p.splits,
                           a.scale_log2, d.out_dtype);
    };
    // Two row groups read the same pages: loads that leave them in the L2 (128 requests of 72 rows at 8 kv heads, head_dim 128,
    // window 1024: 139 us, streaming loads 160; window 4096, 64 requests: 222 and 282).  Head_dim 64 gains nothing (93 us either
    // way), and one group alone loses by them (32 rows, window 1024: 102 us instead of 91).
    auto with_rt = [&](auto tag, auto dim) {
        constexpr bool kMay = decltype(dim)::value == 128;
        auto with_form = [&](auto rt) {
            if constexpr (decltype(rt)::value < 4) {
                if (p.alone) { launch(tag, dim, rt, std::true_type{}, std::false_type{}); return; }
            }
            if constexpr (kMay && decltype(rt)::value > 2) {        // (more than one group: of three or four tiles)
                if (p.groups > 1) { launch(tag, dim, rt, std::false_type{}, std::true_type{}); return; }
            }
            launch(tag, dim, rt, std::false_type{}, std::false_type{});
        };
        switch (p.rows_per_group / 16) {
        case 1: with_form(std::integral_constant<int, 1>{}); break;
        case 2: with_form(std::integral_constant<int, 2>{}); break;
        case 3: with_form(std::integral_constant<int, 3>{}); break;
        default: with_form(std::integral_constant<int, 4>{}); break;
        }
    };
    auto with_dim = [&](auto tag) {
        if (d.head_dim == 128) with_rt(tag, std::integral_constant<int, 128>{});
        else with_rt(tag, std::integral_constant<int, 64>{});
    };
    if (d.dtype == ADASPEC_F16) with_dim(F16{});
    else with_dim(BF16{});
    return hipGetLastError();
}

}  // namespace adaspec
