// Positions: queries turned, keys turned and appended to the paged cache with the values, in one launch.
//
// Row j of request i stands at p = L_i - n_i + j (in a draft tree at L_i - n_i + depth of node j).  Pair f of a head's first
// rot_dim entries, (x[f], x[f + rot_dim / 2]) or, interleaved, (x[2f], x[2f + 1]), becomes
//     (a cos - b sin, b cos + a sin),   angle = p * inv_freq[f],   cos and sin times attn_factor.
// The angle is taken in 64 bits and reduced to a fraction of a turn before it is rounded: in 32 bits the angle of position
// 10^6 is off by a sixteenth of a radian.  The rest is in 32 bits, rounded once to what is stored.
//
// A workgroup takes up to 16 consecutive rows of a request (for a cache of 8 bits: those of one page, whose scale they
// decide together) and some of the kv heads with their query heads; cosines and sines of its rows are worked out once.
//
// Small calls are bound by latency: two memory round trips (lengths, rows), three into a cache of 8 bits (the page's scale), with
// the angles worked out while the rows travel: 128 requests of up to 7 rows, 32/8 heads of 128, 6.8 us, into 8 bits 8.9, where a wavefront's second head
// is requested when its first is written: one round trip more.  Large ones by HBM: 16 prompts of 100-4000 rows 169 us for 806 MB,
// 4.8 TB/s; into 8 bits, 64/8 heads, 256 for 1276 MB, 5.0 TB/s (a large copy: 5.07).
#include <type_traits>

#include "adaspec_internal.h"
#include "attn_mfma_common.h"
#include "device_utils.h"
#include "e4m3.h"

namespace adaspec {

constexpr int kRopeThreads = 256;
constexpr int kRopeRows = 16;
static_assert(kRopeRows == kPageTokens, "a workgroup's rows are those of a page");
constexpr int kRopeMaxHalf = 128;       // pairs of a head
// MI355X, us, into 8 bits, chunk by chunk / request by request: 128 requests of up to 7 rows (2 chunks) 9.5 / 8.9, 128 prompts of up to 100 (8)
// 77 / 62, 64 of up to 250 (17) 68.5 / 82, 16 of up to 4000 (251) 243 / 304.
constexpr int kFewChunks = 8;

struct RopeArgs {
    const void *q, *k, *v;
    const float *inv_freq;
    void *q_out, *k_pages, *v_pages;
    float *k_scales, *v_scales;
    const int32_t *block_table, *ctx_lens, *spec_lens, *parents;
    adaspec_rope_dims d;
    int chunks;                 // of up to 16 rows that a request may have
    int heads;                  // heads (kv heads with their query heads; query heads where nothing is appended) per workgroup
};

// x / n for 0 <= x < 2^21 and 1 <= n, by the rounded reciprocal: (x + 1/2) / n is at least 1 / (2 n) away from an integer, and off by
// less than x / n * 2^-22
struct Divider {
    int n;
    float inv;
    __device__ __forceinline__ explicit Divider(int n_) : n(n_), inv(1.0f / (float)n_) {}
    __device__ __forceinline__ int operator()(int x, int &rest) const
    {
        const int q = (int)(((float)x + 0.5f) * inv);
        rest = x - q * n;
        return q;
    }
};

// kBytes at an address aligned to them (to 16 bytes, if there are more), in words
template <int kBytes> struct Words { uint32_t w[kBytes / 4]; };
template <int kBytes>
__device__ __forceinline__ Words<kBytes> load_words(const void *at)
{
    Words<kBytes> r;
    if constexpr (kBytes == 4) {
        r.w[0] = *static_cast<const uint32_t *>(at);
    } else if constexpr (kBytes == 8) {
        const uint2 v = *static_cast<const uint2 *>(at);
        r.w[0] = v.x, r.w[1] = v.y;
    } else {
#pragma unroll
        for (int e = 0; e < kBytes / 16; ++e) {
            const uint4 v = static_cast<const uint4 *>(at)[e];
            r.w[4 * e] = v.x, r.w[4 * e + 1] = v.y, r.w[4 * e + 2] = v.z, r.w[4 * e + 3] = v.w;
        }
    }
    return r;
}
template <int kBytes>
__device__ __forceinline__ void store_words(void *at, const Words<kBytes> &r)
{
    if constexpr (kBytes == 4) {
        *static_cast<uint32_t *>(at) = r.w[0];
    } else if constexpr (kBytes == 8) {
        *static_cast<uint2 *>(at) = make_uint2(r.w[0], r.w[1]);
    } else {
#pragma unroll
        for (int e = 0; e < kBytes / 16; ++e) static_cast<uint4 *>(at)[e] = make_uint4(r.w[4 * e], r.w[4 * e + 1], r.w[4 * e + 2], r.w[4 * e + 3]);
    }
}
// W consecutive elements as they are stored, in words (an array of 16-bit elements would take a register each), or a single one
template <class T, int W> struct Raw {
    static constexpr int kBytes = W * sizeof(typename T::storage);
    std::conditional_t<kBytes >= 4, Words<kBytes < 4 ? 4 : kBytes>, uint16_t> x;
    __device__ __forceinline__ void load(const void *base, int64_t at)
    {
        const typename T::storage *p = static_cast<const typename T::storage *>(base) + at;
        if constexpr (kBytes >= 4) x = load_words<kBytes>(p);
        else x = *p;
    }
    __device__ __forceinline__ float operator[](int e) const
    {
        if constexpr (kBytes < 4) return load_as_float<T>(&x, 0);
        else if constexpr (T::id == ADASPEC_F32) return __uint_as_float(x.w[e]);
        else if constexpr (T::id == ADASPEC_BF16) return __uint_as_float(e & 1 ? x.w[e / 2] & 0xffff0000u : x.w[e / 2] << 16);
        else return f16_bits_to_float((uint16_t)(x.w[e / 2] >> (16 * (e & 1))));
    }
};
template <class T, int W>
__device__ __forceinline__ void store_unit(void *base, int64_t at, const float (&x)[W])
{
    typename T::storage *p = static_cast<typename T::storage *>(base) + at;
    if constexpr (W == 1) {
        store_out(p, 0, x[0], T::id);
    } else {
        Words<W * sizeof(*p)> r;
        if constexpr (T::id == ADASPEC_F32) {
#pragma unroll
            for (int e = 0; e < W; ++e) r.w[e] = __float_as_uint(x[e]);
        } else {
#pragma unroll
            for (int e = 0; e < W / 2; ++e) r.w[e] = Mma<T>::pack2(x[2 * e], x[2 * e + 1]);
        }
        store_words(p, r);
    }
}
template <int W>
__device__ __forceinline__ void store_unit8(void *base, int64_t at, const float (&x)[W], float inv)
{
    uint8_t *p = static_cast<uint8_t *>(base) + at;
    if constexpr (W == 8) {
        *reinterpret_cast<uint2 *>(p) = make_uint2(float4_to_e4m3(x[0] * inv, x[1] * inv, x[2] * inv, x[3] * inv),
                                                   float4_to_e4m3(x[4] * inv, x[5] * inv, x[6] * inv, x[7] * inv));
    } else if constexpr (W == 4) {
        *reinterpret_cast<uint32_t *>(p) = float4_to_e4m3(x[0] * inv, x[1] * inv, x[2] * inv, x[3] * inv);
    } else if constexpr (W == 2) {
        *reinterpret_cast<uint16_t *>(p) = (uint16_t)float2_to_e4m3(x[0] * inv, x[1] * inv);
    } else {
        *p = (uint8_t)float2_to_e4m3(x[0] * inv, 0.f);
    }
}

// A head's row in units: with the halves paired a unit is W entries of the first half and their partners, interleaved it is W
// entries; behind them, W at a time, those that are not turned.
template <class T, int W, bool kInter>
struct Units {
    struct Item { Raw<T, W> a, b; };    // (b: the partners)
    int rot, turned, count;
    __device__ __forceinline__ Units(int rot_, int d) : rot(rot_), turned(kInter ? rot / W : rot / (2 * W)), count(turned + (d - rot) / W) {}

    __device__ __forceinline__ int place(int u) const { return u < turned ? u * W : rot + (u - turned) * W; }
    // unit u of the row at `src`
    __device__ __forceinline__ void fetch(Item &it, const void *base, int64_t src, int u) const
    {
        it.a.load(base, src + place(u));
        if constexpr (!kInter)
            if (u < turned) it.b.load(base, src + u * W + rot / 2);
    }
    // turned (cs: the row's cosines and sines): put(place in the row, values)
    template <class Put>
    __device__ __forceinline__ void turn(const Item &it, int u, const float2 *cs, Put &&put) const
    {
        float a[W];
#pragma unroll
        for (int e = 0; e < W; ++e) a[e] = it.a[e];
        if (u < turned) {
            if constexpr (kInter) {
#pragma unroll
                for (int e = 0; e + 1 < W; e += 2) {
                    const float2 r = cs[(u * W + e) / 2];
                    const float x = a[e], y = a[e + 1];
                    a[e] = x * r.x - y * r.y;
                    a[e + 1] = y * r.x + x * r.y;
                }
            } else {
                float b[W];
#pragma unroll
                for (int e = 0; e < W; ++e) {
                    const float2 r = cs[u * W + e];
                    const float x = a[e], y = it.b[e];
                    a[e] = x * r.x - y * r.y;
                    b[e] = y * r.x + x * r.y;
                }
                put(u * W + rot / 2, b);
            }
        }
        put(place(u), a);
    }
    // the largest squared length of the unit's pairs and of its other entries, in F; what is not a number does not count
    template <class F>
    __device__ __forceinline__ void longest(const Item &it, int u, F &pairs, F &rest) const
    {
        // (selected values, no branches: the compiler would select what to write to by its address, in scratch memory, which cost every launch:
        // 16 trees of up to 61 rows, 32/8 heads of 128, 12.6 us, 8.8 without; 128 requests of up to 7 rows 10.0, 8.9)
        const bool turns = u < turned;
#pragma unroll
        for (int e = 0; e < W; e += kInter ? 2 : 1) {
            const F x = it.a[e], y = kInter ? F(it.a[e + 1]) : turns ? F(it.b[e]) : F(0), pair = x * x + y * y;
            pairs = larger(pairs, turns ? pair : F(0));
            rest = larger(rest, turns ? F(0) : x * x);
            if constexpr (kInter) rest = larger(rest, turns ? F(0) : y * y);
        }
    }
    static __device__ __forceinline__ float larger(float most, float s) { return fmaxf(most, s); }
    // (in 64 bits squares of floats are finite, infinities do not count)
    static __device__ __forceinline__ double larger(double most, double s) { return fmax(most, s < 1e200 ? s : 0.0); }
};

// The new tokens of one (page, kv head) of K or of V, by one wavefront: rows src, src + stride, ... go to slots [lo, hi).
// begin() requests what it can (the rows stay in registers up to kHeld units per lane, more are read twice); finish() finds the
// scale, rounds the page's earlier tokens to it where it has grown, and writes the new ones.
template <class T, int W, bool kInter>
struct PageAppend {
    using U = Units<T, W, kInter>;
    static constexpr int kHeld = kInter ? 4 : 2;        // 16 rows of 128 channels
    U units;
    const void *x;
    int64_t src, stride;
    uint8_t *block;
    float *scale_at;
    int d, lo, work, lane;
    bool held_all;
    float old;
    typename U::Item held[kHeld];

    __device__ __forceinline__ PageAppend(const U &units_) : units(units_) {}
    __device__ __forceinline__ void begin(const void *x_, int64_t src_, int64_t stride_, int d_, uint8_t *block_, float *scale_at_, int lo_, int n, int lane_)
    {
        x = x_, src = src_, stride = stride_, d = d_, block = block_, scale_at = scale_at_, lo = lo_, lane = lane_;
        work = n * units.count;
        held_all = work <= kHeld * kWave;
        old = lo > 0 ? *scale_at : 0.f;
        if (held_all) {
#pragma unroll
            for (int e = 0; e < kHeld; ++e)
                if (lane + e * kWave < work) fetch(held[e], lane + e * kWave);
        }
    }
    __device__ __forceinline__ int of(int idx, int &u) const { return Divider(units.count)(idx, u); }
    __device__ __forceinline__ void fetch(typename U::Item &it, int idx) const
    {
        int u;
        const int j = of(idx, u);
        units.fetch(it, x, src + j * stride, u);
    }
    // f(unit of the page in registers, its number)
    template <class Fn>
    __device__ __forceinline__ void each(Fn &&f)
    {
        if (held_all) {
#pragma unroll
            for (int e = 0; e < kHeld; ++e)
                if (lane + e * kWave < work) f(held[e], lane + e * kWave);
        } else {
            for (int idx = lane; idx < work; idx += kWave) {
                fetch(held[0], idx);
                f(held[0], idx);
            }
        }
    }
    // log2 of the scale that the new tokens need.  Squares and their sums in 32 bits are off by a few units in the last place; where
    // that leaves the scale in doubt (near a border, 1.53125 * 2^odd, or where they overflow or underflow) it is worked out in 64,
    // where the products are exact, so that it never depends on a rounding.
    __device__ __forceinline__ int scale_log2(float gain)
    {
        float pairs = 0.f, rest = 0.f;
        each([&](const typename U::Item &it, int idx) {
            int u;
            of(idx, u);
            units.longest(it, u, pairs, rest);
        });
        const float most = wave_max(fmaxf(pairs * (gain * gain), rest));
        const uint32_t fraction = (__float_as_uint(most) & 0x7fffffu) - 0x440000u;              // of 1.53125
        if (most > 1e-30f && most < 1e37f && (fraction + 32u) > 64u) return scale_log2_for(most);
        double pairs64 = 0.0, rest64 = 0.0;
        each([&](const typename U::Item &it, int idx) {
            int u;
            of(idx, u);
            units.longest(it, u, pairs64, rest64);
        });
        const double gain64 = gain, most64 = fmax(pairs64 * (gain64 * gain64), rest64);
        return scale_log2_for(last_lane(wave_scan(most64, 0.0, [](double a, double b) { return fmax(a, b); })));
    }
    __device__ __forceinline__ void finish(float gain, const float2 *cs, int cs_stride)
    {
        float scale = power_of_two(scale_log2(gain));
        if (lo > 0) {                                   // the page keeps earlier tokens: their scale never falls
            scale = fmaxf(old, scale);
            if (scale != old) {
                const float ratio = old / scale;
                for (int c = lane; c < lo * d / 8; c += kWave) e4m3_rescale8(block + 8 * c, block + 8 * c, ratio);
            }
        }
        const float inv = 1.0f / scale;
        each([&](const typename U::Item &it, int idx) {
            int u;
            const int j = of(idx, u);
            units.turn(it, u, cs + j * cs_stride, [&](int c, const float (&y)[W]) { store_unit8<W>(block, (int64_t)(lo + j) * d + c, y, inv); });
        });
        if (lane == 0) *scale_at = scale;
    }
};

template <class T, int W, bool kInter, bool k8>
__global__ __launch_bounds__(kRopeThreads) void rope_append_kernel(RopeArgs a)
{
    extern __shared__ float2 cs[];                      // [rows][pairs]
    __shared__ float freq[kRopeMaxHalf];
    __shared__ int wsum[kRopeThreads / kWave];
    __shared__ int depth[kWave];
    __shared__ int pages[2];
    using U = Units<T, W, kInter>;
    const adaspec_rope_dims &D = a.d;
    const int tid = threadIdx.x, lane = tid & 63, wv = __builtin_amdgcn_readfirstlane(tid >> 6);
    // (neighbours in memory side by side; where most requests have fewer rows than chunks, the chunks that have none come last)
    const bool by_request = a.chunks <= kFewChunks;
    const int i = by_request ? blockIdx.x % D.batch : blockIdx.x / a.chunks, chunk = by_request ? blockIdx.x / D.batch : blockIdx.x % a.chunks;
    const int d = D.head_dim, half = D.rot_dim / 2, Hkv = D.n_kv_heads;

    const int n = min(max(a.spec_lens[i], 0), D.max_spec_len) + 1;
    const int L = a.ctx_lens[i], first = L - n;
    // its rows [j0, j1) here: tokens [t0, t1) of the request (counted from the first row: a length may be anything)
    const int in_page = k8 ? first % kPageTokens : 0;
    const int j0 = max(0, chunk * kRopeRows - in_page), j1 = min(n, (chunk + 1) * kRopeRows - in_page);
    const int t0 = first + j0, t1 = first + j1;
    int part = 0;
    for (int j = tid; j < i; j += kRopeThreads) part += min(max(a.spec_lens[j], 0), D.max_spec_len) + 1;
    if (tid < half) freq[tid] = a.inv_freq[tid];
    if (L < n || j0 >= j1) return;
    if (a.k && tid < 2) {
        const int at = t0 / kPageTokens + tid;
        int page = -1;
        if (at <= (t1 - 1) / kPageTokens && at < D.max_pages_per_req) page = a.block_table[(int64_t)i * D.max_pages_per_req + at];
        pages[tid] = page >= 0 && page < D.num_pages ? page : -1;
    }
    part = wave_sum(part);
    if (lane == 0) wsum[wv] = part;
    lds_barrier();
    int row0 = 0;
#pragma unroll
    for (int w = 0; w < kRopeThreads / kWave; ++w) row0 += wsum[w];
    if (row0 + n > D.total_q) return;                   // inconsistent metadata: touch nothing
    const int nt = j1 - j0;
    const int64_t row = (int64_t)row0 + j0;

    // Rows of heads in the order of memory, unit by unit: the query heads of this workgroup and, 16-bit and fp32 caches, its kv heads.
    const U units(D.rot_dim, d);
    const int per = a.k ? (a.q ? D.n_q_heads / Hkv : 0) : 1;        // query heads per head of the grid
    const int h0 = blockIdx.y * a.heads, nh = min(a.heads, (a.k ? Hkv : D.n_q_heads) - h0);
    const int nq = nh * per, nk = a.k && !k8 ? nh : 0, both = nq + nk;
    const int work = both * nt * units.count;
    // Cosines and sines of the rows' pairs, by all wavefronts (each of which comes here once, with its own rows on their way).
    const auto angles = [&] {
        if (half == 0) return;
        if (a.parents) {
            // depths by doubling: every node looks at the node that its jumps so far have led to (the root at itself)
            if (wv == 0) {
                int up = lane > 0 && lane < n ? min(max(a.parents[row0 + lane], 0), lane - 1) : 0, dep = lane > 0 && lane < n ? 1 : 0;
#pragma unroll
                for (int s = 0; s < 6; ++s) {
                    dep += __shfl(dep, up, kWave);
                    up = __shfl(up, up, kWave);
                }
                depth[lane] = dep;
            }
            lds_barrier();
        }
        const Divider by_half(half);
        for (int idx = tid; idx < nt * half; idx += kRopeThreads) {
            int f;
            const int j = by_half(idx, f);
            const int pos = first + (a.parents ? depth[j0 + j] : j0 + j);
            const double turns = (double)pos * (double)freq[f] * 0.15915494309189533577;        // 1 / (2 pi)
            // (half turns, in two floats: what the first leaves turns the result by that little further)
            const double halves = 2.0 * (turns - rint(turns));
            const float r = (float)halves, more = (float)(halves - r) * 3.14159265f;
            float s, c;
            sincospif(r, &s, &c);
            cs[idx] = make_float2(fmaf(-s, more, c) * D.attn_factor, fmaf(c, more, s) * D.attn_factor);
        }
        lds_barrier();
    };
    // (into a cache of 8 bits two wavefronts take the keys and values, where there are queries: one the keys, one the values)
    const int kv_waves = k8 ? (a.q ? 2 : 4) : 0, threads = kRopeThreads - kv_waves * kWave, me = tid - kv_waves * kWave;
    if constexpr (k8) {
        if (wv < kv_waves) {
            const int page = pages[0], lo = t0 % kPageTokens, last = page < 0 ? 0 : h0 + nh;
            const auto append = [&](auto part, const void *x, int64_t stride, void *pages_of, float *scales, float gain, int cs_stride) {
                const auto begin = [&](int h) {
                    const int64_t at = (int64_t)page * Hkv + h;
                    part.begin(x, row * stride + (int64_t)h * d, stride, d, static_cast<uint8_t *>(pages_of) + at * kPageTokens * d, scales + at, lo, nt, lane);
                };
                int h = h0 + wv / 2;
                if (h < last) begin(h);
                angles();
                while (h < last) {
                    part.finish(gain, cs, cs_stride);
                    h += kv_waves / 2;
                    if (h < last) begin(h);
                }
            };
            if (wv & 1) append(PageAppend<T, 8, true>(Units<T, 8, true>(0, d)), a.v, D.v_row_stride, a.v_pages, a.v_scales, 1.f, 0);
            else append(PageAppend<T, W, kInter>(units), a.k, D.k_row_stride, a.k_pages, a.k_scales, D.attn_factor, half);
            return;
        }
    }
    const Divider by_units(units.count), by_heads(both);
    constexpr int kAhead = 2;
    typename U::Item item[kAhead];
    const auto where = [&](int idx, int &j, int &h, int &u) { j = by_heads(by_units(idx, u), h); };
    const auto fetch = [&](typename U::Item &it, int idx) {
        int j, h, u;
        where(idx, j, h, u);
        if (k8 || h < nq) units.fetch(it, a.q, (row + j) * D.q_row_stride + (int64_t)(h0 * per + h) * d, u);
        else units.fetch(it, a.k, (row + j) * D.k_row_stride + (int64_t)(h0 + h - nq) * d, u);
    };
#pragma unroll
    for (int e = 0; e < kAhead; ++e)
        if (me + e * threads < work) fetch(item[e], me + e * threads);
    angles();
    for (int idx = me; idx < work; idx += kAhead * threads) {
#pragma unroll
        for (int e = 0; e < kAhead; ++e) {
            if (idx + e * threads >= work) continue;
            int j, h, u;
            where(idx + e * threads, j, h, u);
            void *out = a.q_out;
            int64_t dst = (row + j) * D.q_out_row_stride + (int64_t)(h0 * per + h) * d;
            if (!k8 && h >= nq) {
                const int t = t0 + j, page = pages[t / kPageTokens - t0 / kPageTokens];
                if (page < 0) continue;
                out = a.k_pages;
                dst = (((int64_t)page * Hkv + h0 + h - nq) * kPageTokens + t % kPageTokens) * d;
            }
            units.turn(item[e], u, cs + j * half, [&](int c, const float (&y)[W]) { store_unit<T, W>(out, dst + c, y); });
        }
#pragma unroll
        for (int e = 0; e < kAhead; ++e)
            if (idx + (kAhead + e) * threads < work) fetch(item[e], idx + (kAhead + e) * threads);
    }
    if constexpr (!k8) {
        // values as they are, 16 bytes at a time
        constexpr int kSize = sizeof(typename T::storage);
        const int vecs = d * kSize / 16, copies = nk * nt * vecs;
        const Divider by_vecs(vecs), by_kv(max(nk, 1));
        for (int idx = tid; idx < copies; idx += kRopeThreads) {
            int u, h;
            const int j = by_kv(by_vecs(idx, u), h), t = t0 + j;
            const int page = pages[t / kPageTokens - t0 / kPageTokens];
            if (page < 0) continue;
            const int64_t dst = (((int64_t)page * Hkv + h0 + h) * kPageTokens + t % kPageTokens) * d;
            reinterpret_cast<uint4 *>(static_cast<char *>(a.v_pages) + dst * kSize)[u] =
                reinterpret_cast<const uint4 *>(static_cast<const char *>(a.v) + ((row + j) * D.v_row_stride + (int64_t)(h0 + h) * d) * kSize)[u];
        }
    }
}

static int rope_chunks(const adaspec_rope_dims &d, bool fp8)
{
    return fp8 ? (d.max_spec_len + kPageTokens - 1) / kPageTokens + 1 : (d.max_spec_len + kRopeRows) / kRopeRows;
}

bool rope_grid_fits(const adaspec_rope_dims &d, bool fp8) { return (int64_t)d.batch * rope_chunks(d, fp8) < 1 << 23; }

hipError_t launch_rope_append(const void *q, const void *k, const void *v, const float *inv_freq, void *q_out, void *k_pages, void *v_pages,
                              float *k_scales, float *v_scales, const int32_t *block_table, const int32_t *ctx_lens,
                              const int32_t *spec_lens, const int32_t *parents, const adaspec_rope_dims &d, hipStream_t stream)
{
    const bool fp8 = k_scales != nullptr;
    RopeArgs a{q, k, v, inv_freq, q_out, k_pages, v_pages, k_scales, v_scales, block_table, ctx_lens, spec_lens, parents, d, rope_chunks(d, fp8), 1};
    if (!inv_freq) a.d.rot_dim = 0;
    const int heads = k ? d.n_kv_heads : d.n_q_heads;
    // Heads per workgroup: enough for its angles to be shared (20 rows of heads per row; into 8 bits, where a wavefront takes a head's keys
    // or values, 2 kv heads, or 4 without shared ones), fewer where that leaves less than two workgroups per compute unit.
    // MI355X, us, 1 / 2 / 4 / 8 kv heads of 32/8: 128 requests of up to 7 rows 7.4 / 6.8 / 7.9 / 10.7, into 8 bits 9.6 / 9.0 / 9.8 /
    // 13.8; prompts of 32000 rows 184 / 190 / 169 / 177, into 8 bits 180 / 181 / 153 / 159, of 64/8 heads 307 / 256 / 264 / 274; 16 trees of
    // up to 61 rows into 8 bits 8.8 / 10.3 / 13.1 / 21.0; without shared heads (32/32), 128 of up to 7 into 8 bits 28.8 / 20.6 / 17.6 / 17.9, without
    // queries 18.1 / 12.9 / 10.9 / 12.1; query heads alone, 17400 rows of 32 94 / 60 / 51 / 52.
    const int shared = k && q ? d.n_q_heads / d.n_kv_heads : 1;
    a.heads = !k ? 4 : !fp8 ? 20 / (shared + 1) : shared > 1 ? 2 : 4;
    a.heads = a.heads < 1 ? 1 : a.heads > heads ? heads : a.heads;
    while (a.heads > 1 && (int64_t)d.batch * a.chunks * ceil_div(heads, a.heads) < 512) a.heads = (a.heads + 1) / 2;
    const size_t lds = (size_t)kRopeRows * (a.d.rot_dim / 2) * sizeof(float2);
    const dim3 grid((unsigned)((int64_t)d.batch * a.chunks), ceil_div(heads, a.heads));
    auto launch = [&](auto tag) {
        using T = decltype(tag);
        auto with = [&](auto w, auto inter) {
            constexpr int W = decltype(w)::value;
            constexpr bool kInter = decltype(inter)::value;
            if (fp8) hipLaunchKernelGGL((rope_append_kernel<T, W, kInter, true>), grid, dim3(kRopeThreads), lds, stream, a);
            else hipLaunchKernelGGL((rope_append_kernel<T, W, kInter, false>), grid, dim3(kRopeThreads), lds, stream, a);
        };
        if (d.interleaved || a.d.rot_dim == 0) {
            if (a.d.rot_dim % 8 == 0) with(std::integral_constant<int, 8>{}, std::true_type{});
            else if (a.d.rot_dim % 4 == 0) with(std::integral_constant<int, 4>{}, std::true_type{});
            else with(std::integral_constant<int, 2>{}, std::true_type{});
        } else {
            if (a.d.rot_dim % 16 == 0) with(std::integral_constant<int, 8>{}, std::false_type{});
            else if (a.d.rot_dim % 8 == 0) with(std::integral_constant<int, 4>{}, std::false_type{});
            else if (a.d.rot_dim % 4 == 0) with(std::integral_constant<int, 2>{}, std::false_type{});
            else with(std::integral_constant<int, 1>{}, std::false_type{});
        }
    };
    if (d.dtype == ADASPEC_F32) launch(F32{});
    else if (d.dtype == ADASPEC_F16) launch(F16{});
    else launch(BF16{});
    return hipGetLastError();
}

}  // namespace adaspec
