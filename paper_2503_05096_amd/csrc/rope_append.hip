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
#include <type_traits>

#include "adaspec_internal.h"
#include "device_utils.h"
#include "e4m3.h"

namespace adaspec {

constexpr int kRopeThreads = 256;
constexpr int kRopeRows = 16;
constexpr int kRopeMaxHalf = 128;       // pairs of a head

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

// W consecutive elements
template <class T, int W>
__device__ __forceinline__ void load_unit(const void *base, int64_t at, float (&x)[W])
{
    using S = typename T::storage;
    const S *p = static_cast<const S *>(base) + at;
    if constexpr (W == 8) {
        S raw[8];
        if constexpr (sizeof(S) == 2) {
            *reinterpret_cast<uint4 *>(raw) = *reinterpret_cast<const uint4 *>(p);
        } else {
            reinterpret_cast<uint4 *>(raw)[0] = reinterpret_cast<const uint4 *>(p)[0];
            reinterpret_cast<uint4 *>(raw)[1] = reinterpret_cast<const uint4 *>(p)[1];
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = load_as_float<T>(raw, e);
    } else {
#pragma unroll
        for (int e = 0; e < W; ++e) x[e] = load_as_float<T>(p, e);
    }
}
template <class T, int W>
__device__ __forceinline__ void store_unit(void *base, int64_t at, const float (&x)[W])
{
    using S = typename T::storage;
    S *p = static_cast<S *>(base) + at;
    if constexpr (W == 8) {
        S raw[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) store_out(raw, e, x[e], T::id);
        if constexpr (sizeof(S) == 2) {
            *reinterpret_cast<uint4 *>(p) = *reinterpret_cast<const uint4 *>(raw);
        } else {
            reinterpret_cast<uint4 *>(p)[0] = reinterpret_cast<const uint4 *>(raw)[0];
            reinterpret_cast<uint4 *>(p)[1] = reinterpret_cast<const uint4 *>(raw)[1];
        }
    } else {
#pragma unroll
        for (int e = 0; e < W; ++e) store_out(p, e, x[e], T::id);
    }
}
template <int W>
__device__ __forceinline__ void store_unit8(void *base, int64_t at, const float (&x)[W], float inv)
{
    uint8_t *p = static_cast<uint8_t *>(base) + at;
    if constexpr (W == 8) {
        *reinterpret_cast<uint2 *>(p) = make_uint2(float4_to_e4m3(x[0] * inv, x[1] * inv, x[2] * inv, x[3] * inv),
                                                   float4_to_e4m3(x[4] * inv, x[5] * inv, x[6] * inv, x[7] * inv));
    } else if constexpr (W == 2) {
        const uint32_t w = float2_to_e4m3(x[0] * inv, x[1] * inv);
        p[0] = (uint8_t)w;
        p[1] = (uint8_t)(w >> 8);
    } else {
        *p = (uint8_t)float2_to_e4m3(x[0] * inv, 0.f);
    }
}

// A head's row in units: with the halves paired a unit is W entries of the first half and their partners, interleaved it is W
// entries; behind them, W at a time, those that are not turned.
template <class T, int W, bool kInter>
struct Units {
    static __device__ __forceinline__ int turned(int rot) { return kInter ? rot / W : rot / (2 * W); }
    static __device__ __forceinline__ int count(int rot, int d) { return turned(rot) + (d - rot) / W; }

    // unit u of the row that starts at `src`, turned (cs: the row's cosines and sines): put(place in the row, values)
    template <class Put>
    static __device__ __forceinline__ void turn(const void *base, int64_t src, int u, int rot, const float2 *cs, Put &&put)
    {
        const int n = turned(rot);
        float a[W];
        if (u >= n) {
            const int c = rot + (u - n) * W;
            load_unit<T, W>(base, src + c, a);
            put(c, a);
        } else if constexpr (kInter) {
            load_unit<T, W>(base, src + u * W, a);
#pragma unroll
            for (int e = 0; e < W; e += 2) {
                const float2 r = cs[(u * W + e) / 2];
                const float x = a[e], y = a[e + 1];
                a[e] = x * r.x - y * r.y;
                a[e + 1] = y * r.x + x * r.y;
            }
            put(u * W, a);
        } else {
            float b[W];
            load_unit<T, W>(base, src + u * W, a);
            load_unit<T, W>(base, src + u * W + rot / 2, b);
#pragma unroll
            for (int e = 0; e < W; ++e) {
                const float2 r = cs[u * W + e];
                const float x = a[e], y = b[e];
                a[e] = x * r.x - y * r.y;
                b[e] = y * r.x + x * r.y;
            }
            put(u * W, a);
            put(u * W + rot / 2, b);
        }
    }
    // the largest squared length of the unit's pairs, in 64 bits; pairs with something that is not finite do not count
    static __device__ __forceinline__ void longest(const void *base, int64_t src, int u, int rot, double &pairs, double &rest)
    {
        const auto count = [](double s, double &most) { if (s < 1e200) most = fmax(most, s); };
        const int n = turned(rot);
        float a[W];
        if (u >= n) {
            load_unit<T, W>(base, src + rot + (u - n) * W, a);
#pragma unroll
            for (int e = 0; e < W; ++e) count((double)a[e] * a[e], rest);
        } else if constexpr (kInter) {
            load_unit<T, W>(base, src + u * W, a);
#pragma unroll
            for (int e = 0; e < W; e += 2) count((double)a[e] * a[e] + (double)a[e + 1] * a[e + 1], pairs);
        } else {
            float b[W];
            load_unit<T, W>(base, src + u * W, a);
            load_unit<T, W>(base, src + u * W + rot / 2, b);
#pragma unroll
            for (int e = 0; e < W; ++e) count((double)a[e] * a[e] + (double)b[e] * b[e], pairs);
        }
    }
};

// The new tokens of one (page, kv head) of K or of V, by one wavefront: rows src, src + stride, ... go to slots [lo, hi).
template <class T, int W, bool kInter>
__device__ __forceinline__ void append_page8(const void *x, int64_t src, int64_t stride, int d, int rot, double gain2, const float2 *cs,
                                             int cs_stride, uint8_t *block, float *scale_at, int lo, int hi, int lane)
{
    using U = Units<T, W, kInter>;
    const int units = U::count(rot, d), n = hi - lo;
    double pairs = 0.0, rest = 0.0;
    for (int idx = lane; idx < n * units; idx += kWave) U::longest(x, src + (idx / units) * stride, idx % units, rot, pairs, rest);
    const double most = last_lane(wave_scan(fmax(pairs * gain2, rest), 0.0, [](double a, double b) { return fmax(a, b); }));
    float scale = power_of_two(scale_log2_for(most));
    if (lo > 0) {                                       // the page keeps earlier tokens: their scale never falls
        const float old = *scale_at;
        scale = fmaxf(old, scale);
        if (scale != old) {
            const float ratio = old / scale;
            for (int idx = lane; idx < lo * d / 8; idx += kWave) e4m3_rescale8(block + 8 * idx, block + 8 * idx, ratio);
        }
    }
    const float inv = 1.0f / scale;
    for (int idx = lane; idx < n * units; idx += kWave) {
        const int j = idx / units;
        U::turn(x, src + j * stride, idx % units, rot, cs + j * cs_stride, [&](int c, const float (&y)[W]) {
            store_unit8<W>(block, (int64_t)(lo + j) * d + c, y, inv);
        });
    }
    if (lane == 0) *scale_at = scale;
}

template <class T, int W, bool kInter, bool k8>
__global__ __launch_bounds__(kRopeThreads) void rope_append_kernel(RopeArgs a)
{
    __shared__ float2 cs[kRopeRows * kRopeMaxHalf];
    __shared__ int wsum[kRopeThreads / kWave];
    __shared__ int depth[kWave];
    __shared__ int pages[2];
    using U = Units<T, W, kInter>;
    const adaspec_rope_dims &D = a.d;
    const int tid = threadIdx.x, lane = tid & 63, wv = tid >> 6;
    const int i = blockIdx.x / a.chunks, chunk = blockIdx.x % a.chunks;
    const int d = D.head_dim, rot = D.rot_dim, half = rot / 2, Hkv = D.n_kv_heads;

    int part = 0;
    for (int j = tid; j < i; j += kRopeThreads) part += min(max(a.spec_lens[j], 0), D.max_spec_len) + 1;
    part = wave_sum(part);
    if (lane == 0) wsum[wv] = part;
    const int n = min(max(a.spec_lens[i], 0), D.max_spec_len) + 1;
    const int L = a.ctx_lens[i], first = L - n;
    // tokens [t0, t1) of the request
    const int t0 = k8 ? max(first, (first / kPageTokens + chunk) * kPageTokens) : first + chunk * kRopeRows;
    const int t1 = k8 ? min(L, (first / kPageTokens + chunk + 1) * kPageTokens) : min(L, t0 + kRopeRows);
    if (first < 0 || t0 >= t1) return;
    const int nt = t1 - t0, j0 = t0 - first;
    if (a.k && tid < 2) {
        const int at = t0 / kPageTokens + tid;
        int page = -1;
        if (at <= (t1 - 1) / kPageTokens && at < D.max_pages_per_req) page = a.block_table[(int64_t)i * D.max_pages_per_req + at];
        pages[tid] = page >= 0 && page < D.num_pages ? page : -1;
    }
    __syncthreads();
    int row0 = 0;
#pragma unroll
    for (int w = 0; w < kRopeThreads / kWave; ++w) row0 += wsum[w];
    if (row0 + n > D.total_q) return;                   // inconsistent metadata: touch nothing
    if (a.parents && half > 0) {
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
        __syncthreads();
    }
    for (int idx = tid; idx < nt * half; idx += kRopeThreads) {
        const int j = idx / half, f = idx - j * half;
        const int pos = first + (a.parents ? depth[j0 + j] : j0 + j);
        const double turns = (double)pos * (double)a.inv_freq[f] * 0.15915494309189533577;      // 1 / (2 pi)
        const float r = (float)(2.0 * (turns - rint(turns)));
        float s, c;
        sincospif(r, &s, &c);
        cs[j * half + f] = make_float2(c * D.attn_factor, s * D.attn_factor);
    }
    __syncthreads();

    const int units = U::count(rot, d);
    const int64_t row = (int64_t)row0 + j0;
    if (a.q) {
        const int per = a.k ? D.n_q_heads / Hkv : 1;    // query heads per head of the grid
        const int h0 = blockIdx.y * a.heads * per, h1 = min(h0 + a.heads * per, D.n_q_heads);
        const int work = (h1 - h0) * nt * units;
        for (int idx = tid; idx < work; idx += kRopeThreads) {
            const int u = idx % units, hj = idx / units, h = h0 + hj % (h1 - h0), j = hj / (h1 - h0);
            U::turn(a.q, (row + j) * D.q_row_stride + (int64_t)h * d, u, rot, cs + j * half, [&](int c, const float (&y)[W]) {
                store_unit<T, W>(a.q_out, (row + j) * D.q_out_row_stride + (int64_t)h * d + c, y);
            });
        }
    }
    if (!a.k) return;
    const int h0 = blockIdx.y * a.heads, h1 = min(h0 + a.heads, Hkv);
    if constexpr (k8) {
        const int page = pages[0], lo = t0 % kPageTokens;
        if (page < 0) return;
        const double gain2 = (double)D.attn_factor * (double)D.attn_factor;
        for (int task = wv; task < 2 * (h1 - h0); task += kRopeThreads / kWave) {
            const int h = h0 + task / 2;
            const int64_t at = (int64_t)page * Hkv + h, off = at * kPageTokens * d;
            if (task & 1)
                append_page8<T, 8, true>(a.v, row * D.v_row_stride + (int64_t)h * d, D.v_row_stride, d, 0, 1.0, cs, 0,
                                         static_cast<uint8_t *>(a.v_pages) + off, a.v_scales + at, lo, lo + nt, lane);
            else
                append_page8<T, W, kInter>(a.k, row * D.k_row_stride + (int64_t)h * d, D.k_row_stride, d, rot, gain2, cs, half,
                                           static_cast<uint8_t *>(a.k_pages) + off, a.k_scales + at, lo, lo + nt, lane);
        }
    } else {
        const int nh = h1 - h0, work = nh * nt * units;
        for (int idx = tid; idx < work; idx += kRopeThreads) {
            const int u = idx % units, hj = idx / units, h = h0 + hj % nh, j = hj / nh, t = t0 + j;
            const int page = pages[t / kPageTokens - t0 / kPageTokens];
            if (page < 0) continue;
            const int64_t dst = (((int64_t)page * Hkv + h) * kPageTokens + t % kPageTokens) * d;
            U::turn(a.k, (row + j) * D.k_row_stride + (int64_t)h * d, u, rot, cs + j * half, [&](int c, const float (&y)[W]) {
                store_unit<T, W>(a.k_pages, dst + c, y);
            });
        }
        // values as they are, 16 bytes at a time
        constexpr int kSize = sizeof(typename T::storage);
        const int vecs = d * kSize / 16, copies = nh * nt * vecs;
        for (int idx = tid; idx < copies; idx += kRopeThreads) {
            const int u = idx % vecs, hj = idx / vecs, h = h0 + hj % nh, j = hj / nh, t = t0 + j;
            const int page = pages[t / kPageTokens - t0 / kPageTokens];
            if (page < 0) continue;
            const int64_t dst = (((int64_t)page * Hkv + h) * kPageTokens + t % kPageTokens) * d;
            reinterpret_cast<uint4 *>(static_cast<char *>(a.v_pages) + dst * kSize)[u] =
                reinterpret_cast<const uint4 *>(static_cast<const char *>(a.v) + ((row + j) * D.v_row_stride + (int64_t)h * d) * kSize)[u];
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
    a.heads = heads;
    const dim3 grid((unsigned)((int64_t)d.batch * a.chunks), ceil_div(heads, a.heads));
    auto launch = [&](auto tag) {
        using T = decltype(tag);
        auto with = [&](auto w, auto inter) {
            constexpr int W = decltype(w)::value;
            constexpr bool kInter = decltype(inter)::value;
            if (fp8) hipLaunchKernelGGL((rope_append_kernel<T, W, kInter, true>), grid, dim3(kRopeThreads), 0, stream, a);
            else hipLaunchKernelGGL((rope_append_kernel<T, W, kInter, false>), grid, dim3(kRopeThreads), 0, stream, a);
        };
        if (d.interleaved || a.d.rot_dim == 0) {
            if (a.d.rot_dim % 8 == 0) with(std::integral_constant<int, 8>{}, std::true_type{});
            else with(std::integral_constant<int, 2>{}, std::true_type{});
        } else {
            if (a.d.rot_dim % 16 == 0) with(std::integral_constant<int, 8>{}, std::false_type{});
            else with(std::integral_constant<int, 1>{}, std::false_type{});
        }
    };
    if (d.dtype == ADASPEC_F32) launch(F32{});
    else if (d.dtype == ADASPEC_F16) launch(F16{});
    else launch(BF16{});
    return hipGetLastError();
}

}  // namespace adaspec
