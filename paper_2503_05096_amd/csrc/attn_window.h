// Windowed verification attention: what its kernels share.
//
// Row j of request i, at pos = L - n + j, sees token t iff  t <= pos  and  (t > pos - window  or  t < sinks).  The tokens that
// some row of a unit (request, kv head, group of rows) sees lie in two runs of pages: the sinks' and the window's.  The
// kernels walk the pages of both as one list: entry v is page v of the request for v < first, page v + skip behind that.
// Pages between the runs are never looked up: their places in the block table may hold anything.
#pragma once
#include "adaspec_internal.h"
#include "device_utils.h"

namespace adaspec {

struct WindowDims {                 // what every kernel needs to find its unit
    const int32_t *block_table, *ctx_lens, *spec_lens;
    int batch, total_q, max_spec_len, max_pages, Hq, Hkv, window, sinks, groups, rows_per_group;      // (16 max_pages is at most 2^30)
};

struct WindowUnit {                 // wave-uniform
    int i, rg, gkv, L, n, rows, r0, first_pos, window, sinks;
    int first, skip, pages;         // pages of the sinks' run, pages left out behind it, entries of the list
    int64_t qrow0, bt_off;
    // page of the request that entry v of the list is; its first token is 16 times that
    __device__ __forceinline__ int page_of(int v) const { return v < first ? v : v + skip; }
};

// Rows of the requests before request i, added up by the lanes of a whole wavefront.  Two steps, so that the loads are under way
// while the unit's first pages are looked up: nothing but Q and the results needs the sum.
struct RowsBefore {
    static constexpr int kAhead = 4;
    int k[kAhead];
    __device__ __forceinline__ RowsBefore(const WindowDims &d, int i, int lane)
    {
#pragma unroll
        for (int c = 0; c < kAhead; ++c) k[c] = c * kWave + lane < i ? d.spec_lens[c * kWave + lane] : -1;
    }
    __device__ __forceinline__ int sum(const WindowDims &d, int i, int lane) const
    {
        int part = 0;
#pragma unroll
        for (int c = 0; c < kAhead; ++c) part += c * kWave + lane < i ? min(max(k[c], 0), d.max_spec_len) + 1 : 0;
        for (int j = kAhead * kWave + lane; j < i; j += kWave) part += min(max(d.spec_lens[j], 0), d.max_spec_len) + 1;
        return wave_sum(part);
    }
};

// Unit (i, rg, gkv) but for its first row; false: the request has fewer rows.
__device__ __forceinline__ bool window_unit(WindowUnit &u, const WindowDims &d, int i, int rg, int gkv)
{
    u.i = i; u.rg = rg; u.gkv = gkv;
    u.bt_off = (int64_t)i * d.max_pages;
    const int G = d.Hq / d.Hkv;
    u.L = min(max(d.ctx_lens[i], 1), d.max_pages * 16);
    u.n = min(max(d.spec_lens[i], 0), d.max_spec_len) + 1;
    u.rows = u.n * G;
    u.r0 = rg * d.rows_per_group;
    u.window = d.window; u.sinks = d.sinks;
    u.first_pos = u.L - u.n;
    const int j0 = u.r0 / G, j1 = min(u.r0 + d.rows_per_group, u.rows) - 1;
    const int low = max(u.first_pos + j0 - u.window + 1, 0) >> 4;                   // page of the oldest token in a window
    const int end = max(u.first_pos + j1 / G + 16, 0) >> 4;                          // behind the page of the newest row
    u.first = min((u.sinks + 15) >> 4, low);
    u.skip = low - u.first;
    u.pages = max(end - u.skip, 0);
    return u.r0 < u.rows;
}

// Request and row group of workgroup x of batch * groups.  Workgroups go round the eight XCDs in turn: the groups of a request,
// which read the same K and V, are eight apart, so that they run on one XCD at about the same time and share its L2.
__device__ __forceinline__ void window_place(const WindowDims &d, int x, int &i, int &rg)
{
    if (d.groups == 1) { i = x; rg = 0; return; }
    const int first = x / (8 * d.groups) * 8, rest = x - first * d.groups, n = min(8, d.batch - first);
    rg = rest / n;
    i = first + rest - rg * n;
}

// whether the row at position `pos` sees token t
__device__ __forceinline__ bool window_sees(const WindowUnit &u, int pos, int t)
{
    return t <= pos && (pos - t < u.window || t < u.sinks);
}

hipError_t launch_attn_window_mfma(const WindowArgs &a, const WindowDims &w);      // 16 bits
hipError_t launch_attn_window_f32(const WindowArgs &a, const WindowDims &w);

}  // namespace adaspec
