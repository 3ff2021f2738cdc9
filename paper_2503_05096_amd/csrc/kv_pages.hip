// The pages of the cache: which request holds which (remap, compact: integers only, on the block table and a count of
// holders per page), and the copies that follow from it (copy_pages: the bytes).
//
// Every result is independent of the order in which workgroups run: counts change by integer atomics, free pages are handed
// out by their rank in ascending order, requests by theirs.
//
// The id calls move little (remap of 128 requests 0.8 MB, compaction of 262144 pages 5.2 MB): launches and chains of dependent
// accesses bound them, so they are few launches with everything in flight that can be.  Whole calls from Python: remap of
// 128 requests of up to 8192 tokens 13-16 us (four kernels of 3.0, 4.0, 2.8 and 4.8), of 16 into 256 forks 10.7 (5.8 and 5.4),
// compaction of 2048 pages 5.3-5.9 us (one of 5.3), of 262144 pages 9.5-9.8 us (2.4 and 8.5).  (Kernels under the profiler, in a busy
// stream: about 3 us of each are its boundary, and they overlap a little.)
#include "adaspec_internal.h"
#include "device_utils.h"

namespace adaspec {

constexpr int kPagesThreads = 256;
constexpr int kPerThread = 4;
constexpr int kChunk = kPagesThreads * kPerThread;          // pages, or table entries, of one workgroup

// four counts from p on (behind the last page: `past`)
__device__ __forceinline__ int4 four(const int32_t *__restrict__ a, int p, int n, int past)
{
    int4 v;
    if (p + 4 <= n) {
        __builtin_memcpy(&v, a + p, sizeof v);              // (4-byte aligned)
    } else {
        v.x = p < n ? a[p] : past;
        v.y = p + 1 < n ? a[p + 1] : past;
        v.z = p + 2 < n ? a[p + 2] : past;
        v.w = past;
    }
    return v;
}

// sum over the workgroup, in all threads
__device__ __forceinline__ int block_sum(int v, int *s /* [kPagesThreads / kWave] */)
{
    v = wave_sum(v);
    __syncthreads();
    if ((threadIdx.x & 63) == 0) s[threadIdx.x >> 6] = v;
    __syncthreads();
    int t = 0;
#pragma unroll
    for (int w = 0; w < kPagesThreads / kWave; ++w) t += s[w];
    return t;
}
// exclusive scan over the workgroup; *total in all threads
__device__ __forceinline__ int block_scan(int v, int *s, int *total)
{
    const int inc = wave_scan_incl_dpp(v), wv = threadIdx.x >> 6;
    __syncthreads();
    if ((threadIdx.x & 63) == 63) s[wv] = inc;
    __syncthreads();
    int pre = 0, t = 0;
#pragma unroll
    for (int w = 0; w < kPagesThreads / kWave; ++w) {
        pre += w < wv ? s[w] : 0;
        t += s[w];
    }
    *total = t;
    return pre + inc - v;
}

// ---- remap ---------------------------------------------------------------------------------------------------------

// What a row keeps of an old row of `len` tokens: entries of its pages that are not behind the window.
struct Kept {
    int pages, first, low;      // pages of len tokens; those of the sinks; first one that the window reaches
    __device__ __forceinline__ Kept(int len, const adaspec_pages_dims &d)
    {
        pages = ceil_div(len, d.page_size);
        first = d.window > 0 ? ceil_div(d.sinks, d.page_size) : pages;
        low = d.window > 0 ? max(len - d.window + 1, 0) / d.page_size : 0;
    }
    __device__ __forceinline__ bool keeps(int j) const { return j < pages && (j < first || j >= low); }
};

// tokens of old row s (0 for a row that starts empty), cut to what the row can hold
__device__ __forceinline__ int len_of(const RemapArgs &a, int s)
{
    return s >= 0 ? min(max(a.lens[s], 0), a.dims.max_pages_per_req * a.dims.page_size) : 0;
}
__device__ __forceinline__ int source_of(const RemapArgs &a, int i)
{
    const int s = a.sources[i];
    return s >= 0 && s < a.dims.old_batch ? s : -1;
}

constexpr int kRowPart = 2048;              // entries of a row that one workgroup takes

// The counts, and nobody about to write into a page.
__global__ __launch_bounds__(kPagesThreads) void remap_start_kernel(RemapArgs a)
{
    const int n = a.dims.num_pages, p = blockIdx.x * kChunk + kPerThread * threadIdx.x;
    int4 v = make_int4(0, 0, 0, 0);
    if (a.out_refs != a.page_refs) v = four(a.page_refs, p, n, 0);
    const int refs[kPerThread] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int e = 0; e < kPerThread; ++e) {
        if (p + e >= n) break;
        if (a.out_refs != a.page_refs) a.out_refs[p + e] = refs[e];
        a.writers[p + e] = make_int2(0, -1);
    }
}

// Rows 0 .. old_batch - 1: every entry of the old row is released, and held again by each new row that keeps it; what is left of
// both goes into the counts.  Rows behind: the new row, with what it keeps; whether it is about to write into a page that
// holds tokens, and how many rows are and which is the last.
__global__ __launch_bounds__(kPagesThreads) void remap_rows_kernel(RemapArgs a)
{
    __shared__ int s_sum[kPagesThreads / kWave];
    const adaspec_pages_dims &d = a.dims;
    const int row = blockIdx.y, at = blockIdx.x * kRowPart, end = min(at + kRowPart, d.max_pages_per_req);
    if (row < d.old_batch) {
        int c = 0;
        for (int i = threadIdx.x; i < d.batch; i += kPagesThreads) c += a.sources[i] == row;
        c = block_sum(c, s_sum);
        const Kept kept(len_of(a, row), d);
        const int32_t *t = a.block_table + (int64_t)row * d.max_pages_per_req;
        for (int j = at + threadIdx.x; j < end; j += kPagesThreads) {
            const int p = t[j], delta = (kept.keeps(j) ? c : 0) - 1;
            if (p >= 0 && p < d.num_pages && delta != 0) atomicAdd(a.out_refs + p, delta);
        }
    } else {
        const int i = row - d.old_batch, s = source_of(a, i), len = len_of(a, s);
        const bool writes = len % d.page_size != 0 && a.new_lens[i] > len;
        const Kept kept(len, d);
        const int32_t *t = a.block_table + (int64_t)max(s, 0) * d.max_pages_per_req;
        int32_t *o = a.out_table + (int64_t)i * d.max_pages_per_req;
        if (at == 0 && threadIdx.x == 0 && !writes) a.rows[i] = make_int2(len, -1);
        for (int j = at + threadIdx.x; j < end; j += kPagesThreads) {
            int p = s >= 0 && kept.keeps(j) ? t[j] : -1;
            if (p >= d.num_pages) p = -1;
            o[j] = max(p, -1);
            if (writes && j == len / d.page_size) {
                a.rows[i] = make_int2(len, max(p, -1));
                if (p >= 0) {
                    atomicAdd(&a.writers[p].x, 1);
                    atomicMax(&a.writers[p].y, i);
                }
            }
        }
    }
}

// Workgroups 0 .. chunks - 1: free pages of a chunk.  Those behind, for 256 rows each: what a row wants, as a record of
// (its first want's number among these rows', the entry that it is for, the page to copy into it or -1, how many).
__global__ __launch_bounds__(kPagesThreads) void remap_count_kernel(RemapArgs a)
{
    __shared__ int s_sum[kPagesThreads / kWave];
    const adaspec_pages_dims &d = a.dims;
    const int tid = threadIdx.x;
    if ((int)blockIdx.x < a.chunks) {
        const int4 r = four(a.out_refs, blockIdx.x * kChunk + kPerThread * tid, d.num_pages, 1);
        const int n = block_sum((r.x == 0) + (r.y == 0) + (r.z == 0) + (r.w == 0), s_sum);
        if (tid == 0) a.chunk_free[blockIdx.x] = n;
        return;
    }
    const int tile = blockIdx.x - a.chunks, i = tile * kPagesThreads + tid, P = d.page_size;
    int want = 0, start = 0, from = -1;
    if (i < d.batch) {
        const int2 row = a.rows[i];
        const int len = row.x, p = row.y;
        if (p >= 0) {           // shared, unless this row is the last of those who hold it, all of which are about to write
            const int refs = a.out_refs[p];
            const int2 w = a.writers[p];
            if (refs > 1 && !(w.x == refs && w.y == i)) from = p;
        }
        start = from >= 0 ? len / P : ceil_div(len, P);
        want = max(ceil_div(min(max(a.new_lens[i], 0), d.max_pages_per_req * P), P) - start, 0);
        a.copy_src[i] = -1;
        a.copy_dst[i] = -1;
    }
    int total;
    const int first = block_scan(want, s_sum, &total);
    if (i < d.batch) a.want[i] = make_int4(first, start, from, want);
    if (tid == 0) a.tile_wants[tile] = total;
}

// Everything up to here in one launch, where the old table and both batches are small: a workgroup per 1024 pages goes through the
// whole old table and keeps the counts of its own pages in LDS, so that nobody has to wait for anybody.  It also decides what
// those rows want that are about to write into one of its pages (the first workgroup: into none that holds tokens).  The
// workgroups behind write a new row each.
//
// Up to 512 of these workgroups, two per compute unit, run at once, and the table's length decides; beyond that each further
// round of them reads the table again, and its length times the number of workgroups does.  Rows count a little: every workgroup
// looks up where each of them writes.  The look-ups of one workgroup are shared out by the table's places: short rows in a wide
// table, all in one workgroup's pages, crowd in few threads (64 rows of 8 pages in 512 entries, a pool of 1024: 17.8/14.1).
// Whole calls (us), this way / in three launches, all rows in use as far as the pool goes:
//   table entries                   2048       12288      24576      36864      49152      65536
//     64 rows, pool of   65536   8.8/14.5   8.8/14.2   9.2/14.1  10.5/14.8  10.8/14.9  12.7/14.6
//     64 rows, pool of  524288   8.8/14.5   9.7/14.3  10.0/14.4  12.0/14.4  12.9/14.6  15.0/14.5
//     64 rows, pool of 1048576  11.1/16.2  13.4/15.8  15.3/16.0  18.8/16.1  20.8/16.1  24.5/16.5
//     64 rows, pool of 2097152  17.3/21.6  21.8/22.3  25.1/22.2  31.6/22.1  35.4/22.5  42.5/23.1
//     64 rows, pool of 8388608  67.8/69.6  85.5/69.7  95.9/69.7   117/70.2   131/69.7   158/70.2
//   1024 rows, pool of   65536   9.2/13.9   9.4/14.0  10.4/14.0  11.6/14.0  12.5/14.4  13.6/14.7
//   1024 rows, pool of  524288  11.0/15.2  12.2/14.7  13.6/15.3  15.7/15.1  16.8/14.9  18.4/15.1
//   1024 rows, pool of 1048576  14.7/18.6  17.7/18.5  20.5/18.6  24.4/18.7  26.8/18.6  29.9/18.5
constexpr int kSmallRows = 1024;
constexpr int64_t kSmallEntries = 49152, kSmallReads = 26 << 20;
static bool remap_is_small(const adaspec_pages_dims &d, int chunks)
{
    const int64_t entries = (int64_t)d.old_batch * d.max_pages_per_req;
    return d.old_batch <= kSmallRows && d.batch <= kSmallRows && entries <= kSmallEntries && chunks * entries + 8192 * (int64_t)d.batch <= kSmallReads;
}
constexpr int kScan = 2;                    // loads of four entries that a thread has under way
static_assert(kSmallRows == kChunk, "a thread per row");
__global__ __launch_bounds__(kChunk) void remap_small_kernel(RemapArgs a)
{
    __shared__ int s_refs[kChunk], s_writers[kChunk], s_last[kChunk], s_sum[kChunk / kWave];
    __shared__ int s_children[kSmallRows], s_pages[kSmallRows], s_low[kSmallRows];
    const adaspec_pages_dims &d = a.dims;
    const int tid = threadIdx.x, width = d.max_pages_per_req, P = d.page_size;
    if ((int)blockIdx.x >= a.chunks) {
        const int i = blockIdx.x - a.chunks, s = source_of(a, i);
        const Kept kept(len_of(a, s), d);
        const int32_t *t = a.block_table + (int64_t)max(s, 0) * width;
        int32_t *o = a.out_table + (int64_t)i * width;
        for (int j = tid; j < width; j += kChunk) {
            const int p = s >= 0 && kept.keeps(j) ? t[j] : -1;
            o[j] = p < d.num_pages ? max(p, -1) : -1;
        }
        if (tid == 0) {
            a.copy_src[i] = -1;
            a.copy_dst[i] = -1;
        }
        return;
    }
    const int p0 = blockIdx.x * kChunk, p = p0 + tid;
    const int old = p < d.num_pages ? a.page_refs[p] : 1;
    // new row tid: the page that it is about to write into
    int len = 0, grown = 0, part = -1;
    const int src = tid < d.batch ? source_of(a, tid) : -1;
    if (tid < d.batch) grown = a.new_lens[tid];
    s_refs[tid] = 0; s_writers[tid] = 0; s_last[tid] = -1; s_children[tid] = 0;
    __syncthreads();
    if (src >= 0) atomicAdd(&s_children[src], 1);
    if (tid < d.old_batch) {
        const Kept kept(len_of(a, tid), d);
        s_pages[tid] = kept.pages;
        s_low[tid] = kept.low;
    }
    if (src >= 0) {
        len = len_of(a, src);
        if (len % P != 0 && grown > len) part = a.block_table[(int64_t)src * width + len / P];
        if (part >= d.num_pages) part = -1;
    }
    __syncthreads();
    const int first = d.window > 0 ? ceil_div(d.sinks, P) : 0;      // (entries of the sinks; without a window s_low is 0)
    const int entries = d.old_batch * width;
    auto count = [&](int e, int q) {                                // entry e of the table, which holds page q of this chunk
        const int row = e / width, j = e - row * width;
        const bool keeps = j < s_pages[row] && (j < first || j >= s_low[row]);
        const int delta = (keeps ? s_children[row] : 0) - 1;
        if (delta != 0) atomicAdd(&s_refs[q - p0], delta);
    };
    // About one entry per thread holds one of the chunk's pages: they are put aside, and looked at by all threads together.
    const unsigned mine = min(kChunk, d.num_pages - p0);
    int aside[4] = {-1, -1, -1, -1}, held[4] = {0, 0, 0, 0};
    for (int e0 = 4 * tid; e0 < entries; e0 += kScan * 4 * kChunk) {
        int4 q[kScan];
#pragma unroll
        for (int k = 0; k < kScan; ++k) q[k] = four(a.block_table, e0 + k * 4 * kChunk, entries, -1);
#pragma unroll
        for (int k = 0; k < kScan; ++k) {
            const int v[4] = {q[k].x, q[k].y, q[k].z, q[k].w};
#pragma unroll
            for (int c = 0; c < 4; ++c) {
                if ((unsigned)(v[c] - p0) >= mine) continue;
                if (aside[3] >= 0) count(aside[3], held[3]);
#pragma unroll
                for (int i = 3; i > 0; --i) { aside[i] = aside[i - 1]; held[i] = held[i - 1]; }
                aside[0] = e0 + k * 4 * kChunk + c;
                held[0] = v[c];
            }
        }
    }
#pragma unroll
    for (int i = 0; i < 4; ++i)
        if (aside[i] >= 0) count(aside[i], held[i]);
    const bool here = part >= p0 && part < p0 + kChunk;
    if (here) {
        atomicAdd(&s_writers[part - p0], 1);
        atomicMax(&s_last[part - p0], tid);
    }
    __syncthreads();
    const int now = old + s_refs[tid];
    if (p < d.num_pages) a.out_refs[p] = now;
    const unsigned long long free = __ballot(p < d.num_pages && now == 0);
    if ((tid & 63) == 0) s_sum[tid >> 6] = __popcll(free);
    s_refs[tid] = now;                                              // (every thread reads its own before)
    __syncthreads();
    if (tid == 0) {
        int n = 0;
#pragma unroll
        for (int w = 0; w < kChunk / kWave; ++w) n += s_sum[w];
        a.chunk_free[blockIdx.x] = n;
    }
    if (tid < d.batch && (here || (part < 0 && blockIdx.x == 0))) {
        int from = -1;
        if (here) {             // shared, unless this row is the last of those who hold it, all of which are about to write
            const int q = part - p0, refs = s_refs[q];
            if (refs > 1 && !(s_writers[q] == refs && s_last[q] == tid)) from = part;
        }
        const int start = from >= 0 ? len / P : ceil_div(len, P);
        a.want[tid] = make_int4(0, start, from, max(ceil_div(min(max(grown, 0), width * P), P) - start, 0));
    }
}

// Free page number f of the pool goes to want number f.  kFew: at most kFewRows rows, whose wants every workgroup adds up itself.
constexpr int kFewRows = 2048;
template <bool kFew>
__global__ __launch_bounds__(kPagesThreads) void remap_assign_kernel(RemapArgs a)
{
    constexpr int kRows = kFew ? kFewRows / kPagesThreads : 1;
    __shared__ int s_sum[kPagesThreads / kWave];
    __shared__ int s_first[kFew ? kFewRows : kPagesThreads];        // where the wants of every row, or of every 256 rows, begin
    const adaspec_pages_dims &d = a.dims;
    const int tid = threadIdx.x, p0 = blockIdx.x * kChunk + kPerThread * tid;
    const int4 r = four(a.out_refs, p0, d.num_pages, 1);
    const bool free[kPerThread] = {r.x == 0, r.y == 0, r.z == 0, r.w == 0};
    int n[kRows], mine = 0;
#pragma unroll
    for (int k = 0; k < kRows; ++k) {
        if constexpr (kFew) n[k] = tid * kRows + k < d.batch ? a.want[tid * kRows + k].w : 0;
        else n[k] = tid < a.tiles ? a.tile_wants[tid] : 0;          // (at most 256 tiles: 65535 rows)
        mine += n[k];
    }
    int before = 0, all = 0;
    for (int c = tid; c < a.chunks; c += kPagesThreads) {
        const int m = a.chunk_free[c];
        before += c < (int)blockIdx.x ? m : 0;
        all += m;
    }
    int wants, here;
    int at = block_scan(mine, s_sum, &wants);
#pragma unroll
    for (int k = 0; k < kRows; ++k) {
        s_first[tid * kRows + k] = at;
        at += n[k];
    }
    before = block_sum(before, s_sum);
    if (blockIdx.x == 0) {
        all = block_sum(all, s_sum);
        if (tid == 0) {
            a.status[0] = max(all - wants, 0);
            a.status[1] = max(wants - all, 0);
        }
    }
    // (wants that no page is left for: their entries are -1 already, a shared page stays shared)
    if (before >= wants) return;
    int f[kPerThread];
    f[0] = before + block_scan(free[0] + free[1] + free[2] + free[3], s_sum, &here);
#pragma unroll
    for (int e = 1; e < kPerThread; ++e) f[e] = f[e - 1] + free[e - 1];
    // The row, or the rows and then the row, whose wants f is among: the last one whose wants begin at or before it.  All four
    // pages' look-ups step by step together.
    bool takes[kPerThread], any = false;
    int lo[kPerThread] = {}, nth[kPerThread];
#pragma unroll
    for (int e = 0; e < kPerThread; ++e) any |= takes[e] = free[e] && f[e] < wants;
    if (!any) return;
    const int size = kFew ? d.batch : a.tiles;
    for (int step = 1 << (31 - __builtin_clz(size)); step > 0; step >>= 1) {
#pragma unroll
        for (int e = 0; e < kPerThread; ++e) {
            const int at = min(lo[e] + step, size - 1);
            lo[e] = s_first[at] <= f[e] ? at : lo[e];
        }
    }
    int4 w[kPerThread];
#pragma unroll
    for (int e = 0; e < kPerThread; ++e) {
        nth[e] = f[e] - s_first[lo[e]];
        if constexpr (!kFew) {
            int hi = min((lo[e] + 1) * kPagesThreads, d.batch);
            lo[e] *= kPagesThreads;
            while (takes[e] && hi - lo[e] > 1) {
                const int mid = (lo[e] + hi) >> 1;
                if (a.want[mid].x <= nth[e]) lo[e] = mid;
                else hi = mid;
            }
        }
        w[e] = a.want[lo[e]];
        if constexpr (!kFew) nth[e] -= w[e].x;
    }
#pragma unroll
    for (int e = 0; e < kPerThread; ++e) {
        if (!takes[e]) continue;
        const int p = p0 + e;
        a.out_refs[p] = 1;
        a.out_table[(int64_t)lo[e] * d.max_pages_per_req + w[e].y + nth[e]] = p;
        if (w[e].z >= 0 && nth[e] == 0) {
            atomicAdd(a.out_refs + w[e].z, -1);
            a.copy_src[lo[e]] = w[e].z;
            a.copy_dst[lo[e]] = p;
        }
    }
}

size_t remap_workspace(const adaspec_pages_dims &d, RemapArgs *a, char *ws)
{
    const int chunks = ceil_div(d.num_pages, kChunk), tiles = ceil_div(d.batch, kPagesThreads);
    size_t off = 0;
    auto take = [&](size_t n) {
        int32_t *p = reinterpret_cast<int32_t *>(ws + off);
        off = align_up(off + n * 4, 256);
        return p;
    };
    int32_t *free = take(chunks), *wants = take(tiles), *want = take(4 * (size_t)d.batch), *rows = take(2 * (size_t)d.batch);
    int32_t *writers = take(2 * (size_t)d.num_pages);
    if (a) {
        a->chunks = chunks; a->tiles = tiles;
        a->chunk_free = free; a->tile_wants = wants;
        a->want = reinterpret_cast<int4 *>(want); a->rows = reinterpret_cast<int2 *>(rows); a->writers = reinterpret_cast<int2 *>(writers);
    }
    return off;
}

hipError_t launch_kv_remap(const RemapArgs &a, hipStream_t stream)
{
    const adaspec_pages_dims &d = a.dims;
    if (remap_is_small(d, a.chunks)) {
        hipLaunchKernelGGL(remap_small_kernel, dim3(a.chunks + d.batch), dim3(kChunk), 0, stream, a);
    } else {
        hipLaunchKernelGGL(remap_start_kernel, dim3(a.chunks), dim3(kPagesThreads), 0, stream, a);
        if (d.old_batch + d.batch > 0)
            hipLaunchKernelGGL(remap_rows_kernel, dim3(ceil_div(d.max_pages_per_req, kRowPart), d.old_batch + d.batch), dim3(kPagesThreads), 0,
                               stream, a);
        hipLaunchKernelGGL(remap_count_kernel, dim3(a.chunks + a.tiles), dim3(kPagesThreads), 0, stream, a);
    }
    if (d.batch <= kFewRows) hipLaunchKernelGGL(remap_assign_kernel<true>, dim3(a.chunks), dim3(kPagesThreads), 0, stream, a);
    else hipLaunchKernelGGL(remap_assign_kernel<false>, dim3(a.chunks), dim3(kPagesThreads), 0, stream, a);
    return hipGetLastError();
}

// ---- compact -------------------------------------------------------------------------------------------------------
// N pages are used (counts above 0).  The m-th used page at or behind N moves to the m-th free page below N, for the first
// `max_moves` of them.

//
// Which pages are used is one bit per page, in words of 32 with the number of used pages before them; everything else follows
// from the number of used pages below a page and from where the m-th free page is, which are two or three look-ups each.

// A thread's four bits and those of its seven neighbours: within four lanes, then the other four by mirroring the eight
__device__ __forceinline__ uint32_t word_of(const int4 &r)
{
    uint32_t w = ((r.x > 0) | (r.y > 0) << 1 | (r.z > 0) << 2 | (r.w > 0) << 3) << (4 * (threadIdx.x & 7));
    w |= dpp_move<0xb1, 0xf>(0, w);
    w |= dpp_move<0x4e, 0xf>(0, w);
    w |= dpp_move<0x141, 0xf>(0, w);
    return w;
}

// Words of a wavefront's 256 pages, counted from their beginning, and how many of these are used.
constexpr int kGrain = kWave * kPerThread;
__global__ __launch_bounds__(kPagesThreads) void compact_words_kernel(CompactArgs a)
{
    const int tid = threadIdx.x, lane = tid & 63, grain = blockIdx.x * (kChunk / kGrain) + (tid >> 6);
    const uint32_t w = word_of(four(a.page_refs, blockIdx.x * kChunk + kPerThread * tid, a.dims.num_pages, 0));
    const int n = (lane & 7) == 0 ? __popc(w) : 0, upto = wave_scan_incl_dpp(n);
    if ((lane & 7) == 0) a.words[grain * (kGrain / 32) + (lane >> 3)] = make_int2((int)w, upto - n);
    if (lane == 63) a.grain_used[grain] = upto;
}

// Workgroups 0 .. chunks - 1: counts, map and moves of a chunk of pages; those behind: the table.  Every count is read and
// written by one thread each, so that the new counts may lie over the old ones (not with kSelf).
// kSelf: small pools, whose words every workgroup works out itself, from 16 loads of a thread: one launch (whole calls 5.3 us for
// 2048 pages, 6.8 for 16384) instead of two (8.0, 9.2).  The new counts must not lie over the old ones then.
constexpr int kSelfPages = 16384;
template <bool kSelf>
__global__ __launch_bounds__(kPagesThreads) void compact_write_kernel(CompactArgs a)
{
    extern __shared__ int s_base[];                                 // used pages before every 256; behind the last: all
    __shared__ int2 s_words[kSelf ? kSelfPages / 32 : 1];
    __shared__ int s_sum[kPagesThreads / kWave];
    const adaspec_pages_dims &d = a.dims;
    const int tid = threadIdx.x, grains = a.chunks * (kChunk / kGrain);
    // the workgroup's counts, or its first entries of the table: under way while the bases are worked out
    const bool on_counts = (int)blockIdx.x < a.chunks;
    const int64_t entries = (int64_t)d.old_batch * d.max_pages_per_req;
    int got[kPerThread];
    auto table_entries = [&](int64_t e0) {
#pragma unroll
        for (int k = 0; k < kPerThread; ++k) got[k] = e0 + k * kPagesThreads + tid < entries ? a.block_table[e0 + k * kPagesThreads + tid] : -1;
    };
    if (on_counts) {
#pragma unroll
        for (int k = 0; k < kPerThread; ++k) {
            const int p = blockIdx.x * kChunk + k * kPagesThreads + tid;
            got[k] = p < d.num_pages ? a.page_refs[p] : 0;
        }
    } else {
        table_entries((int64_t)(blockIdx.x - a.chunks) * kChunk);
    }
    // the words of those pages, which the bases are not needed for either (kSelf: there are none yet)
    int2 own[kPerThread];
    auto page_at = [&](int k) { return on_counts ? (int)blockIdx.x * kChunk + k * kPagesThreads + tid : got[k]; };
    auto own_words = [&]() {
#pragma unroll
        for (int k = 0; k < kPerThread; ++k) {
            const int p = page_at(k), w = p >= 0 && p < d.num_pages ? p / 32 : 0;
            if constexpr (kSelf) own[k] = s_words[w];
            else own[k] = a.words[w];
        }
    };
    if constexpr (!kSelf) own_words();
    if constexpr (kSelf) {
        constexpr int kMost = kSelfPages / kChunk;
        int4 r[kMost];
#pragma unroll
        for (int c = 0; c < kMost; ++c) r[c] = c < a.chunks ? four(a.page_refs, c * kChunk + kPerThread * tid, d.num_pages, 0) : make_int4(0, 0, 0, 0);
#pragma unroll
        for (int c = 0; c < kMost; ++c) {
            const uint32_t w = c < a.chunks ? word_of(r[c]) : 0;
            if ((tid & 7) == 0) s_words[c * (kChunk / 32) + (tid >> 3)].x = (int)w;
        }
        __syncthreads();
        const int w0 = s_words[2 * tid].x, w1 = s_words[2 * tid + 1].x;
        int total;
        const int before = block_scan(__popc(w0) + __popc(w1), s_sum, &total);
        s_words[2 * tid].y = before;                                // (from the pool's beginning: no bases of chunks)
        s_words[2 * tid + 1].y = before + __popc(w0);
        if (tid <= grains) s_base[tid] = tid < grains ? 0 : total;
        __syncthreads();
    } else {
        int base = 0;
        for (int c0 = 0; c0 < grains; c0 += 4 * kPagesThreads) {
            const int c = c0 + 4 * tid;
            const int4 n = four(a.grain_used, c, grains, 0);
            int total;
            const int at = base + block_scan((n.x + n.y) + (n.z + n.w), s_sum, &total);
            if (c < grains) {                                       // (a multiple of four)
                s_base[c] = at;
                s_base[c + 1] = at + n.x;
                s_base[c + 2] = at + n.x + n.y;
                s_base[c + 3] = at + n.x + n.y + n.z;
            }
            base += total;
        }
        if (tid == 0) s_base[grains] = base;
        __syncthreads();
    }
    const int N = s_base[grains];
    auto word = [&](int w) -> int2 {
        if constexpr (kSelf) return s_words[w];
        else return a.words[w];
    };
    auto used_before = [&](int p, int2 w) { return s_base[p / kGrain] + w.y + __popc((uint32_t)w.x & ((1u << (p & 31)) - 1u)); };
    int low = N;                                                    // used pages below N
    if (N < a.chunks * kChunk) low = used_before(N, word(N / 32));
    const int moves = N - low;
    // to[k] = the m[k]-th free page, for m[k] < moves (m[k] < 0: as it is); the four look-ups step by step together
    auto free_pages = [&](const int (&of)[kPerThread], int (&to)[kPerThread]) {
        bool any = false;
#pragma unroll
        for (int k = 0; k < kPerThread; ++k) any |= of[k] >= 0;
        if (__ballot(any) == 0) return;
        int m[kPerThread], lo[kPerThread];
#pragma unroll
        for (int k = 0; k < kPerThread; ++k) { m[k] = max(of[k], 0); lo[k] = 0; }
        const int size = kSelf ? a.chunks * (kChunk / 32) : grains;
        for (int step = 1 << (31 - __builtin_clz(size)); step > 0; step >>= 1) {
#pragma unroll
            for (int k = 0; k < kPerThread; ++k) {
                const int at = min(lo[k] + step, size - 1);
                int before;                                         // free pages in front of word, or grain, `at`
                if constexpr (kSelf) before = 32 * at - s_words[at].y;
                else before = at * kGrain - s_base[at];
                lo[k] = before <= m[k] ? at : lo[k];
            }
        }
#pragma unroll
        for (int k = 0; k < kPerThread; ++k) {
            if constexpr (kSelf) {
                m[k] -= 32 * lo[k] - s_words[lo[k]].y;
            } else {
                m[k] -= lo[k] * kGrain - s_base[lo[k]];
                lo[k] *= kGrain / 32;
            }
        }
        uint32_t mask[kPerThread];
        if constexpr (kSelf) {
#pragma unroll
            for (int k = 0; k < kPerThread; ++k) mask[k] = (uint32_t)s_words[lo[k]].x;
        } else {                                                    // which of the grain's eight words
            int4 w[kPerThread][4];
#pragma unroll
            for (int k = 0; k < kPerThread; ++k)
#pragma unroll
                for (int i = 0; i < 4; ++i) w[k][i] = reinterpret_cast<const int4 *>(a.words + lo[k])[i];
#pragma unroll
            for (int k = 0; k < kPerThread; ++k) {
                int at = 0, before = 0;
                mask[k] = (uint32_t)w[k][0].x;
#pragma unroll
                for (int i = 1; i < 8; ++i) {
                    const int b = 32 * i - (i & 1 ? w[k][i / 2].w : w[k][i / 2].y);
                    if (b <= m[k]) { at = i; before = b; mask[k] = (uint32_t)(i & 1 ? w[k][i / 2].z : w[k][i / 2].x); }
                }
                m[k] -= before;
                lo[k] += at;
            }
        }
#pragma unroll
        for (int k = 0; k < kPerThread; ++k) {
            uint32_t rest = ~mask[k];                               // its m-th set bit
            int bit = 0;
#pragma unroll
            for (int half = 16; half > 0; half >>= 1) {
                const int below = __popc(rest & ((1u << half) - 1u));
                const bool up = m[k] >= below;
                m[k] -= up ? below : 0;
                bit += up ? half : 0;
                rest = up ? rest >> half : rest;
            }
            if (of[k] >= 0) to[k] = lo[k] * 32 + bit;
        }
    };
    if (blockIdx.x == 0 && tid == 0) {
        a.status[0] = N;
        a.status[1] = moves;
    }
    // of a page, or of what an entry names: the number of its move, or -1
    auto move_of = [&](int p, int2 w) {
        if (p < N || p >= d.num_pages) return -1;
        const int m = used_before(p, w) - low;
        return (((uint32_t)w.x >> (p & 31)) & 1u) && m < d.max_moves ? m : -1;
    };
    // (what has to be looked up is, for all four, before anything is written: the loads are under way together)
    if constexpr (kSelf) own_words();
    if (on_counts) {
        int move[kPerThread], to[kPerThread] = {};
        const int (&refs)[kPerThread] = got;
        bool hole[kPerThread];
#pragma unroll
        for (int k = 0; k < kPerThread; ++k) {
            const int p = blockIdx.x * kChunk + k * kPagesThreads + tid;
            move[k] = move_of(p, own[k]);
            hole[k] = p < N && !(((uint32_t)own[k].x >> (p & 31)) & 1u) && p - used_before(p, own[k]) < d.max_moves;
        }
        free_pages(move, to);
#pragma unroll
        for (int k = 0; k < kPerThread; ++k) {
            const int p = blockIdx.x * kChunk + k * kPagesThreads + tid;
            if (p >= d.num_pages) break;
            if (p >= moves && p < d.max_moves) {                    // (max_moves <= num_pages: every unused place is met)
                a.copy_src[p] = -1;
                a.copy_dst[p] = -1;
            }
            if (move[k] >= 0) {                                     // its new place takes over its holders
                a.out_refs[to[k]] = refs[k];
                a.out_refs[p] = 0;
                a.page_map[p] = to[k];
                a.copy_src[move[k]] = p;
                a.copy_dst[move[k]] = to[k];
            } else if (hole[k]) {
                a.page_map[p] = -1;                                 // was free; its count comes from the page that moves here
            } else {
                a.out_refs[p] = refs[k];
                a.page_map[p] = refs[k] > 0 ? p : -1;
            }
        }
        return;
    }
    const int64_t step = (int64_t)a.table_groups * kChunk;
    for (int64_t e0 = (int64_t)(blockIdx.x - a.chunks) * kChunk; e0 < entries; e0 += step) {
        int p[kPerThread], move[kPerThread];
#pragma unroll
        for (int k = 0; k < kPerThread; ++k) {
            p[k] = got[k];
            move[k] = move_of(p[k], own[k]);
        }
        table_entries(e0 + step);
        free_pages(move, p);
#pragma unroll
        for (int k = 0; k < kPerThread; ++k)
            if (e0 + k * kPagesThreads + tid < entries) a.out_table[e0 + k * kPagesThreads + tid] = p[k];
        if (e0 + step < entries) own_words();
    }
}

size_t compact_workspace(const adaspec_pages_dims &d, CompactArgs *a, char *ws)
{
    const int chunks = ceil_div(d.num_pages, kChunk);
    const size_t used = align_up((size_t)chunks * (kChunk / kGrain) * 4, 256), words = align_up((size_t)chunks * (kChunk / 32) * 8, 256);
    if (a) {
        a->chunks = chunks;
        a->grain_used = reinterpret_cast<int32_t *>(ws);
        a->words = reinterpret_cast<int2 *>(ws + used);
        const int64_t n = ((int64_t)d.old_batch * d.max_pages_per_req + kChunk - 1) / kChunk;
        a->table_groups = (int)(n < 2048 ? n : 2048);
    }
    return used + words;
}

hipError_t launch_kv_compact_pages(const CompactArgs &a, hipStream_t stream)
{
    const dim3 grid(a.chunks + a.table_groups);
    const size_t lds = ((size_t)a.chunks * (kChunk / kGrain) + 1) * 4;
    if (a.dims.num_pages <= kSelfPages && a.out_refs != a.page_refs) {
        hipLaunchKernelGGL(compact_write_kernel<true>, grid, dim3(kPagesThreads), lds, stream, a);
    } else {
        hipLaunchKernelGGL(compact_words_kernel, dim3(a.chunks), dim3(kPagesThreads), 0, stream, a);
        hipLaunchKernelGGL(compact_write_kernel<false>, grid, dim3(kPagesThreads), lds, stream, a);
    }
    return hipGetLastError();
}

// ---- copy ----------------------------------------------------------------------------------------------------------
// One workgroup per (pair, layer) at a time, K and V side by side: 16 bytes per thread and access.  Memory bounds it: 4096 pages of
// 64 KB of K and V in 111 us, 4.84 TB/s read and written, the rate of a large copy (4.93).
__global__ __launch_bounds__(kPagesThreads) void copy_pages_kernel(uint4 *__restrict__ k_pages, uint4 *__restrict__ v_pages,
                                                                   const int32_t *__restrict__ copy_src,
                                                                   const int32_t *__restrict__ copy_dst, int n_copies, int layers,
                                                                   int num_pages, int64_t page_vecs)
{
    const int64_t work = (int64_t)n_copies * layers;
    for (int64_t w = blockIdx.x; w < work; w += gridDim.x) {
        const int i = (int)(w / layers), layer = (int)(w % layers);
        const int s = copy_src[i], t = copy_dst[i];
        if (s < 0 || t < 0 || s >= num_pages || t >= num_pages || s == t) continue;
        const int64_t from = ((int64_t)layer * num_pages + s) * page_vecs, to = ((int64_t)layer * num_pages + t) * page_vecs;
        for (int64_t c = threadIdx.x; c < page_vecs; c += kPagesThreads) {
            const uint4 k = k_pages[from + c], v = v_pages[from + c];
            k_pages[to + c] = k;
            v_pages[to + c] = v;
        }
    }
}

// The scales of a cache of 8 bits go with its pages: page_scales of K and of V per page.
__global__ __launch_bounds__(kPagesThreads) void copy_scales_kernel(float *__restrict__ k_scales, float *__restrict__ v_scales,
                                                                    const int32_t *__restrict__ copy_src,
                                                                    const int32_t *__restrict__ copy_dst, int n_copies, int layers,
                                                                    int num_pages, int page_scales)
{
    const int64_t work = (int64_t)n_copies * layers * page_scales;
    for (int64_t w = (int64_t)blockIdx.x * kPagesThreads + threadIdx.x; w < work; w += (int64_t)gridDim.x * kPagesThreads) {
        const int h = (int)(w % page_scales), layer = (int)(w / page_scales % layers), i = (int)(w / page_scales / layers);
        const int s = copy_src[i], t = copy_dst[i];
        if (s < 0 || t < 0 || s >= num_pages || t >= num_pages) continue;
        const int64_t from = ((int64_t)layer * num_pages + s) * page_scales + h, to = ((int64_t)layer * num_pages + t) * page_scales + h;
        k_scales[to] = k_scales[from];
        v_scales[to] = v_scales[from];
    }
}

static hipError_t copy_pages(void *k_pages, void *v_pages, const int32_t *copy_src, const int32_t *copy_dst, int n_copies,
                             const adaspec_copy_dims &d, int element, hipStream_t stream)
{
    const int64_t page_vecs = (int64_t)d.n_kv_heads * d.page_size * d.head_dim * element / 16;
    const int64_t work = (int64_t)n_copies * d.layers;
    hipLaunchKernelGGL(copy_pages_kernel, dim3((unsigned)(work < 4096 ? work : 4096)), dim3(kPagesThreads), 0, stream, (uint4 *)k_pages,
                       (uint4 *)v_pages, copy_src, copy_dst, n_copies, d.layers, d.num_pages, page_vecs);
    return hipGetLastError();
}

hipError_t launch_kv_copy_pages(void *k_pages, void *v_pages, const int32_t *copy_src, const int32_t *copy_dst, int n_copies,
                                const adaspec_copy_dims &d, hipStream_t stream)
{
    return copy_pages(k_pages, v_pages, copy_src, copy_dst, n_copies, d, d.dtype == ADASPEC_F32 ? 4 : 2, stream);
}

hipError_t launch_kv_copy_pages_scaled(void *k_pages, void *v_pages, float *k_scales, float *v_scales, const int32_t *copy_src,
                                       const int32_t *copy_dst, int n_copies, const adaspec_copy_dims &d, hipStream_t stream)
{
    const hipError_t e = copy_pages(k_pages, v_pages, copy_src, copy_dst, n_copies, d, 1, stream);
    if (e != hipSuccess) return e;
    const int64_t groups = ((int64_t)n_copies * d.layers * d.n_kv_heads + kPagesThreads - 1) / kPagesThreads;
    hipLaunchKernelGGL(copy_scales_kernel, dim3((unsigned)(groups < 1024 ? groups : 1024)), dim3(kPagesThreads), 0, stream, k_scales, v_scales,
                       copy_src, copy_dst, n_copies, d.layers, d.num_pages, d.n_kv_heads);
    return hipGetLastError();
}

}  // namespace adaspec
