// The pages of the cache: which request holds which (remap, compact: integers only, on the block table and a count of
// holders per page), and the copies that follow from it (copy_pages: the bytes).
//
// Every result is independent of the order in which workgroups run: counts change by integer atomics, free pages are handed
// out by their rank in ascending order, requests by theirs.
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
// (its first want's number among these rows', the entry that it is for, the page to copy into it or -1).
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
    if (i < d.batch) a.want[i] = make_int4(first, start, from, 0);
    if (tid == 0) a.tile_wants[tile] = total;
}

// Free page number f of the pool goes to want number f.
constexpr int kFirstRows = 2048;            // rows whose first wants are looked up in LDS
__global__ __launch_bounds__(kPagesThreads) void remap_assign_kernel(RemapArgs a)
{
    __shared__ int s_sum[kPagesThreads / kWave];
    __shared__ int s_tile[kPagesThreads];                   // where the wants of every 256 rows begin
    __shared__ int s_first[kFirstRows];
    const adaspec_pages_dims &d = a.dims;
    const int tid = threadIdx.x, p0 = blockIdx.x * kChunk + kPerThread * tid;
    const int4 r = four(a.out_refs, p0, d.num_pages, 1);
    const bool free[kPerThread] = {r.x == 0, r.y == 0, r.z == 0, r.w == 0};
    const bool in_lds = d.batch <= kFirstRows;
    if (in_lds)
        for (int i = tid; i < d.batch; i += kPagesThreads) s_first[i] = a.want[i].x;
    int before = 0, all = 0;
    for (int c = tid; c < a.chunks; c += kPagesThreads) {
        const int n = a.chunk_free[c];
        before += c < (int)blockIdx.x ? n : 0;
        all += n;
    }
    int wants, here;
    s_tile[tid] = block_scan(tid < a.tiles ? a.tile_wants[tid] : 0, s_sum, &wants);         // (at most 256 tiles: 65535 rows)
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
    int f = before + block_scan(free[0] + free[1] + free[2] + free[3], s_sum, &here);
#pragma unroll
    for (int e = 0; e < kPerThread; ++e) {
        if (!free[e] || f >= wants) continue;
        const int p = p0 + e;
        int lo = 0, hi = a.tiles;                           // the rows, then the row, whose wants f is among
        while (hi - lo > 1) {
            const int mid = (lo + hi) >> 1;
            if (s_tile[mid] <= f) lo = mid;
            else hi = mid;
        }
        const int in_tile = f - s_tile[lo];
        ++f;
        hi = min((lo + 1) * kPagesThreads, d.batch);
        lo *= kPagesThreads;
        while (hi - lo > 1) {
            const int mid = (lo + hi) >> 1;
            if ((in_lds ? s_first[mid] : a.want[mid].x) <= in_tile) lo = mid;
            else hi = mid;
        }
        const int4 w = a.want[lo];
        const int nth = in_tile - w.x;
        a.out_refs[p] = 1;
        a.out_table[(int64_t)lo * d.max_pages_per_req + w.y + nth] = p;
        if (w.z >= 0 && nth == 0) {
            atomicAdd(a.out_refs + w.z, -1);
            a.copy_src[lo] = w.z;
            a.copy_dst[lo] = p;
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
    hipLaunchKernelGGL(remap_start_kernel, dim3(a.chunks), dim3(kPagesThreads), 0, stream, a);
    if (d.old_batch + d.batch > 0)
        hipLaunchKernelGGL(remap_rows_kernel, dim3(ceil_div(d.max_pages_per_req, kRowPart), d.old_batch + d.batch), dim3(kPagesThreads), 0,
                           stream, a);
    hipLaunchKernelGGL(remap_count_kernel, dim3(a.chunks + a.tiles), dim3(kPagesThreads), 0, stream, a);
    hipLaunchKernelGGL(remap_assign_kernel, dim3(a.chunks), dim3(kPagesThreads), 0, stream, a);
    return hipGetLastError();
}

// ---- compact -------------------------------------------------------------------------------------------------------
// N pages are used (counts above 0).  The m-th used page at or behind N moves to the m-th free page below N, for the first
// `max_moves` of them.

__global__ __launch_bounds__(kPagesThreads) void compact_count_kernel(CompactArgs a)
{
    __shared__ int s_sum[kPagesThreads / kWave];
    const int4 r = four(a.page_refs, blockIdx.x * kChunk + kPerThread * threadIdx.x, a.dims.num_pages, 0);
    const int n = block_sum((r.x > 0) + (r.y > 0) + (r.z > 0) + (r.w > 0), s_sum);
    if (threadIdx.x == 0) a.chunk_used[blockIdx.x] = n;
}

// rank[p]: of a page that moves or is moved to, the number of its move; -1 otherwise.  Both lists of moves.
__global__ __launch_bounds__(kPagesThreads) void compact_rank_kernel(CompactArgs a)
{
    __shared__ int s_sum[kPagesThreads / kWave];
    const adaspec_pages_dims &d = a.dims;
    const int tid = threadIdx.x, p0 = blockIdx.x * kChunk + kPerThread * tid;
    const int4 r = four(a.page_refs, p0, d.num_pages, 0);
    const bool used[kPerThread] = {r.x > 0, r.y > 0, r.z > 0, r.w > 0};
    int N = 0, before = 0;
    for (int c = tid; c < a.chunks; c += kPagesThreads) {
        const int n = a.chunk_used[c];
        N += n;
        before += c < (int)blockIdx.x ? n : 0;
    }
    N = block_sum(N, s_sum);
    before = block_sum(before, s_sum);
    // used pages below N: whole chunks, and the part of the one that N lies in
    int low = 0;
    const int last = N / kChunk, q0 = last * kChunk + kPerThread * tid;
    for (int c = tid; c < last; c += kPagesThreads) low += a.chunk_used[c];
    const int4 q = four(a.page_refs, q0, N, 0);
    low = block_sum(low + (q.x > 0) + (q.y > 0) + (q.z > 0) + (q.w > 0), s_sum);
    const int moves = N - low;
    if (blockIdx.x == 0 && tid == 0) {
        a.status[0] = N;
        a.status[1] = moves;
    }
    int total;
    int u = before + block_scan(used[0] + used[1] + used[2] + used[3], s_sum, &total);      // used pages below p
#pragma unroll
    for (int e = 0; e < kPerThread; ++e) {
        const int p = p0 + e;
        if (p >= d.num_pages) break;
        int rank = -1;
        if (used[e] && p >= N) rank = u - low;
        else if (!used[e] && p < N) rank = p - u;
        u += used[e];
        if (rank >= d.max_moves) rank = -1;
        if (rank >= 0) (used[e] ? a.copy_src : a.copy_dst)[rank] = p;
        a.rank[p] = rank;
        if (p >= moves && p < d.max_moves) {                        // (max_moves <= num_pages: every unused place is met)
            a.copy_src[p] = -1;
            a.copy_dst[p] = -1;
        }
    }
}

// Workgroups 0 .. chunks - 1: counts and map of a chunk of pages; those behind: the table.  Every count is read and written by
// one thread each, so that the new counts may lie over the old ones.
__global__ __launch_bounds__(kPagesThreads) void compact_write_kernel(CompactArgs a)
{
    const adaspec_pages_dims &d = a.dims;
    const int N = a.status[0];
    const int tid = threadIdx.x;
    if ((int)blockIdx.x < a.chunks) {
        int r[kPerThread], to[kPerThread];
#pragma unroll
        for (int k = 0; k < kPerThread; ++k) {                      // (all of them under way together)
            const int p = blockIdx.x * kChunk + k * kPagesThreads + tid;
            r[k] = p < d.num_pages ? a.rank[p] : -1;
        }
#pragma unroll
        for (int k = 0; k < kPerThread; ++k) {
            const int p = blockIdx.x * kChunk + k * kPagesThreads + tid;
            to[k] = r[k] >= 0 && p >= N ? a.copy_dst[r[k]] : p;
        }
#pragma unroll
        for (int k = 0; k < kPerThread; ++k) {
            const int p = blockIdx.x * kChunk + k * kPagesThreads + tid;
            if (p >= d.num_pages) break;
            if (r[k] >= 0 && p < N) {
                a.page_map[p] = -1;             // was free; its count comes from the page that moves here
            } else {
                const int refs = a.page_refs[p];
                a.out_refs[to[k]] = refs;
                if (to[k] != p) a.out_refs[p] = 0;
                a.page_map[p] = refs > 0 ? to[k] : -1;
            }
        }
        return;
    }
    const int64_t n = (int64_t)d.old_batch * d.max_pages_per_req;
    for (int64_t e0 = (int64_t)(blockIdx.x - a.chunks) * kChunk; e0 < n; e0 += (int64_t)a.table_groups * kChunk) {
        int p[kPerThread], r[kPerThread];
#pragma unroll
        for (int k = 0; k < kPerThread; ++k) p[k] = e0 + k * kPagesThreads + tid < n ? a.block_table[e0 + k * kPagesThreads + tid] : -1;
#pragma unroll
        for (int k = 0; k < kPerThread; ++k) r[k] = p[k] >= N && p[k] < d.num_pages ? a.rank[p[k]] : -1;
#pragma unroll
        for (int k = 0; k < kPerThread; ++k)
            if (r[k] >= 0) p[k] = a.copy_dst[r[k]];
#pragma unroll
        for (int k = 0; k < kPerThread; ++k)
            if (e0 + k * kPagesThreads + tid < n) a.out_table[e0 + k * kPagesThreads + tid] = p[k];
    }
}

size_t compact_workspace(const adaspec_pages_dims &d, CompactArgs *a, char *ws)
{
    const int chunks = ceil_div(d.num_pages, kChunk);
    const size_t used = align_up((size_t)chunks * 4, 256), rank = align_up((size_t)d.num_pages * 4, 256);
    if (a) {
        a->chunks = chunks;
        a->chunk_used = reinterpret_cast<int32_t *>(ws);
        a->rank = reinterpret_cast<int32_t *>(ws + used);
        const int64_t n = ((int64_t)d.old_batch * d.max_pages_per_req + kChunk - 1) / kChunk;
        a->table_groups = (int)(n < 2048 ? n : 2048);
    }
    return used + rank;
}

hipError_t launch_kv_compact_pages(const CompactArgs &a, hipStream_t stream)
{
    hipLaunchKernelGGL(compact_count_kernel, dim3(a.chunks), dim3(kPagesThreads), 0, stream, a);
    hipLaunchKernelGGL(compact_rank_kernel, dim3(a.chunks), dim3(kPagesThreads), 0, stream, a);
    hipLaunchKernelGGL(compact_write_kernel, dim3(a.chunks + a.table_groups), dim3(kPagesThreads), 0, stream, a);
    return hipGetLastError();
}

// ---- copy ----------------------------------------------------------------------------------------------------------
// One workgroup per (pair, layer, tensor) at a time: 16 bytes per thread and access.
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

hipError_t launch_kv_copy_pages(void *k_pages, void *v_pages, const int32_t *copy_src, const int32_t *copy_dst, int n_copies,
                                const adaspec_copy_dims &d, hipStream_t stream)
{
    const int64_t page_vecs = (int64_t)d.n_kv_heads * d.page_size * d.head_dim * (d.dtype == ADASPEC_F32 ? 4 : 2) / 16;
    const int64_t work = (int64_t)n_copies * d.layers;
    hipLaunchKernelGGL(copy_pages_kernel, dim3((unsigned)(work < 4096 ? work : 4096)), dim3(kPagesThreads), 0, stream, (uint4 *)k_pages,
                       (uint4 *)v_pages, copy_src, copy_dst, n_copies, d.layers, d.num_pages, page_vecs);
    return hipGetLastError();
}

}  // namespace adaspec
