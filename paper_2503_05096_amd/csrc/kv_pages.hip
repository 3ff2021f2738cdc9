// The pages of the cache: which request holds which (remap, compact: integers only, on the block table and a count of
// holders per page), and the copies that follow from it (copy_pages: the bytes).
//
// Every result is independent of the order in which workgroups run: counts change by integer atomics, free pages are handed
// out by their rank in ascending order, requests by theirs.
#include "adaspec_internal.h"
#include "device_utils.h"

namespace adaspec {

constexpr int kPagesThreads = 256;
constexpr int kChunk = 4096;                // pages whose holders one workgroup counts
constexpr int kPerThread = kChunk / kPagesThreads;

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

__global__ __launch_bounds__(kPagesThreads) void copy_ints_kernel(const int32_t *__restrict__ from, int32_t *__restrict__ to, int n)
{
    for (int i = blockIdx.x * kPagesThreads + threadIdx.x; i < n; i += gridDim.x * kPagesThreads) to[i] = from[i];
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

// Rows 0 .. old_batch - 1: every entry of the old row is released, and held again by each new row that keeps it; what is left of
// both goes into the counts.  Rows behind: the new row, with what it keeps.
__global__ __launch_bounds__(kPagesThreads) void remap_rows_kernel(RemapArgs a)
{
    __shared__ int s_sum[kPagesThreads / kWave];
    const adaspec_pages_dims &d = a.dims;
    const int row = blockIdx.y, at = blockIdx.x * kChunk, end = min(at + kChunk, d.max_pages_per_req);
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
        const int i = row - d.old_batch, s = source_of(a, i);
        const Kept kept(len_of(a, s), d);
        const int32_t *t = a.block_table + (int64_t)max(s, 0) * d.max_pages_per_req;
        int32_t *o = a.out_table + (int64_t)i * d.max_pages_per_req;
        for (int j = at + threadIdx.x; j < end; j += kPagesThreads) {
            const int p = s >= 0 && kept.keeps(j) ? t[j] : -1;
            o[j] = p >= 0 && p < d.num_pages ? p : -1;
        }
    }
}

// Workgroups 0 .. chunks - 1: free pages of a chunk.  The last one: what every row wants, and where its wants begin.
__global__ __launch_bounds__(kPagesThreads) void remap_count_kernel(RemapArgs a)
{
    __shared__ int s_sum[kPagesThreads / kWave];
    const adaspec_pages_dims &d = a.dims;
    if ((int)blockIdx.x < a.chunks) {
        int n = 0;
        for (int k = 0; k < kPerThread; ++k) {
            const int p = blockIdx.x * kChunk + k * kPagesThreads + threadIdx.x;
            n += p < d.num_pages && a.out_refs[p] == 0;
        }
        n = block_sum(n, s_sum);
        if (threadIdx.x == 0) a.chunk_free[blockIdx.x] = n;
        return;
    }
    // the page that every row is about to write into, if others may hold it
    for (int i = threadIdx.x; i < d.batch; i += kPagesThreads) {
        const int len = len_of(a, source_of(a, i)), j = len / d.page_size;
        int p = -1;
        if (len % d.page_size != 0 && a.new_lens[i] > len) p = a.out_table[(int64_t)i * d.max_pages_per_req + j];
        a.part[i] = p >= 0 && a.out_refs[p] > 1 ? p : -1;
    }
    __syncthreads();
    int base = 0;
    for (int i0 = 0; i0 < d.batch; i0 += kPagesThreads) {
        const int i = i0 + threadIdx.x;
        int want = 0, copies = 0;
        if (i < d.batch) {
            const int len = len_of(a, source_of(a, i)), p = a.part[i];
            if (p >= 0) {               // of those who share it the last keeps it
                int before = 0;
                for (int k = 0; k < i; ++k) before += a.part[k] == p;
                copies = before < a.out_refs[p] - 1;
            }
            const int from = ceil_div(len, d.page_size), to = ceil_div(min(max(a.new_lens[i], 0), d.max_pages_per_req * d.page_size), d.page_size);
            want = copies + max(to - from, 0);
            a.copy_src[i] = -1;
            a.copy_dst[i] = -1;
        }
        int total;
        const int mine = base + block_scan(want, s_sum, &total);
        if (i < d.batch) {
            a.want_base[i] = mine;
            a.copies[i] = copies;
        }
        base += total;
    }
    if (threadIdx.x == 0) a.want_base[d.batch] = base;
}

// Free page number f of the pool goes to want number f.
__global__ __launch_bounds__(kPagesThreads) void remap_assign_kernel(RemapArgs a)
{
    __shared__ int s_sum[kPagesThreads / kWave];
    const adaspec_pages_dims &d = a.dims;
    int before = 0, all = 0;
    for (int c = threadIdx.x; c < a.chunks; c += kPagesThreads) {
        const int n = a.chunk_free[c];
        before += c < (int)blockIdx.x ? n : 0;
        all += n;
    }
    before = block_sum(before, s_sum);
    all = block_sum(all, s_sum);
    const int wants = a.want_base[d.batch];
    if (blockIdx.x == 0 && threadIdx.x == 0) {
        a.status[0] = max(all - wants, 0);
        a.status[1] = max(wants - all, 0);
    }
    // (wants that no page is left for: their entries are -1 already, a shared page stays shared)
    for (int k = 0; k < kPerThread; ++k) {
        const int p = blockIdx.x * kChunk + k * kPagesThreads + threadIdx.x;
        const bool free = p < d.num_pages && a.out_refs[p] == 0;
        int total;
        const int f = before + block_scan(free, s_sum, &total);
        before += total;
        if (!free || f >= wants) continue;
        int lo = 0, hi = d.batch;                   // the row whose wants f is among
        while (hi - lo > 1) {
            const int mid = (lo + hi) >> 1;
            if (a.want_base[mid] <= f) lo = mid;
            else hi = mid;
        }
        const int i = lo, len = len_of(a, source_of(a, i)), nth = f - a.want_base[i], copies = a.copies[i];
        int32_t *o = a.out_table + (int64_t)i * d.max_pages_per_req;
        a.out_refs[p] = 1;
        if (copies && nth == 0) {
            const int from = o[len / d.page_size];
            o[len / d.page_size] = p;
            atomicAdd(a.out_refs + from, -1);
            a.copy_src[i] = from;
            a.copy_dst[i] = p;
        } else {
            o[ceil_div(len, d.page_size) + nth - copies] = p;
        }
    }
}

size_t remap_workspace(const adaspec_pages_dims &d, RemapArgs *a, char *ws)
{
    const int chunks = ceil_div(d.num_pages, kChunk);
    size_t off = 0;
    auto take = [&](size_t n) {
        int32_t *p = reinterpret_cast<int32_t *>(ws + off);
        off = align_up(off + n * 4, 256);
        return p;
    };
    int32_t *free = take(chunks), *part = take(d.batch), *base = take((size_t)d.batch + 1), *copies = take(d.batch);
    if (a) { a->chunks = chunks; a->chunk_free = free; a->part = part; a->want_base = base; a->copies = copies; }
    return off;
}

hipError_t launch_kv_remap(const RemapArgs &a, hipStream_t stream)
{
    const adaspec_pages_dims &d = a.dims;
    if (a.out_refs != a.page_refs)
        hipLaunchKernelGGL(copy_ints_kernel, dim3(ceil_div(d.num_pages, kChunk)), dim3(kPagesThreads), 0, stream, a.page_refs, a.out_refs,
                           d.num_pages);
    if (d.old_batch + d.batch > 0)
        hipLaunchKernelGGL(remap_rows_kernel, dim3(ceil_div(d.max_pages_per_req, kChunk), d.old_batch + d.batch), dim3(kPagesThreads), 0,
                           stream, a);
    hipLaunchKernelGGL(remap_count_kernel, dim3(a.chunks + 1), dim3(kPagesThreads), 0, stream, a);
    hipLaunchKernelGGL(remap_assign_kernel, dim3(a.chunks), dim3(kPagesThreads), 0, stream, a);
    return hipGetLastError();
}

// ---- compact -------------------------------------------------------------------------------------------------------
// N pages are used (counts above 0).  The m-th used page at or behind N moves to the m-th free page below N, for the first
// `max_moves` of them.

__global__ __launch_bounds__(kPagesThreads) void compact_count_kernel(CompactArgs a)
{
    __shared__ int s_sum[kPagesThreads / kWave];
    int n = 0;
    for (int k = 0; k < kPerThread; ++k) {
        const int p = blockIdx.x * kChunk + k * kPagesThreads + threadIdx.x;
        n += p < a.dims.num_pages && a.page_refs[p] > 0;
    }
    n = block_sum(n, s_sum);
    if (threadIdx.x == 0) a.chunk_used[blockIdx.x] = n;
}

// rank[p]: of a page that moves or is moved to, the number of its move; -1 otherwise.  Both lists of moves.
__global__ __launch_bounds__(kPagesThreads) void compact_rank_kernel(CompactArgs a)
{
    __shared__ int s_sum[kPagesThreads / kWave];
    const adaspec_pages_dims &d = a.dims;
    int N = 0, before = 0;
    for (int c = threadIdx.x; c < a.chunks; c += kPagesThreads) {
        const int n = a.chunk_used[c];
        N += n;
        before += c < (int)blockIdx.x ? n : 0;
    }
    N = block_sum(N, s_sum);
    before = block_sum(before, s_sum);
    // used pages below N: whole chunks, and the part of the one that N lies in
    int low = 0;
    const int last = N / kChunk;
    for (int c = threadIdx.x; c < last; c += kPagesThreads) low += a.chunk_used[c];
    for (int p = last * kChunk + threadIdx.x; p < N; p += kPagesThreads) low += a.page_refs[p] > 0;
    low = block_sum(low, s_sum);
    const int moves = N - low;
    if (blockIdx.x == 0 && threadIdx.x == 0) {
        a.status[0] = N;
        a.status[1] = moves;
    }
    for (int k = 0; k < kPerThread; ++k) {
        const int p = blockIdx.x * kChunk + k * kPagesThreads + threadIdx.x;
        const bool used = p < d.num_pages && a.page_refs[p] > 0;
        int total;
        const int u = before + block_scan(used, s_sum, &total);     // used pages below p
        before += total;
        if (p >= d.num_pages) continue;
        int rank = -1;
        if (used && p >= N) rank = u - low;
        else if (!used && p < N) rank = p - u;
        if (rank >= d.max_moves) rank = -1;
        if (rank >= 0) (used ? a.copy_src : a.copy_dst)[rank] = p;
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
    if ((int)blockIdx.x < a.chunks) {
        for (int k = 0; k < kPerThread; ++k) {
            const int p = blockIdx.x * kChunk + k * kPagesThreads + threadIdx.x;
            if (p >= d.num_pages) break;
            const int r = a.rank[p];
            if (r < 0) {
                const int refs = a.page_refs[p];
                a.out_refs[p] = refs;
                a.page_map[p] = refs > 0 ? p : -1;
            } else if (p >= N) {                // moves: its new place takes over its holders
                const int to = a.copy_dst[r];
                a.out_refs[to] = a.page_refs[p];
                a.out_refs[p] = 0;
                a.page_map[p] = to;
            } else {
                a.page_map[p] = -1;             // (was free; its count is written above)
            }
        }
        return;
    }
    const int64_t n = (int64_t)d.old_batch * d.max_pages_per_req;
    for (int64_t e = (int64_t)(blockIdx.x - a.chunks) * kPagesThreads + threadIdx.x; e < n; e += (int64_t)a.table_groups * kPagesThreads) {
        const int p = a.block_table[e];
        const int r = p >= N && p < d.num_pages ? a.rank[p] : -1;
        a.out_table[e] = r >= 0 ? a.copy_dst[r] : p;
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
