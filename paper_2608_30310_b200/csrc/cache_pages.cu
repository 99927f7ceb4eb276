// Pages of a cache: copied, shared by forks, given back, brought to the front.
//
// The bookkeeping (which pages are free, which page moves where) is the work of a single CTA or a cluster of eight: it is a few prefix sums over
// num_pages counts, whose steps need barriers between them.  The kernel after it moves the pages with the whole GPU, in pieces of 4 KB
// per warp, eight 16-byte loads in flight per lane; it is bound by HBM.  Nothing depends on the order in which threads run: free pages
// are ranked by number, counts change by atomic integer additions.
//
// 400 pages of 12 pools, 64 KB each: 102 us, 6.1 TB/s, 95 % of the measured copy rate; 512 of 2,048 pages moved by a compaction 135 us (92 %, planning
// included).  64 forks of prefixes of 2,048 pages: 18 us for 24 MB, three dependent kernels.  A fork reads its parent's row once, and the count
// of each page there: 64 rows of 32,768 entries 81 us.
#include <cooperative_groups.h>
#include "cache_pages.cuh"

namespace cg = cooperative_groups;

namespace gdn {
namespace {

constexpr int kCluster = 8, kThreads = 512;
constexpr int64_t kPiece = 4096;       // bytes that a warp moves at a time
constexpr int kPoolsPerLaunch = 64;

struct Pools {
    void* base[kPoolsPerLaunch];
    int64_t bytes[kPoolsPerLaunch];                  // of a page
    uint32_t pieces[kPoolsPerLaunch + 1];            // of a page in the pools before this one
    int32_t count;
};

__device__ __forceinline__ void report(int32_t* status_word, int32_t what)
{
    if (status_word) *status_word = what;
}

// Item i of `pairs` x pieces: one warp moves one piece of page src[k] to page dst[k].  The CTAs from `first_cta` on share the items.
__device__ void copy_pages(const Pools& pools, const int32_t* src, const int32_t* dst, uint32_t pairs, int32_t num_pages, bool check, int32_t* status_word,
                           uint32_t first_cta)
{
    const uint32_t per = pools.pieces[pools.count], lane = threadIdx.x % 32;
    const uint64_t items = (uint64_t)pairs * per;
    uint64_t i = ((uint64_t)(blockIdx.x - first_cta) * blockDim.x + threadIdx.x) / 32;
    const uint64_t warps = (uint64_t)(gridDim.x - first_cta) * blockDim.x / 32;
    for (; i < items; i += warps) {
        const uint32_t k = items >> 32 ? (uint32_t)(i / per) : (uint32_t)i / per, piece = (uint32_t)(i - (uint64_t)k * per);
        const int from = src[k], to = dst[k];
        if (from < 0 || from >= num_pages || to < 0 || to >= num_pages) {
            if (check) report(status_word, GDN_ERR_BAD_INDEX);
            continue;
        }
        int lo = 0;
        for (int hi = pools.count; hi - lo > 1;) {
            const int mid = (lo + hi) / 2;
            if (pools.pieces[mid] <= piece) lo = mid; else hi = mid;
        }
        const int64_t bytes = pools.bytes[lo], at = (int64_t)(piece - pools.pieces[lo]) * kPiece + lane * 16;
        const char* s = (const char*)pools.base[lo] + from * bytes;
        char* d = (char*)pools.base[lo] + to * bytes;
        int4 v[kPiece / 512];
#pragma unroll
        for (int j = 0; j < kPiece / 512; ++j)
            if (at + j * 512 < bytes) v[j] = *reinterpret_cast<const int4*>(s + at + j * 512);
#pragma unroll
        for (int j = 0; j < kPiece / 512; ++j)
            if (at + j * 512 < bytes) *reinterpret_cast<int4*>(d + at + j * 512) = v[j];
    }
}

__global__ void __launch_bounds__(256) copy_kernel(const Pools pools, const int32_t* src, const int32_t* dst, const uint32_t pairs, const int32_t num_pages, int32_t* status_word)
{
    allow_successor();
    wait_for_predecessor();
    copy_pages(pools, src, dst, pairs, num_pages, true, status_word, 0);
}

// Sum over the threads before this one, and over all of the CTA.
__device__ int scan_cta(int v, int* total, int* part)
{
    const int lane = threadIdx.x % 32, warp = threadIdx.x / 32;
    int x = v;
#pragma unroll
    for (int m = 1; m < 32; m *= 2) {
        const int y = __shfl_up_sync(0xffffffffu, x, m);
        if (lane >= m) x += y;
    }
    if (lane == 31) part[warp] = x;
    __syncthreads();
    const int w = lane < kThreads / 32 ? part[lane] : 0;
    const int before_warp = __reduce_add_sync(0xffffffffu, lane < warp ? w : 0);
    *total = __reduce_add_sync(0xffffffffu, w);
    __syncthreads();
    return before_warp + x - v;
}

// Each CTA's number to all CTAs of the cluster: the sum over the CTAs before this one, and over all.
__device__ int scan_cluster(int mine, int* total, int* box)
{
    cg::cluster_group cluster = cg::this_cluster();
    const int rank = (int)cluster.block_rank(), ctas = (int)cluster.num_blocks();
    if (threadIdx.x < ctas) cluster.map_shared_rank(box, threadIdx.x)[rank] = mine;
    cluster.sync();
    int before = 0, all = 0;
    for (int r = 0; r < ctas; ++r) {
        before += r < rank ? box[r] : 0;
        all += box[r];
    }
    *total = all;
    return before;
}

// ---- fork

struct ForkPlan {                  // in the workspace, [count] each
    int32_t *need, *src, *dst, *share, *free;
};
struct ForkArgs {
    int32_t *refcounts, *tables;
    const int32_t *parents, *children, *tokens;
    int32_t count, num_pages, num_rows, row_pages, page_tokens;
    int32_t* status_word;
    ForkPlan plan;
};

// Entries of a row in a thread's hands, all of them on their way at once: kHand, `step` apart from entry j0 on.
constexpr int kHand = 8;
__device__ __forceinline__ void entries_of(const int32_t* row, int64_t j0, int step, int end, int beyond, int (&page)[kHand])
{
#pragma unroll
    for (int u = 0; u < kHand; ++u) page[u] = j0 + u * step < end ? row[j0 + u * step] : beyond;
}

// Whether entries of a parent's row before `end` name pages that are held.  A page that the row holds in earnest keeps its count above 0 whoever
// gives back meanwhile; one that is free could be handed to another fork.
__device__ __forceinline__ bool all_held(const ForkArgs& a, const int32_t* row, int64_t j0, int step, int end)
{
    int page[kHand], count[kHand];
    bool ok = true;
    entries_of(row, j0, step, end, 0, page);
#pragma unroll
    for (int u = 0; u < kHand; ++u) {
        const bool real = page[u] >= 0 && page[u] < a.num_pages;
        count[u] = j0 + u * step < end ? (real ? __ldcg(&a.refcounts[page[u]]) : 0) : 1;
    }
#pragma unroll
    for (int u = 0; u < kHand; ++u) ok &= count[u] > 0;
    return ok;
}

// entries_of a child's row (beyond it -1), given back
__device__ __forceinline__ void give_back(const ForkArgs& a, int32_t* row, int64_t j0, int step, const int (&page)[kHand])
{
    int held[kHand];
#pragma unroll
    for (int u = 0; u < kHand; ++u) {
        if (page[u] != -1) row[j0 + u * step] = -1;
        held[u] = page[u] >= 0 && page[u] < a.num_pages ? atomicSub(&a.refcounts[page[u]], 1) : page[u] == -1;
    }
#pragma unroll
    for (int u = 0; u < kHand; ++u) {
        if (held[u] > 0) continue;                   // (an entry that names no page, or a free one)
        if (page[u] >= 0 && page[u] < a.num_pages) atomicAdd(&a.refcounts[page[u]], 1);
        report(a.status_word, GDN_ERR_BAD_INDEX);
    }
}

// The checks of the forks and the giving back, a CTA or a cluster for each fork: its atomics want more SMs than the planning cluster has.
// (No parent is a child: the rows that are checked here are not those that change.)
__global__ void __launch_bounds__(kThreads) give_back_kernel(const ForkArgs a)
{
    __shared__ int box[kCluster];
    cg::cluster_group cluster = cg::this_cluster();
    const int ctas = (int)cluster.num_blocks(), i = blockIdx.x / ctas, W = a.row_pages;
    const int me = (int)(cluster.block_rank() * blockDim.x + threadIdx.x), all = (int)(ctas * blockDim.x);
    allow_successor();
    cluster.sync();                                  // (all CTAs are there: they write to each other's memory)
    wait_for_predecessor();
    const int p = a.parents[i], c = a.children[i], n = a.tokens[i];
    const int need = n < 0 ? -1 : n / a.page_tokens + (n % a.page_tokens > 0);
    const bool there = p >= 0 && p < a.num_rows && c >= 0 && c < a.num_rows && need >= 0 && need <= W;
    const int32_t* from = a.tables + (int64_t)(there ? p : 0) * W;
    int32_t* row = a.tables + (int64_t)(there ? c : 0) * W;
    bool bad = !there;
    for (int k = threadIdx.x; k < a.count; k += blockDim.x) {
        const int other = a.children[k];
        bad |= other == p || (other == c && k != i);
    }
    for (int64_t j0 = me; there && j0 < need; j0 += (int64_t)all * kHand) bad |= !all_held(a, from, j0, all, need);
    bad = __syncthreads_or(bad);
    if (ctas > 1) {                                  // (a fork's checks are all made before any of its entries changes)
        int wrong;
        scan_cluster(bad, &wrong, box);
        bad = wrong > 0;
    }
    if (me == 0) {
        a.plan.need[i] = bad ? -1 : need;
        if (bad) report(a.status_word, GDN_ERR_BAD_INDEX);
    }
    if (bad) return;
    for (int64_t j0 = me; j0 < W; j0 += (int64_t)all * kHand) {
        int page[kHand];                             // (read ahead of the checks the children of many forks keep each other waiting)
        entries_of(row, j0, all, W, -1, page);
        give_back(a, row, j0, all, page);
    }
}

// The pages that forks take: the free ones, ranked by number.
__global__ void __launch_bounds__(kThreads) fork_plan_kernel(const ForkArgs a)
{
    extern __shared__ int32_t forks[];               // [count] each: parent, child, pages that the child takes (the last one in part; -1: no
    __shared__ int part[kThreads / 32], box[kCluster];          // fork), whole pages
    cg::cluster_group cluster = cg::this_cluster();
    const int rank = (int)cluster.block_rank(), ctas = (int)cluster.num_blocks(), tid = threadIdx.x, F = a.count, W = a.row_pages;
    int32_t *parent = forks, *child = forks + F, *need = forks + 2 * F, *whole = forks + 3 * F;
    cluster.sync();                                  // (all CTAs are there: they write to each other's memory)
    wait_for_predecessor();
    for (int i = tid; i < F; i += kThreads) {
        const int n = a.tokens[i];
        parent[i] = a.parents[i];
        child[i] = a.children[i];
        need[i] = a.plan.need[i];
        whole[i] = n < 0 ? 0 : n / a.page_tokens;
    }
    int wanted = 0;                                  // (a thread reads what it wrote itself)
    for (int i = tid; i - tid < F; i += kThreads) wanted += __syncthreads_count(i < F && need[i] > whole[i]);
    allow_successor();                               // (earlier, its CTAs take the SMs where the giving back still runs)
    // each CTA counts the free pages of its share, then lists the first `wanted`
    const int slice = (a.num_pages + ctas - 1) / ctas, lo = min(rank * slice, a.num_pages), hi = min(lo + slice, a.num_pages);
    int mine = 0, there, all_free;
    for (int p = lo + tid; p < hi; p += kThreads) mine += __ldcg(&a.refcounts[p]) <= 0;
    scan_cta(mine, &there, part);
    int before = scan_cluster(there, &all_free, box);
    for (int p0 = lo; p0 < hi && before < wanted; p0 += kThreads) {
        const int p = p0 + tid;
        const bool is_free = p < hi && __ldcg(&a.refcounts[p]) <= 0;
        const int at = before + scan_cta(is_free, &there, part);
        if (is_free && at < wanted) a.plan.free[at] = p;
        before += there;
    }
    cluster.sync();
    if (rank) return;
    int given = 0;
    for (int i0 = 0; i0 < F; i0 += kThreads) {
        const int i = i0 + tid;
        const bool partial = i < F && need[i] > whole[i];
        int taken;
        const int at = given + scan_cta(partial, &taken, part);
        given += taken;
        if (i >= F) continue;
        int share = need[i] < 0 ? 0 : whole[i], src = -1, dst = -1;
        if (partial && at < all_free) {
            src = a.tables[(int64_t)parent[i] * W + share];
            dst = __ldcg(&a.plan.free[at]);
            a.tables[(int64_t)child[i] * W + share] = dst;
            a.refcounts[dst] = 1;
        } else if (partial) {
            share = 0;
            report(a.status_word, GDN_ERR_NO_PAGES);
        }
        a.plan.src[i] = src; a.plan.dst[i] = dst; a.plan.share[i] = share;
    }
}

// The first `sharing` CTAs enter the shared pages, the others copy the partial ones.
__global__ void __launch_bounds__(256) fork_kernel(const Pools pools, const ForkArgs a, const uint32_t sharing)
{
    allow_successor();
    wait_for_predecessor();
    if (blockIdx.x < sharing) {
        const int W = a.row_pages;
        const uint32_t entries = (uint32_t)a.count * W;
        for (uint32_t e = blockIdx.x * blockDim.x + threadIdx.x; e < entries; e += sharing * blockDim.x) {
            const int i = e / (uint32_t)W, j = e - i * W;
            if (j >= a.plan.share[i]) continue;
            const int page = a.tables[(int64_t)a.parents[i] * W + j];
            a.tables[(int64_t)a.children[i] * W + j] = page;
            atomicAdd(&a.refcounts[page], 1);
        }
    } else {
        copy_pages(pools, a.plan.src, a.plan.dst, a.count, a.num_pages, false, nullptr, sharing);
    }
}

// ---- free

__global__ void __launch_bounds__(256) free_kernel(int32_t* refcounts, int32_t* tables, const int32_t* rows, int32_t count, int32_t num_pages,
                                                   int32_t num_rows, int32_t row_pages, int32_t* status_word)
{
    allow_successor();
    wait_for_predecessor();
    const uint32_t entries = (uint32_t)count * row_pages;
    for (uint32_t e = blockIdx.x * blockDim.x + threadIdx.x; e < entries; e += gridDim.x * blockDim.x) {
        const int i = e / (uint32_t)row_pages, j = e - i * row_pages, r = rows[i];
        if (r < 0 || r >= num_rows) {
            if (j == 0) report(status_word, GDN_ERR_BAD_INDEX);
            continue;
        }
        int32_t* at = tables + (int64_t)r * row_pages + j;
        if (*(volatile int32_t*)at == -1) continue;
        const int page = atomicExch(at, -1);         // (of a row named twice, one finds it)
        if (page == -1) continue;
        if (page < 0 || page >= num_pages) report(status_word, GDN_ERR_BAD_INDEX);
        else if (atomicSub(&refcounts[page], 1) <= 0) {
            atomicAdd(&refcounts[page], 1);
            report(status_word, GDN_ERR_BAD_INDEX);
        }
    }
}

// ---- compact

struct CompactPlan {               // in the workspace: how many pages move and where their list of sources begins; holes, sources, their counts
    int32_t *header, *holes, *src, *src_count;
};
struct CompactArgs {
    const int32_t *refcounts, *tables;
    int32_t *out_refcounts, *out_tables, *page_map, *live;
    int32_t num_pages, num_rows, row_pages;
    int32_t* status_word;
    CompactPlan plan;
};

__global__ void __launch_bounds__(kThreads) compact_plan_kernel(const CompactArgs a)
{
    __shared__ int part[kThreads / 32], box[kCluster];
    cg::cluster_group cluster = cg::this_cluster();
    const int rank = (int)cluster.block_rank(), tid = threadIdx.x, P = a.num_pages;
    cluster.sync();                                  // (all CTAs are there: they write to each other's memory)
    wait_for_predecessor();
    const int slice = (P + (int)cluster.num_blocks() - 1) / (int)cluster.num_blocks(), lo = min(rank * slice, P), hi = min(lo + slice, P);
    int mine = 0, there, all_free;
    for (int p = lo + tid; p < hi; p += kThreads) mine += a.refcounts[p] <= 0;
    scan_cta(mine, &there, part);
    int before = scan_cluster(there, &all_free, box);
    const int M = P - all_free;
    // with f free pages before page p, p is hole f (below M) or live page p - f (at or after M); M has H holes before it
    for (int p0 = lo; p0 < hi; p0 += kThreads) {
        const int p = p0 + tid, count = p < hi ? a.refcounts[p] : 1;
        const int f = before + scan_cta(count <= 0, &there, part);
        before += there;
        if (p >= hi) continue;
        a.page_map[p] = f;
        if (p < M && count <= 0) a.plan.holes[f] = p;
        if (p >= M && count > 0) { a.plan.src[p - f] = p; a.plan.src_count[p - f] = count; }
        if (p == M) { a.plan.header[0] = f; a.plan.header[1] = M - f; }
    }
    if (rank == 0 && tid == 0) {
        *a.live = M;
        if (M == P) { a.plan.header[0] = 0; a.plan.header[1] = 0; }
    }
    cluster.sync();
    allow_successor();
    const int first = __ldcg(&a.plan.header[1]);     // rank among the live pages of the first one that moves
    for (int p = lo + tid; p < hi; p += kThreads) {
        const int count = a.refcounts[p], f = a.page_map[p];
        int to = -1, now = 0;
        if (count > 0) to = p < M ? p : __ldcg(&a.plan.holes[p - f - first]);
        if (p < M) now = count > 0 ? count : __ldcg(&a.plan.src_count[first + f]);
        a.page_map[p] = to;
        a.out_refcounts[p] = now;
    }
}

// The first `renaming` CTAs rewrite the tables, the others move the pages.
__global__ void __launch_bounds__(256) compact_kernel(const Pools pools, const CompactArgs a, const uint32_t renaming)
{
    allow_successor();
    wait_for_predecessor();
    if (blockIdx.x < renaming) {
        const uint32_t entries = (uint32_t)a.num_rows * a.row_pages;
        for (uint32_t e = blockIdx.x * blockDim.x + threadIdx.x; e < entries; e += renaming * blockDim.x) {
            const int page = a.tables[e];
            int to = -1;
            if (page >= 0 && page < a.num_pages) to = a.page_map[page];
            if (page != -1 && to < 0) report(a.status_word, GDN_ERR_BAD_INDEX);
            a.out_tables[e] = to;
        }
    } else {
        copy_pages(pools, a.plan.src + a.plan.header[1], a.plan.holes, a.plan.header[0], a.num_pages, false, nullptr, renaming);
    }
}

// ---- host

Pools pools_from(const gdn_cache_desc* d, int first)
{
    Pools p = {};
    for (int i = first; i < d->num_pools && p.count < kPoolsPerLaunch; ++i, ++p.count) {
        p.base[p.count] = d->pools[i].base;
        p.bytes[p.count] = d->pools[i].page_bytes;
        p.pieces[p.count + 1] = p.pieces[p.count] + (uint32_t)((d->pools[i].page_bytes + kPiece - 1) / kPiece);
    }
    return p;
}

// CTAs of eight warps: enough for the items, at most as many as fit the GPU at once
unsigned grid_for(uint64_t pieces, uint64_t entries)
{
    const uint64_t ctas = pieces / 8 > entries / 1024 ? (pieces + 7) / 8 : (entries + 1023) / 1024;
    return (unsigned)(ctas < 1 ? 1 : ctas > 148 * 4 ? 148 * 4 : ctas);
}

// CTAs of a planning kernel: one where few counts are to be read, whose barriers cost least, else a cluster.  (us with one / a cluster: a
// compaction of 600 pages 5.4 / 6.0, 1,024 5.7 / 5.9, 1,500 6.6 / 6.2, 8,192 17.1 / 7.3; a fork among 929 pages 8.0 / 8.4, 64 among 4,224
// 12.6 / 12.3, among 65,664 53 / 31.)
unsigned plan_ctas(int64_t pages) { return pages <= 1024 ? 1 : kCluster; }
}  // namespace

int fork_launches(const gdn_cache_desc* d) { return 2 + pool_launches(d); }

int pool_launches(const gdn_cache_desc* d) { return d->num_pools > 0 ? (d->num_pools + kPoolsPerLaunch - 1) / kPoolsPerLaunch : 1; }

cudaError_t launch_cache_copy(const gdn_cache_desc* d, const int32_t* src, const int32_t* dst, int32_t count)
{
    for (int first = 0; first < d->num_pools; first += kPoolsPerLaunch) {
        const Pools p = pools_from(d, first);
        const cudaError_t e = launch_kernel(copy_kernel, grid_for((uint64_t)count * p.pieces[p.count], 0), 256, 0, (cudaStream_t)d->stream, 1, p, src, dst,
                                            (uint32_t)count, d->num_pages, d->status_word);
        if (e != cudaSuccess) return e;
    }
    return cudaSuccess;
}

cudaError_t launch_cache_fork(const gdn_cache_desc* d, int32_t* refcounts, int32_t* tables, const int32_t* parents, const int32_t* children,
                              const int32_t* tokens, int32_t count)
{
    ForkArgs a = {refcounts, tables, parents, children, tokens, count, d->num_pages, d->num_rows, d->row_pages, d->page_tokens, d->status_word, {}};
    int32_t* w = (int32_t*)d->workspace;
    a.plan = {w, w + count, w + 2 * (int64_t)count, w + 3 * (int64_t)count, w + 4 * (int64_t)count};
    const int64_t entries = (int64_t)count * d->row_pages;
    const size_t smem = 4 * sizeof(int32_t) * (size_t)count;
    cudaStream_t stream = (cudaStream_t)d->stream;
    // A fork's CTAs and their threads: one small one for short rows, of which an SM runs more at once, a cluster for long rows.  (us of a call,
    // 128 / 512 threads: 4,096 forks with rows of 64 entries 46 / 62, 512 of 64 13.1 / 15.1, 32 of 256 10.6 / 10.4, 64 of 1,024 15.1 / 13.4.
    // One CTA / a cluster: 64 forks with rows of 4,096 20.4 / 23.5, of 8,192 38 / 31; 16 of 16,384 38 / 20.)
    const unsigned per_fork = d->row_pages <= 4096 ? 1 : kCluster, threads = d->row_pages <= 256 ? 128 : kThreads, ctas = plan_ctas(d->num_pages);
    cudaError_t e = cudaSuccess;
    // (the most that any call needs: another thread's call may set it too)
    if (smem > 40 * 1024) e = cudaFuncSetAttribute(fork_plan_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, 4 * sizeof(int32_t) * GDN_CACHE_MAX_FORKS);
    if (e == cudaSuccess) e = launch_kernel(give_back_kernel, count * per_fork, threads, 0, stream, per_fork, a);
    if (e == cudaSuccess) e = launch_kernel(fork_plan_kernel, ctas, kThreads, smem, stream, ctas, a);
    for (int i = 0; i < pool_launches(d) && e == cudaSuccess; ++i) {
        const Pools p = pools_from(d, i * kPoolsPerLaunch);
        const unsigned sharing = i == 0 ? grid_for(0, entries) : 0;
        e = launch_kernel(fork_kernel, sharing + grid_for((uint64_t)count * p.pieces[p.count], 0), 256, 0, stream, 1, p, a, sharing);
    }
    return e;
}

cudaError_t launch_cache_free(const gdn_cache_desc* d, int32_t* refcounts, int32_t* tables, const int32_t* rows, int32_t count)
{
    return launch_kernel(free_kernel, grid_for(0, 4 * (uint64_t)count * d->row_pages), 256, 0, (cudaStream_t)d->stream, 1, refcounts, tables, rows, count,
                         d->num_pages, d->num_rows, d->row_pages, d->status_word);
}

cudaError_t launch_cache_compact(const gdn_cache_desc* d, const int32_t* refcounts, const int32_t* tables, int32_t* out_refcounts, int32_t* out_tables,
                                 int32_t* page_map, int32_t* live)
{
    CompactArgs a = {refcounts, tables, out_refcounts, out_tables, page_map, live, d->num_pages, d->num_rows, d->row_pages, d->status_word, {}};
    int32_t* w = (int32_t*)d->workspace;
    a.plan = {w, w + 64, w + 64 + (int64_t)d->num_pages, w + 64 + 2 * (int64_t)d->num_pages};
    cudaStream_t stream = (cudaStream_t)d->stream;
    const unsigned ctas = plan_ctas(d->num_pages);
    cudaError_t e = launch_kernel(compact_plan_kernel, ctas, kThreads, 0, stream, ctas, a);
    for (int i = 0; i < pool_launches(d) && e == cudaSuccess; ++i) {
        const Pools p = pools_from(d, i * kPoolsPerLaunch);
        const unsigned renaming = i == 0 ? grid_for(0, (uint64_t)d->num_rows * d->row_pages) : 0;
        // (half the pages at most move)
        e = launch_kernel(compact_kernel, renaming + grid_for((uint64_t)d->num_pages / 2 * p.pieces[p.count], 0), 256, 0, stream, 1, p, a, renaming);
    }
    return e;
}

}  // namespace gdn
