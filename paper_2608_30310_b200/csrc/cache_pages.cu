// Pages of a cache: copied, shared by forks, given back, brought to the front.
//
// The bookkeeping (which pages are free, which page moves where) is the work of a single CTA or a cluster of eight: it is a few prefix sums over
// num_pages counts, whose steps need barriers between them.  The kernel after it moves the pages with the whole GPU, in pieces of 4 KB
// per warp, eight 16-byte loads in flight per lane; it is bound by HBM.  Nothing depends on the order in which threads run: free pages
// are ranked by number, counts change by atomic integer additions.
//
// 400 pages of 12 pools, 64 KB each: 102 us, 6.1 TB/s, 95 % of the measured copy rate; 512 of 2,048 pages moved by a compaction 136 us (92 %, planning
// included).  64 forks of prefixes of 2,048 pages: 20 us for 24 MB, three dependent kernels.
#include <cooperative_groups.h>
#include "cache_pages.cuh"

namespace cg = cooperative_groups;

namespace gdn {
namespace {

constexpr int kCluster = 8, kThreads = 512, kChunk = 256;
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

// kChunk entries of the child's row of fork i, from its entry j0 on (lanes 32 apart), given back
__device__ __forceinline__ void give_back(const ForkArgs& a, int child, int j0)
{
    int32_t* row = a.tables + (int64_t)child * a.row_pages;
    int page[kChunk / 32], held[kChunk / 32];
#pragma unroll
    for (int u = 0; u < kChunk / 32; ++u) page[u] = j0 + 32 * u < a.row_pages ? row[j0 + 32 * u] : -1;
#pragma unroll
    for (int u = 0; u < kChunk / 32; ++u) {
        if (page[u] != -1) row[j0 + 32 * u] = -1;
        held[u] = page[u] >= 0 && page[u] < a.num_pages ? atomicSub(&a.refcounts[page[u]], 1) : page[u] == -1;
    }
#pragma unroll
    for (int u = 0; u < kChunk / 32; ++u) {
        if (held[u] > 0) continue;                   // (an entry that names no page, or a free one)
        if (page[u] >= 0 && page[u] < a.num_pages) atomicAdd(&a.refcounts[page[u]], 1);
        report(a.status_word, GDN_ERR_BAD_INDEX);
    }
}

// The pages that forks take.  ALL: with the checks of the forks and the giving back before it, where there are few entries; many are given
// back by a kernel of their own, as their atomics want more SMs than a cluster has.
template <bool ALL>
__global__ void __launch_bounds__(kThreads) fork_plan_kernel(const ForkArgs a)
{
    extern __shared__ int32_t forks[];               // [count] each: parent, child, pages that the child takes (the last one in part; -1: no
    __shared__ int part[kThreads / 32], box[kCluster];          // fork), whole pages; then the rows that are children: once or more; more than once
    cg::cluster_group cluster = cg::this_cluster();
    const int rank = (int)cluster.block_rank(), ctas = (int)cluster.num_blocks(), tid = threadIdx.x, lane = tid % 32, F = a.count, W = a.row_pages;
    int32_t *parent = forks, *child = forks + F, *need = forks + 2 * F, *whole = forks + 3 * F;
    uint32_t *named = reinterpret_cast<uint32_t*>(forks + 4 * F), *twice = named + (a.num_rows + 31) / 32;
    if (ALL)
        for (int i = tid; i < (a.num_rows + 31) / 32; i += kThreads) named[i] = twice[i] = 0;
    cluster.sync();                                  // (all CTAs are there: they write to each other's memory)
    wait_for_predecessor();
    for (int i = tid; i < F; i += kThreads) {
        const int p = a.parents[i], c = a.children[i], n = a.tokens[i];
        parent[i] = p;
        child[i] = c;
        whole[i] = n < 0 ? 0 : n / a.page_tokens;
        if (ALL) {
            need[i] = n < 0 ? -1 : whole[i] + (n % a.page_tokens > 0);
            if (c < 0 || c >= a.num_rows) continue;
            const uint32_t bit = 1u << (c & 31);
            if (atomicOr(&named[c >> 5], bit) & bit) atomicOr(&twice[c >> 5], bit);
        } else {
            need[i] = a.plan.need[i];
        }
    }
    __syncthreads();
    const int chunks = (W + kChunk - 1) / kChunk, items = F * chunks, warps = ctas * (kThreads / 32), first = rank * (kThreads / 32) + tid / 32;
    if (ALL) {
        auto has = [](const uint32_t* set, int r) { return (set[r >> 5] >> (r & 31)) & 1u; };
        for (int i = tid; i < F; i += kThreads) {
            const int p = parent[i], c = child[i];
            if (!(p >= 0 && p < a.num_rows && c >= 0 && c < a.num_rows && need[i] <= W && !has(twice, c) && !has(named, p))) need[i] = -1;
        }
        cluster.sync();
        // a warp takes kChunk entries of a parent's row at a time, all of them on their way at once
        for (int e = first; e < items; e += warps) {
            const int i = e / chunks, j0 = (e - i * chunks) * kChunk + lane, n = need[i];
            const int32_t* row = a.tables + (int64_t)(n > 0 ? parent[i] : 0) * W;
            int page[kChunk / 32];
#pragma unroll
            for (int u = 0; u < kChunk / 32; ++u) page[u] = j0 + 32 * u < n ? row[j0 + 32 * u] : 0;
            bool bad = false;
#pragma unroll
            for (int u = 0; u < kChunk / 32; ++u) bad |= page[u] < 0 || page[u] >= a.num_pages;
            if (bad)                                 // (others may read either: the fork is left out by then)
                for (int r = 0; r < ctas; ++r) *(volatile int32_t*)(cluster.map_shared_rank(need, r) + i) = -1;
        }
        cluster.sync();
        for (int i = rank * kThreads + tid; i < F; i += ctas * kThreads)
            if (need[i] < 0) report(a.status_word, GDN_ERR_BAD_INDEX);
        for (int e = first; e < items; e += warps) {
            const int i = e / chunks;
            if (need[i] >= 0) give_back(a, child[i], (e - i * chunks) * kChunk + lane);
        }
        cluster.sync();
    }
    allow_successor();
    // free pages, ranked by number: each CTA counts those of its share of the pages, then lists the first `wanted`
    int wanted = 0;
    for (int i = tid; i - tid < F; i += kThreads) wanted += __syncthreads_count(i < F && need[i] > whole[i]);
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

// The giving back of many entries, each warp for kChunk of a fork's, with the checks of the fork that fork_plan_kernel makes otherwise.
// (No parent is a child: the rows that are checked here are not those that change.)
__global__ void __launch_bounds__(256) give_back_kernel(const ForkArgs a)
{
    allow_successor();
    wait_for_predecessor();
    const int W = a.row_pages, chunks = (W + kChunk - 1) / kChunk, items = a.count * chunks, lane = threadIdx.x % 32;
    for (int e = (blockIdx.x * blockDim.x + threadIdx.x) / 32; e < items; e += gridDim.x * blockDim.x / 32) {
        const int i = e / chunks, p = a.parents[i], c = a.children[i], n = a.tokens[i];
        const int need = n < 0 ? -1 : n / a.page_tokens + (n % a.page_tokens > 0);
        bool ok = p >= 0 && p < a.num_rows && c >= 0 && c < a.num_rows && need >= 0 && need <= W;
        int times = 0;
        bool named = false;
        for (int k = lane; k < a.count; k += 32) {
            const int other = a.children[k];
            times += other == c;
            named |= other == p;
        }
        ok = ok && __reduce_add_sync(0xffffffffu, times) == 1 && !__any_sync(0xffffffffu, named);
        bool bad = false;
        for (int j0 = lane; ok && j0 < need; j0 += kChunk) {
            int page[kChunk / 32];
#pragma unroll
            for (int u = 0; u < kChunk / 32; ++u) page[u] = j0 + 32 * u < need ? a.tables[(int64_t)p * W + j0 + 32 * u] : 0;
#pragma unroll
            for (int u = 0; u < kChunk / 32; ++u) bad |= page[u] < 0 || page[u] >= a.num_pages;
        }
        ok = ok && !__any_sync(0xffffffffu, bad);
        if (e == i * chunks && lane == 0) {
            a.plan.need[i] = ok ? need : -1;
            if (!ok) report(a.status_word, GDN_ERR_BAD_INDEX);
        }
        if (ok) give_back(a, c, (e - i * chunks) * kChunk + lane);
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

// CTAs of a planning kernel: one where little is to be read, whose barriers cost least, else a cluster
unsigned plan_ctas(int64_t pages, int64_t entries) { return pages <= 8192 && entries <= 8192 ? 1 : kCluster; }
constexpr int64_t kFewEntries = 16384;

}  // namespace

int fork_launches(const gdn_cache_desc* d, int32_t count) { return ((int64_t)count * d->row_pages <= kFewEntries ? 1 : 2) + pool_launches(d); }

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
    const bool all = entries <= kFewEntries;
    const size_t smem = 4 * sizeof(int32_t) * (size_t)count + (all ? 2 * sizeof(uint32_t) * ((d->num_rows + 31) / 32) : 0);
    cudaStream_t stream = (cudaStream_t)d->stream;
    cudaError_t e = cudaSuccess;
    auto plan = all ? fork_plan_kernel<true> : fork_plan_kernel<false>;
    // (the most that any call needs: another thread's call may set it too)
    constexpr int most = 4 * sizeof(int32_t) * GDN_CACHE_MAX_FORKS + 2 * sizeof(uint32_t) * (GDN_CACHE_MAX_ROWS / 32);
    if (smem > 40 * 1024) e = cudaFuncSetAttribute(plan, cudaFuncAttributeMaxDynamicSharedMemorySize, most);
    const unsigned ctas = plan_ctas(d->num_pages, all ? entries : 0);
    if (e == cudaSuccess && !all) e = launch_kernel(give_back_kernel, grid_for(0, entries), 256, 0, stream, 1, a);
    if (e == cudaSuccess) e = launch_kernel(plan, ctas, kThreads, smem, stream, ctas, a);
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
    const unsigned ctas = plan_ctas(d->num_pages, 0);
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
