// The page operations of the key/value cache: pages for new tokens, writing keys and values into them, freeing, forking, copying and compacting.
//
// Which page goes where is decided on the device, so that a captured graph can do it: one block scans the reference counts for free pages, lowest first, and
// deals them out in the order of the askers (a scan of their needs), which makes the numbers a function of the input alone (4.3 us: two loads and two scans, one
// behind the other).  The data moves in 16-byte pieces, 16 KiB a block; those launches are bound by HBM: 64 partial pages of 32 layers, 537 MB read and written, 99 us (5.4 TB/s; a
// large copy 4.9 to 5.1), compaction of 403 MB 81, keys and values of 4267 tokens appended, 140 MB, 29 us.
#include "fbq_cache.h"
#include "fbq_internal.h"

namespace fbq {

typedef unsigned int word4_t __attribute__((ext_vector_type(4)));

constexpr int kPlanThreads = 1024;            // the block that deals out pages
constexpr int kRefsPerThread = 4;
constexpr int kRefsChunk = kPlanThreads * kRefsPerThread;
constexpr int kCopyThreads = 256, kCopyPieces = 4;
constexpr int kCopyBytes = kCopyThreads * kCopyPieces * 16;   // 16 KiB a block

constexpr int kGridChunks = 65534;            // chunks of a page in all its layers that a grid has blocks for; a block goes on with every so manieth

static int chunks_of(long page_bytes) { return (int)((page_bytes + kCopyBytes - 1) / kCopyBytes); }

// Sum over the block and of the threads before this one; `scratch` a word a wave.  All threads call it.
__device__ __forceinline__ int block_scan(int v, int *scratch, int *total)
{
    constexpr int kWaves = kPlanThreads / 64;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, s = wave_scan(v);
    __syncthreads();                                          // (scratch may still be read from the scan before)
    if (lane == 63) scratch[wave] = s;
    __syncthreads();
    const int mine = lane < kWaves ? scratch[lane] : 0, sums = wave_scan(mine);
    *total = __builtin_amdgcn_readlane(sums, 63);
    return __builtin_amdgcn_readlane(sums - mine, __builtin_amdgcn_readfirstlane(wave)) + s - v;
}

__device__ __forceinline__ void copy_chunk(const unsigned char *src, unsigned char *dst, long page_bytes, int chunk)
{
    const long at = (long)chunk * kCopyBytes + threadIdx.x * 16;
    word4_t v[kCopyPieces];
#pragma unroll
    for (int i = 0; i < kCopyPieces; ++i)
        if (at + i * (kCopyThreads * 16) < page_bytes) v[i] = *reinterpret_cast<const word4_t *>(src + at + i * (kCopyThreads * 16));
#pragma unroll
    for (int i = 0; i < kCopyPieces; ++i)
        if (at + i * (kCopyThreads * 16) < page_bytes) *reinterpret_cast<word4_t *>(dst + at + i * (kCopyThreads * 16)) = v[i];
}

// The free ones of this thread's pages of the chunk that begins with page p0, a bit each.
__device__ __forceinline__ unsigned free_pages_of(const CacheArgs &c, int p0)
{
    unsigned is_free = 0;
#pragma unroll
    for (int k = 0; k < kRefsPerThread; ++k) {
        const int p = p0 + threadIdx.x * kRefsPerThread + k;
        is_free |= (p < c.pages && c.refs[p] == 0 ? 1u : 0u) << k;
    }
    return is_free;
}

// Deals out free pages, lowest first, to askers 0 .. n-1 that want need(i) each; who does not fit among the free ones together with all before it gets none.
// give(i, k, page): asker i's k-th page;  done(i, served) once for every asker, after its need() calls and before any give().  Returns the pages lacking.
// A chain of loads and scans in one block: the first chunk's reference counts are asked for before anything else, since they mostly suffice.
template <class Need, class Give, class Done>
__device__ __forceinline__ int deal_pages(const CacheArgs &c, int n, Need need, Give give, Done done)
{
    __shared__ int scratch[kPlanThreads / 64];
    __shared__ int first[kPlanThreads];
    const int tid = threadIdx.x;
    const unsigned free0 = free_pages_of(c, 0);
    int mine = tid < n ? need(tid) : 0, all, before = block_scan(mine, scratch, &all);
    long wanted = all;
    for (int i0 = kPlanThreads; i0 < n; i0 += kPlanThreads) {
        int some;
        block_scan(i0 + tid < n ? need(i0 + tid) : 0, scratch, &some);
        wanted += some;
    }
    long free_pages = 0;                                      // found; counted on only while fewer than wanted
    int rank_of0 = 0, found0 = 0;
    if (wanted > 0) {
        rank_of0 = block_scan(__popc(free0), scratch, &found0);
        free_pages = found0;
        for (int p0 = kRefsChunk; p0 < c.pages && free_pages < wanted; p0 += kRefsChunk) {
            int some;
            block_scan(__popc(free_pages_of(c, p0)), scratch, &some);
            free_pages += some;
        }
    }
    long dealt = 0;
    int p0 = 0;                                               // pages before this chunk are all taken
    for (int i0 = 0; i0 < n; i0 += kPlanThreads) {
        const int i = i0 + tid;
        if (i0) {
            mine = i < n ? need(i) : 0;
            before = block_scan(mine, scratch, &all);
        }
        const bool served = mine == 0 || dealt + before + mine <= free_pages;
        int give_total = all;                                        // who is served comes first: their ranks are `first`'s
        if (wanted > free_pages) block_scan(served ? mine : 0, scratch, &give_total);
        first[tid] = before;
        if (i < n) done(i, served);
        __syncthreads();
        int rank0 = 0;
        while (rank0 < give_total && p0 < c.pages) {
            const bool again = i0 > 0 || p0 > 0;                     // (the first chunk, before anything was dealt from it, is known)
            const unsigned is_free = again ? free_pages_of(c, p0) : free0;
            int found = found0, rank = rank0 + (again ? block_scan(__popc(is_free), scratch, &found) : rank_of0);   // (its barriers lie between reads of refs and writes)
#pragma unroll
            for (int k = 0; k < kRefsPerThread; ++k) {
                if (!(is_free >> k & 1)) continue;
                if (rank < give_total) {
                    int lo = 0, hi = min(kPlanThreads, n - i0);      // the last asker with first[lo] <= rank
                    while (hi - lo > 1) {
                        const int mid = (lo + hi) >> 1;
                        if (first[mid] <= rank) lo = mid;
                        else hi = mid;
                    }
                    const int p = p0 + tid * kRefsPerThread + k;
                    c.refs[p] = 1;
                    give(i0 + lo, rank - first[lo], p);
                }
                ++rank;
            }
            rank0 += found;
            if (rank0 < give_total) p0 += kRefsChunk;                // (else the rest of this chunk serves the next askers)
            __syncthreads();
        }
        dealt += all;
    }
    return (int)(wanted > free_pages ? wanted - free_pages : 0);
}

__global__ __launch_bounds__(kPlanThreads) void fbq_reserve_kernel(CacheArgs c, const int32_t *__restrict__ count, int32_t *__restrict__ start, int32_t *info)
{
    const int ps1 = (1 << c.log_ps) - 1, most = c.max_pages << c.log_ps;
    const auto held = [&](int i) { return tokens_of(c.lengths[i], most); };
    const auto fits = [&](int i) { return max(count[i], 0) <= most - held(i); };
    const auto need = [&](int i) { return fits(i) ? ((held(i) + max(count[i], 0) + ps1) >> c.log_ps) - ((held(i) + ps1) >> c.log_ps) : 0; };
    // lengths change only behind the last use: need() of an asker's chunk comes before its done(), give() looks at start
    const int lacking = deal_pages(
        c, c.rows, need,
        [&](int i, int k, int page) { c.table[(long)i * c.max_pages + ((start[i] + ps1) >> c.log_ps) + k] = page; },
        [&](int i, bool served) {
            const int n = held(i);
            served = served && fits(i);
            start[i] = served ? n : -1;
            c.lengths[i] = served ? n + max(count[i], 0) : n;
        });
    if (info && threadIdx.x == 0) info[0] = lacking;
}

// One block a token and 256 pieces: its row, its place there, and the pieces of all heads.
__global__ __launch_bounds__(256) void fbq_append_kernel(CacheArgs c, long layer_offset, const int32_t *__restrict__ q_start, const int32_t *__restrict__ start,
                                                         const uint16_t *__restrict__ k, long k_stride, const uint16_t *__restrict__ v, long v_stride)
{
    const int t = blockIdx.x;
    const int b = q_start ? row_of_token(q_start, c.rows, t) : t;
    if (b < 0) return;
    const int s = start[b];
    if (s < 0) return;
    const long pos = (long)s + (q_start ? t - q_start[b] : 0);
    if (pos >= (long)c.max_pages << c.log_ps) return;
    const int page = c.table[(long)b * c.max_pages + (pos >> c.log_ps)];
    if ((unsigned)page >= (unsigned)c.pages) return;
    const int pieces = c.D >> 3, slot = (int)pos & ((1 << c.log_ps) - 1);
    unsigned char *const to = c.pool + layer_offset + page * c.page_bytes;
    const word4_t *const ks = reinterpret_cast<const word4_t *>(k + t * k_stride), *const vs = reinterpret_cast<const word4_t *>(v + t * v_stride);
    for (int i = threadIdx.x; i < c.kv_heads * pieces; i += 256) {
        const int h = i / pieces, p = i - h * pieces;
        const long at = ((((long)h << c.log_ps) + slot) * c.D + p * 8) * 2;
        *reinterpret_cast<word4_t *>(to + at) = ks[i];
        *reinterpret_cast<word4_t *>(to + (c.page_bytes >> 1) + at) = vs[i];
    }
}

constexpr int kFreeEntries = 1024;            // of the table, a block

__global__ __launch_bounds__(256) void fbq_free_kernel(CacheArgs c, const int32_t *__restrict__ rows)
{
    const int b = rows[blockIdx.x];
    if ((unsigned)b >= (unsigned)c.rows) return;
    const int e1 = min(c.max_pages, (int)(blockIdx.y + 1) * kFreeEntries);
    for (int e = blockIdx.y * kFreeEntries + threadIdx.x; e < e1; e += 256) {
        int32_t *const at = c.table + (long)b * c.max_pages + e;
        const int page = *at;
        if ((unsigned)page < (unsigned)c.pages) atomicSub(c.refs + page, 1);
        *at = -1;
    }
    if (blockIdx.y == 0 && threadIdx.x == 0) c.lengths[b] = 0;
}

// Fork, first launch: which pairs are served, the page each partial last page is copied to.  plan[i] = {tokens, page or -1}; tokens -1: skipped.
__global__ __launch_bounds__(kPlanThreads) void fbq_fork_plan_kernel(CacheArgs c, int n, const int32_t *__restrict__ parent, const int32_t *__restrict__ child,
                                                                     int2 *__restrict__ plan, int32_t *info)
{
    __shared__ int skipped;
    const int ps1 = (1 << c.log_ps) - 1, most = c.max_pages << c.log_ps;
    if (threadIdx.x == 0) skipped = 0;
    for (int i = threadIdx.x; i < n; i += kPlanThreads) {     // lengths as they are before the call, also where a child is another pair's parent
        const int p = parent[i], q = child[i];
        const bool ok = (unsigned)p < (unsigned)c.rows && (unsigned)q < (unsigned)c.rows && p != q && c.lengths[q] == 0;
        plan[i] = make_int2(ok ? tokens_of(c.lengths[p], most) : -1, -1);
    }
    __syncthreads();
    const int lacking = deal_pages(
        c, n, [&](int i) { return plan[i].x > 0 && (plan[i].x & ps1) != 0 ? 1 : 0; }, [&](int i, int, int page) { plan[i].y = page; },
        [&](int i, bool served) {
            if (plan[i].x >= 0 && served) c.lengths[child[i]] = plan[i].x;
            else atomicAdd(&skipped, 1);
        });
    __syncthreads();
    if (info && threadIdx.x == 0) {
        info[0] = lacking;
        info[1] = skipped;
    }
}

// Second launch: block y = 0 of a pair shares the full pages, the others copy the partial last one, one chunk of one layer each.
__global__ __launch_bounds__(kCopyThreads) void fbq_fork_kernel(CacheArgs c, const int32_t *__restrict__ parent, const int32_t *__restrict__ child,
                                                                const int2 *__restrict__ plan, int chunks)
{
    const int i = blockIdx.x;
    const int2 pl = plan[i];
    if (pl.x <= 0) return;
    const int full = pl.x >> c.log_ps;
    const bool part = (pl.x & ((1 << c.log_ps) - 1)) != 0;
    if (part && pl.y < 0) return;                             // no page was left for it
    const int32_t *const from = c.table + (long)parent[i] * c.max_pages;
    if (blockIdx.y == 0) {
        int32_t *const to = c.table + (long)child[i] * c.max_pages;
        for (int e = threadIdx.x; e < full; e += kCopyThreads) {
            const int page = from[e];
            to[e] = page;
            if ((unsigned)page < (unsigned)c.pages) atomicAdd(c.refs + page, 1);
        }
        if (part && threadIdx.x == 0) to[full] = pl.y;
        return;
    }
    if (!part) return;
    const int src = from[full];
    if ((unsigned)src >= (unsigned)c.pages) return;
    for (int y = blockIdx.y - 1; y < c.layers * chunks; y += kGridChunks) {
        unsigned char *const layer = c.pool + (y / chunks) * c.layer_bytes;
        copy_chunk(layer + src * c.page_bytes, layer + pl.y * c.page_bytes, c.page_bytes, y % chunks);
    }
}

__global__ __launch_bounds__(kCopyThreads) void fbq_copy_pages_kernel(CacheArgs c, const int32_t *__restrict__ src, const int32_t *__restrict__ dst, int chunks)
{
    const int s = src[blockIdx.x], d = dst[blockIdx.x];
    if ((unsigned)s >= (unsigned)c.pages || (unsigned)d >= (unsigned)c.pages) return;
    for (int y = blockIdx.y; y < c.layers * chunks; y += kGridChunks) {
        unsigned char *const layer = c.pool + (y / chunks) * c.layer_bytes;
        copy_chunk(layer + s * c.page_bytes, layer + d * c.page_bytes, c.page_bytes, y % chunks);
    }
}

// Compaction.  With n pages in use: the k-th free page below n (a hole) gets the k-th page in use from n up (a mover).
// Workspace: {n, moves}, then pages in use by chunk of kRefsChunk, then holes [pages], movers [pages], rank of a mover by page [pages].
struct CompactPlan {
    int32_t *head, *chunk, *holes, *movers, *rank;
    int chunks;
};

__global__ __launch_bounds__(kPlanThreads) void fbq_count_pages_kernel(CacheArgs c, CompactPlan w)
{
    __shared__ int scratch[kPlanThreads / 64];
    int mine = 0, all;
#pragma unroll
    for (int k = 0; k < kRefsPerThread; ++k) {
        const int p = blockIdx.x * kRefsChunk + threadIdx.x * kRefsPerThread + k;
        mine += p < c.pages && c.refs[p] > 0;
    }
    block_scan(mine, scratch, &all);
    if (threadIdx.x == 0) w.chunk[blockIdx.x] = all;
}

__global__ __launch_bounds__(kPlanThreads) void fbq_compact_plan_kernel(CacheArgs c, CompactPlan w, int32_t *refs_out, int32_t *info)
{
    __shared__ int scratch[kPlanThreads / 64];
    const int tid = threadIdx.x;
    int live = 0, before = 0;                                 // pages in use in all, and below this chunk
    bool used[kRefsPerThread];
    int refs[kRefsPerThread], mine = 0, all;
#pragma unroll
    for (int k = 0; k < kRefsPerThread; ++k) {
        const int p = blockIdx.x * kRefsChunk + tid * kRefsPerThread + k;
        refs[k] = p < c.pages ? c.refs[p] : 0;
        used[k] = refs[k] > 0;
        mine += used[k];
    }
    int at = block_scan(mine, scratch, &live);                // pages in use below this thread's, in this chunk
    if (w.chunks > 1) live = 0;
    for (int i0 = 0; w.chunks > 1 && i0 < w.chunks; i0 += kPlanThreads) {
        const int x = i0 + tid < w.chunks ? w.chunk[i0 + tid] : 0;
        int all, below;
        block_scan(x, scratch, &all);
        block_scan(i0 + tid < (int)blockIdx.x ? x : 0, scratch, &below);
        live += all;
        before += below;
    }
    // pages in use below n: whole chunks, and the part of the one that n lies in (a single chunk has not been counted: all of it is the part)
    const int cut = w.chunks > 1 ? live / kRefsChunk : 0;
    int low = 0;
    for (int i0 = 0; i0 < cut; i0 += kPlanThreads) {
        int all;
        block_scan(i0 + tid < cut ? w.chunk[i0 + tid] : 0, scratch, &all);
        low += all;
    }
    mine = 0;
#pragma unroll
    for (int k = 0; k < kRefsPerThread; ++k) {
        const int p = cut * kRefsChunk + tid * kRefsPerThread + k;
        mine += p < live && p < c.pages && c.refs[p] > 0;
    }
    block_scan(mine, scratch, &all);
    low += all;
    at += before;                                             // ... of all
#pragma unroll
    for (int k = 0; k < kRefsPerThread; ++k) {
        const int p = blockIdx.x * kRefsChunk + tid * kRefsPerThread + k;
        if (p < c.pages) {
            if (p < live && !used[k]) w.holes[p - at] = p;
            else if (p >= live && used[k]) {
                w.movers[at - low] = p;
                w.rank[p] = at - low;
            } else refs_out[p] = used[k] ? refs[k] : 0;       // (a page that stays, or a free one: in place, what it already is)
        }
        at += used[k];
    }
    if (blockIdx.x == 0 && tid == 0) {
        w.head[0] = live;
        w.head[1] = live - low;
        if (info) {
            info[0] = live;
            info[1] = live - low;
        }
    }
}

// Blocks 0 .. table_blocks - 1 rewrite the table and the movers' reference counts, the others move data.
__global__ __launch_bounds__(kCopyThreads) void fbq_compact_kernel(CacheArgs c, CompactPlan w, int32_t *table_out, int32_t *refs_out, int table_blocks, int chunks)
{
    const int live = w.head[0], moves = w.head[1];
    if ((int)blockIdx.x < table_blocks) {
        const long entries = (long)c.rows * c.max_pages, step = (long)table_blocks * kCopyThreads;
        for (long e = (long)blockIdx.x * kCopyThreads + threadIdx.x; e < entries; e += step) {
            const int page = c.table[e];
            int to = page;
            if (page >= live && page < c.pages) {
                const int k = w.rank[page];                   // (not written for a page that no row should hold: then any number)
                to = (unsigned)k < (unsigned)moves && w.movers[k] == page ? w.holes[k] : page;
            }
            table_out[e] = to;
        }
        for (int k = blockIdx.x * kCopyThreads + threadIdx.x; k < moves; k += (int)step) {
            const int v = c.refs[w.movers[k]];
            refs_out[w.holes[k]] = v;
            refs_out[w.movers[k]] = 0;
        }
        return;
    }
    const long pieces = (long)moves * c.layers * chunks;
    for (long i = blockIdx.x - table_blocks; i < pieces; i += gridDim.x - table_blocks) {
        const long q = i / chunks;
        const int chunk = (int)(i - q * chunks), k = (int)(q / c.layers), l = (int)(q - (long)k * c.layers);
        unsigned char *const layer = c.pool + l * c.layer_bytes;
        copy_chunk(layer + w.movers[k] * c.page_bytes, layer + w.holes[k] * c.page_bytes, c.page_bytes, chunk);
    }
}

static CompactPlan compact_plan(const fbq_cache_desc &d, void *workspace)
{
    CompactPlan w{};
    w.chunks = ceil_div(d.pages, kRefsChunk);
    w.head = (int32_t *)workspace;
    w.chunk = w.head + 4;
    w.holes = w.chunk + ceil_div(w.chunks, 4) * 4;
    w.movers = w.holes + d.pages;
    w.rank = w.movers + d.pages;
    return w;
}

fbq_status check_cache(const fbq_cache *c, bool refs)
{
    if (!c) return FBQ_ERR_NULL;
    const fbq_status st = fbq_check_cache(&c->desc);
    if (st != FBQ_OK) return st;
    if (c->rows < 1 || c->rows > 65536 || c->max_pages < 1) return FBQ_ERR_SHAPE;
    const long tokens = (long)c->max_pages * c->desc.page_size;
    if (tokens > (1L << 24) || (c->rows + 1L) * c->desc.kv_heads * (tokens / 32 + 1) >= (1L << 30)) return FBQ_ERR_UNSUPPORTED;
    if (!c->pool || !c->table || !c->lengths || (refs && !c->refs)) return FBQ_ERR_NULL;
    if (!aligned(c->pool, 16) || !aligned(c->table, 4) || !aligned(c->lengths, 4) || !aligned(c->refs, 4)) return FBQ_ERR_ALIGN;
    return FBQ_OK;
}

static fbq_status launched() { return hipGetLastError() == hipSuccess ? FBQ_OK : FBQ_ERR_HIP; }

}  // namespace fbq

using namespace fbq;

extern "C" fbq_status fbq_check_cache(const fbq_cache_desc *d)
{
    if (!d) return FBQ_ERR_NULL;
    if (d->layers < 1 || d->layers > 4096 || d->pages < 1 || d->pages > (1 << 22) || d->kv_heads < 1 || d->kv_heads > 1024) return FBQ_ERR_SHAPE;
    if (d->head_dim < 16 || d->head_dim > 256 || d->head_dim % 8) return FBQ_ERR_SHAPE;
    if (d->page_size < 16 || d->page_size > 256 || (d->page_size & (d->page_size - 1))) return FBQ_ERR_UNSUPPORTED;
    if (d->type != FBQ_F16 && d->type != FBQ_BF16) return FBQ_ERR_UNSUPPORTED;
    return FBQ_OK;
}

extern "C" size_t fbq_cache_bytes(const fbq_cache_desc *d)
{
    if (fbq_check_cache(d) != FBQ_OK) return 0;
    return 4 * (size_t)d->kv_heads * d->page_size * d->head_dim * d->pages * d->layers;
}

extern "C" size_t fbq_cache_workspace_bytes(const fbq_cache_desc *d, int n)
{
    if (fbq_check_cache(d) != FBQ_OK || n < 0) return 0;
    if (n > 0) return (size_t)n * sizeof(int2);
    return 4 * (4 + (size_t)ceil_div(ceil_div(d->pages, kRefsChunk), 4) * 4 + 3 * (size_t)d->pages);   // (see compact_plan)
}

extern "C" fbq_status fbq_cache_reserve(const fbq_cache *c, const int32_t *count, int32_t *start, int32_t *info, fbq_stream stream)
{
    const fbq_status st = check_cache(c, true);
    if (st != FBQ_OK) return st;
    if (!count || !start) return FBQ_ERR_NULL;
    if (!aligned(count, 4) || !aligned(start, 4) || !aligned(info, 4)) return FBQ_ERR_ALIGN;
    hipLaunchKernelGGL(fbq_reserve_kernel, dim3(1), dim3(kPlanThreads), 0, (hipStream_t)stream, cache_args(*c), count, start, info);
    return launched();
}

extern "C" fbq_status fbq_cache_append(const fbq_cache *c, int layer, int T, const int32_t *q_start, const int32_t *start, const void *k, int64_t k_stride,
                                       const void *v, int64_t v_stride, fbq_stream stream)
{
    const fbq_status st = check_cache(c, false);
    if (st != FBQ_OK) return st;
    const int64_t row = (int64_t)c->desc.kv_heads * c->desc.head_dim;
    if (layer < 0 || layer >= c->desc.layers || T < 1 || T > (1 << 23) || (!q_start && T != c->rows)) return FBQ_ERR_SHAPE;
    if (k_stride < row || v_stride < row || k_stride % 8 || v_stride % 8 || k_stride > (1L << 32) || v_stride > (1L << 32)) return FBQ_ERR_SHAPE;
    if (!start || !k || !v) return FBQ_ERR_NULL;
    if (!aligned(q_start, 4) || !aligned(start, 4) || !aligned(k, 16) || !aligned(v, 16)) return FBQ_ERR_ALIGN;
    const CacheArgs a = cache_args(*c);
    hipLaunchKernelGGL(fbq_append_kernel, dim3(T), dim3(256), 0, (hipStream_t)stream, a, layer * a.layer_bytes, q_start, start, (const uint16_t *)k, (long)k_stride,
                       (const uint16_t *)v, (long)v_stride);
    return launched();
}

extern "C" fbq_status fbq_cache_free(const fbq_cache *c, int n, const int32_t *rows, fbq_stream stream)
{
    const fbq_status st = check_cache(c, true);
    if (st != FBQ_OK) return st;
    if (n < 1 || n > 65536) return FBQ_ERR_SHAPE;
    if (!rows) return FBQ_ERR_NULL;
    if (!aligned(rows, 4)) return FBQ_ERR_ALIGN;
    hipLaunchKernelGGL(fbq_free_kernel, dim3(n, ceil_div(c->max_pages, kFreeEntries)), dim3(256), 0, (hipStream_t)stream, cache_args(*c), rows);
    return launched();
}

extern "C" fbq_status fbq_cache_fork(const fbq_cache *c, int n, const int32_t *parent, const int32_t *child, int32_t *info, void *workspace, size_t workspace_bytes,
                                     fbq_stream stream)
{
    const fbq_status st = check_cache(c, true);
    if (st != FBQ_OK) return st;
    if (n < 1 || n > 65536) return FBQ_ERR_SHAPE;
    if (!parent || !child || !workspace) return FBQ_ERR_NULL;
    if (!aligned(parent, 4) || !aligned(child, 4) || !aligned(info, 4) || !aligned(workspace, 16)) return FBQ_ERR_ALIGN;
    if (workspace_bytes < fbq_cache_workspace_bytes(&c->desc, n)) return FBQ_ERR_WORKSPACE;
    const CacheArgs a = cache_args(*c);
    const int chunks = chunks_of(a.page_bytes);
    hipLaunchKernelGGL(fbq_fork_plan_kernel, dim3(1), dim3(kPlanThreads), 0, (hipStream_t)stream, a, n, parent, child, (int2 *)workspace, info);
    hipLaunchKernelGGL(fbq_fork_kernel, dim3(n, 1 + std::min(a.layers * chunks, kGridChunks)), dim3(kCopyThreads), 0, (hipStream_t)stream, a, parent, child, (const int2 *)workspace, chunks);
    return launched();
}

extern "C" fbq_status fbq_cache_copy(const fbq_cache *c, int n, const int32_t *src, const int32_t *dst, fbq_stream stream)
{
    const fbq_status st = check_cache(c, false);
    if (st != FBQ_OK) return st;
    if (n < 1 || n > (1 << 22)) return FBQ_ERR_SHAPE;
    if (!src || !dst) return FBQ_ERR_NULL;
    if (!aligned(src, 4) || !aligned(dst, 4)) return FBQ_ERR_ALIGN;
    const CacheArgs a = cache_args(*c);
    const int chunks = chunks_of(a.page_bytes);
    hipLaunchKernelGGL(fbq_copy_pages_kernel, dim3(n, std::min(a.layers * chunks, kGridChunks)), dim3(kCopyThreads), 0, (hipStream_t)stream, a, src, dst, chunks);
    return launched();
}

extern "C" fbq_status fbq_cache_compact(const fbq_cache *c, int32_t *table_out, int32_t *refs_out, int32_t *info, void *workspace, size_t workspace_bytes,
                                        fbq_stream stream)
{
    const fbq_status st = check_cache(c, true);
    if (st != FBQ_OK) return st;
    if (!table_out || !refs_out || !workspace) return FBQ_ERR_NULL;
    if (!aligned(table_out, 4) || !aligned(refs_out, 4) || !aligned(info, 4) || !aligned(workspace, 16)) return FBQ_ERR_ALIGN;
    if (workspace_bytes < fbq_cache_workspace_bytes(&c->desc, 0)) return FBQ_ERR_WORKSPACE;
    const CacheArgs a = cache_args(*c);
    const CompactPlan w = compact_plan(c->desc, workspace);
    const int chunks = chunks_of(a.page_bytes);
    const int table_blocks = (int)std::min<long>(256, (std::max((long)a.rows * a.max_pages, (long)a.pages) + kCopyThreads * 4 - 1) / (kCopyThreads * 4));
    const long most = (long)(a.pages / 2) * a.layers * chunks;
    if (w.chunks > 1) hipLaunchKernelGGL(fbq_count_pages_kernel, dim3(w.chunks), dim3(kPlanThreads), 0, (hipStream_t)stream, a, w);
    hipLaunchKernelGGL(fbq_compact_plan_kernel, dim3(w.chunks), dim3(kPlanThreads), 0, (hipStream_t)stream, a, w, refs_out, info);
    hipLaunchKernelGGL(fbq_compact_kernel, dim3(table_blocks + (unsigned)std::min<long>(2048, most)), dim3(kCopyThreads), 0, (hipStream_t)stream, a, w, table_out,
                       refs_out, table_blocks, chunks);
    return launched();
}
