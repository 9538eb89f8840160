// fbq_cache_evict: rows cut back to the tokens that matter, each layer and key/value head by its own weights.
//
// Three launches: which tokens of each layer, row and head stay, and their weights; the tokens moved; tables, lengths and pages.  What is cut back is decided by the first from the pages as they
// are before the call, by every block for its row.
// Choosing: the least weight that stays is found 11 bits at a time from counts of the digits in LDS (whole numbers: their order does not matter); of those equal to it the earliest stay.
// Moving is in place: position i takes token src[i] >= i.  A block has some columns - 128 bytes of every key, say - of one row and head to itself and goes through the positions upwards: a
// round's tokens are read before the round before it is written, and all that is written lies before all that is still to be read.  Bound by HBM: every token that moves is read and written
// once.  16 rows of up to 1280 tokens to 1024, 4 layers of 8 heads of 128 in 16 bits: 105 us for 533 MB (5.0 TB/s, as a large copy).  3 rows of up to 8500 to 6000, heads of 80: 89 for 370 MB, few
// blocks that go through long rows.  In 4 bits 59 for 149 MB and 73 for 129 MB: pieces of 64 bytes, scales of 4, value codes byte by byte.  One token a row over 1024 of the 16 rows, what a decode loop cuts
// back each step, takes 65 and 57: all tokens are read, those behind the one that goes are written.  Choosing takes 9 to 15 us for rows up to 2048, 22 for 8500: three passes over the digits and one over the tokens, each a few barriers.
#include <algorithm>

#include "fbq_attend.h"
#include "fbq_cache4.h"
#include "fbq_internal.h"

namespace fbq {

constexpr int kChooseEach = 4;           // weights a thread and round of the choosing
constexpr int kShortRows = 2048;         // up to so many weights a row a block of 256 chooses, else one of 1024
constexpr int kDigits = 2048;
template <bool FOUR>
constexpr int kMoveThreads = FOUR ? 256 : 512;                // (4 bits: what four threads a token, and sixteen four tokens, count on)
constexpr int kEvictBlocks = 1 << 20;    // of a grid at most; they go on with every so manieth item

struct EvictArgs {
    CacheArgs c;
    const float *weights;
    float *weights_out;
    long layer_stride;
    const int32_t *keep;
    int width, first, recent;
    int32_t *rows;                       // tokens of a row that is cut back, -1: left as it is, -2: skipped
    int32_t *src;                        // [items][width]: where the tokens that stay lie, page * page_size + place in it
    long items;                          // layers x rows x heads
};

// Tokens of row b if it is to be cut back, else -1, or -2 if it cannot be (see fbq.h).  The whole block calls it.
template <int THREADS>
__device__ __forceinline__ int tokens_to_cut(const EvictArgs &e, int b, int *scratch)
{
    const CacheArgs &c = e.c;
    const int tokens = tokens_of(c.lengths[b], c.max_pages << c.log_ps), keep = e.keep[b];
    if (keep < 0 || keep >= tokens) return -1;
    if (tokens > e.width || (long)e.first + e.recent > keep) return -2;
    const int pages = (tokens + (1 << c.log_ps) - 1) >> c.log_ps;
    bool bad = false;
    for (int i = (e.first >> c.log_ps) + threadIdx.x; i < pages; i += THREADS) {
        const int page = c.table[(long)b * c.max_pages + i];
        bad |= (unsigned)page >= (unsigned)c.pages || c.refs[page] != 1;
    }
    __syncthreads();                                          // (scratch may still be read)
    if ((threadIdx.x & 63) == 0) scratch[threadIdx.x >> 6] = 0;
    if (__ballot(bad) && (threadIdx.x & 63) == 0) scratch[threadIdx.x >> 6] = 1;
    __syncthreads();
    for (int w = 0; w < THREADS / 64; ++w)
        if (scratch[w]) return -2;
    return tokens;
}

// Sum over the threads before this one, and of all; all threads call it.
template <int THREADS>
__device__ __forceinline__ int block_before(int v, int *scratch, int *total)
{
    constexpr int kWaves = THREADS / 64;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, s = wave_scan(v);
    __syncthreads();
    if (lane == 63) scratch[wave] = s;
    __syncthreads();
    const int mine = lane < kWaves ? scratch[lane] : 0, sums = wave_scan(mine);
    *total = __builtin_amdgcn_readlane(sums, 63);
    return __builtin_amdgcn_readlane(sums - mine, uniform(wave)) + s - v;
}

// A weight as a whole number in the order of weights; what is no number is the least.
__device__ __forceinline__ uint32_t order_of(float x)
{
    if (!(x == x)) return 0;
    const uint32_t u = __builtin_bit_cast(uint32_t, x + 0.0f);             // (no zero with a sign)
    return u >> 31 ? ~u : u | 0x80000000u;
}

template <int THREADS>
__global__ __launch_bounds__(THREADS) void fbq_evict_choose_kernel(const EvictArgs e)
{
    constexpr int kHeld = THREADS == 256 ? kShortRows : 16384, kOwn = kDigits / THREADS;   // weights kept in LDS; digits of a thread
    __shared__ int counts[kDigits], scratch[THREADS / 64], found[2];
    __shared__ uint32_t held[kHeld];
    const CacheArgs &c = e.c;
    const int tid = threadIdx.x;
    for (long item = blockIdx.x; item < e.items; item += gridDim.x) {
        const long of_layer = (long)c.rows * c.kv_heads, layer = item / of_layer, rest = item - layer * of_layer;
        const int b = (int)(rest / c.kv_heads), tokens = tokens_to_cut<THREADS>(e, b, scratch);
        if (layer == 0 && rest == (long)b * c.kv_heads && tid == 0) e.rows[b] = tokens;
        if (tokens < 0) continue;
        const long at = layer * e.layer_stride + rest * e.width;
        const float *const from = e.weights + at;
        float *const to = e.weights_out + at;
        int32_t *const src = e.src + item * e.width;
        const int32_t *const list = c.table + (long)b * c.max_pages;
        const int first = e.first, end = tokens - e.recent, keep = e.keep[b];
        int wanted = keep - first - e.recent;                 // of the middle, first <= j < end (more than those: some go)
        uint32_t least = wanted > 0 ? 0 : 0xffffffffu, mask = 0;           // what all weights that may still be the least one that stays begin with (or above every weight)
        for (int shift = 21; wanted > 0 && shift >= -1; shift -= 11) {
            const int low = max(shift, 0);                    // the last digit has ten bits
#pragma unroll
            for (int i = 0; i < kOwn; ++i) counts[tid + i * THREADS] = 0;
            __syncthreads();
            for (int j = first + tid; j < end; j += THREADS) {
                uint32_t u;
                if (shift == 21) {
                    u = order_of(from[j]);
                    if (j - first < kHeld) held[j - first] = u;
                } else {
                    u = j - first < kHeld ? held[j - first] : order_of(from[j]);
                }
                if ((u & mask) == least) atomicAdd(&counts[u >> low & (shift < 0 ? 1023 : 2047)], 1);
            }
            __syncthreads();
            int own[kOwn], mine = 0, total;                   // digits from the largest down
#pragma unroll
            for (int i = 0; i < kOwn; ++i) mine += own[i] = counts[kDigits - 1 - (tid * kOwn + i)];
            int above = block_before<THREADS>(mine, scratch, &total);
#pragma unroll
            for (int i = 0; i < kOwn; ++i) {
                if (above < wanted && above + own[i] >= wanted) {
                    found[0] = kDigits - 1 - (tid * kOwn + i);
                    found[1] = above;
                }
                above += own[i];
            }
            __syncthreads();
            least |= (uint32_t)found[0] << low;
            mask |= (shift < 0 ? 1023u : 2047u) << low;
            wanted -= found[1];
            __syncthreads();
        }
        // those larger than `least` stay, and the first `wanted` of those equal to it
        int larger = 0, equal = 0;                            // so far
        for (int j0 = 0; j0 < tokens; j0 += THREADS * kChooseEach) {
            float w[kChooseEach];
            bool over[kChooseEach], same[kChooseEach];
            int mine = 0, all;
#pragma unroll
            for (int i = 0; i < kChooseEach; ++i) {
                const int j = j0 + tid * kChooseEach + i;
                w[i] = j < tokens ? from[j] : 0;
                const bool always = j < first || (j >= end && j < tokens), middle = j >= first && j < end;
                const uint32_t u = order_of(w[i]);
                over[i] = always || (middle && u > least);
                same[i] = middle && u == least && wanted > 0;
                mine += over[i] + (same[i] << 16);
            }
            const int before = block_before<THREADS>(mine, scratch, &all);    // (all reads of the chunk are done behind it)
            int o = larger + (before & 0xffff), s = equal + (before >> 16);
#pragma unroll
            for (int i = 0; i < kChooseEach; ++i) {
                const int j = j0 + tid * kChooseEach + i;
                if (over[i] || (same[i] && s < wanted)) {
                    const int place = o + min(s, max(wanted, 0));
                    src[place] = list[j >> c.log_ps] << c.log_ps | (j & ((1 << c.log_ps) - 1));
                    to[place] = w[i];
                }
                o += over[i];
                s += same[i];
            }
            larger += all & 0xffff;
            equal += all >> 16;
        }
        __syncthreads();
        for (int j = keep + tid; j < tokens; j += THREADS) to[j] = 0;
        __syncthreads();
    }
}

// What a block has to itself of an item.  16 bits: 128 bytes of every key, or value, where they are so many lines of 128, else all of it: a line that two blocks write in parts goes out twice (in pieces of
// 64 bytes 16 rows of 1280 to 1024 tokens, 128 features, took 110 us for 105, 3 of 8500 to 6000, 80 features, 116 for 89).  4 bits, where wider pieces leave too few blocks (112 for 85 and 211 for
// 103, calls as a whole): 64 bytes of a key's codes, the four bytes each of a token's scales, or, of value codes, 16 words of every four tokens.
struct MovePart {
    bool values, codes;                  // codes: the value codes of 4 bits
    int at, end, row;                    // bytes at .. end of rows of `row` bytes (16 bits) or at .. at + 64 of it (4); of value codes the first word
    bool scales;
};
template <bool FOUR>
__host__ __device__ __forceinline__ int move_parts(int D)
{
    if (!FOUR) return 2 * (D % 64 ? 1 : D / 64);
    const int DS = features4(D);
    return (DS / 2 + 63) / 64 + DS / 32 + 2;
}
__host__ __device__ __forceinline__ long move_jobs(long items, int parts) { return (items + 7) / 8 * 8 * parts; }
template <bool FOUR>
__device__ __forceinline__ MovePart move_part(int D, int i)
{
    if (!FOUR) {
        const int n = D % 64 ? 1 : D / 64, width = 2 * D / n, at = i % n * width;
        return MovePart{i >= n, false, at, at + width, 2 * D, false};
    }
    const int DS = features4(D), n = (DS / 2 + 63) / 64;
    if (i < n) return MovePart{false, false, 64 * i, DS / 2, DS / 2, false};
    if (i < n + DS / 32) return MovePart{true, true, 16 * (i - n), 0, 0, false};
    return MovePart{i > n + DS / 32, false, 0, 4 * groups4(DS), 4 * groups4(DS), true};
}

// Rows of a token each: `step` tokens a pass, this thread's token of them `mine`, a piece W of it; EACH passes a round; two rounds' at a time.  place: of a token by where it lies; where: position i's.
template <class W, int EACH, class Place, class Where>
__device__ __forceinline__ void move_rows(const int32_t *__restrict__ src, int lowest, int keep, int step, int mine, bool there, Place place, Where where)
{
    constexpr int kEach = EACH;
    struct Round { int from[kEach]; W v[kEach]; };
    const auto read = [&](Round &x, int i0) __attribute__((always_inline)) {
#pragma unroll
        for (int y = 0; y < kEach; ++y) x.from[y] = src[min(i0 + y * step + mine, keep - 1)];
#pragma unroll
        for (int y = 0; y < kEach; ++y)
            if (there) x.v[y] = *reinterpret_cast<const W *>(place(x.from[y]));
    };
    const auto write = [&](const Round &x, int i0) __attribute__((always_inline)) {
#pragma unroll
        for (int y = 0; y < kEach; ++y) {
            const int i = i0 + y * step + mine, to = where(min(i, keep - 1));
            if (there && i < keep && to != x.from[y]) *reinterpret_cast<W *>(place(to)) = x.v[y];
        }
    };
    Round a, b;
    read(a, lowest);
    for (int i0 = lowest; i0 < keep; i0 += 2 * step * kEach) {
        read(b, i0 + step * kEach);
        __syncthreads();                                      // (all have read the round that is written, and those behind it read later lie behind it)
        write(a, i0);
        read(a, i0 + 2 * step * kEach);
        __syncthreads();
        write(b, i0 + step * kEach);
    }
}

template <bool FOUR>
__global__ __launch_bounds__(kMoveThreads<FOUR>, FOUR ? 2 : 4) void fbq_evict_move_kernel(const EvictArgs e)
{
    const CacheArgs &c = e.c;
    const int tid = threadIdx.x, ps1 = (1 << c.log_ps) - 1, parts = move_parts<FOUR>(c.D), DS = features4(c.D);
    const long head_bytes = (c.page_bytes >> 1) / c.kv_heads, jobs = move_jobs(e.items, parts);
    for (long job = blockIdx.x; job < jobs; job += gridDim.x) {
        // The parts of an item on one XCD: they share lines of 128 bytes in its L2.  Blocks go round the eight in turn, so eight items' parts are dealt out part by part.
        const long eight = job / (8 * parts);
        const int in_eight = (int)(job - eight * (8 * parts));
        const long item = eight * 8 + (in_eight & 7);
        if (item >= e.items) continue;
        const long of_layer = (long)c.rows * c.kv_heads, layer = item / of_layer, rest = item - layer * of_layer;
        const int b = (int)(rest / c.kv_heads), h = (int)(rest - (long)b * c.kv_heads);
        if (e.rows[b] < 0) continue;
        const MovePart part = move_part<FOUR>(c.D, in_eight >> 3);
        const int keep = e.keep[b];
        if (keep <= e.first) continue;                        // (nothing moves; with none kept there is no src, either)
        const int32_t *const src = e.src + item * e.width, *const list = c.table + (long)b * c.max_pages;
        unsigned char *const heads = c.pool + layer * c.layer_bytes + (part.values ? c.page_bytes >> 1 : 0) + h * head_bytes;
        const auto head_of = [&](int at) { return heads + (long)(at >> c.log_ps) * c.page_bytes; };                 // of a token by where it lies
        const auto where = [&](int i) { return list[i >> c.log_ps] << c.log_ps | (i & ps1); };
        if (!FOUR) {
            const int pieces = (part.end - part.at) / 16, step = kMoveThreads<FOUR> / pieces, mine = tid / pieces, at = part.at + (tid - mine * pieces) * 16;
            move_rows<word4_t, 6>(src, e.first, keep, step, mine, mine < step, [&](int token) { return head_of(token) + (long)(token & ps1) * part.row + at; }, where);
        } else if (part.scales) {
            const int at = (tid & 3) * 4;
            move_rows<uint32_t, 8>(src, e.first, keep, kMoveThreads<FOUR> / 4, tid >> 2, at < part.end, [&](int token) { return head_of(token) + scales_at4(c.log_ps, token & ps1, DS) + at; }, where);
        } else if (!part.codes) {
            const int at = part.at + (tid & 3) * 16;
            move_rows<word4_t, 8>(src, e.first, keep, kMoveThreads<FOUR> / 4, tid >> 2, at < part.end,
                                  [&](int token) { return head_of(token) + codes_at4(token & ps1, DS) + (token & 15) * part.row + at; }, where);
        } else {
            // four tokens' codes a word: each byte from where its token's is
            constexpr int kStep = kMoveThreads<FOUR> / 16, kEach = 4;
            const int word = part.at + (tid & 15), words = DS / 2;            // of each four tokens
            const auto place = [&](int token) {
                const int slot = token & ps1;
                return reinterpret_cast<uint32_t *>(head_of(token) + codes_at4(slot, DS)) + (slot >> 2 & 3) * words + word;
            };
            for (int q0 = e.first >> 2; 4 * q0 < keep; q0 += kStep * kEach) {
                uint32_t v[kEach][4], old[kEach];
                int j[kEach][4];
#pragma unroll
                for (int y = 0; y < kEach; ++y)
#pragma unroll
                    for (int k = 0; k < 4; ++k) j[y][k] = src[min(4 * (q0 + y * kStep + (tid >> 4)) + k, keep - 1)];
#pragma unroll
                for (int y = 0; y < kEach; ++y) {
                    const int i = 4 * (q0 + y * kStep + (tid >> 4));
                    old[y] = i < keep && i + 4 > keep ? *place(where(i)) : 0; // (places behind the last token stay as they are)
#pragma unroll
                    for (int k = 0; k < 4; ++k) v[y][k] = *place(j[y][k]);
                }
                __syncthreads();
#pragma unroll
                for (int y = 0; y < kEach; ++y) {
                    const int i = 4 * (q0 + y * kStep + (tid >> 4));
                    if (i >= keep) continue;
                    uint32_t to = 0;
#pragma unroll
                    for (int k = 0; k < 4; ++k) {
                        const int at = 8 * byte_of_token4(k);
                        to |= i + k < keep ? (v[y][k] >> 8 * byte_of_token4(j[y][k] & 3) & 0xff) << at : old[y] & 0xffu << at;
                    }
                    *place(where(i)) = to;
                }
            }
        }
    }
}

__global__ __launch_bounds__(256) void fbq_evict_rows_done_kernel(const EvictArgs e, int32_t *info)
{
    const CacheArgs &c = e.c;
    const int b = blockIdx.x;
    if (info && b == 0) {                                     // rows cut back, rows skipped
        __shared__ int done, skipped;
        if (threadIdx.x == 0) done = skipped = 0;
        __syncthreads();
        int d = 0, s = 0;
        for (int i = threadIdx.x; i < c.rows; i += 256) {
            d += e.rows[i] >= 0;
            s += e.rows[i] == -2;
        }
        if (d) atomicAdd(&done, d);
        if (s) atomicAdd(&skipped, s);
        __syncthreads();
        if (threadIdx.x == 0) {
            info[0] = done;
            info[1] = skipped;
        }
    }
    const int tokens = e.rows[b];
    if (tokens < 0) return;
    const int keep = e.keep[b], pages = (tokens + (1 << c.log_ps) - 1) >> c.log_ps;
    for (int i = ((keep + (1 << c.log_ps) - 1) >> c.log_ps) + threadIdx.x; i < pages; i += 256) {
        int32_t *const at = c.table + (long)b * c.max_pages + i;
        const int page = *at;
        if ((unsigned)page < (unsigned)c.pages) atomicSub(c.refs + page, 1);
        *at = -1;
    }
    if (threadIdx.x == 0) c.lengths[b] = keep;
}

}  // namespace fbq

using namespace fbq;

extern "C" size_t fbq_cache_evict_workspace_bytes(const fbq_cache *c, int32_t width)
{
    if (!c || fbq_check_cache(&c->desc) != FBQ_OK || c->rows < 1 || c->rows > 65536 || width < 1 || width > (1 << 24)) return 0;
    const long items = (long)c->desc.layers * c->rows * c->desc.kv_heads;
    return items > (1L << 31) ? 0 : ((size_t)c->rows * 4 + 255) / 256 * 256 + (size_t)items * width * 4;
}

extern "C" fbq_status fbq_cache_evict(const fbq_cache *c, const float *weights, float *weights_out, int64_t layer_stride, int32_t width, const int32_t *keep, int32_t first, int32_t recent,
                                      int32_t *info, void *workspace, size_t workspace_bytes, fbq_stream stream)
{
    const fbq_status st = check_cache(c, true);
    if (st != FBQ_OK) return st;
    const int64_t of_layer = (int64_t)c->rows * c->desc.kv_heads, items = of_layer * c->desc.layers;
    if (width < 1 || width > (1 << 24) || first < 0 || recent < 0 || first > (1 << 24) || recent > (1 << 24) || layer_stride < of_layer * width) return FBQ_ERR_SHAPE;
    if (items > (1L << 31) || layer_stride > (1L << 48)) return FBQ_ERR_UNSUPPORTED;
    if (!weights || !weights_out || !keep || !workspace) return FBQ_ERR_NULL;
    if (!aligned(weights, 4) || !aligned(weights_out, 4) || !aligned(keep, 4) || !aligned(info, 4) || !aligned(workspace, 16)) return FBQ_ERR_ALIGN;
    if (workspace_bytes < fbq_cache_evict_workspace_bytes(c, width)) return FBQ_ERR_WORKSPACE;
    const uintptr_t a_layer = (uintptr_t)of_layer * width * 4, apart = (uintptr_t)layer_stride * 4, all = (c->desc.layers - 1) * apart + a_layer, a = (uintptr_t)weights, b = (uintptr_t)weights_out;
    if (a != b && a < b + all && b < a + all) {               // one over a part of the other, unless each one's layers lie between the other's (rows of the same tensor)
        const uintptr_t on = (a < b ? b - a : a - b) % apart;
        if (on < a_layer || apart - on < a_layer) return FBQ_ERR_UNSUPPORTED;
    }
    EvictArgs e{};
    e.c = cache_args(*c);
    e.weights = weights; e.weights_out = weights_out; e.layer_stride = layer_stride; e.keep = keep; e.width = width; e.first = first; e.recent = recent;
    e.rows = (int32_t *)workspace;
    e.src = (int32_t *)((char *)workspace + ((size_t)c->rows * 4 + 255) / 256 * 256);
    e.items = items;
    const bool four = in_4_bits(c->desc.type);
    const long jobs = move_jobs(items, four ? move_parts<true>(e.c.D) : move_parts<false>(e.c.D));
    const hipStream_t s = (hipStream_t)stream;
    const unsigned blocks = (unsigned)std::min<long>(items, kEvictBlocks);
    if (std::min((long)width, (long)c->max_pages * c->desc.page_size) <= kShortRows) hipLaunchKernelGGL(fbq_evict_choose_kernel<256>, dim3(blocks), dim3(256), 0, s, e);
    else hipLaunchKernelGGL(fbq_evict_choose_kernel<1024>, dim3(blocks), dim3(1024), 0, s, e);
    hipError_t err = hipGetLastError();
    if (err == hipSuccess) {
        const dim3 grid((unsigned)std::min<long>(jobs, kEvictBlocks));
        if (four) hipLaunchKernelGGL(fbq_evict_move_kernel<true>, grid, dim3(kMoveThreads<true>), 0, s, e);
        else hipLaunchKernelGGL(fbq_evict_move_kernel<false>, grid, dim3(kMoveThreads<false>), 0, s, e);
        err = hipGetLastError();
    }
    if (err == hipSuccess) {
        hipLaunchKernelGGL(fbq_evict_rows_done_kernel, dim3(c->rows), dim3(256), 0, s, e, info);
        err = hipGetLastError();
    }
    return err == hipSuccess ? FBQ_OK : FBQ_ERR_HIP;
}
