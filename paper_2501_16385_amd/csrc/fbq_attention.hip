// fbq_attention: which kernels serve a call, where their partial results lie, and the kernel that joins these.
#include "fbq_attend.h"

namespace fbq {

constexpr int kJoinThreads = 256;

// The partial results of one query row, added up in an order that depends on their number alone, so that equal calls give equal bits:
//     out = sum_p o_p 2^(m_p - m) / sum_p l_p 2^(m_p - m),   m the largest m_p.   A part whose sum l is 0 saw nothing and has no o.
// Bound by the latency of a chain of loads - where the parts lie, then their m, l and o at once - so as many as possible are under way together: 64 rows of 67 parts 5.5 us (71.6 with a wave
// going through 256 one after the other), 4096 rows of 9 parts 8.8.

// The parts of an item of the few-row kernel's line: pieces of the workers first .. last, those of a whole block of workers as one (see few_together).
struct FewParts {
    int u0, first, last, block0, blocks, count;               // its first step; whole blocks from block0 on
    __device__ __forceinline__ void of(int u, int steps, int share)
    {
        u0 = u;
        first = u / share;
        last = steps ? (u + steps - 1) / share : first;
        block0 = (first + kFewWaves - 1) / kFewWaves;
        if (!few_together(block0, share, u0, u0 + steps)) ++block0;                       // (the first worker of it may have begun before the item)
        int end = (last + 1) / kFewWaves;                                                // behind the last block that lies before `last`'s end
        if (end > block0 && !few_together(end - 1, share, u0, u0 + steps)) --end;         // (the last worker may have less than its share of it)
        blocks = max(0, end - block0);
        count = steps ? last - first + 1 - (kFewWaves - 1) * blocks : 0;
    }
    // part p's place among the workers' places, two a worker
    __device__ __forceinline__ long place(int p, int share) const
    {
        const int before = blocks ? block0 * kFewWaves - first : count;                   // single ones in front of the blocks
        const int w = p < before ? first + p : p < before + blocks ? (block0 + p - before) * kFewWaves : first + p + (kFewWaves - 1) * blocks;
        return (long)w * 2 + ((long)w * share < u0 ? 1 : 0);
    }
};

// A block a row, LANES lanes a part, four features each.  The row's own part is either whole (written by its one piece: nothing left to do unless shared tokens come with it)
// or cut into the pieces of the few-row kernel's workers w0 .. w1, or of the many-row kernel.  THREADS: 256, or a wave where there are rows enough to fill the GPU with.
template <class TY, int LANES, int THREADS>
__global__ __launch_bounds__(THREADS) void fbq_join_pieces_kernel(const AttendArgs a, const bool few)
{
    constexpr int kGroups = THREADS / LANES, kAtOnce = 8;
    __shared__ float2 group_ml[kGroups];
    __shared__ float4_t group_o[kGroups][LANES];
    const int tid = threadIdx.x, lane = tid & 63;
    const int t = blockIdx.x / a.heads, head = blockIdx.x - t * a.heads, h = head / a.group, j = head - h * a.group;
    const int b = a.q_start ? row_of_token(a.q_start, a.rows, t) : t;
    if (b < 0) return;
    const int2 q = queries_of(a, b);
    const int i = t - q.x;
    if (i >= q.y) return;

    const long row = (long)t * a.heads + head, rows = (long)a.T * a.heads;
    int n_own, n_shared = a.part_shared.o ? a.shared_splits : 0;
    bool one_own;
    int share = 1;                                            // few-row kernel: steps a worker
    FewParts own{}, of_shared{};
    if (few) {
        int before = 0, all = 0;                              // steps of the rows before b, of all rows
        for (int x = lane; x < a.rows; x += 64) {
            const int steps = few_steps(a, x);
            all += steps;
            before += x < b ? steps : 0;
        }
        all = __builtin_amdgcn_readlane(wave_scan(all), 63);
        before = __builtin_amdgcn_readlane(wave_scan(before), 63);
        const int shared_steps = a.shared_here ? (a.n_shared + kFewTile - 1) / kFewTile : 0, steps = few_steps(a, b);
        share = few_share(a, (all + shared_steps) * a.kv_heads);
        own.of((shared_steps + before) * a.kv_heads + h * steps, steps, share);
        n_own = own.count;
        if (a.shared_here) {
            of_shared.of(h * shared_steps, shared_steps, share);
            n_shared = of_shared.count;
        }
        one_own = own.last == own.first && steps > 0;
        if (one_own && !a.whole.o) return;
    } else {
        n_own = many_pieces(a, many_steps(a, many_limit(a, row_tokens(a, b), q.y, (i * a.group + j) / kManyRows)), a.splits == 1 ? 1 << 30 : many_share(a));
        one_own = false;
        if (n_own == 1 && !n_shared) return;
    }
    const int n = n_shared + n_own;
    const auto part = [&](int p, long *at) {                  // where part p of the n lies
        if (p < n_shared) {
            if (!a.shared_here) return *at = p * rows + row, a.part_shared;
            if (of_shared.first == of_shared.last) return *at = row, a.whole_shared;
            return *at = of_shared.place(p, share) * a.slot_rows + t * a.group + j, a.piece;
        }
        if (!few) return *at = (p - n_shared) * rows + row, a.part;
        if (one_own) return *at = row, a.whole;
        return *at = own.place(p - n_shared, share) * a.slot_rows + i * a.group + j, a.piece;
    };

    float m = kNoScore, l = 0;
    float4_t o{0, 0, 0, 0};
    const int group = tid / LANES, d = (tid % LANES) * 4;
    for (int p0 = group; p0 < n; p0 += kGroups * kAtOnce) {
        float2 ml[kAtOnce];
        float4_t v[kAtOnce];
#pragma unroll
        for (int k = 0; k < kAtOnce; ++k) {                   // (past the end the last one again, without weight)
            long at;
            const Partials from = part(min(p0 + k * kGroups, n - 1), &at);
            ml[k] = from.ml[at];
            v[k] = *reinterpret_cast<const float4_t *>(from.o + at * a.D + min(d, a.D - 4));
            if (p0 + k * kGroups >= n) ml[k] = make_float2(kNoScore, 0.0f);
        }
        float to = m;
#pragma unroll
        for (int k = 0; k < kAtOnce; ++k) to = fmaxf(to, ml[k].x);
        const float by = __builtin_amdgcn_exp2f(m - to);
        m = to;
        l *= by;
        o *= by;
#pragma unroll
        for (int k = 0; k < kAtOnce; ++k) {
            const float times = __builtin_amdgcn_exp2f(ml[k].x - m);
            if (ml[k].y != 0) {                               // (not a number counts)
                l += ml[k].y * times;
                o += v[k] * times;
            }
        }
    }
    group_o[group][tid % LANES] = o;
    if (tid % LANES == 0) group_ml[group] = make_float2(m, l);
    __syncthreads();
    if (tid >= LANES || d >= a.D) return;
    m = kNoScore;
    for (int g = 0; g < kGroups; ++g) m = fmaxf(m, group_ml[g].x);
    l = 0;
    o = float4_t{0, 0, 0, 0};
    for (int g = 0; g < kGroups; ++g) {
        const float times = __builtin_amdgcn_exp2f(group_ml[g].x - m);
        l += group_ml[g].y * times;
        o += group_o[g][tid] * times;
    }
    o *= l == 0 ? 0.0f : 1.0f / l;
    *reinterpret_cast<word2_t *>(a.out + t * a.out_stride + head * a.D + d) = word2_t{TY::pack(o[0], o[1]), TY::pack(o[2], o[3])};
    if (a.lse && tid == 0) a.lse[row] = l == 0 ? -INFINITY : (m + __builtin_amdgcn_logf(l)) * 0.6931471805599453f;
}

// Many-row kernel, many rows: LANES lanes a row, four features each, its pieces one behind the other.  No more blocks than the GPU holds: what is cut they work out once, and in most
// calls of many rows it is nothing.
constexpr int kJoinBlocks = 2048;
template <class TY, int LANES>
__global__ __launch_bounds__(kJoinThreads) void fbq_join_splits_kernel(const AttendArgs a)
{
    const int share = a.splits == 1 ? 1 << 30 : many_share(a), n_shared = a.part_shared.o ? a.shared_splits : 0;
    if (!n_shared) {
        int longest = 0;                                      // steps of any row's last tile
        for (int b = threadIdx.x & 63; b < a.rows; b += 64) longest = max(longest, queries_of(a, b).y ? many_steps(a, row_tokens(a, b)) : 0);
        if (__ballot(longest > share) == 0) return;
    }
    const long rows = (long)a.T * a.heads;
    const int d = (threadIdx.x % LANES) * 4;
    if (d >= a.D) return;
    for (long row = (long)blockIdx.x * (kJoinThreads / LANES) + threadIdx.x / LANES; row < rows; row += (long)gridDim.x * (kJoinThreads / LANES)) {
        const int t = (int)(row / a.heads), b = a.q_start ? row_of_token(a.q_start, a.rows, t) : t;
        if (b < 0) continue;                                  // a token of no row
        const int2 q = queries_of(a, b);
        if (t - q.x >= q.y) continue;
        const int head = (int)(row - (long)t * a.heads), tile = ((t - q.x) * a.group + head % a.group) / kManyRows;
        const int n = n_shared + many_pieces(a, many_steps(a, many_limit(a, row_tokens(a, b), q.y, tile)), share);
        if (n == 1) continue;                                 // written by its one piece
        const auto part = [&](int p, long *at) { return p < n_shared ? (*at = p * rows + row, a.part_shared) : (*at = (p - n_shared) * rows + row, a.part); };
        float m = kNoScore, l = 0;
#pragma unroll 4
        for (int p = 0; p < n; ++p) {
            long at;
            const Partials from = part(p, &at);
            m = fmaxf(m, from.ml[at].x);
        }
        float4_t o{0, 0, 0, 0};
#pragma unroll 4
        for (int p = 0; p < n; ++p) {
            long at;
            const Partials from = part(p, &at);
            const float2 ml = from.ml[at];
            if (ml.y == 0) continue;
            const float by = __builtin_amdgcn_exp2f(ml.x - m);
            l += ml.y * by;
            o += *reinterpret_cast<const float4_t *>(from.o + at * a.D + d) * by;
        }
        o *= l == 0 ? 0.0f : 1.0f / l;
        *reinterpret_cast<word2_t *>(a.out + t * a.out_stride + head * a.D + d) = word2_t{TY::pack(o[0], o[1]), TY::pack(o[2], o[3])};
        if (a.lse && d == 0) a.lse[row] = l == 0 ? -INFINITY : (m + __builtin_amdgcn_logf(l)) * 0.6931471805599453f;
    }
}

template <class TY, int LANES>
static hipError_t launch_join(const AttendArgs &a, bool few, hipStream_t stream)
{
    const long rows = (long)a.T * a.heads, a_block = kJoinThreads / LANES;
    if (rows < 2048) hipLaunchKernelGGL((fbq_join_pieces_kernel<TY, LANES, kJoinThreads>), dim3((unsigned)rows), dim3(kJoinThreads), 0, stream, a, few);
    else if (few) hipLaunchKernelGGL((fbq_join_pieces_kernel<TY, LANES, 64>), dim3((unsigned)rows), dim3(64), 0, stream, a, few);
    else hipLaunchKernelGGL((fbq_join_splits_kernel<TY, LANES>), dim3((unsigned)std::min<long>(kJoinBlocks, (rows + a_block - 1) / a_block)), dim3(kJoinThreads), 0, stream, a);
    return hipGetLastError();
}

template <class TY>
static hipError_t launch_join(const AttendArgs &a, bool few, hipStream_t stream)
{
    return a.D <= 64 ? launch_join<TY, 16>(a, few, stream) : a.D <= 128 ? launch_join<TY, 32>(a, few, stream) : launch_join<TY, 64>(a, few, stream);
}

// Few-row kernel: whether an item goes whole to a wave (1) or a block (2), with nothing to join, or the steps of all are dealt out (0), by the room that a row of the table has.
// us, 64 query heads on 32 of 128 features, 1 / 2 / 0 (r: rows of 0.25 to 1.75 times as many tokens).  60 tokens: 2 rows 7.1 / 7.3 / 12.1, 32 rows 9.5 / 14.9 / 16.1, 128 r 29 / 52 / 43.
// 200: 2 rows 14.2 / 9.2 / 14.9, 16 17.2 / 13.6 / 22.8, 32 19.6 / 24.9 / 30.4, 64 r 43.5 / 47.5 / 50.3.  500: 2 rows 29 / 13.0 / 15.1, 16 35 / 25 / 33, 64 r 103 / 95 / 98.  1000: 2 rows
// 56 / 20.1 / 16.9, 8 62 / 25 / 32, 32 80 / 86 / 89, 16 r 101 / 57.5 / 55.7.  2000: 8 rows 119 / 44 / 55, but 16 r 198 / 110 / 96, where one row is all that is left at the end.
// In 4 bits, where what is streamed is a third and the join costs the same (a wave / a block / dealt out).  60 tokens: 256 items 8.9 / 9.1 / 13.2, 1024 8.9 / 16.9 / 15.5.  500: 256 22.6 / 12.5 /
// 18.2, 512 22.4 / 15.2 / 21.7, 1024 23.1 / 27.9 / 26.6.  1000: 256 38 / 16.4 / 21.5, 512 38 / 21.0 / 27.8, 1024 38.3 / 39.3 / 38.6; r 512 58 / 28.5 / 30.7.  2000: 128 68 / 24.4 / 22.8, 256 68 /
// 24.7 / 30.3, 512 68 / 33.4 / 42.8, but r 256 109 / 35.8 / 32.0.  4000: 128 129 / 40.6 / 29.5, 256 131 / 42 / 45.
static int few_direct(long items, long tokens, bool four)
{
    if (items > 1L << 22) return 0;                           // (a grid counts its threads in 32 bits)
    if (four) return tokens <= 1024 ? (items >= 1024 ? 1 : 2) : tokens <= 2048 && items >= 256 ? 2 : 0;
    if (tokens <= 256 && items >= 1024) return 1;
    return tokens <= 512 || (tokens <= 1024 && items >= 128) ? 2 : 0;
}

// Whether the shared tokens are taken apart from the rows' own: where few queries come with a row, and what is then not read again, `saved`, is worth the launches and joins.
// us apart / not, 128 features, 32 heads of 8 keys' unless stated.  Many-row kernel: 8 rows of 16 tokens behind 16384 shared 75 / 84, of 32 106 / 101, of 64 174 / 167; 4 of 16 behind 4096
// (50 MB) 40 / 35; 32 heads of 32, 32 rows of 20 behind 4096 97 / 195, of 64 210 / 220, of 128 410 / 303; 11 of 15, 16 heads of 96, behind 64 (5 MB) 23.6 / 8.9.  Few-row kernel: 8 of 4 behind 16384
// 33 / 97, 2 of 4 23 / 35, 4 of 4 behind 4096 18 / 21; 64 rows of 2000 behind 512 (129 MB) 97 / 106, behind 64 (17 MB) 94.0 / 93.7, but of 600 behind 64 38 / 28: there a row is a block's
// without a join.
// In 4 bits what is not read again is less than a third, and the many-row kernel makes its operands first; fp16, bf16, rows of 300 tokens of their own unless stated.  Many-row kernel for the shared tokens,
// single tokens in the same launch (up to 128 features): what it costs is a launch's time and the queries', so it is the shared tokens that count, 2048 and more: 8 rows behind 1024 17.7 / 17.3, 20.3 / 18.2,
// behind 2048 18.0 / 21.2, 20.4 / 21.2; 16 behind 1024 19.1 / 19.3, 21.7 / 20.2, behind 4096 (240 MiB as 16 bits) 20.7 / 29.6, 23.1 / 29.8; 64 behind 1024 (252 MiB) 27.5 / 22.6, 27.2 / 23.8, behind 2048
// 36.0 / 43.7, 36.7 / 43.8; where they save something: 16 of 8 heads to 1 behind 4096 (30 MiB) 18.9 / 17.3, behind 8192 (60) 19.1 / 21.0, 5 behind 2048 (32) 17.6 / 17.4; and the rows' own are few beside
// them: 16 of 2000 behind 2048 31.8 / 28.7, behind 4096 33.2 / 33.8, 35.5 / 33.6, but 64 of 2000 behind 2048 (504 MiB) 56.6 / 59.2.  Others by bytes: 4 tokens a row, 16 rows behind 4096 (240 MiB) 39.1 /
// 32.9, behind 8192 39.1 / 42.7; 8 tokens, 16 behind 4096 63.6 / 56.3, behind 8192 72 / 87; 20 tokens, 32 heads of 32, 16 behind 1024 (240 MiB) 59 / 57, 67 / 71, behind 2048 67 / 89; 256 features, 16 behind
// 2048 (240 MiB) 52 / 41, behind 4096 57 / 55, 54 / 55.  Few-row kernel: 2 of 4 behind 512 13.6 / 13.6, behind 2048 14.4 / 15.5, 4 of 4 behind 4096 16.4 / 18.4.
static bool worth_sharing(const fbq_attention_call &c, bool few, long row_queries)
{
    const fbq_cache_desc &d = c.cache.desc;
    const long tokens = (long)c.n_shared * d.page_size, saved = 4L * tokens * d.kv_heads * d.head_dim * (c.cache.rows - 1);
    if (saved == 0 || row_queries > 64) return false;
    if (in_4_bits(d.type) && (long)c.T * (c.heads / d.kv_heads) > kFewRows) {
        const long own = (long)c.cache.max_pages * d.page_size - tokens;      // room for a row's own
        return saved >= 256L << 20 || (few && row_queries == c.heads / d.kv_heads && d.head_dim <= 128 && tokens >= 2048 && tokens >= 4 * own && saved >= 48L << 20);
    }
    if (!few) return saved >= (row_queries > 32 ? 96L : 32L) << 20;
    return saved >= (few_direct((long)c.cache.rows * d.kv_heads, (long)c.cache.max_pages * d.page_size, in_4_bits(d.type)) ? 24L : 2L) << 20;
}

struct AttendPlan {
    AttendArgs a;
    bool few, shared_many, join;
    size_t bytes;
};

// From the call's sizes alone: its lengths are the device's.
static AttendPlan attend_plan(const fbq_attention_call &c, void *workspace)
{
    AttendPlan p{};
    AttendArgs &a = p.a;
    const CacheArgs cache = cache_args(c.cache);
    a.kv = cache.pool + c.layer * cache.layer_bytes;
    a.table = c.cache.table; a.lengths = c.cache.lengths; a.q_start = c.q_start; a.shared = c.shared;
    a.q = (const uint16_t *)c.q; a.out = (uint16_t *)c.out; a.lse = c.lse;
    a.page_bytes = cache.page_bytes; a.q_stride = c.q_stride; a.out_stride = c.out_stride;
    a.pages = cache.pages; a.log_ps = cache.log_ps; a.max_pages = cache.max_pages; a.rows = cache.rows; a.kv_heads = cache.kv_heads; a.D = cache.D;
    a.heads = c.heads; a.group = c.heads / a.kv_heads; a.T = c.T; a.max_q = c.q_start ? c.max_q : 1;
    a.scale = c.scale == 0 ? 1.0f : std::fabs(c.scale) * 1.4426950408889634f;
    a.q_and = c.scale == 0 ? 0u : 0xffffffffu;
    a.q_xor = c.scale < 0 ? 0x80008000u : 0u;

    const long row_queries = (long)a.max_q * a.group, all_queries = (long)a.T * a.group;   // of one key/value head
    p.few = row_queries <= kFewRows;
    if (worth_sharing(c, p.few, row_queries)) a.n_shared = c.n_shared << a.log_ps;
    const long own_tokens = std::max(((long)a.max_pages << a.log_ps) - a.n_shared, 0L), results = (long)a.T * a.heads;

    size_t at = 0;
    const auto room = [&](Partials *to, long n) {
        to->o = (float *)((char *)workspace + at);
        at += ((size_t)n * a.D * 4 + 255) / 256 * 256;
        to->ml = (float2 *)((char *)workspace + at);
        at += ((size_t)n * 8 + 255) / 256 * 256;
    };
    const auto splits_of = [](long blocks, long tokens, long room_for) {   // so that the GPU is about filled, with 256 keys or more each
        return (int)std::max(1L, std::min({(room_for + blocks / 2) / blocks, (tokens + 255) / 256, 64L}));
    };
    if (a.n_shared) {
        a.shared_here = p.few && all_queries <= kFewRows;
        p.shared_many = !a.shared_here;
        if (p.shared_many) {
            a.shared_splits = splits_of((all_queries + kManyRows - 1) / kManyRows * a.kv_heads, a.n_shared, p.few ? 256 : many_blocks(a.D));   // (few: a block a CU, see fbq_attend_both.hip)
            room(&a.part_shared, a.shared_splits * results);
        } else {
            room(&a.whole_shared, results);
        }
    }
    a.direct = p.few && !a.n_shared ? few_direct((long)a.rows * a.kv_heads, own_tokens, in_4_bits(c.cache.desc.type)) : 0;
    if (p.few && !a.direct) {
        const long steps = ((own_tokens + kFewTile - 1) / kFewTile * a.rows + (a.shared_here ? a.n_shared / kFewTile + 1 : 0)) * a.kv_heads;
        a.workers = (int)std::min(a.D > 128 ? 1024L : 2048L, (steps + kFewWaves - 1) / kFewWaves * kFewWaves);
        a.workers = std::max(a.workers, kFewWaves);
        a.slot_rows = (int)(a.shared_here ? std::max(row_queries, all_queries) : row_queries);
        room(&a.piece, 2L * a.workers * a.slot_rows);
        if (a.n_shared) room(&a.whole, results);
        p.join = true;
    } else if (!p.few) {
        const long per_row = (a.group + kManyRows - 1) / kManyRows;
        const long tiles = a.q_start ? (all_queries + kManyRows - 1) / kManyRows : a.rows * per_row;
        a.splits = (int)std::max(1L, std::min({(2L * many_blocks(a.D) - 1) / (tiles * a.kv_heads), (own_tokens + 255) / 256, 128L, 65535 / (tiles + a.rows)}));
        p.join = a.splits > 1 || a.n_shared;
        if (p.join) room(&a.part, a.splits * results);
    }
    p.bytes = at;
    return p;
}

static fbq_status check_attention(const fbq_attention_call *c, bool pointers)
{
    if (!c) return FBQ_ERR_NULL;
    fbq_cache cache = c->cache;
    if (!pointers) {                                          // (any that pass)
        cache.pool = (void *)(uintptr_t)256;
        cache.table = cache.lengths = (int32_t *)(uintptr_t)256;
    }
    const fbq_status st = check_cache(&cache, false);
    if (st != FBQ_OK) return st;
    const fbq_cache_desc &d = c->cache.desc;
    if (c->layer < 0 || c->layer >= d.layers || c->heads < 1 || c->heads % d.kv_heads || c->T < 1 || c->max_q < 1 || c->max_q > c->T) return FBQ_ERR_SHAPE;
    if (!c->q_start && (c->T != c->cache.rows || c->max_q != 1)) return FBQ_ERR_SHAPE;
    if (c->n_shared < 0 || c->n_shared > c->cache.max_pages) return FBQ_ERR_SHAPE;
    const int64_t row = (int64_t)c->heads * d.head_dim;
    if (c->q_stride < row || c->out_stride < row || c->q_stride % 8 || c->out_stride % 8) return FBQ_ERR_SHAPE;
    if (c->heads > 8192 || c->T > (1 << 20) || c->q_stride > (1L << 32) || c->out_stride > (1L << 32)) return FBQ_ERR_UNSUPPORTED;
    if ((int64_t)c->T * c->heads > (1L << 25)) return FBQ_ERR_UNSUPPORTED;
    if (!pointers) return FBQ_OK;
    if (!c->q || !c->out || (c->n_shared && !c->shared)) return FBQ_ERR_NULL;
    if (!aligned(c->q, 16) || !aligned(c->out, 16) || !aligned(c->lse, 4) || !aligned(c->q_start, 4) || !aligned(c->shared, 4)) return FBQ_ERR_ALIGN;
    return FBQ_OK;
}

}  // namespace fbq

using namespace fbq;

extern "C" size_t fbq_attention_workspace_bytes(const fbq_attention_call *a)
{
    return check_attention(a, false) == FBQ_OK ? attend_plan(*a, nullptr).bytes : 0;
}

extern "C" fbq_status fbq_attention(const fbq_attention_call *c, void *workspace, size_t workspace_bytes, fbq_stream stream)
{
    const fbq_status st = check_attention(c, true);
    if (st != FBQ_OK) return st;
    const AttendPlan p = attend_plan(*c, workspace);
    if (p.bytes && !workspace) return FBQ_ERR_NULL;
    if (!aligned(workspace, 16)) return FBQ_ERR_ALIGN;
    if (workspace_bytes < p.bytes) return FBQ_ERR_WORKSPACE;
    const int type = c->cache.desc.type;
    const hipStream_t s = (hipStream_t)stream;
    hipError_t e = hipSuccess;
    const bool four = in_4_bits(type), both = p.shared_many && p.few && p.a.D <= 128;
    const auto launch_few = four ? launch_attend4_few : launch_attend_few;
    const auto launch_many = four ? launch_attend4_many : launch_attend_many;
    if (both) e = (four ? launch_attend4_both : launch_attend_both)(p.a, type, s);
    else if (p.shared_many) e = launch_many(p.a, type, true, s);
    if (e == hipSuccess && !both) e = p.few ? launch_few(p.a, type, s) : launch_many(p.a, type, false, s);
    if (e == hipSuccess && p.join) e = (type & ~4) == FBQ_F16 ? launch_join<TypeF16>(p.a, p.few, s) : launch_join<TypeBf16>(p.a, p.few, s);
    return e == hipSuccess ? FBQ_OK : FBQ_ERR_HIP;
}
