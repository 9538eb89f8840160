// fbq_attention: which kernels serve a call, where their partial results lie, and the kernel that joins these.
#include "fbq_attend.h"

namespace fbq {

constexpr int kJoinWaves = 4;

// out = sum over the partial results of a query row, one block a row; in the order of their numbers, so that equal calls give equal bits.  A row's own part is either
// whole (written by its one piece: nothing left to do unless shared tokens come with it), or cut into the pieces of the waves w0 .. w1 of the few-row kernel, or
// into the splits of the many-row kernel.
template <class TY>
__global__ __launch_bounds__(64 * kJoinWaves) void fbq_attend_join_kernel(const AttendArgs a, const bool few)
{
    __shared__ int sums[2][kJoinWaves];
    __shared__ float2 wave_ml[kJoinWaves];
    __shared__ float wave_o[kJoinWaves][256];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int t = blockIdx.x / a.heads, head = blockIdx.x - t * a.heads, h = head / a.group, j = head - h * a.group;
    const int b = a.q_start ? row_of_token(a.q_start, a.rows, t) : t;
    if (b < 0) return;
    const int2 q = queries_of(a, b);
    const int i = t - q.x;
    if (i >= q.y) return;

    const long row = (long)t * a.heads + head, rows = (long)a.T * a.heads;
    int share = 1, own0 = 0, own1 = 0, shared0 = 0, shared1 = 0;              // few: the item's steps in the line
    if (few) {
        int before = 0, all = 0;
        for (int x = threadIdx.x; x < a.rows; x += 64 * kJoinWaves) {
            const int steps = few_steps(a, x);
            all += steps;
            before += x < b ? steps : 0;
        }
#pragma unroll
        for (int o = 32; o; o >>= 1) {
            all += __shfl_xor(all, o);
            before += __shfl_xor(before, o);
        }
        if (lane == 0) {
            sums[0][wave] = all;
            sums[1][wave] = before;
        }
        __syncthreads();
        all = before = 0;
        for (int w = 0; w < kJoinWaves; ++w) {
            all += sums[0][w];
            before += sums[1][w];
        }
        const int shared_steps = a.shared_here ? (a.n_shared + kFewTile - 1) / kFewTile : 0, steps = few_steps(a, b);
        share = few_share(a, (all + shared_steps) * a.kv_heads);
        own0 = (shared_steps + before) * a.kv_heads + h * steps;
        own1 = own0 + steps;
        shared0 = h * shared_steps;
        shared1 = shared0 + shared_steps;
    }
    const bool one_own = few && own1 > own0 && own0 / share == (own1 - 1) / share;
    if (one_own && !a.whole.o) return;                        // written by its piece
    const int n_own = !few ? a.splits : own1 == own0 ? 0 : (own1 - 1) / share - own0 / share + 1;
    const int n_shared = a.shared_here ? (shared1 - 1) / share - shared0 / share + 1 : a.part_shared.o ? a.shared_splits : 0;
    const auto piece = [&](int u0, int x, int r) {            // the x-th piece of the item that begins with step u0, its row r
        const int w = u0 / share + x;
        return ((long)w * 2 + ((long)w * share < u0 ? 1 : 0)) * a.slot_rows + r;
    };

    float m = kNoScore, l = 0, acc[4] = {0, 0, 0, 0};
    for (int p = wave; p < n_shared + n_own; p += kJoinWaves) {
        Partials from;
        long at;
        if (p < n_shared) {
            if (!a.shared_here) from = a.part_shared, at = p * rows + row;
            else if (n_shared == 1) from = a.whole_shared, at = row;
            else from = a.piece, at = piece(shared0, p, t * a.group + j);
        } else {
            const int x = p - n_shared;
            if (!few) from = a.part, at = x * rows + row;
            else if (one_own) from = a.whole, at = row;
            else from = a.piece, at = piece(own0, x, i * a.group + j);
        }
        const float2 ml = from.ml[at];
        if (ml.y == 0) continue;
        const float to = fmaxf(m, ml.x), by = __builtin_amdgcn_exp2f(m - to), times = __builtin_amdgcn_exp2f(ml.x - to);
        m = to;
        l = l * by + ml.y * times;
#pragma unroll
        for (int k = 0; k < 4; ++k)
            if (lane + 64 * k < a.D) acc[k] = acc[k] * by + from.o[at * a.D + lane + 64 * k] * times;
    }
    if (lane == 0) wave_ml[wave] = make_float2(m, l);
#pragma unroll
    for (int k = 0; k < 4; ++k) wave_o[wave][lane + 64 * k] = acc[k];
    __syncthreads();
    float top = kNoScore, sum = 0, o = 0;
    for (int w = 0; w < kJoinWaves; ++w) top = fmaxf(top, wave_ml[w].x);
    const int d = threadIdx.x;
    for (int w = 0; w < kJoinWaves; ++w) {
        const float by = __builtin_amdgcn_exp2f(wave_ml[w].x - top);
        sum += wave_ml[w].y * by;
        o += wave_o[w][d] * by;
    }
    if (d < a.D) a.out[t * a.out_stride + head * a.D + d] = TY::one(sum == 0 ? 0.0f : o / sum);
    if (a.lse && d == 0) a.lse[row] = sum == 0 ? -INFINITY : (top + __builtin_amdgcn_logf(sum)) * 0.6931471805599453f;
}

static hipError_t launch_join(const AttendArgs &a, int type, bool few, hipStream_t stream)
{
    const dim3 grid((unsigned)((long)a.T * a.heads)), block(64 * kJoinWaves);
    if (type == FBQ_F16) hipLaunchKernelGGL(fbq_attend_join_kernel<TypeF16>, grid, block, 0, stream, a, few);
    else hipLaunchKernelGGL(fbq_attend_join_kernel<TypeBf16>, grid, block, 0, stream, a, few);
    return hipGetLastError();
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
    a.scale = c.scale * 1.4426950408889634f;

    const long row_queries = (long)a.max_q * a.group, all_queries = (long)a.T * a.group;   // of one key/value head
    p.few = row_queries <= kFewRows;
    // shared tokens are taken apart from the rows' own where that saves reading them: several rows, and few queries a row
    if (a.rows > 1 && row_queries <= 64) a.n_shared = c.n_shared << a.log_ps;
    const long own_tokens = std::max(((long)a.max_pages << a.log_ps) - a.n_shared, 0L), results = (long)a.T * a.heads;

    size_t at = 0;
    const auto room = [&](Partials *to, long n) {
        to->o = (float *)((char *)workspace + at);
        at += ((size_t)n * a.D * 4 + 255) / 256 * 256;
        to->ml = (float2 *)((char *)workspace + at);
        at += ((size_t)n * 8 + 255) / 256 * 256;
    };
    const auto splits_of = [](long blocks, long tokens) {     // so that the GPU, two blocks a CU, is filled, with 256 keys or more each
        return (int)std::max(1L, std::min({(512 + blocks - 1) / blocks, (tokens + 255) / 256, 32L}));
    };
    if (a.n_shared) {
        a.shared_here = p.few && all_queries <= kFewRows;
        p.shared_many = !a.shared_here;
        if (p.shared_many) {
            a.shared_splits = splits_of((all_queries + kManyRows - 1) / kManyRows * a.kv_heads, a.n_shared);
            room(&a.part_shared, a.shared_splits * results);
        } else {
            room(&a.whole_shared, results);
        }
    }
    if (p.few) {
        const long steps = ((own_tokens + kFewTile - 1) / kFewTile * a.rows + (a.shared_here ? a.n_shared / kFewTile + 1 : 0)) * a.kv_heads;
        a.workers = (int)std::min(a.D > 128 ? 1024L : 2048L, (steps + kFewWaves - 1) / kFewWaves * kFewWaves);
        a.workers = std::max(a.workers, kFewWaves);
        a.slot_rows = (int)(a.shared_here ? std::max(row_queries, all_queries) : row_queries);
        room(&a.piece, 2L * a.workers * a.slot_rows);
        if (a.n_shared) room(&a.whole, results);
        p.join = true;
    } else {
        const long per_row = (a.group + kManyRows - 1) / kManyRows;
        const long tiles = a.q_start ? (all_queries + kManyRows - 1) / kManyRows : a.rows * per_row;
        a.splits = splits_of(tiles * a.kv_heads, own_tokens);
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
    if ((int64_t)c->T * c->heads > (1L << 30) || ((int64_t)c->T * (c->heads / d.kv_heads)) / kManyRows + c->cache.rows > 65535) return FBQ_ERR_UNSUPPORTED;
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
    if (p.shared_many) e = launch_attend_many(p.a, type, true, s);
    if (e == hipSuccess) e = p.few ? launch_attend_few(p.a, type, s) : launch_attend_many(p.a, type, false, s);
    if (e == hipSuccess && p.join) e = launch_join(p.a, type, p.few, s);
    return e == hipSuccess ? FBQ_OK : FBQ_ERR_HIP;
}
