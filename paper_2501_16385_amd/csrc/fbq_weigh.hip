// fbq_attention_weights: what attention's softmax gave each key, added up over the queries and heads of a key/value head.
//
// The softmax's sums are known (lse), so a key's weights are exp(scale q . k - lse) and nothing runs along the keys: a wave keeps 64 keys as operands of the matrix cores and goes through the query
// rows 16 at a time, S^T = K Q^T in v_mfma 16x16x32 as in fbq_attend_few.h, adds the exponentials up in the lane and over its 16 columns at the end.  Bound by reading the keys where rows are few
// (half of what attention reads), by the exponentials and the products where they are many.
// A block's four waves have 64 keys each, or, where a row of the table has many query rows, the same 64 keys and a fourth of the query tiles each, added up in LDS in a fixed order.
// Codes of 4 bits are small whole numbers of the queries' type, exactly; a group's scale and lowest value come in behind the product, in 32 bits, with the sums of q over the group.
#include <algorithm>
#include <cmath>

#include "fbq_attend.h"
#include "fbq_cache4.h"
#include "fbq_internal.h"
#include "fbq_lds_copy.h"

namespace fbq {

constexpr int kWeighKeys = 64;           // of a wave at a time
constexpr int kWeighWaves = 4;
constexpr int kWeighBlocks = 16384;      // about as many blocks at most: those of one row and head go along its keys

struct WeighArgs {
    AttendArgs a;
    const float *weights;                // null: nothing
    float *out;
    int width, parts;                    // blocks of a row and head
    float decay;
    bool together;                       // a block's waves have the same keys
};

// Eight codes of a word as numbers of the type, features in their order.
struct WholeF16 : TypeF16 {
    typedef NumberF16 Number;
    static constexpr uint32_t kOne = 0x3c003c00u;
    static __device__ __forceinline__ word4_t codes(uint32_t w)
    {
        typedef _Float16 half2_t __attribute__((ext_vector_type(2)));
        const auto low = [](uint32_t c) { return __builtin_bit_cast(uint32_t, __builtin_bit_cast(half2_t, (c & kLowCodes) | 0x64006400u) - half2_t{(_Float16)1024.0f, (_Float16)1024.0f}); };
        return word4_t{low(w), low(w >> 8), low(w >> 4), low(w >> 12)};
    }
};
struct WholeBf16 : TypeBf16 {
    typedef NumberBf16 Number;
    static constexpr uint32_t kOne = 0x3f803f80u;
    static __device__ __forceinline__ word4_t codes(uint32_t w)
    {
        const auto low = [](uint32_t c) { return pack((float)(c & 15), (float)(c >> 16 & 15)); };
        return word4_t{low(w), low(w >> 8), low(w >> 4), low(w >> 12)};
    }
};

// Sum over the 16 lanes of a row, in all of them.
__device__ __forceinline__ float row_sum(float x)
{
    const auto turn = [](float x, auto by) {
        return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, x), decltype(by)::value, 0xf, 0xf, false));
    };
    x += turn(x, std::integral_constant<int, 0x128>());       // row_ror 8, 4, 2, 1
    x += turn(x, std::integral_constant<int, 0x124>());
    x += turn(x, std::integral_constant<int, 0x122>());
    x += turn(x, std::integral_constant<int, 0x121>());
    return x;
}

template <class TY, bool FOUR, int NW>
__global__ __launch_bounds__(64 * kWeighWaves, NW > 4 ? 1 : 2) void fbq_weigh_kernel(const WeighArgs w)
{
    constexpr int DS = 32 * NW, G = FOUR ? groups4(DS) : 1, kTiles = kWeighKeys / 16;
    typedef typename TY::Number NT;
    __shared__ float sums[kWeighWaves][kWeighKeys];
    const AttendArgs &a = w.a;
    const int lane = threadIdx.x & 63, col = lane & 15, grp = lane >> 4, wave = uniform(threadIdx.x >> 6);
    const int h = blockIdx.x % a.kv_heads, b = blockIdx.x / a.kv_heads, D = a.D, ps1 = (1 << a.log_ps) - 1;
    const int2 of = queries_of(a, b);
    const int q0 = uniform(of.x), nq = uniform(of.y), tokens = uniform(row_tokens(a, b)), limit = min(tokens, w.width);
    const long head_bytes = (a.page_bytes >> 1) / a.kv_heads, at = ((long)b * a.kv_heads + h) * w.width;
    const int32_t *const list = a.table + (long)b * a.max_pages;
    const int a_block = w.together ? kWeighKeys : kWeighWaves * kWeighKeys, stride = w.parts * a_block;
    const int rows = nq * a.group, tiles = (rows + 15) / 16;

    for (int base = blockIdx.y * a_block; base < limit; base += stride) {
        const int key0 = base + (w.together ? 0 : wave * kWeighKeys);
        word4_t k[kTiles][NW], scales[kTiles][FOUR ? G : 1];
#pragma unroll
        for (int t = 0; t < kTiles; ++t) {
            const int key = key0 + 16 * t;
            int valid = min(max(tokens - key, 0), 16);
            const int id = valid ? uniform(list[key >> a.log_ps]) : 0;
            if ((unsigned)id >= (unsigned)a.pages) valid = 0;
            const unsigned char *const head = a.kv + (valid ? id : 0) * a.page_bytes + h * head_bytes;
            if constexpr (FOUR) {
                const __amdgpu_buffer_rsrc_t codes = buffer_of(head + codes_at4(key & ps1, DS), valid ? 8 * DS : 0);
                const __amdgpu_buffer_rsrc_t words = buffer_of(head + scales_at4(a.log_ps, key & ps1, DS), valid * 4 * G);
#pragma unroll
                for (int x = 0; x < NW; ++x) k[t][x][0] = __builtin_amdgcn_raw_buffer_load_b32(codes, ((col * 4 + grp) * NW + x) * 4, 0, 0);
#pragma unroll
                for (int y = 0; y < G; ++y) scales[t][y] = __builtin_amdgcn_raw_buffer_load_b128(words, grp * 16 * G + 16 * y, 0, 0);
            } else {
                const __amdgpu_buffer_rsrc_t from = buffer_of(head + (long)(key & ps1) * D * 2, valid * D * 2);
#pragma unroll
                for (int x = 0; x < NW; ++x) k[t][x] = __builtin_amdgcn_raw_buffer_load_b128(from, 32 * x + 8 * grp < D ? (col * D + 32 * x + 8 * grp) * 2 : kNowhere, 0, 0);
            }
        }
        if constexpr (FOUR) {
#pragma unroll
            for (int t = 0; t < kTiles; ++t)
#pragma unroll
                for (int x = 0; x < NW; ++x) k[t][x] = TY::codes(k[t][x][0]);
        }
        float4_t sum[kTiles];
#pragma unroll
        for (int t = 0; t < kTiles; ++t) sum[t] = float4_t{0, 0, 0, 0};

        struct Queries { word4_t q[NW]; float lse; int sees; };
        auto ask = [&](Queries &x, int tile) __attribute__((always_inline)) {
            const int r = tile * 16 + col, i = r / a.group, head = h * a.group + r - i * a.group, t = q0 + i;
            const bool there = r < rows;
            x.sees = there ? tokens - nq + i + 1 : 0;
            x.lse = there ? a.lse[(long)t * a.heads + head] : 0;
#pragma unroll
            for (int y = 0; y < NW; ++y) {
                const int d = 32 * y + 8 * grp;
                x.q[y] = word4_t{0, 0, 0, 0};
                if (there && d < D) x.q[y] = *reinterpret_cast<const word4_t *>(a.q + t * a.q_stride + head * D + d);
            }
        };
        auto add = [&](Queries &x) __attribute__((always_inline)) {
            float group_sum[G];
#pragma unroll
            for (int y = 0; y < NW; ++y) x.q[y] = (x.q[y] & a.q_and) ^ a.q_xor;
            if constexpr (FOUR) {
                const word4_t one{TY::kOne, TY::kOne, TY::kOne, TY::kOne};
#pragma unroll
                for (int y = 0; y < G; ++y) {
                    float4_t s = TY::mfma(one, x.q[2 * y], float4_t{0, 0, 0, 0});
                    if (2 * y + 1 < NW) s = TY::mfma(one, x.q[std::min(2 * y + 1, NW - 1)], s);
                    group_sum[y] = s[0];
                }
            }
            const float less = x.lse * 1.4426950408889634f;
#pragma unroll
            for (int t = 0; t < kTiles; ++t) {
                float4_t z{0, 0, 0, 0};
                if constexpr (FOUR) {
#pragma unroll
                    for (int y = 0; y < G; ++y) {
                        float4_t c = TY::mfma(k[t][2 * y], x.q[2 * y], float4_t{0, 0, 0, 0});
                        if (2 * y + 1 < NW) c = TY::mfma(k[t][std::min(2 * y + 1, NW - 1)], x.q[std::min(2 * y + 1, NW - 1)], c);
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            const uint32_t word = scales[t][(i * G + y) / 4][(i * G + y) % 4];
                            z[i] = __builtin_fmaf(NT::of_upper(word), c[i], __builtin_fmaf(NT::of(word & 0xffff), group_sum[y], z[i]));
                        }
                    }
                } else {
#pragma unroll
                    for (int y = 0; y < NW; ++y) z = TY::mfma(k[t][y], x.q[y], z);
                }
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const float p = __builtin_amdgcn_exp2f(__builtin_fmaf(z[i], a.scale, -less));
                    sum[t][i] += key0 + 16 * t + 4 * grp + i < x.sees ? p : 0.0f;
                }
            }
        };
        // the first tile with a row that sees the first key; those before see none of these
        const int first = uniform(max(0, (int)((long)max(key0 - (tokens - nq), 0) * a.group / 16)));
        const int step = w.together ? kWeighWaves : 1;
        int tile = first + (w.together ? wave : 0);
        if (key0 < limit && tile < tiles) {
            Queries x0, x1;
            ask(x0, tile);
            while (true) {
                if (tile + step < tiles) ask(x1, tile + step);
                add(x0);
                tile += step;
                if (tile >= tiles) break;
                if (tile + step < tiles) ask(x0, tile + step);
                add(x1);
                tile += step;
                if (tile >= tiles) break;
            }
        }
        // lane (grp, col) takes key 16 (col / 4) + 4 grp + col % 4
        float mine = 0;
#pragma unroll
        for (int t = 0; t < kTiles; ++t)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float all = row_sum(sum[t][i]);
                mine = col == 4 * t + i ? all : mine;
            }
        const int key = key0 + 16 * (col >> 2) + 4 * grp + (col & 3);
        if (w.together) {
            __syncthreads();                                  // (the sums may still be read from the keys before)
            sums[wave][lane] = mine;
            __syncthreads();
            if (wave) continue;
            mine = (sums[0][lane] + sums[1][lane]) + (sums[2][lane] + sums[3][lane]);
        }
        if (key < limit) {
            if (w.weights && key < tokens - nq) mine = __builtin_fmaf(w.weights[at + key], w.decay, mine);
            w.out[at + key] = mine;
        }
    }
}

template <class TY, bool FOUR>
static hipError_t launch_weigh(const WeighArgs &w, hipStream_t stream)
{
    const dim3 grid(w.a.kv_heads * w.a.rows, w.parts), block(64 * kWeighWaves);
    switch (features4(w.a.D) / 32) {
    case 2: hipLaunchKernelGGL((fbq_weigh_kernel<TY, FOUR, 2>), grid, block, 0, stream, w); break;
    case 3: hipLaunchKernelGGL((fbq_weigh_kernel<TY, FOUR, 3>), grid, block, 0, stream, w); break;
    case 4: hipLaunchKernelGGL((fbq_weigh_kernel<TY, FOUR, 4>), grid, block, 0, stream, w); break;
    case 6: hipLaunchKernelGGL((fbq_weigh_kernel<TY, FOUR, 6>), grid, block, 0, stream, w); break;
    default: hipLaunchKernelGGL((fbq_weigh_kernel<TY, FOUR, 8>), grid, block, 0, stream, w); break;
    }
    return hipGetLastError();
}

}  // namespace fbq

using namespace fbq;

extern "C" fbq_status fbq_attention_weights(const fbq_attention_call *c, const float *weights, float *out, int32_t width, float decay, fbq_stream stream)
{
    if (!c) return FBQ_ERR_NULL;
    const fbq_status st = check_cache(&c->cache, false);
    if (st != FBQ_OK) return st;
    const fbq_cache_desc &d = c->cache.desc;
    if (c->layer < 0 || c->layer >= d.layers || c->heads < 1 || c->heads % d.kv_heads || c->T < 1 || c->max_q < 1 || c->max_q > c->T) return FBQ_ERR_SHAPE;
    if (!c->q_start && (c->T != c->cache.rows || c->max_q != 1)) return FBQ_ERR_SHAPE;
    if (c->q_stride < (int64_t)c->heads * d.head_dim || c->q_stride % 8 || width < 1 || width > (1 << 24) || !(decay >= 0 && decay <= 1)) return FBQ_ERR_SHAPE;
    if (c->heads > 8192 || c->T > (1 << 20) || c->q_stride > (1L << 32) || (int64_t)c->T * c->heads > (1L << 25)) return FBQ_ERR_UNSUPPORTED;
    if ((int64_t)d.kv_heads * c->cache.rows > (1L << 23)) return FBQ_ERR_UNSUPPORTED;     // (a grid counts its threads in 32 bits)
    if (!c->q || !c->lse || !out) return FBQ_ERR_NULL;
    if (!aligned(c->q, 16) || !aligned(c->lse, 4) || !aligned(c->q_start, 4) || !aligned(weights, 4) || !aligned(out, 4)) return FBQ_ERR_ALIGN;
    const uintptr_t all = (uintptr_t)d.kv_heads * c->cache.rows * width * 4, from = (uintptr_t)weights, to = (uintptr_t)out;
    if (weights && from != to && from < to + all && to < from + all) return FBQ_ERR_UNSUPPORTED;          // (one over a part of the other)
    const CacheArgs cache = cache_args(c->cache);
    WeighArgs w{};
    AttendArgs &a = w.a;
    a.kv = cache.pool + c->layer * cache.layer_bytes;
    a.table = c->cache.table; a.lengths = c->cache.lengths; a.q_start = c->q_start;
    a.q = (const uint16_t *)c->q; a.lse = c->lse;
    a.page_bytes = cache.page_bytes; a.q_stride = c->q_stride;
    a.pages = cache.pages; a.log_ps = cache.log_ps; a.max_pages = cache.max_pages; a.rows = cache.rows; a.kv_heads = cache.kv_heads; a.D = cache.D;
    a.heads = c->heads; a.group = c->heads / a.kv_heads; a.T = c->T; a.max_q = c->q_start ? c->max_q : 1;
    a.scale = c->scale == 0 ? 1.0f : std::fabs(c->scale) * 1.4426950408889634f;
    a.q_and = c->scale == 0 ? 0u : 0xffffffffu;
    a.q_xor = c->scale < 0 ? 0x80008000u : 0u;
    w.weights = decay == 0 ? nullptr : weights;
    w.out = out; w.width = width; w.decay = decay;
    w.together = (long)a.max_q * a.group > 16 * kWeighWaves;
    const long most = std::min((long)a.max_pages << a.log_ps, (long)width), items = (long)a.rows * a.kv_heads;
    const int a_block = w.together ? kWeighKeys : kWeighWaves * kWeighKeys;
    w.parts = (int)std::max(1L, std::min({(most + a_block - 1) / a_block, (kWeighBlocks + items - 1) / items, 65535L}));
    hipError_t e;
    switch (d.type) {
    case FBQ_F16: e = launch_weigh<WholeF16, false>(w, (hipStream_t)stream); break;
    case FBQ_BF16: e = launch_weigh<WholeBf16, false>(w, (hipStream_t)stream); break;
    case FBQ_F16_4BIT: e = launch_weigh<WholeF16, true>(w, (hipStream_t)stream); break;
    default: e = launch_weigh<WholeBf16, true>(w, (hipStream_t)stream); break;
    }
    return e == hipSuccess ? FBQ_OK : FBQ_ERR_HIP;
}
