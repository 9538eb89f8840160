// Attention over the paged cache: what its kernels share (device code, launch arguments).
//
// Two kinds of work read keys and values.  fbq_attend_few.h: up to 16 query rows of one key/value head (query tokens times the heads that share it) against its
// tokens, in registers.  fbq_attend_many.h: 128 rows a block, key and value tiles in LDS.  Both can leave partial results - sum of p v, its maximum
// exponent, sum of p - for the join kernels (fbq_attention.hip), which add them up in a fixed order.
//
// What has fewer than 32 bits: the result, rounded once at the end, and the probabilities p where they are an operand of the matrix cores, which take v in its 16 bits and would take
// 32-bit p at a sixteenth of the rate.  p is rounded to the cache's type (relative error 2^-11, 2^-8 for bf16); the sum that the result is divided by is of the unrounded ones, in 32
// bits.  Relative L2 against 64 bits 2.2 to 2.8e-4 (fp16) and 2.1 to 2.3e-3 (bf16); rounding the result alone makes 2.1e-4 and 1.7e-3.
#ifndef FBQ_ATTEND_H
#define FBQ_ATTEND_H

#include "fbq_attend_plan.h"
#include "fbq_cache.h"
#include "fbq_internal.h"

namespace fbq {

typedef _Float16 half8_t __attribute__((ext_vector_type(8)));
typedef __bf16 bfloat8_t __attribute__((ext_vector_type(8)));
typedef float float4_t __attribute__((ext_vector_type(4)));
typedef float float16_t __attribute__((ext_vector_type(16)));
typedef uint32_t word2_t __attribute__((ext_vector_type(2)));
typedef uint32_t word4_t __attribute__((ext_vector_type(4)));

constexpr int kFewRows = 16;             // query rows of the few-row kernel
constexpr int kFewTile = 32;             // its keys a step of a wave
constexpr int kFewWaves = 4;             // waves a block; each has its own piece, and they join those of one item
constexpr int kManyRows = 128;           // query rows of a block of the many-row kernel
constexpr int kManyTile = 64;            // keys a step
constexpr float kNoScore = -3.0e38f;     // running maximum before any score (finite, so that differences with it are)
// The maximum that exponents are relative to follows the scores' only when they pass it by this much: rescaling what was summed is then rare.  Probabilities reach
// 2^8 instead of 1, far from what fp16 holds, and rounding is relative.
constexpr float kSlack = 8.0f;

// A set of partial results: o [n][D], {maximum, sum} [n]; the maximum is an exponent of two.
struct Partials {
    float *o;
    float2 *ml;
};

struct AttendArgs {
    const unsigned char *kv;             // the layer's pages
    const int32_t *table, *lengths, *q_start, *shared;
    const uint16_t *q;
    uint16_t *out;
    float *lse;
    long page_bytes, q_stride, out_stride;
    int pages, log_ps, max_pages, rows, kv_heads, group, D, T, max_q, heads;
    int n_shared;                        // tokens read through `shared` for all rows together; a row's own tokens start there
    float scale;                         // > 0, times log2 e: scores are exponents of two.  The sign of the call's scale, and a scale of zero, are taken into the queries:
    uint32_t q_and, q_xor;               // their words & q_and ^ q_xor
    // few-row kernel: `workers` waves; the partial results of pieces of items, two a worker ([workers][2][slot_rows]); those of whole items where something else
    // has to be added ([T heads]), null: out is written
    int workers, slot_rows;
    int direct;                          // 1: an item a worker, 2: an item a block; no partial results
    bool shared_here;                    // the shared tokens are items of this kernel's own, for the rows of all sequences together
    Partials piece, whole, whole_shared;
    // many-row kernel: at most `splits` pieces of a tile's keys, partial results [splits][T heads] (null: out is written); shared_splits of the shared tokens
    int splits, shared_splits;
    Partials part, part_shared;
};

// The two types: operands of the matrix cores, and two floats rounded to a word of them (to nearest, ties to even).
struct TypeF16 {
    static __device__ __forceinline__ float4_t mfma(word2_t a, word2_t b, float4_t c)       // 16 x 16 x 16
    {
        typedef _Float16 half4_t __attribute__((ext_vector_type(4)));
        return __builtin_amdgcn_mfma_f32_16x16x16f16(__builtin_bit_cast(half4_t, a), __builtin_bit_cast(half4_t, b), c, 0, 0, 0);
    }
    static __device__ __forceinline__ float4_t mfma(word4_t a, word4_t b, float4_t c)
    {
        return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(half8_t, a), __builtin_bit_cast(half8_t, b), c, 0, 0, 0);
    }
    static __device__ __forceinline__ float16_t mfma(word4_t a, word4_t b, float16_t c)
    {
        return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(half8_t, a), __builtin_bit_cast(half8_t, b), c, 0, 0, 0);
    }
    static __device__ __forceinline__ uint32_t pack(float x, float y)
    {
        typedef _Float16 half2_t __attribute__((ext_vector_type(2)));
        return __builtin_bit_cast(uint32_t, half2_t{(_Float16)x, (_Float16)y});
    }
};
struct TypeBf16 {
    static __device__ __forceinline__ float4_t mfma(word2_t a, word2_t b, float4_t c)
    {
        typedef short short4_t __attribute__((ext_vector_type(4)));
        return __builtin_amdgcn_mfma_f32_16x16x16bf16_1k(__builtin_bit_cast(short4_t, a), __builtin_bit_cast(short4_t, b), c, 0, 0, 0);
    }
    static __device__ __forceinline__ float4_t mfma(word4_t a, word4_t b, float4_t c)
    {
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bfloat8_t, a), __builtin_bit_cast(bfloat8_t, b), c, 0, 0, 0);
    }
    static __device__ __forceinline__ float16_t mfma(word4_t a, word4_t b, float16_t c)
    {
        return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bfloat8_t, a), __builtin_bit_cast(bfloat8_t, b), c, 0, 0, 0);
    }
    static __device__ __forceinline__ uint32_t pack(float x, float y)
    {
        typedef __bf16 bf2_t __attribute__((ext_vector_type(2)));
        return __builtin_bit_cast(uint32_t, bf2_t{(__bf16)x, (__bf16)y});
    }
};

// A value that is the same in all lanes, as one the compiler knows to be.
__device__ __forceinline__ int uniform(int v) { return __builtin_amdgcn_readfirstlane(v); }

// Query tokens of a row: the first one and how many (whatever q_start holds, inside [0, T) and at most max_q).
__device__ __forceinline__ int2 queries_of(const AttendArgs &a, int b)
{
    if (!a.q_start) return make_int2(b, 1);
    const int q0 = min(max(a.q_start[b], 0), a.T), q1 = min(max(a.q_start[b + 1], q0), a.T);
    return make_int2(q0, min(q1 - q0, a.max_q));
}

__device__ __forceinline__ int row_tokens(const AttendArgs &a, int b) { return tokens_of(a.lengths[b], a.max_pages << a.log_ps); }

// Steps of a row's own tokens in the few-row kernel, of which it has `tokens` with the shared ones; none if it has no query tokens.
__device__ __forceinline__ int few_steps(const AttendArgs &a, int b, int tokens)
{
    const int steps = (max(tokens - a.n_shared, 0) + kFewTile - 1) / kFewTile;
    return a.q_start && queries_of(a, b).y == 0 ? 0 : steps;
}
__device__ __forceinline__ int few_steps(const AttendArgs &a, int b) { return few_steps(a, b, row_tokens(a, b)); }

// How many steps each worker takes, from all there are: the last ones may have none.
__device__ __forceinline__ int few_share(const AttendArgs &a, int steps) { return max(1, (steps + a.workers - 1) / a.workers); }

// Whether all workers of a block have their whole share of the item that reaches from step u0 to u1: they join their results before they write them, as the first one's.
__device__ __forceinline__ bool few_together(int block, int share, int u0, int u1)
{
    return (long)block * kFewWaves * share >= u0 && (long)(block + 1) * kFewWaves * share <= u1;
}

// Many-row kernel: tiles of a row's queries; keys that a tile's last query sees; steps to there.
__device__ __forceinline__ int many_tiles(const AttendArgs &a, int queries) { return (queries * a.group + kManyRows - 1) / kManyRows; }
__device__ __forceinline__ int many_limit(const AttendArgs &a, int tokens, int queries, int tile)
{
    return max(0, min(tokens, tokens - queries + min(queries - 1, ((tile + 1) * kManyRows - 1) / a.group) + 1));
}
__device__ __forceinline__ int many_steps(const AttendArgs &a, int limit) { return (max(limit - a.n_shared, 0) + kManyTile - 1) / kManyTile; }

// How many steps a piece of a tile has at most (see fbq_attend_plan.h).  The whole wave calls it.
__host__ __device__ __forceinline__ constexpr int many_blocks(int D) { return D > 128 ? 256 : 512; }
__device__ __forceinline__ int many_share(const AttendArgs &a)
{
    uint64_t twice = 0;
    int tiles = 0;
    for (int b = threadIdx.x & 63; b < a.rows; b += 64) {
        const int n = queries_of(a, b).y, of_row = many_tiles(a, n), tokens = row_tokens(a, b);
        if (of_row) twice += (uint64_t)of_row * (uint32_t)(many_steps(a, many_limit(a, tokens, n, 0)) + many_steps(a, tokens));
        tiles += of_row;
    }
    // (2^18 tiles and 2^16 rows' begun ones, 2^19 steps each: the lower 20 bits and the others apart)
    const uint32_t low = __builtin_amdgcn_readlane(wave_scan((int)(twice & 0xfffff)), 63), high = __builtin_amdgcn_readlane(wave_scan((int)(twice >> 20)), 63);
    return uniform(share_of_steps(((uint64_t)high << 20) + low, __builtin_amdgcn_readlane(wave_scan(tiles), 63), a.kv_heads, many_blocks(a.D)));
}
// Pieces of a tile of so many steps.
__device__ __forceinline__ int many_pieces(const AttendArgs &a, int steps, int share) { return max(1, min(a.splits, (steps + share - 1) / share)); }

// The larger of x and the x of the lane 16, or 32, further round in pairs of rows of 16, or 32.
__device__ __forceinline__ float larger_of_16(float x)
{
    const auto r = __builtin_amdgcn_permlane16_swap(__builtin_bit_cast(uint32_t, x), __builtin_bit_cast(uint32_t, x), false, false);
    return fmaxf(__builtin_bit_cast(float, (uint32_t)r[0]), __builtin_bit_cast(float, (uint32_t)r[1]));
}
__device__ __forceinline__ float larger_of_32(float x)
{
    const auto r = __builtin_amdgcn_permlane32_swap(__builtin_bit_cast(uint32_t, x), __builtin_bit_cast(uint32_t, x), false, false);
    return fmaxf(__builtin_bit_cast(float, (uint32_t)r[0]), __builtin_bit_cast(float, (uint32_t)r[1]));
}

// The page list that a wave goes along: 64 entries a register, the next 64 under way.
struct PageList {
    const int32_t *list;
    int count, base, ids, next;
    __device__ __forceinline__ int load(int at) const { return list[min(at, count - 1)]; }
    __device__ __forceinline__ void begin(const int32_t *l, int n, int first)
    {
        list = l; count = n; base = first;
        const int lane = threadIdx.x & 63;
        ids = load(base + lane);
        next = load(base + 64 + lane);
    }
    __device__ __forceinline__ int at(int index)              // index: the same in all lanes, never going back, at most 64 further than the last
    {
        if (index - base >= 64) {
            ids = next;
            base += 64;
            next = load(base + 64 + (threadIdx.x & 63));
        }
        return __builtin_amdgcn_readlane(ids, index - base);
    }
};

// A page number by a scalar load: vector loads are waited for in their order, and one among a step's would hold up those behind it.
__device__ __forceinline__ int page_of(const int32_t *list, int index, int count)
{
    typedef const __attribute__((address_space(4))) int32_t *scalar_t;
    return ((scalar_t)(uintptr_t)list)[uniform(max(min(index, count - 1), 0))];
}

constexpr int kNowhere = 1 << 30;        // an offset behind every descriptor's end: loads answer zero

hipError_t launch_attend_few(const AttendArgs &a, int type, hipStream_t stream);
hipError_t launch_attend_many(const AttendArgs &a, int type, bool shared, hipStream_t stream);   // shared: the shared tokens for all rows, else the rows' own

// of a cache in 4 bits
hipError_t launch_attend4_few(const AttendArgs &a, int type, hipStream_t stream);
hipError_t launch_attend4_many(const AttendArgs &a, int type, bool shared, hipStream_t stream);
hipError_t launch_attend4_both(const AttendArgs &a, int type, hipStream_t stream);

hipError_t launch_attend_both(const AttendArgs &a, int type, hipStream_t stream);                // the shared tokens many-row, the rows' own few-row

}  // namespace fbq

#endif
