// fbq_attention_weights: what attention's softmax gave each key, added up over the queries and heads of a key/value head.
//
// The softmax's sums are known (lse), so a key's weights are exp(scale q . k - lse) and nothing runs along the keys.  S^T = K Q^T in v_mfma 16x16x32 as in fbq_attend_few.h; the exponentials are
// added up in the lane and over its 16 columns at the end.
//   few   up to 16 query rows of a key/value head (fbq_weigh_few_kernel): bound by reading the keys, half of what attention reads.  The waves of the grid share the steps of all rows and heads
//         as attention's do (FewLine), a step's keys asked for a step ahead; there is nothing to join, since a key's sum is a wave's own.  us from card to card, 16 rows
//         of about 1000 tokens, 32 heads of 128: 28 to 32 in 16 bits (136 MB), 18.4 in 4 (41 MB); 64 of 4096, 64 heads to 8 of the keys': 119 (555 MB), 45 (169 MB); one of 65537: 35, 19.  (Written as
//         attention's loop, two steps at a time, the same.)
//   many  (fbq_weigh_many_kernel) bound by vector instructions and matrix products one behind the other in two waves a SIMD.  A wave keeps 64 keys as operands and goes through the query rows 16
//         at a time, which come through LDS.  One, two or all four of a block's waves have the same 64 keys, and share the query tiles; their sums are added up in LDS in a fixed order.  Two
//         rows of 4000 tokens, 512 of them queries, 32 heads of 128 to 8 of the keys', us from card to card: 45 to 50 in 16 bits, 55 to 59 in 4 of bf16, 65 in 4 of fp16 (a card that took 63 for bf16
//         and 45 for 16 bits: queries from memory as operands 75 and 68, all four waves with the same keys, too, 78 and 72).  16000 tokens: 181 to 184, 208 and 226; heads of 256, 4000 tokens: 104, 151, 156.
// Codes of 4 bits: few, as in fbq_attend4_few.h; many, as small whole numbers of the queries' type, exactly, and scales come in behind the product, in 32 bits: the matrix cores spread them over
// the lanes once for 64 keys, and make m sum(q) of the sums of q over a group in parts of 16 bits, three of them (what bf16 leaves is 2^-24 of a sum), so that weights are as exact as lse is.
#include <algorithm>
#include <cmath>

#include "fbq_attend4_few.h"
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
    bool few;                            // the few-row kernel
    int log_share;                       // many rows: 2 to this waves of a block have the same keys, and a share of the query tiles each
};

// Eight codes of a word as numbers of the type, features in their order.
struct WholeF16 : TypeF16 {
    typedef NumberF16 Number;
    static constexpr uint32_t kOne = 0x3c003c00u;
    static constexpr bool kWide = false;
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
    static constexpr bool kWide = true;                       // has fp32's range
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

// A step's keys, 16 a part, on their way to a wave: in 16 bits operands, in 4 bits codes and scale words; and what the sums begin with.
template <bool FOUR, int NW>
struct WeighStep {
    word4_t k[kFew4Parts][FOUR ? 1 : NW];
    uint32_t codes[kFew4Parts][FOUR ? NW : 1], scales[kFew4Parts];
    float before;
};

template <class TY, bool FOUR, int NW>
__global__ __launch_bounds__(64 * kFewWaves, 2) void fbq_weigh_few_kernel(const WeighArgs w)
{
    constexpr int DS = 32 * NW, G = groups4(DS), kParts = kFew4Parts;
    typedef typename TY::Number NT;
    const AttendArgs &a = w.a;
    const int lane = threadIdx.x & 63, col = lane & 15, grp = lane >> 4, D = a.D, ps1 = (1 << a.log_ps) - 1;
    const int worker = uniform(blockIdx.x * kFewWaves + (threadIdx.x >> 6)), member = col % a.group;
    const long head_bytes = (a.page_bytes >> 1) / a.kv_heads;
    const int mine = 16 * (col >> 2) + 4 * grp + (col & 3);   // this lane's key of a step, of those lanes that have one
    const bool has = col < 4 * kParts;

    Piece4<NW> cur, behind;
    float lse = 0, lse_behind = 0;
    FewLine line;
    if (!line.first(a, blockIdx.x, worker, cur)) return;
    auto prepare = [&](Piece4<NW> &x, float &l) __attribute__((always_inline)) {
        few_sight(a, x, col);
#pragma unroll
        for (int part = 0; part < kParts; ++part) x.pages[part] = page_of(few_pages(a, x), (x.key0 + 16 * part) >> a.log_ps, few_page_count(a, x));
        const int head = x.h * a.group + member;
        l = x.t >= 0 ? a.lse[(long)x.t * a.heads + head] : 0;
#pragma unroll
        for (int y = 0; y < NW; ++y) {
            const int d = 32 * y + 8 * grp;
            x.q[y] = word4_t{0, 0, 0, 0};
            if (x.t >= 0 && d < D) x.q[y] = *reinterpret_cast<const word4_t *>(a.q + x.t * a.q_stride + head * D + d);
        }
    };
    int k_off[FOUR ? 1 : NW];
    if constexpr (!FOUR) {
#pragma unroll
        for (int y = 0; y < NW; ++y) k_off[y] = 32 * y + 8 * grp < D ? (col * D + 32 * y + 8 * grp) * 2 : kNowhere;
    }
    const int scale_off = grp < G ? (col * G + grp) * 4 : kNowhere;
    int ask_key = 0, ask_end = 0, ask_h = 0, ask_b = 0, ask_old = 0, ask_pages[kParts];
    auto aim = [&](const Piece4<NW> &x, bool there) __attribute__((always_inline)) {
        ask_key = x.key0;
        ask_end = there ? min(x.limit, x.key0 + x.n * kFewTile) : 0;
        ask_h = x.h;
        ask_b = x.b;
        ask_old = w.weights ? min(min(ask_end, w.width), x.limit - queries_of(a, x.b).y) : 0;        // where tokens that are there begin to be new
#pragma unroll
        for (int part = 0; part < kParts; ++part) ask_pages[part] = x.pages[part];
    };
    auto load = [&](WeighStep<FOUR, NW> &to) __attribute__((always_inline)) {     // always as many loads: see attend4_few
#pragma unroll
        for (int part = 0; part < kParts; ++part) {
            const int key = ask_key + 16 * part, id = ask_pages[part];
            const int valid = (unsigned)id < (unsigned)a.pages ? min(max(ask_end - key, 0), 16) : 0;
            const unsigned char *const keys = a.kv + (valid ? id : 0) * a.page_bytes + ask_h * head_bytes;
            if constexpr (FOUR) {
                load_words<NW, kOnce>(to.codes[part], buffer_of(keys + codes_at4(key & ps1, DS), valid ? 8 * DS : 0), (col * 4 + grp) * NW * 4);
                to.scales[part] = __builtin_amdgcn_raw_buffer_load_b32(buffer_of(keys + scales_at4(a.log_ps, key & ps1, DS), valid * 4 * G), scale_off, 0, 0);
            } else {
                const __amdgpu_buffer_rsrc_t from = buffer_of(keys + (long)(key & ps1) * D * 2, valid * D * 2);
#pragma unroll
                for (int y = 0; y < NW; ++y) to.k[part][y] = __builtin_amdgcn_raw_buffer_load_b128(from, k_off[y], 0, kOnce);
            }
        }
        const float *const row = w.weights + ((long)ask_b * a.kv_heads + ask_h) * w.width + ask_key;
        to.before = __builtin_bit_cast(float, __builtin_amdgcn_raw_buffer_load_b32(buffer_of(w.weights ? row : w.out, max(min(ask_old - ask_key, kFewTile), 0) * 4), has ? mine * 4 : kNowhere, 0, 0));
        ask_key += kFewTile;
        const int32_t *const list = a.table + (long)ask_b * a.max_pages;
#pragma unroll
        for (int part = 0; part < kParts; ++part) ask_pages[part] = page_of(list, (ask_key + 16 * part) >> a.log_ps, a.max_pages);
    };

    Queries4<TY, NT, NW> codes_q;
    word4_t q[FOUR ? 1 : NW];
    float unit = a.scale, less = 0;
    auto begin = [&]() __attribute__((always_inline)) {
#pragma unroll
        for (int y = 0; y < NW; ++y) cur.q[y] = (cur.q[y] & a.q_and) ^ a.q_xor;
        if constexpr (FOUR) {
            codes_q.of(cur.q, a.scale);
            unit = codes_q.unit;
        } else {
#pragma unroll
            for (int y = 0; y < NW; ++y) q[y] = cur.q[y];
        }
        less = lse * 1.4426950408889634f;
    };
    auto compute = [&](const WeighStep<FOUR, NW> &x, int s) __attribute__((always_inline)) {
        const int key = cur.key0 + s * kFewTile, sees = cur.sees - key - 4 * grp;
        float sum = 0;
#pragma unroll
        for (int part = 0; part < kParts; ++part) {
            float4_t z{0, 0, 0, 0};
            if constexpr (FOUR) {
                z = scores4<TY, NT, NW>(x.codes[part], x.scales[part], codes_q);
            } else {
#pragma unroll
                for (int y = 0; y < NW; ++y) z = TY::mfma(x.k[part][y], q[y], z);
            }
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float p = __builtin_amdgcn_exp2f(__builtin_fmaf(z[i], unit, -less));
                const float all = row_sum(16 * part + i < sees ? p : 0.0f);
                sum = col == 4 * part + i ? all : sum;
            }
        }
        if (has && key + mine < min(min(cur.limit, cur.key0 + cur.n * kFewTile), w.width))
            w.out[((long)cur.b * a.kv_heads + cur.h) * w.width + key + mine] = __builtin_fmaf(x.before, w.decay, sum);
    };

    prepare(cur, lse);
    behind = cur;                                             // (where there is none, something that is one)
    bool more = line.follow(a, cur, behind);
    if (more) prepare(behind, lse_behind);
    WeighStep<FOUR, NW> x0, x1;
    aim(cur, true);
    load(x0);
    begin();
    int s = 0;
    auto turn = [&](const WeighStep<FOUR, NW> &now, WeighStep<FOUR, NW> &next) __attribute__((always_inline)) {
        if (s + 1 == cur.n) aim(behind, more);
        load(next);
        compute(now, s);
        if (++s < cur.n) return false;
        if (!more) return true;
        cur = behind;
        lse = lse_behind;
        s = 0;
        more = line.follow(a, cur, behind);
        if (more) prepare(behind, lse_behind);
        begin();
        return false;
    };
    while (!turn(x0, x1) && !turn(x1, x0)) {}
}

template <class TY, bool FOUR, int NW>
__global__ __launch_bounds__(64 * kWeighWaves, NW > 4 ? 1 : 2) void fbq_weigh_many_kernel(const WeighArgs w)
{
    constexpr int DS = 32 * NW, G = groups4(DS), kTiles = kWeighKeys / 16;
    typedef typename TY::Number NT;
    constexpr int kPieces = 4 * NW, kBuffer = 1024 * NW + 256;                // a tile's queries, 16 bytes a piece, and their lse
    __shared__ float sums[kWeighWaves][kWeighKeys];
    __shared__ __attribute__((aligned(16))) unsigned char room[kWeighWaves][2][kBuffer];
    const AttendArgs &a = w.a;
    const int lane = threadIdx.x & 63, col = lane & 15, grp = lane >> 4, wave = uniform(threadIdx.x >> 6);
    const int h = blockIdx.x % a.kv_heads, b = blockIdx.x / a.kv_heads, D = a.D, ps1 = (1 << a.log_ps) - 1;
    const int2 of = queries_of(a, b);
    if (of.y == 0) return;                                    // (no queries: left as it is)
    const int q0 = uniform(of.x), nq = uniform(of.y), tokens = uniform(row_tokens(a, b)), limit = min(tokens, w.width);
    const long head_bytes = (a.page_bytes >> 1) / a.kv_heads, at = ((long)b * a.kv_heads + h) * w.width;
    const int32_t *const list = a.table + (long)b * a.max_pages;
    // (A sign is the scale's here.)  Codes of bf16: the scale goes into the keys' scales and the sums of q, and sums begin at -lse.  In fp16, whose range an arbitrary scale would leave, it comes
    // in with lse, sums of q are 2^-7 of them, and what is left of them 2^12.
    constexpr bool kFolded = FOUR && TY::kWide;
    const float unit = (a.q_xor ? -a.scale : a.scale) * (FOUR && !kFolded ? 128.0f : 1.0f);
    const int share = 1 << w.log_share, part = wave & (share - 1), a_block = kWeighKeys * (kWeighWaves >> w.log_share), stride = w.parts * a_block;
    const int rows = nq * a.group, tiles = (rows + 15) / 16;

    for (int base = blockIdx.y * a_block; base < limit; base += stride) {
        const int key0 = base + (wave >> w.log_share) * kWeighKeys;
        word4_t k[kTiles][NW];
        uint32_t words[kTiles];                               // 4 bits: scale word of key l % 16, group l / 16
#pragma unroll
        for (int t = 0; t < kTiles; ++t) {
            const int key = key0 + 16 * t;
            int valid = min(max(tokens - key, 0), 16);
            const int id = valid ? uniform(list[key >> a.log_ps]) : 0;
            if ((unsigned)id >= (unsigned)a.pages) valid = 0;
            const unsigned char *const head = a.kv + (valid ? id : 0) * a.page_bytes + h * head_bytes;
            if constexpr (FOUR) {
                const __amdgpu_buffer_rsrc_t codes = buffer_of(head + codes_at4(key & ps1, DS), valid ? 8 * DS : 0);
                uint32_t of[NW];
                load_words<NW, 0>(of, codes, (col * 4 + grp) * NW * 4);
#pragma unroll
                for (int x = 0; x < NW; ++x) k[t][x][0] = of[x];
                words[t] = __builtin_amdgcn_raw_buffer_load_b32(buffer_of(head + scales_at4(a.log_ps, key & ps1, DS), valid * 4 * G), grp < G ? (col * G + grp) * 4 : kNowhere, 0, 0);
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
        float4_t scales[kTiles][FOUR ? G : 1];                // of the lane's four keys, 2^-7 of them as of the sums of q, or times the scale
        if constexpr (FOUR) {
#pragma unroll
            for (int t = 0; t < kTiles; ++t)
#pragma unroll
                for (int y = 0; y < G; ++y) {
                    scales[t][y] = scales_of<TY>(words[t], word2_t{grp == y ? NT::bits(kFolded ? 1.0f : 0x1p-7f) << 16 : 0u, 0u});
                    if (kFolded) scales[t][y] *= unit;
                }
        }
        float4_t sum[kTiles];
#pragma unroll
        for (int t = 0; t < kTiles; ++t) sum[t] = float4_t{0, 0, 0, 0};

        // Tiles of queries come through LDS, two ahead: a row's sixteen pieces are neighbours' copies, where operands read from memory are sixteen rows' pieces and take four times as long.
        // Piece p of a row lies at p ^ swap.  (Rows past the last one are that one; words from kSure on can have features past the last: these are zeros.)
        constexpr int kSure = NW == 2 ? 0 : NW == 8 ? 6 : NW == 6 ? 4 : NW - 1;
        const auto swap = [](int row) { return kPieces == 8 ? piece_key(row) : kPieces == 12 ? row >> 2 & 3 : kPieces == 24 ? row & 7 : row & 15; };
        const int first = uniform(max(0, (int)((long)max(key0 - (tokens - nq), 0) * a.group / 16)));   // the first tile with a row that sees the first key; those before see none of these
        const int clear = uniform((int)(((long)max(key0 + kWeighKeys - 1 - (tokens - nq), 0) * a.group + 15) / 16));   // from this one on all rows see all keys
        const long tokens_on = 16 * share / a.group;          // from a wave's tile to its next, where it is whole tokens
        const bool even = 16 * share % a.group == 0;
        int tile = first + part;
        const unsigned char *from[NW];
        const float *lse_from;
        auto place = [&](int tile) __attribute__((always_inline)) {
            const auto row = [&](int r, long *token) { r = min(16 * tile + r, rows - 1); const int i = r / a.group; *token = q0 + i; return h * a.group + r - i * a.group; };
            long t;
#pragma unroll
            for (int x = 0; x < NW; ++x) {
                const int r = (64 * x + lane) / kPieces, p = (64 * x + lane) % kPieces ^ swap(r), head = row(r, &t);
                from[x] = reinterpret_cast<const unsigned char *>(a.q + t * a.q_stride + head * D + (8 * p < D ? 8 * p : 0));
            }
            const int head = row(col, &t);
            lse_from = a.lse + t * a.heads + head;
        };
        auto copy = [&](int to) __attribute__((always_inline)) {
            const uint32_t at = uniform(lds_offset(room[wave][to]));
#pragma unroll
            for (int x = 0; x < NW; ++x) copy16_to_lds(from[x], at + 1024 * x);
            copy4_to_lds(lse_from, at + 1024 * NW);
        };
        struct { word4_t q[NW]; float lse; } x;
        auto add = [&](int in) __attribute__((always_inline)) {
            if (tile + share < tiles) asm volatile("s_waitcnt vmcnt(%0)" ::"n"(NW + 1) : "memory");
            else asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
#pragma unroll
            for (int y = 0; y < NW; ++y) x.q[y] = *reinterpret_cast<const word4_t *>(room[wave][in] + (col * kPieces + ((4 * y + grp) ^ swap(col))) * 16);
            x.lse = *reinterpret_cast<const float *>(room[wave][in] + 1024 * NW + lane * 4);
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
            const int next = tile + 2 * share;
            if (next < tiles) {
                if (even && 16 * next + 16 <= rows) {
#pragma unroll
                    for (int y = 0; y < NW; ++y) from[y] += tokens_on * a.q_stride * 2;
                    lse_from += tokens_on * a.heads;
                } else {
                    place(next);
                }
                copy(in);
            }
#pragma unroll
            for (int y = kSure; y < NW; ++y)
                if (32 * y + 8 * grp >= D) x.q[y] = word4_t{0, 0, 0, 0};
            if (a.q_and == 0) {                               // (scale 0)
                asm volatile("");
#pragma unroll
                for (int y = 0; y < NW; ++y) x.q[y] = word4_t{0, 0, 0, 0};
            }
            float4_t z[kTiles];
            const float less = x.lse * 1.4426950408889634f;
            if constexpr (FOUR) {
                // the sum of q over group l / 16, times the scale or 2^-7, and what is left of it in two parts
                const word4_t one{TY::kOne, TY::kOne, TY::kOne, TY::kOne};
                word2_t high{0, 0}, rest{0, 0};
                float4_t sums[G];
                float sum = 0;
#pragma unroll
                for (int y = 0; y < G; ++y) {
                    sums[y] = TY::mfma(one, x.q[2 * y], float4_t{0, 0, 0, 0});
                    if (2 * y + 1 < NW) sums[y] = TY::mfma(one, x.q[std::min(2 * y + 1, NW - 1)], sums[y]);
                }
                // (products that follow from each other stand apart)
                float4_t c[kTiles][G], lower[kTiles];
#pragma unroll
                for (int half = 0; half < 2; ++half)
#pragma unroll
                    for (int y = 0; y < G; ++y)
#pragma unroll
                        for (int t = 0; t < kTiles; ++t) {
                            if (half == 0) c[t][y] = TY::mfma(k[t][2 * y], x.q[2 * y], float4_t{0, 0, 0, 0});
                            else if (2 * y + 1 < NW) c[t][y] = TY::mfma(k[t][std::min(2 * y + 1, NW - 1)], x.q[std::min(2 * y + 1, NW - 1)], c[t][y]);
                        }
#pragma unroll
                for (int y = 0; y < G; ++y) sum = grp == y ? sums[y][0] * (kFolded ? unit : 0x1p-7f) : sum;
                high[0] = NT::bits(sum);
                const float left = (sum - NT::of(high[0])) * (kFolded ? 1.0f : 0x1p12f);
                rest[0] = NT::bits(left);
                rest[1] = NT::bits(left - NT::of(rest[0]));
#pragma unroll
                for (int t = 0; t < kTiles; ++t) {
                    z[t] = TY::mfma(word2_t{words[t], 0u}, high, kFolded ? float4_t{-less, -less, -less, -less} : float4_t{0, 0, 0, 0});
                    lower[t] = TY::mfma(word2_t{words[t], words[t]}, rest, kFolded ? z[t] : float4_t{0, 0, 0, 0});
                }
                __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                for (int t = 0; t < kTiles; ++t)
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        float x = kFolded ? lower[t][i] : z[t][i];
#pragma unroll
                        for (int y = 0; y < G; ++y) x = __builtin_fmaf(scales[t][y][i], c[t][y][i], x);
                        if (!kFolded) x = __builtin_fmaf(__builtin_fmaf(lower[t][i], 0x1p-12f, x), unit, -less);
                        z[t][i] = __builtin_amdgcn_exp2f(x);
                    }
            } else {
#pragma unroll
                for (int y = 0; y < NW; ++y)
#pragma unroll
                    for (int t = 0; t < kTiles; ++t) z[t] = TY::mfma(k[t][y], x.q[y], y ? z[t] : float4_t{0, 0, 0, 0});
                __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                for (int t = 0; t < kTiles; ++t)
#pragma unroll
                    for (int i = 0; i < 4; ++i) z[t][i] = __builtin_amdgcn_exp2f(__builtin_fmaf(z[t][i], unit, -less));
            }
            if (tile < clear || 16 * tile + 16 > rows) {      // some row does not see all of the keys
                const int r = 16 * tile + col, sees = (r < rows ? tokens - nq + r / a.group + 1 : 0) - key0 - 4 * grp;
                asm volatile("");
#pragma unroll
                for (int t = 0; t < kTiles; ++t)
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        if (16 * t + i >= sees) z[t][i] = 0;
            }
#pragma unroll
            for (int t = 0; t < kTiles; ++t) sum[t] += z[t];
        };
        if (key0 < limit && tile < tiles) {
            place(tile);
            copy(0);
            if (tile + share < tiles) {
                place(tile + share);
                copy(1);
            }
            for (int in = 0; tile < tiles; tile += share, in ^= 1) add(in);
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
        if (share > 1) {
            __syncthreads();                                  // (the sums may still be read from the keys before)
            sums[wave][lane] = mine;
            __syncthreads();
            if (part) continue;
            mine += sums[wave + 1][lane];
            if (share == 4) mine += sums[2][lane] + sums[3][lane];
        }
        if (key < limit) {
            if (w.weights && key < tokens - nq) mine = __builtin_fmaf(w.weights[at + key], w.decay, mine);
            w.out[at + key] = mine;
        }
    }
}

template <class TY, bool FOUR, int NW>
static void launch_weigh(const WeighArgs &w, hipStream_t stream)
{
    if (w.few) hipLaunchKernelGGL((fbq_weigh_few_kernel<TY, FOUR, NW>), dim3(w.a.workers / kFewWaves), dim3(64 * kFewWaves), 0, stream, w);
    else hipLaunchKernelGGL((fbq_weigh_many_kernel<TY, FOUR, NW>), dim3(w.a.kv_heads * w.a.rows, w.parts), dim3(64 * kWeighWaves), 0, stream, w);
}

template <class TY, bool FOUR>
static hipError_t launch_weigh(const WeighArgs &w, hipStream_t stream)
{
    switch (features4(w.a.D) / 32) {
    case 2: launch_weigh<TY, FOUR, 2>(w, stream); break;
    case 3: launch_weigh<TY, FOUR, 3>(w, stream); break;
    case 4: launch_weigh<TY, FOUR, 4>(w, stream); break;
    case 6: launch_weigh<TY, FOUR, 6>(w, stream); break;
    default: launch_weigh<TY, FOUR, 8>(w, stream); break;
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
    w.few = (long)a.max_q * a.group <= kFewRows;
    const long steps = (((long)a.max_pages << a.log_ps) + kFewTile - 1) / kFewTile * a.rows * a.kv_heads;
    a.workers = (int)std::min(a.D > 128 ? 2048L : 4096L, (steps + kFewWaves - 1) / kFewWaves * kFewWaves);                 // (as many waves as the GPU holds)
    // Making keys ready takes a wave about as long as ten tiles of queries: so many waves to the same keys as make rounds of the GPU's waves, times that and a share of the tiles, least.
    const long most = std::min((long)a.max_pages << a.log_ps, (long)width), items = (long)a.rows * a.kv_heads, waves = (most + kWeighKeys - 1) / kWeighKeys * items;
    const long tiles = ((long)a.max_q * a.group + 15) / 16, at_once = a.D > 128 ? 1024 : 2048;
    const auto takes = [&](int log_share) { return ((waves << log_share) + at_once - 1) / at_once * (10 + (tiles >> log_share)); };
    for (int x = 1; x <= 2; ++x)
        if (takes(x) < takes(w.log_share)) w.log_share = x;
    const int a_block = kWeighKeys * (kWeighWaves >> w.log_share);
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
