// The cache in 4 bits: new keys and values quantized into their pages, and tokens of a cache read back as numbers.
#include <algorithm>

#include "fbq_attend.h"
#include "fbq_cache4.h"
#include "fbq_internal.h"

namespace fbq {

// Append: a wave takes one head's new tokens of one block of 16.  Lane l has token l % 16, features 32 w + 8 g .. of g = l / 16: a group's least and largest
// are over a lane's own and three neighbours'.  Key codes are then the lane's own words.  Values lie four tokens to a word: their codes go through LDS, one byte each, and where some of a
// word's tokens are not of this call the rest of the word is kept.  Nobody else writes the word: a partial page has one holder.
// Of a block of 16's new tokens the first is the one that it is done for.  A grid block looks at WINDOW tokens for such ones: at one where rows have few, and its keys and values are then on their
// way before it knows where they go; at 16 where they have many (16 times as many blocks that find nothing: 62 us for 4267 tokens of 32 heads, 33 this way).  At one a wave has the keys or the
// values alone: 16 tokens of 32 heads 5.0 us for 6.6, a chain of loads, minima and quotients that no size shortens.  At 16, 70 MB read and 20 written in
// 28 to 33 us from card to card.  Counters: vector instructions, 1364 a wave of a block of 16, keep the units busy 55 % of that; the waves, 2.5 a SIMD, wait for loads 36 % of theirs and as long for each other's
// instructions: loads, codes, LDS and stores of a block follow each other, and the few waves hide only a part.
template <class NT, int NW, int WINDOW>
__global__ __launch_bounds__(256) void fbq_append4_kernel(CacheArgs c, long layer_offset, int T, const int32_t *__restrict__ q_start, const int32_t *__restrict__ start,
                                                          const uint16_t *__restrict__ k, long k_stride, const uint16_t *__restrict__ v, long v_stride)
{
    constexpr int DS = 32 * NW, G = groups4(DS), kRow = DS + 16;
    constexpr int kSure = NW == 2 ? 0 : NW == 8 ? 6 : NW == 6 ? 4 : NW - 1;       // words before it have no feature past the last
    __shared__ __attribute__((aligned(16))) unsigned char room[4][16 * kRow];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, slot = lane & 15, g = lane >> 4;
    // (at one token a wave makes the keys or the values alone: half as long a chain)
    const int h = WINDOW == 1 ? blockIdx.y * 2 + (wave >> 1) : blockIdx.y * 4 + wave, head = min(h, c.kv_heads - 1);
    const bool has_keys = WINDOW > 1 || (wave & 1) == 0, has_values = WINDOW > 1 || (wave & 1);
    const long head_bytes = (c.page_bytes >> 1) / c.kv_heads;

    word4_t x[2][NW];
    const auto ask = [&](int token, bool mine) __attribute__((always_inline)) {
#pragma unroll
        for (int which = 0; which < 2; ++which) {
            const uint16_t *const from = (which ? v + token * v_stride : k + token * k_stride) + (long)head * c.D;
#pragma unroll
            for (int w = 0; w < NW; ++w) {
                x[which][w] = word4_t{0, 0, 0, 0};
                if (mine && 32 * w + 8 * g < c.D) x[which][w] = *reinterpret_cast<const word4_t *>(from + 32 * w + 8 * g);
            }
        }
    };
    if (WINDOW == 1) ask(blockIdx.x, true);                   // (of the first token in every lane: of others later, where there are any)

    // which of the window's tokens blocks of 16 are done for: a lane each
    const int mine_t = blockIdx.x * WINDOW + lane % WINDOW;
    int of_row = -1, of_count = 0, of_page = -1;
    long of_pos = 0;
    if (mine_t < T) {
        const int b = q_start ? row_of_token(q_start, c.rows, mine_t) : mine_t;
        const int first = b < 0 ? -1 : start[b];
        if (first >= 0) {
            const int i = q_start ? mine_t - q_start[b] : 0;
            of_pos = (long)first + i;
            of_count = (q_start ? q_start[b + 1] - q_start[b] : 1) - i;
            if ((i == 0 || (of_pos & 15) == 0) && of_pos < (long)c.max_pages << c.log_ps) of_row = b;
            if (of_row >= 0) of_page = c.table[(long)b * c.max_pages + (of_pos >> c.log_ps)];
            if ((unsigned)of_page >= (unsigned)c.pages) of_row = -1;
        }
    }
    for (unsigned long long left = __ballot(of_row >= 0) & ((1ull << WINDOW) - 1); left; left &= left - 1) {
        const int who = __builtin_ctzll(left), t = blockIdx.x * WINDOW + who;
        const int page = __builtin_amdgcn_readlane(of_page, who), low = __builtin_amdgcn_readlane((int)of_pos, who);      // (below 2^24)
        const int s0 = low & 15, s1 = min(16, s0 + min(__builtin_amdgcn_readlane(of_count, who), T - t));             // slots of the block that get a token
        const bool mine = h < c.kv_heads && slot >= s0 && slot < s1;
        const int place = low & ((1 << c.log_ps) - 1) & ~15;                          // of the block, in its page
        unsigned char *const keys = c.pool + layer_offset + page * c.page_bytes + head * head_bytes, *const values = keys + (c.page_bytes >> 1);
        if (WINDOW > 1 || s1 - s0 > 1) ask(t + slot - s0, mine);

        // values: lane r = l % 16 of tokens 4 g .. 4 g + 3 writes its words of all products; `keep` has the bits of the tokens that are not this call's
        uint32_t keep = 0, old[NW];
#pragma unroll
        for (int j = 0; j < 4; ++j)
            if (4 * g + j < s0 || 4 * g + j >= s1) keep |= 0xffu << 8 * byte_of_token4(j);
        const bool writes = has_values && h < c.kv_heads && keep != 0xffffffffu;
        uint32_t *const words = reinterpret_cast<uint32_t *>(values + codes_at4(place, DS)) + lane * NW;          // (lane = 16 g + r)
#pragma unroll
        for (int w = 0; w < NW; ++w) old[w] = writes && keep ? words[w] : 0;

        uint32_t above = 0;                                   // halves with an exponent of ones are not finite
#pragma unroll
        for (int which = 0; which < 2; ++which)
#pragma unroll
            for (int w = 0; w < NW; ++w)
#pragma unroll
                for (int y = 0; y < 4; ++y) {
                    typedef uint16_t short2_t __attribute__((ext_vector_type(2)));
                    above = __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(short2_t, above), __builtin_bit_cast(short2_t, x[which][w][y] & 0x7fff7fffu)));
                }
        bool odd = mine && ((above & 0xffff) >= NT::kExponent || above >> 16 >= NT::kExponent);
        const unsigned long long bad = __ballot(odd);
        odd = ((bad | bad >> 16 | bad >> 32 | bad >> 48) >> slot & 1) != 0;           // ... in any of the token's four lanes

        uint32_t key_codes[NW];
#pragma unroll
        for (int which = 0; which < 2; ++which) {
            if (!(which ? has_values : has_keys)) continue;
#pragma unroll
            for (int y = 0; y < G; ++y) {
                // halves throughout, so that no difference is beyond fp32 (of bf16 numbers)
                float low = INFINITY, high = -INFINITY;
#pragma unroll
                for (int w = 2 * y; w < std::min(2 * y + 2, NW); ++w)
                    if (32 * w + 8 * g < c.D)
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            const float x0 = NT::of(x[which][w][e] & 0xffff) * 0.5f, x1 = NT::of_upper(x[which][w][e]) * 0.5f;
                            low = fminf(low, fminf(x0, x1));
                            high = fmaxf(high, fmaxf(x0, x1));
                        }
                low = -larger_of_32(larger_of_16(-low)) + 0.0f;       // (no zero with a sign)
                high = larger_of_32(larger_of_16(high));
                const float d = high - low;                           // (head_dim reaches into every group of DS)
                uint32_t s = NT::bits(d / 7.5f);
                if (NT::of(s) * 7.5f < d) ++s;
                if (s && __builtin_fmaf(NT::of(s), 15.0f, 2.0f * low) > NT::kMost) --s;
                // x / half to the nearest number: x times the reciprocal, itself the nearest, and one step of correction, which is exact; where the reciprocal is no number, by division
                const float half = NT::of(s) * 0.5f, by = half > 0 ? 1.0f / half : 0.0f;
                const bool plain = __ballot(half > 0 && half < 0x1p-120f) == 0;
                uint32_t word = s << 16 | NT::bits(2.0f * low);
                if (odd) word = which ? 0u : NT::kNaN << 16;
                if (mine && g == y) *reinterpret_cast<uint32_t *>((which ? values : keys) + scales_at4(c.log_ps, place + slot, DS) + 4 * y) = word;
                const auto make = [&](auto quotient) __attribute__((always_inline)) {
#pragma unroll
                    for (int w = 2 * y; w < std::min(2 * y + 2, NW); ++w) {
                        // keys: nibble n is feature e, n with its bits in reverse; values: a byte each
                        uint32_t lower = 0, upper = 0;        // features 0 .. 3 and 4 .. 7
#pragma unroll
                        for (int e = 0; e < 8; ++e) {
                            const uint32_t word = x[which][w][e >> 1];
                            const float at = __builtin_fmaf(e & 1 ? NT::of_upper(word) : NT::of(word & 0xffff), 0.5f, -low), code = fminf(fmaxf(rintf(quotient(at)), 0.0f), 15.0f);
                            const int byte = which ? e & 3 : (e & 1) << 1 | (e >> 1 & 1);
                            if (e < 4) lower = __builtin_amdgcn_cvt_pk_u8_f32(code, byte, lower);
                            else upper = __builtin_amdgcn_cvt_pk_u8_f32(code, byte, upper);
                        }
                        if (w >= kSure && 32 * w + 8 * g >= c.D) lower = upper = 0;
                        if (which == 0) key_codes[w] = lower | upper << 4;
                        else *reinterpret_cast<word2_t *>(&room[wave][slot * kRow + 32 * w + 8 * g]) = word2_t{lower, upper};
                    }
                };
                if (plain) make([&](float at) { const float near = at * by; return __builtin_fmaf(__builtin_fmaf(-near, half, at), by, near); });
                else make([&](float at) { return half > 0 ? at / half : 0.0f; });
            }
        }
        if (mine && has_keys) {
            uint32_t *const to = reinterpret_cast<uint32_t *>(keys + codes_at4(place, DS)) + (slot * 4 + g) * NW;
#pragma unroll
            for (int w = 0; w < NW; ++w) to[w] = key_codes[w];
        }
        __syncthreads();
#pragma unroll
        for (int y = 0; y < G; ++y) {
            const int z = lane_features4(DS, y);
            uint32_t pairs[4];                                // two codes of a token in bits 0 .. 7, two more in bits 16 .. 23
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const unsigned char *const at = &room[wave][(4 * g + j) * kRow + 64 * y + z * slot];
                const uint32_t codes = z == 4 ? *reinterpret_cast<const uint32_t *>(at) : *reinterpret_cast<const uint16_t *>(at);
                pairs[j] = codes | codes >> 4;
            }
#pragma unroll
            for (int w = 2 * y; w < 2 * y + z / 2; ++w) {
                uint32_t word = 0;
#pragma unroll
                for (int j = 0; j < 4; ++j) word |= (pairs[j] >> 16 * (w & 1) & 0xff) << 8 * byte_of_token4(j);
                if (writes) words[w] = (word & ~keep) | (old[w] & keep);
            }
        }
        __syncthreads();
    }
}

template <class NT>
static hipError_t launch_append(const CacheArgs &c, long layer_offset, int T, const int32_t *q_start, const int32_t *start, const void *k, long k_stride, const void *v, long v_stride,
                                hipStream_t stream)
{
    const auto go = [&](auto few, auto many) {
        const bool wide = q_start && T > 4L * c.rows;
        hipLaunchKernelGGL(wide ? many : few, dim3(wide ? ceil_div(T, 16) : T, ceil_div(c.kv_heads, wide ? 4 : 2)), dim3(256), 0, stream, c, layer_offset, T, q_start, start, (const uint16_t *)k, k_stride,
                           (const uint16_t *)v, v_stride);
    };
    switch (features4(c.D) / 32) {
    case 2: go(fbq_append4_kernel<NT, 2, 1>, fbq_append4_kernel<NT, 2, 16>); break;
    case 3: go(fbq_append4_kernel<NT, 3, 1>, fbq_append4_kernel<NT, 3, 16>); break;
    case 4: go(fbq_append4_kernel<NT, 4, 1>, fbq_append4_kernel<NT, 4, 16>); break;
    case 6: go(fbq_append4_kernel<NT, 6, 1>, fbq_append4_kernel<NT, 6, 16>); break;
    default: go(fbq_append4_kernel<NT, 8, 1>, fbq_append4_kernel<NT, 8, 16>); break;
    }
    return hipGetLastError();
}

hipError_t launch_append4(const CacheArgs &c, int type, long layer_offset, int T, const int32_t *q_start, const int32_t *start, const void *k, long k_stride, const void *v, long v_stride,
                          hipStream_t stream)
{
    return type == FBQ_F16_4BIT ? launch_append<NumberF16>(c, layer_offset, T, q_start, start, k, k_stride, v, v_stride, stream)
                                : launch_append<NumberBf16>(c, layer_offset, T, q_start, start, k, k_stride, v, v_stride, stream);
}

// Read: a block a token.  Four features a thread and step; what is written is seven times what is read (16 bits: twice), and bounds it (4270 tokens of 32 heads of 128, 140 MB written and 20 read:
// 29 to 31 us, 5.0 TB/s and more; a large copy moves 4.9.  Of 16 bits, 70 MB read: 34.  16 single tokens 5.2 and 4.3).
template <class NT, bool FOUR>
__global__ __launch_bounds__(256) void fbq_cache_read_kernel(CacheArgs c, long layer_offset, const int32_t *__restrict__ q_start, const int32_t *__restrict__ start, float *__restrict__ k,
                                                             float *__restrict__ v)
{
    // Sixteen tokens in a row on one XCD (blocks go round the eight in turn): four share words, and lines (36 us without).
    const int of = blockIdx.x & 127, t = blockIdx.x - of + 128 <= gridDim.x ? blockIdx.x - of + (of & 7) * 16 + (of >> 3) : blockIdx.x;
    const int b = q_start ? row_of_token(q_start, c.rows, t) : t;
    if (b < 0) return;
    const int first = start[b];
    if (first < 0) return;
    const long pos = (long)first + (q_start ? t - q_start[b] : 0);
    if (pos >= (long)c.max_pages << c.log_ps) return;
    const int page = c.table[(long)b * c.max_pages + (pos >> c.log_ps)];
    if ((unsigned)page >= (unsigned)c.pages) return;
    const int slot = (int)pos & ((1 << c.log_ps) - 1), fours = c.D >> 2, DS = features4(c.D), token = slot & 15;
    const long head_bytes = (c.page_bytes >> 1) / c.kv_heads;
    const unsigned char *const from = c.pool + layer_offset + page * c.page_bytes;
    for (int i = threadIdx.x; i < 2 * c.kv_heads * fours; i += 256) {
        const int which = i >= c.kv_heads * fours, j = i - which * c.kv_heads * fours, h = j / fours, d = (j - h * fours) * 4;
        float *const to = which ? v : k;
        if (!to) continue;
        const unsigned char *const head = from + which * (c.page_bytes >> 1) + h * head_bytes;
        float4_t x;
        if (!FOUR) {
            const word2_t w = *reinterpret_cast<const word2_t *>(head + ((long)slot * c.D + d) * 2);
            x = float4_t{NT::of(w[0] & 0xffff), NT::of_upper(w[0]), NT::of(w[1] & 0xffff), NT::of_upper(w[1])};
        } else {
            const uint32_t *const codes = reinterpret_cast<const uint32_t *>(head + codes_at4(slot, DS));
            const uint32_t scale = *reinterpret_cast<const uint32_t *>(head + scales_at4(c.log_ps, slot, DS) + 4 * (d >> 6));
            uint32_t four;                                    // codes of features d .. d + 3, a byte each
            if (!which) {
                const uint32_t w = codes[(token * 4 + (d >> 3 & 3)) * (DS / 32) + (d >> 5)] >> (d & 4);          // features e and e + 4 are neighbours
                four = (w & 15) | (w >> 16 & 15) << 8 | (w >> 8 & 15) << 16 | (w >> 24 & 15) << 24;
            } else {
                const int y = d >> 6, z = lane_features4(DS, y), r = (d & 63) / z, at = 8 * byte_of_token4(token & 3);
                const uint32_t *const words = codes + ((token >> 2) * 16 + r) * (DS / 32) + 2 * y;
                const uint32_t lo = words[0] >> at, hi = (z == 4 ? words[1] : words[DS / 32]) >> at;             // (z = 2: the next lane's)
                four = (lo & 15) | (lo >> 4 & 15) << 8 | (hi & 15) << 16 | (hi >> 4 & 15) << 24;
            }
            const float s = NT::of_upper(scale), m = NT::of(scale & 0xffff);
#pragma unroll
            for (int e = 0; e < 4; ++e) x[e] = __builtin_fmaf(s, (float)(four >> 8 * e & 255), m);
        }
        *reinterpret_cast<float4_t *>(to + ((long)t * c.kv_heads + h) * c.D + d) = x;
    }
}

}  // namespace fbq

using namespace fbq;

extern "C" fbq_status fbq_cache_read(const fbq_cache *c, int layer, int T, const int32_t *q_start, const int32_t *start, float *k, float *v, fbq_stream stream)
{
    const fbq_status st = check_cache(c, false);
    if (st != FBQ_OK) return st;
    if (layer < 0 || layer >= c->desc.layers || T < 1 || T > (1 << 23) || (!q_start && T != c->rows)) return FBQ_ERR_SHAPE;
    if (!start || (!k && !v)) return FBQ_ERR_NULL;
    if (!aligned(q_start, 4) || !aligned(start, 4) || !aligned(k, 16) || !aligned(v, 16)) return FBQ_ERR_ALIGN;
    const CacheArgs a = cache_args(*c);
    const auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, dim3(T), dim3(256), 0, (hipStream_t)stream, a, layer * a.layer_bytes, q_start, start, k, v); };
    switch (c->desc.type) {
    case FBQ_F16: go(fbq_cache_read_kernel<NumberF16, false>); break;
    case FBQ_BF16: go(fbq_cache_read_kernel<NumberBf16, false>); break;
    case FBQ_F16_4BIT: go(fbq_cache_read_kernel<NumberF16, true>); break;
    default: go(fbq_cache_read_kernel<NumberBf16, true>); break;
    }
    return hipGetLastError() == hipSuccess ? FBQ_OK : FBQ_ERR_HIP;
}
