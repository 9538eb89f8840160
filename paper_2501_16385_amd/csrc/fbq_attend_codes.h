// Keys and values of a cache in 4 bits on their way to the many-row kernel's LDS (fbq_attend_many.h): asked for in their codes, a step later made into the 16-bit type and put down where that
// kernel reads them.  m + s c is rounded to the type once (relative 2^-11, 2^-8 for bf16: as the operands of a cache in 16 bits are, and less than the codes' own half steps): with
// 128 query rows to a block, rows are too many for scales that come in behind the products, as they do in fbq_attend4_few.h.
// Values are put down turned, [feature][64 keys], since that is how their codes lie: 16 bytes are eight keys of a feature in the order that the probabilities have.
#ifndef FBQ_ATTEND_CODES_H
#define FBQ_ATTEND_CODES_H

#include <algorithm>

#include "fbq_attend.h"
#include "fbq_cache4.h"
#include "fbq_lds_copy.h"

namespace fbq {

__device__ __forceinline__ int key_swap(int row, int pieces);

struct NoCodes {
    __device__ __forceinline__ void begin(const AttendArgs &) {}
};

// Where piece p (16 bytes: eight keys) of a feature's 64 keys lies: equal pieces of eight features in a row, and of every fourth of 32, fall on different banks.
__device__ __forceinline__ int turned_at(int feature, int piece) { return feature * 128 + ((piece ^ (feature & 7) ^ (feature >> 3 & 3)) << 4); }

// Four codes' pairs of a word into numbers of the type: the codes of `word` at low bits (or, HIGH, at high ones), the scales and lowest values of the pair's halves.
struct MakeF16 {
    typedef NumberF16 Number;
    typedef _Float16 half2_t __attribute__((ext_vector_type(2)));
    template <bool HIGH>
    static __device__ __forceinline__ uint32_t two(uint32_t codes, uint32_t s, uint32_t m)
    {
        // 1024 + c, or 1024 + 16 c, exactly; less the 1024 exactly, too
        const half2_t x = __builtin_bit_cast(half2_t, (codes & (HIGH ? kHighCodes : kLowCodes)) | 0x64006400u);
        const half2_t c = HIGH ? __builtin_elementwise_fma(x, half2_t{(_Float16)0.0625f, (_Float16)0.0625f}, half2_t{(_Float16)-64.0f, (_Float16)-64.0f})
                               : x - half2_t{(_Float16)1024.0f, (_Float16)1024.0f};
        return __builtin_bit_cast(uint32_t, __builtin_elementwise_fma(c, __builtin_bit_cast(half2_t, s), __builtin_bit_cast(half2_t, m)));
    }
};
struct MakeBf16 {
    typedef NumberBf16 Number;
    template <bool HIGH>
    static __device__ __forceinline__ uint32_t two(uint32_t codes, uint32_t s, uint32_t m)
    {
        const uint32_t c = HIGH ? codes >> 4 : codes;
        const float lo = __builtin_fmaf((float)(c & 15), Number::of(s & 0xffff), Number::of(m & 0xffff));
        const float hi = __builtin_fmaf((float)(c >> 16 & 15), Number::of_upper(s), Number::of_upper(m));
        return TypeBf16::pack(lo, hi);
    }
};

template <class MAKE, int NW, int DP>
struct Codes {
    static constexpr int DS = 32 * NW, G = groups4(DS);
    uint32_t k[NW], v[NW], ks[G];
    word4_t vs[G];                                            // [4 keys][groups]
    long head_bytes;

    __device__ __forceinline__ void begin(const AttendArgs &a) { head_bytes = (a.page_bytes >> 1) / a.kv_heads; }

    // The codes of 16 keys, or values, from `key` on, in `page` (whatever it is: none of the pool's, then zeros).
    __device__ __forceinline__ void ask(const AttendArgs &a, int h, int page, int key, int limit, bool values)
    {
        const int lane = threadIdx.x & 63, slot = key & ((1 << a.log_ps) - 1);
        const int valid = (unsigned)page < (unsigned)a.pages ? min(max(limit - key, 0), 16) : 0;
        const unsigned char *const head = a.kv + (valid ? page : 0) * a.page_bytes + (values ? a.page_bytes >> 1 : 0) + h * head_bytes;
        const __amdgpu_buffer_rsrc_t codes = buffer_of(head + codes_at4(slot, DS), valid ? 8 * DS : 0), scales = buffer_of(head + scales_at4(a.log_ps, slot, DS), valid * 4 * G);
        uint32_t (&to)[NW] = values ? v : k;
        const int off = (values ? lane : (lane & 15) * 4 + (lane >> 4)) * NW * 4;
#pragma unroll
        for (int w = 0; w < NW; ++w) to[w] = __builtin_amdgcn_raw_buffer_load_b32(codes, off + 4 * w, 0, 0);
        if (values) {
#pragma unroll
            for (int y = 0; y < G; ++y) vs[y] = __builtin_amdgcn_raw_buffer_load_b128(scales, (lane >> 4) * 16 * G + 16 * y, 0, 0);
        } else {
#pragma unroll
            for (int y = 0; y < G; ++y) ks[y] = __builtin_amdgcn_raw_buffer_load_b32(scales, (lane & 15) * 4 * G + 4 * y, 0, 0);
        }
    }
    // Features 32 w + 8 g .. of key 16 wave + l % 16, a piece each.
    template <int PIECES>
    __device__ __forceinline__ void put_keys(unsigned char *tile, int wave) const
    {
        const int lane = threadIdx.x & 63, row = 16 * wave + (lane & 15), g = lane >> 4, swap = key_swap(row, PIECES);
#pragma unroll
        for (int w = 0; w < DP / 32; ++w) {
            word4_t x{0, 0, 0, 0};
            if (w < NW) {
                const uint32_t c = k[std::min(w, NW - 1)], word = ks[std::min(w / 2, G - 1)], s = (word >> 16) | (word & 0xffff0000u), m = (word & 0xffff) | word << 16;
                x = word4_t{MAKE::template two<false>(c, s, m), MAKE::template two<false>(c >> 8, s, m), MAKE::template two<true>(c, s, m), MAKE::template two<true>(c >> 8, s, m)};
            }
            *reinterpret_cast<word4_t *>(tile + row * PIECES * 16 + (((4 * w + g) ^ swap) << 4)) = x;
        }
    }
    // Keys 4 g .. of the wave's sixteen, the features that lane r = l % 16 has of each product.
    __device__ __forceinline__ void put_values(unsigned char *tile, int wave) const
    {
        const int lane = threadIdx.x & 63, r = lane & 15, g = lane >> 4, piece = 2 * wave + (g & 1), half = 8 * (g >> 1);
#pragma unroll
        for (int y = 0; y < G; ++y) {
            const int z = lane_features4(DS, y);
            uint32_t s[2], m[2];
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const uint32_t a = vs[(2 * i * G + y) / 4][(2 * i * G + y) % 4], b = vs[((2 * i + 1) * G + y) / 4][((2 * i + 1) * G + y) % 4];
                s[i] = (a >> 16) | (b & 0xffff0000u);
                m[i] = (a & 0xffff) | b << 16;
            }
#pragma unroll
            for (int x = 0; x < z / 2; ++x) {
                const uint32_t c = v[2 * y + x];
                const int f = 64 * y + z * r + 2 * x;
                *reinterpret_cast<word2_t *>(tile + turned_at(f, piece) + half) = word2_t{MAKE::template two<false>(c, s[0], m[0]), MAKE::template two<false>(c >> 8, s[1], m[1])};
                *reinterpret_cast<word2_t *>(tile + turned_at(f + 1, piece) + half) = word2_t{MAKE::template two<true>(c, s[0], m[0]), MAKE::template two<true>(c >> 8, s[1], m[1])};
            }
        }
        if constexpr (DP > DS) {                              // features that there are not
#pragma unroll
            for (int f = DS; f < DP; f += 16) *reinterpret_cast<word2_t *>(tile + turned_at(f + r, piece) + half) = word2_t{0, 0};
        }
    }
};

}  // namespace fbq

#endif
