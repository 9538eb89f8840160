// Keys and values of a cache in 4 bits on their way to the many-row kernel's LDS (fbq_attend_many.h): asked for in their codes, a step later made into 16 bits and put down where that
// kernel reads them.  With 128 query rows to a block, rows are too many for scales that come in behind the products, as they do in fbq_attend4_few.h: m + s c is rounded to the operand once.  (Whole
// codes of keys as operands, 32 scores a lane times a scale for each group: relative L2 against 64 bits 3.4e-4 instead of 5.7e-4 for scores with a standard deviation of 2 - the codes themselves are 0.19
// off what they stand for there - and 254 us instead of 208 for 1000 tokens each behind 5000 of three rows, heads of 80.)
// The operands are fp16 also for a cache of bf16 - queries too, times a power of two a row - since that is eight times as exact and takes half the instructions: relative L2 against 64 bits
// 1.7e-3 instead of 4.2e-3, of which rounding the result is 1.6e-3.  That wants scales from 2^-13 to 2^11 and lowest values up to 2^15 (or groups of zeros); a block that meets others does
// its work again with operands of bf16, at about twice the time (fbq_attend4_many.h).
// A step's codes are made in shares, among the matrix products of the step before.  Values are put down turned, [feature][64 keys], since that is how their codes lie: 16 bytes are eight
// keys of a feature in the order that the probabilities have.
#ifndef FBQ_ATTEND_CODES_H
#define FBQ_ATTEND_CODES_H

#include <algorithm>

#include "fbq_attend.h"
#include "fbq_cache4.h"
#include "fbq_lds_copy.h"

namespace fbq {

__device__ __forceinline__ int key_swap(int row, int pieces);

// N words in a row of each lane.
template <int N, int POLICY>
__device__ __forceinline__ void load_words(uint32_t (&to)[N], __amdgpu_buffer_rsrc_t from, int off)
{
    typedef uint32_t word3_t __attribute__((ext_vector_type(3)));
#pragma unroll
    for (int i = 0; i < N / 4; ++i) {
        const word4_t w = __builtin_amdgcn_raw_buffer_load_b128(from, off + 16 * i, 0, POLICY);
#pragma unroll
        for (int e = 0; e < 4; ++e) to[4 * i + e] = w[e];
    }
    if constexpr (N % 4 == 1) to[N - 1] = __builtin_amdgcn_raw_buffer_load_b32(from, off + 4 * (N - 1), 0, POLICY);
    if constexpr (N % 4 == 2) {
        const word2_t w = __builtin_amdgcn_raw_buffer_load_b64(from, off + 4 * (N - 2), 0, POLICY);
        to[N - 2] = w[0];
        to[N - 1] = w[1];
    }
    if constexpr (N % 4 == 3) {
        const word3_t w = __builtin_amdgcn_raw_buffer_load_b96(from, off + 4 * (N - 3), 0, POLICY);
        to[N - 3] = w[0];
        to[N - 2] = w[1];
        to[N - 1] = w[2];
    }
}

struct NoCodes {};

// Where piece p (16 bytes: eight keys) of a feature's 64 keys lies: equal pieces of eight features in a row, and of every fourth of 32, fall on different banks.
__device__ __forceinline__ int turned_at(int feature, int piece) { return feature * 128 + ((piece ^ (feature & 7) ^ (feature >> 3 & 3)) << 4); }

// How pairs of codes become pairs of operands: of `codes` those at low bits (or, HIGH, at high ones), with the scales and lowest values of the two, which scale_pair and low_pair make of their
// scale words.  Number: the scale words' type; Operand: the products'.
struct MakeF16 {
    typedef NumberF16 Number;
    typedef TypeF16 Operand;
    typedef _Float16 half2_t __attribute__((ext_vector_type(2)));
    // kChecked: scales may be out of its range; kScaled: queries become fp16 times a power of two a row; kTwice: of a kernel that may do its work again in another form
    static constexpr bool kChecked = false, kScaled = false, kTwice = false;
    static __device__ __forceinline__ uint32_t scale_pair(uint32_t a, uint32_t b) { return (a >> 16) | (b & 0xffff0000u); }
    static __device__ __forceinline__ uint32_t low_pair(uint32_t a, uint32_t b) { return (a & 0xffff) | b << 16; }
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
struct MakeHalf : MakeF16 {              // a cache of bf16 in operands of fp16: its scale words become fp16 on their way to the lanes that need them
    typedef NumberBf16 Number;
    static constexpr bool kChecked = true, kScaled = true, kTwice = true;
    static __device__ __forceinline__ uint32_t halves(uint32_t word) { return TypeF16::pack(Number::of(word & 0xffff), Number::of_upper(word)); }
};
struct MakeBf16 {
    typedef NumberBf16 Number;
    typedef TypeBf16 Operand;
    static constexpr bool kChecked = false, kScaled = false, kTwice = true;
    static __device__ __forceinline__ uint32_t scale_pair(uint32_t a, uint32_t b) { return MakeF16::scale_pair(a, b); }
    static __device__ __forceinline__ uint32_t low_pair(uint32_t a, uint32_t b) { return MakeF16::low_pair(a, b); }
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
    typedef MAKE Make;
    static constexpr int kWords = NW, kLast = lane_features4(DS, G - 1);
    uint32_t k[NW], v[NW], ks, vs;                            // scale words: of key l % 16, group l / 16
    uint32_t of_key[G], of_four[4 * G];                       // while they are put down: of a key, and of four, [key][group]
    uint32_t *room;                                           // 16 G words of the wave's in LDS, where lanes find each other's scale words
    long head_bytes;
    int own_lane;
    int k_at, v_at, last_at;                                  // where this lane's things go in a tile: the others' places follow from these
    unsigned long long met;                                   // lanes that have met a scale word out of range

    // (of two ways to the same number the one that leaves the loop more registers; both were tried for each)
    __device__ __forceinline__ int the_lane() const { return MAKE::kTwice ? own_lane : threadIdx.x & 63; }
    // Features from DS on are zeros for good: nothing else is put there.
    template <int PIECES>
    __device__ __forceinline__ void begin(const AttendArgs &a, unsigned char *keys, unsigned char *values, unsigned char *rooms, int wave, int lane)
    {
        room = reinterpret_cast<uint32_t *>(rooms) + wave * 64;
        own_lane = lane;
        const int r = lane & 15, g = lane >> 4, row = 16 * wave + r, piece = 2 * wave + (g & 1), half = 8 * (g >> 1);
        head_bytes = (a.page_bytes >> 1) / a.kv_heads;
        k_at = row * PIECES * 16 + ((g ^ key_swap(row, PIECES)) << 4);
        v_at = turned_at(4 * r, piece) + half;
        last_at = turned_at(kLast * r, piece) + half;
        met = 0;
        if constexpr (DP > DS) {
#pragma unroll
            for (int p = DS / 8; p < DP / 8; p += 4) *reinterpret_cast<word4_t *>(keys + row * PIECES * 16 + (((p + g) ^ key_swap(row, PIECES)) << 4)) = word4_t{0, 0, 0, 0};
#pragma unroll
            for (int f = DS; f < DP; f += 32) *reinterpret_cast<word4_t *>(values + turned_at(f + (lane & 31), 2 * wave + (lane >> 5))) = word4_t{0, 0, 0, 0};
        }
    }

    // The codes of 16 keys, or values, from `key` on, in `page` (whatever it is: none of the pool's, then zeros).
    __device__ __forceinline__ void ask(const AttendArgs &a, int h, int page, int key, int limit, bool values)
    {
        const int lane = the_lane(), slot = key & ((1 << a.log_ps) - 1);
        const int valid = (unsigned)page < (unsigned)a.pages ? min(max(limit - key, 0), 16) : 0;
        const unsigned char *const head = a.kv + (valid ? page : 0) * a.page_bytes + (values ? a.page_bytes >> 1 : 0) + h * head_bytes;
        const __amdgpu_buffer_rsrc_t codes = buffer_of(head + codes_at4(slot, DS), valid ? 8 * DS : 0), scales = buffer_of(head + scales_at4(a.log_ps, slot, DS), valid * 4 * G);
        uint32_t (&to)[NW] = values ? v : k;
        const int off = (values ? lane : (lane & 15) * 4 + (lane >> 4)) * NW * 4;
        load_words<NW, 0>(to, codes, off);
        (values ? vs : ks) = __builtin_amdgcn_raw_buffer_load_b32(scales, lane >> 4 < G ? ((lane & 15) * G + (lane >> 4)) * 4 : kNowhere, 0, 0);
    }
    // The scale words that are needed for what is put down next.  (All in one wave: LDS serves it in order.)
    __device__ __forceinline__ void spread(bool values)
    {
        const int lane = the_lane();
        uint32_t word = values ? vs : ks;
        if constexpr (MAKE::kChecked) {
            look(word);
            word = MAKE::halves(word);
        }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        if (lane >> 4 < G) room[(lane & 15) * G + (lane >> 4)] = word;
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        if (values) {
#pragma unroll
            for (int i = 0; i < 4 * G; ++i) of_four[i] = room[(lane >> 4) * 4 * G + i];
        } else {
#pragma unroll
            for (int i = 0; i < G; ++i) of_key[i] = room[(lane & 15) * G + i];
        }
    }
    // (addresses anew every step: all of them in registers would push others out)
    __device__ __forceinline__ void step()
    {
        asm volatile("" : "+v"(k_at), "+v"(v_at));
        if (kLast != 4) asm volatile("" : "+v"(last_at));
    }
    // Out of what fp16 operands are made for: neither zeros nor keys that are NaN, and a scale below 2^-13 or from 2^11 + 2^4 on, or a lowest value beyond 2^15.
    __device__ __forceinline__ void look(uint32_t word) { met |= __ballot(word != 0 && word != NumberBf16::kNaN << 16 && (word - 0x39000000u > 0x0c00ffffu || (word & 0x7fff) > 0x4700u)); }
    // Features 32 w + 8 g .. of key 16 wave + l % 16: a piece.
    __device__ __forceinline__ void put_keys(int w, unsigned char *tile)
    {
        const uint32_t c = k[w], word = of_key[w / 2], s = MAKE::scale_pair(word, word), m = MAKE::low_pair(word, word);
        *reinterpret_cast<word4_t *>(tile + (k_at ^ 64 * w)) =
            word4_t{MAKE::template two<false>(c, s, m), MAKE::template two<false>(c >> 8, s, m), MAKE::template two<true>(c, s, m), MAKE::template two<true>(c >> 8, s, m)};
    }
    // Keys 4 g .. of the wave's sixteen: the two features that lane r = l % 16 has of word x.
    __device__ __forceinline__ void put_values(int x, unsigned char *tile)
    {
        const int y = x / 2, j = 2 * (x & 1), at = y == G - 1 ? last_at : v_at;
        const auto word = [&](int key) __attribute__((always_inline)) { return of_four[key * G + y]; };
        const uint32_t c = v[x], s0 = MAKE::scale_pair(word(0), word(1)), s1 = MAKE::scale_pair(word(2), word(3)), m0 = MAKE::low_pair(word(0), word(1)), m1 = MAKE::low_pair(word(2), word(3));
        *reinterpret_cast<word2_t *>(tile + (at ^ j << 4) + (64 * y + j) * 128) = word2_t{MAKE::template two<false>(c, s0, m0), MAKE::template two<false>(c >> 8, s1, m1)};
        *reinterpret_cast<word2_t *>(tile + (at ^ (j + 1) << 4) + (64 * y + j + 1) * 128) = word2_t{MAKE::template two<true>(c, s0, m0), MAKE::template two<true>(c >> 8, s1, m1)};
    }
};

}  // namespace fbq

#endif
