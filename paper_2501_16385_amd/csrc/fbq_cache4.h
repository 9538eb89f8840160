// A cache in 4 bits: where things lie (fbq.h has the layout) and the two 16-bit types' numbers (device code).
//
// The layout is that of the matrix cores' operands, so that attention reads codes straight into them.  A code c between zero bits of an fp16 is the number c 2^-24, at four bits
// higher c 2^-20 (below the normal numbers, which the matrix cores multiply exactly): a mask makes two operand elements of a word, a shift by eight gives the other half.  Nibbles n
// and n + 4 of a word are the two elements of an operand's register; even n are those at the low bits, odd n those four bits higher.
#ifndef FBQ_CACHE4_H
#define FBQ_CACHE4_H

#include "fbq_cache.h"

namespace fbq {

constexpr uint32_t kLowCodes = 0x000f000fu, kHighCodes = 0x00f000f0u;

// Numbers of the cache's 16-bit type in 32 bits, and back (to nearest, ties to even).
struct NumberF16 {
    static constexpr float kMost = 65504.0f;
    static constexpr bool kWide = false;                      // has fp32's range
    static constexpr uint32_t kExponent = 0x7c00u, kNaN = 0x7e00u;
    static __device__ __forceinline__ float of(uint32_t bits) { return (float)__builtin_bit_cast(_Float16, (uint16_t)bits); }
    static __device__ __forceinline__ float of_upper(uint32_t word) { return (float)__builtin_bit_cast(_Float16, (uint16_t)(word >> 16)); }
    static __device__ __forceinline__ uint32_t bits(float x) { return __builtin_bit_cast(uint16_t, (_Float16)x); }
};
struct NumberBf16 {
    static constexpr float kMost = 3.38953139e38f;
    static constexpr bool kWide = true;
    static constexpr uint32_t kExponent = 0x7f80u, kNaN = 0x7fc0u;
    static __device__ __forceinline__ float of(uint32_t bits) { return __builtin_bit_cast(float, bits << 16); }
    static __device__ __forceinline__ float of_upper(uint32_t word) { return __builtin_bit_cast(float, word & 0xffff0000u); }
    static __device__ __forceinline__ uint32_t bits(float x) { return __builtin_bit_cast(uint16_t, (__bf16)x); }
};

// Value products of a group: the z of the layout, features of one of the 16 lanes r.
__host__ __device__ __forceinline__ constexpr int lane_features4(int DS, int group) { return 64 * group + 64 <= DS ? 4 : 2; }

// The byte of a value word that has token 4 g + k.
__host__ __device__ __forceinline__ constexpr int byte_of_token4(int k) { return (k >> 1) | (k & 1) << 1; }

// Codes of a head's 16 tokens, and the scale words behind a page's codes, in bytes from the head's first.
__device__ __forceinline__ long codes_at4(int slot, int DS) { return (long)(slot >> 4) * 8 * DS; }
__device__ __forceinline__ long scales_at4(int log_ps, int slot, int DS) { return ((long)DS << log_ps >> 1) + (long)slot * 4 * groups4(DS); }

}  // namespace fbq

#endif
