// How the keys of a tile of the many-row attention kernel are cut into pieces, from what its rows hold (for the device; the host's tests compile it, too).
#ifndef FBQ_ATTEND_PLAN_H
#define FBQ_ATTEND_PLAN_H

#include <stdint.h>

#include <hip/hip_runtime.h>

namespace fbq {

// How many steps a piece of a tile has at most, for `tiles` tiles a key/value head whose first and last rows' steps add up to `twice` - twice the steps there are - and `blocks` blocks
// that are on the GPU at once.  A piece more writes and reads 128 rows of partial results again, as dear as about six steps, and pieces that do not all fit the GPU at once
// wait for each other: so tiles are cut into as many as there is room for, the average tile and a fifth taken, and where there is none, those twice as long and six.
// (61 tiles of 8 heads and about 100 steps, cut in two where that was above an even share: 243 us; uncut 160.)
// Whole numbers throughout: the kernel that makes the pieces and the one that joins them work this out each for itself, and have to agree.  A tile has at most 2^18 steps, so that
// everything but the `twice` of very many tiles has 32 bits: that and the tiles lose their lowest past 31.
__host__ __device__ inline int share_of_steps(uint64_t twice, int tiles, int kv_heads, int blocks)
{
    uint32_t n = tiles > 1 ? tiles : 1;
    if (2 * (uint64_t)n * (uint32_t)kv_heads <= (uint32_t)blocks) {
        const uint32_t fit = (uint32_t)blocks / (n * (uint32_t)kv_heads), of = 5 * n * fit, share = (3 * (uint32_t)twice + of - 1) / of;      // 1.2 (twice / 2) / (n fit), rounded up
        return share > 4 ? (int)share : 4;
    }
    const int shift = (twice >> 31) ? 33 - __builtin_clzll(twice) : 0;
    n >>= shift;
    return (int)((uint32_t)(twice >> shift) / (n > 1 ? n : 1)) + 6;
}

}  // namespace fbq

#endif
