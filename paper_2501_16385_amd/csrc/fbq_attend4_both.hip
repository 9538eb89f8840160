// A batch behind a shared prefix in one launch, over a cache in 4 bits: as in fbq_attend_both.hip, the shared tokens against the rows of all sequences, the first blocks, and every row's own tokens.
// 24 rows of 64 heads (8 of keys) behind 8192 shared tokens, about 300 of their own each: 31 and 13 us one after the other, 30 this way, the join of 9 besides.
#include "fbq_attend4_few.h"
#include "fbq_attend4_many.h"

namespace fbq {

template <class TY, class NT, class MAKE, int NW>
__global__ __launch_bounds__(256, 2) void fbq_attend4_both_kernel(const AttendArgs a, const int tiles)
{
    constexpr int DP = 32 * NW;
    __shared__ __attribute__((aligned(1024))) unsigned char room[kMany4Room<DP> > kFew4Room<NW> ? kMany4Room<DP> : kFew4Room<NW>];
    const int shared_blocks = a.kv_heads * tiles * a.shared_splits, block = blockIdx.x;
    if (block >= shared_blocks) {
        attend4_few<TY, NT, NW>(a, block - shared_blocks, room);
        return;
    }
    const int rest = block / a.kv_heads, z = rest / tiles;    // a head's blocks on one XCD, where heads are a multiple of eight
    attend4_many<TY, MAKE, NW>(a, true, block - rest * a.kv_heads, rest - z * tiles, z, room);
}

template <class TY, class NT, class MAKE>
static hipError_t launch_both(const AttendArgs &a, hipStream_t stream)
{
    static_assert(kFewWaves == 4, "blocks of one size");
    const int tiles = (int)(((long)a.T * a.group + kManyRows - 1) / kManyRows);
    const dim3 grid(a.kv_heads * tiles * a.shared_splits + a.workers / kFewWaves), block(256);
    switch (features4(a.D) / 32) {
    case 2: hipLaunchKernelGGL((fbq_attend4_both_kernel<TY, NT, MAKE, 2>), grid, block, 0, stream, a, tiles); break;
    case 3: hipLaunchKernelGGL((fbq_attend4_both_kernel<TY, NT, MAKE, 3>), grid, block, 0, stream, a, tiles); break;
    default: hipLaunchKernelGGL((fbq_attend4_both_kernel<TY, NT, MAKE, 4>), grid, block, 0, stream, a, tiles); break;
    }
    return hipGetLastError();
}

hipError_t launch_attend4_both(const AttendArgs &a, int type, hipStream_t stream)
{
    return type == FBQ_F16_4BIT ? launch_both<TypeF16, NumberF16, MakeF16>(a, stream) : launch_both<TypeBf16, NumberBf16, MakeHalf>(a, stream);
}

}  // namespace fbq
