// Launches of the many-row kernel over a cache in 4 bits (fbq_attend4_many.h).
#include "fbq_attend4_many.h"

namespace fbq {

template <class TY, class MAKE, int NW>
__global__ __launch_bounds__(256, NW > 4 ? 1 : 2) void fbq_attend4_many_kernel(const AttendArgs a, const bool shared)
{
    constexpr int DP = NW == 6 ? 256 : 32 * NW;
    __shared__ __attribute__((aligned(1024))) unsigned char room[kMany4Room<DP>];
    const bool pieces = shared && a.shared_splits > 1;
    attend4_many<TY, MAKE, NW>(a, shared, blockIdx.x, pieces ? blockIdx.y : blockIdx.y + blockIdx.z * kGridTiles, pieces ? blockIdx.z : 0, room);
}

template <class TY, class MAKE>
static hipError_t launch_many(const AttendArgs &a, bool shared, hipStream_t stream)
{
    const dim3 grid = many_grid(a, shared), block(256);
    switch (features4(a.D) / 32) {
    case 2: hipLaunchKernelGGL((fbq_attend4_many_kernel<TY, MAKE, 2>), grid, block, 0, stream, a, shared); break;
    case 3: hipLaunchKernelGGL((fbq_attend4_many_kernel<TY, MAKE, 3>), grid, block, 0, stream, a, shared); break;
    case 4: hipLaunchKernelGGL((fbq_attend4_many_kernel<TY, MAKE, 4>), grid, block, 0, stream, a, shared); break;
    case 6: hipLaunchKernelGGL((fbq_attend4_many_kernel<TY, MAKE, 6>), grid, block, 0, stream, a, shared); break;
    default: hipLaunchKernelGGL((fbq_attend4_many_kernel<TY, MAKE, 8>), grid, block, 0, stream, a, shared); break;
    }
    return hipGetLastError();
}

hipError_t launch_attend4_many(const AttendArgs &a, int type, bool shared, hipStream_t stream)
{
    return type == FBQ_F16_4BIT ? launch_many<TypeF16, MakeF16>(a, shared, stream) : launch_many<TypeBf16, MakeHalf>(a, shared, stream);
}

}  // namespace fbq
