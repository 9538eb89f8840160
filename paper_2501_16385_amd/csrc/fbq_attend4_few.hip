// Launches of the few-row kernel of a cache in 4 bits (fbq_attend4_few.h).
#include "fbq_attend4_few.h"

namespace fbq {

template <class TY, class NT, int NW>
__global__ __launch_bounds__(64 * kFewWaves, NW > 4 ? 1 : 2) void fbq_attend4_few_kernel(const AttendArgs a)
{
    __shared__ __attribute__((aligned(16))) unsigned char room[kFew4Room<NW>];
    attend4_few<TY, NT, NW>(a, blockIdx.x, room);
}

template <class TY, class NT>
static hipError_t launch_few(const AttendArgs &a, hipStream_t stream)
{
    const dim3 grid(a.direct == 2 ? a.rows * a.kv_heads : ((a.direct ? a.rows * a.kv_heads : a.workers) + kFewWaves - 1) / kFewWaves), block(64 * kFewWaves);
    switch (features4(a.D) / 32) {
    case 2: hipLaunchKernelGGL((fbq_attend4_few_kernel<TY, NT, 2>), grid, block, 0, stream, a); break;
    case 3: hipLaunchKernelGGL((fbq_attend4_few_kernel<TY, NT, 3>), grid, block, 0, stream, a); break;
    case 4: hipLaunchKernelGGL((fbq_attend4_few_kernel<TY, NT, 4>), grid, block, 0, stream, a); break;
    case 6: hipLaunchKernelGGL((fbq_attend4_few_kernel<TY, NT, 6>), grid, block, 0, stream, a); break;
    default: hipLaunchKernelGGL((fbq_attend4_few_kernel<TY, NT, 8>), grid, block, 0, stream, a); break;
    }
    return hipGetLastError();
}

hipError_t launch_attend4_few(const AttendArgs &a, int type, hipStream_t stream)
{
    return type == FBQ_F16_4BIT ? launch_few<TypeF16, NumberF16>(a, stream) : launch_few<TypeBf16, NumberBf16>(a, stream);
}

}  // namespace fbq
