// Launches of the few-row kernel alone (fbq_attend_few.h).
#include "fbq_attend_few.h"

namespace fbq {

template <class TY, int DP>
__global__ __launch_bounds__(64 * kFewWaves, DP == 256 ? 1 : 2) void fbq_attend_few_kernel(const AttendArgs a)
{
    __shared__ __attribute__((aligned(16))) unsigned char room[kFewRoom<DP>];
    attend_few<TY, DP>(a, blockIdx.x, room);
}

template <class TY>
static hipError_t launch_few(const AttendArgs &a, hipStream_t stream)
{
    const dim3 grid(a.direct == 2 ? a.rows * a.kv_heads : ((a.direct ? a.rows * a.kv_heads : a.workers) + kFewWaves - 1) / kFewWaves), block(64 * kFewWaves);
    if (a.D <= 64) hipLaunchKernelGGL((fbq_attend_few_kernel<TY, 64>), grid, block, 0, stream, a);
    else if (a.D <= 128) hipLaunchKernelGGL((fbq_attend_few_kernel<TY, 128>), grid, block, 0, stream, a);
    else hipLaunchKernelGGL((fbq_attend_few_kernel<TY, 256>), grid, block, 0, stream, a);
    return hipGetLastError();
}

hipError_t launch_attend_few(const AttendArgs &a, int type, hipStream_t stream)
{
    return type == FBQ_F16 ? launch_few<TypeF16>(a, stream) : launch_few<TypeBf16>(a, stream);
}

}  // namespace fbq
