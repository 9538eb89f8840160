// Launches of the many-row kernel alone (fbq_attend_many.h).
#include "fbq_attend_many.h"

namespace fbq {

// A grid has 65535 blocks in y: more tiles than that go on in z, so many at a time.  (That is where a call of shared tokens has their pieces, but not then: it has blocks enough.)
constexpr int kGridTiles = 32768;

template <class TY, int DP>
__global__ __launch_bounds__(256, DP == 256 ? 1 : 2) void fbq_attend_many_kernel(const AttendArgs a, const bool shared)
{
    __shared__ __attribute__((aligned(1024))) unsigned char room[kManyRoom<DP>];
    const bool pieces = shared && a.shared_splits > 1;
    attend_many<TY, DP>(a, shared, blockIdx.x, pieces ? blockIdx.y : blockIdx.y + blockIdx.z * kGridTiles, pieces ? blockIdx.z : 0, room);
}

template <class TY>
static hipError_t launch_many(const AttendArgs &a, bool shared, hipStream_t stream)
{
    const long rows = (long)a.T * a.group, per = (a.group + kManyRows - 1) / kManyRows;
    long tiles = (rows + kManyRows - 1) / kManyRows;          // ragged rows: each may have one more, begun
    if (!shared) tiles = (a.q_start ? std::min(a.T * per, tiles + a.rows) : a.rows * per) * a.splits;
    const bool fits = tiles <= 65535;
    const dim3 grid(a.kv_heads, fits ? (unsigned)tiles : kGridTiles, fits ? (shared ? a.shared_splits : 1) : (unsigned)((tiles + kGridTiles - 1) / kGridTiles)), block(256);
    if (a.D <= 64) hipLaunchKernelGGL((fbq_attend_many_kernel<TY, 64>), grid, block, 0, stream, a, shared);
    else if (a.D <= 96) hipLaunchKernelGGL((fbq_attend_many_kernel<TY, 96>), grid, block, 0, stream, a, shared);
    else if (a.D <= 128) hipLaunchKernelGGL((fbq_attend_many_kernel<TY, 128>), grid, block, 0, stream, a, shared);
    else hipLaunchKernelGGL((fbq_attend_many_kernel<TY, 256>), grid, block, 0, stream, a, shared);
    return hipGetLastError();
}

hipError_t launch_attend_many(const AttendArgs &a, int type, bool shared, hipStream_t stream)
{
    return type == FBQ_F16 ? launch_many<TypeF16>(a, shared, stream) : launch_many<TypeBf16>(a, shared, stream);
}

}  // namespace fbq
