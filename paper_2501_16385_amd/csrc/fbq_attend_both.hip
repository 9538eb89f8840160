// A batch behind a shared prefix in one launch: the shared tokens against the rows of all sequences (many rows, bound by the matrix cores) and every row's own tokens (few
// rows, bound by HBM) at the same time.  The first blocks, one a CU, are the shared tokens' - one block alone on a CU is about as fast as two that share it - and the others,
// as many again at a time, find their places beside them.  us, 64 sequences of 64 heads (8 of keys) behind 16384 shared tokens, about 400 of their own each: 47
// and 27 one after the other, 59 this way, and half as many parts to join (8.5, 11.5).  Up to 128 features: beyond, a block has a
// CU's LDS to itself.
#include "fbq_attend_few.h"
#include "fbq_attend_many.h"

namespace fbq {

template <class TY, int DF, int DM>
__global__ __launch_bounds__(256, 2) void fbq_attend_both_kernel(const AttendArgs a, const int tiles)
{
    __shared__ __attribute__((aligned(1024))) unsigned char room[kManyRoom<DM> > kFewRoom<DF> ? kManyRoom<DM> : kFewRoom<DF>];
    const int shared_blocks = a.kv_heads * tiles * a.shared_splits, block = blockIdx.x;
    if (block >= shared_blocks) {
        attend_few<TY, DF>(a, block - shared_blocks, room);
        return;
    }
    const int rest = block / a.kv_heads, z = rest / tiles;    // a head's blocks on one XCD, where heads are a multiple of eight
    attend_many<TY, DM>(a, true, block - rest * a.kv_heads, rest - z * tiles, z, room);
}

template <class TY>
static hipError_t launch_both(const AttendArgs &a, hipStream_t stream)
{
    static_assert(kFewWaves == 4, "blocks of one size");
    const int tiles = (int)(((long)a.T * a.group + kManyRows - 1) / kManyRows);
    const dim3 grid(a.kv_heads * tiles * a.shared_splits + a.workers / kFewWaves), block(256);
    if (a.D <= 64) hipLaunchKernelGGL((fbq_attend_both_kernel<TY, 64, 64>), grid, block, 0, stream, a, tiles);
    else if (a.D <= 96) hipLaunchKernelGGL((fbq_attend_both_kernel<TY, 128, 96>), grid, block, 0, stream, a, tiles);
    else hipLaunchKernelGGL((fbq_attend_both_kernel<TY, 128, 128>), grid, block, 0, stream, a, tiles);
    return hipGetLastError();
}

hipError_t launch_attend_both(const AttendArgs &a, int type, hipStream_t stream)
{
    return type == FBQ_F16 ? launch_both<TypeF16>(a, stream) : launch_both<TypeBf16>(a, stream);
}

}  // namespace fbq
