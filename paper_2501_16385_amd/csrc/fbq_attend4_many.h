// Attention of many query rows over a cache in 4 bits: the kernel of fbq_attend_many.h with keys and values made on their way to LDS (fbq_attend_codes.h).
// Measured, 32 heads of 128: prompt of 2048 tokens in fp16 66 to 71 us from card to card, in bf16 81 to 86 (of 16 bits 53), 8192 630 to 690 and 715 (540); fp16 heads of 64 46 and 410 to 430 (36, 330), of 80
// 55 and 515 to 535 (45, 425), of 192 130 for 2048 (108), of 256 160 and 2053 (113, 1426).  What making the operands takes is vector instructions, 160 a step of 64 keys beside the kernel's own 360; heads
// of 128 and 256 have 36 to 724 bytes a lane of scratch memory for it, what other loads wait for.  bf16, a token in sixteen with values 2^-20 times the others': 146 and 1422 for 81 and 716, heads of 256
// 652 and 8587 for 141 and 1782: every block does its work twice, the second time in bf16.
#ifndef FBQ_ATTEND4_MANY_H
#define FBQ_ATTEND4_MANY_H

#include "fbq_attend_many.h"

namespace fbq {

// Block (h, y, z) of attend_many over codes.
template <class TY, class MAKE, int NW>
__device__ __forceinline__ void attend4_many(const AttendArgs &a, bool shared, int h, int y, int z, unsigned char *room)
{
    constexpr int DP = NW == 6 ? 256 : 32 * NW;
    bool odd = false;
    attend_many<TY, DP, Codes<MAKE, NW, DP>>(a, shared, h, y, z, room, &odd);
    if constexpr (MAKE::kChecked) {
        if (!odd) return;
        // What follows from the block, the lane and the arguments takes no registers until the second time: the arguments, each such kernel's first parameter, are read again.  (Kept from the first time
        // they push others of the loop out to memory, whose loads wait for the codes under way: 97 us for 86 and 819 for 716, see above, 45 for 41 behind a shared prefix.)
        asm volatile("" : "+s"(h), "+s"(y), "+s"(z) : : "memory");
        typedef const __attribute__((address_space(4))) AttendArgs *Kept;
        Kept again = (Kept)__builtin_amdgcn_kernarg_segment_ptr();
        asm volatile("" : "+s"(again));
        attend_many<TY, DP, Codes<MakeBf16, NW, DP>>(*(const AttendArgs *)again, shared, h, y, z, room);
    }
}

}  // namespace fbq

#endif
