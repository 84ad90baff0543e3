// The W4A16 product on streamed weights, more than 16 tokens: instances of gemm_w4a16_kernel.h, in files of their own so that they build side by side.
#include "gemm_w4a16_kernel.h"

namespace basq {

void launch_w4a16_streamed_many(const W4A16Args& a, hipStream_t s) {
    if (a.unit == 128) launch_many<true, 128>(a, s);
    else if (a.unit == 64) launch_many<true, 64>(a, s);
    else launch_many<true, 32>(a, s);
}

}  // namespace basq
