// The W4A16 product: what its kernels (gemm_w4a16_kernel.h) need to know of a call, and which of them takes it.
#include "basq_internal.h"

namespace basq {

int launch_gemm_w4a16(W4A16Args a, hipStream_t s) {
    a.unit = a.group % 128 == 0 ? 128 : a.group % 64 == 0 ? 64 : 32;
    a.groups = a.K / a.group;
    // group of unit u, in `units` to a group: the upper half of u (2^32 / units + 1), exact as there are fewer than 2^16 units; 0: u
    const unsigned units = (unsigned)(a.group / a.unit);
    a.per_group = units > 1 ? (unsigned)((1ull << 32) / units + 1) : 0;
    if (a.w_layout == BASQ_W_DECODE16) {
        if (a.M <= 16) launch_w4a16_streamed_few(a, s); else launch_w4a16_streamed_many(a, s);
    } else {
        if (a.M <= 16) launch_w4a16_canonical_few(a, s); else launch_w4a16_canonical_many(a, s);
    }
    return check_hip(hipGetLastError(), "w4a16_gemm launch");
}

}  // namespace basq
