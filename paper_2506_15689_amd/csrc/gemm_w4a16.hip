// The W4A16 product: what its kernels (gemm_w4a16_kernel.h) need to know of a call, and which of them takes it.
#include "basq_internal.h"

namespace basq {

int launch_gemm_w4a16(W4A16Args a, hipStream_t s) {
    a.unit = a.group % 128 == 0 ? 128 : a.group % 64 == 0 ? 64 : 32;
    a.groups = a.K / a.group;
    // group of unit u, in `units` to a group: the upper half of u (2^32 / units + 1), exact as there are fewer than 2^16 units; 0: u
    const unsigned units = (unsigned)(a.group / a.unit);
    a.per_group = units > 1 ? (unsigned)((1ull << 32) / units + 1) : 0;
    // A launch has fewer than 2^32 threads along the rows, and the shapes take up to 512 for 16 of them: more than 2^26 rows go in parts.
    constexpr int32_t AT_ONCE = 1 << 26;
    for (int64_t n0 = 0; n0 < a.N; n0 += AT_ONCE) {
        W4A16Args p = a;
        p.N = a.N - n0 < AT_ONCE ? (int32_t)(a.N - n0) : AT_ONCE;
        p.Wq += n0 * (a.K / 2);                            // (whole blocks of the streaming layout)
        p.w_scale += n0 * a.groups;
        p.w_zero += n0 * a.groups;
        if (p.bias) p.bias += n0;
        p.Y = static_cast<uint8_t*>(a.Y) + n0 * (a.y_f32 ? 4 : 2);
        if (a.w_layout == BASQ_W_DECODE16) {
            if (a.M <= 16) launch_w4a16_streamed_few(p, s); else launch_w4a16_streamed_many(p, s);
        } else {
            if (a.M <= 16) launch_w4a16_canonical_few(p, s); else launch_w4a16_canonical_many(p, s);
        }
    }
    return check_hip(hipGetLastError(), "w4a16_gemm launch");
}

}  // namespace basq
