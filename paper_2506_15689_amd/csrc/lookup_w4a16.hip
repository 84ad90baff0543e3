// Rows of a 4-bit matrix with group scales, in bf16: the embeddings of tokens, from the matrix that is the output head's too or
// from one of their own.  Y[t,k] = bf16(scale * (sw (q - zp))), row ids[t]; an id that is no row (padding) gives zeros.
//
// Bound by memory: K/2 bytes of codes and as many as 4 K/G of scales in, 2 K out.  A thread takes 8 channels, 4 bytes of codes, so
// that 64 lanes write 1 KB side by side.
#include "basq_internal.h"

namespace basq {

namespace {

__global__ __launch_bounds__(256) void lookup_w4a16_kernel(LookupArgs a) {
    const int64_t i = (int64_t)workgroup_of_grid() * 256 + threadIdx.x;
    const int pieces = a.K / 8;
    const int64_t t = i / pieces;
    if (t >= a.T) return;
    const int p = (int)(i - t * pieces), k = 8 * p;
    const int id = a.ids[t];
    uint4 out = make_uint4(0, 0, 0, 0);
    if (id >= 0 && id < a.N) {
        const int64_t KB = a.K / 2;
        const int64_t at = a.w_layout == BASQ_W_DECODE16 ? (id & ~15) * KB + (int64_t)(k / 32) * 256 + (id & 15) * 16 + 4 * (p & 3) : id * KB + 4 * p;
        const unsigned q = *reinterpret_cast<const unsigned*>(a.Wq + at);
        const int64_t g = (int64_t)id * a.groups + k / a.group;
        const float s = bf16_to_f32(a.w_scale[g]), z = bf16_to_f32(a.w_zero[g]);
        auto value = [&](int e) { return (unsigned)f32_to_bf16(a.scale * (s * ((float)(q >> (4 * e) & 15) - z))); };
        out = make_uint4(value(0) | value(1) << 16, value(2) | value(3) << 16, value(4) | value(5) << 16, value(6) | value(7) << 16);
    }
    *reinterpret_cast<uint4*>(a.Y + t * a.ldy + k) = out;
}

}  // namespace

int launch_lookup_w4a16(LookupArgs a, hipStream_t s) {
    a.groups = a.K / a.group;
    const int64_t blocks = (a.T * (a.K / 8) + 255) / 256;
    hipLaunchKernelGGL(lookup_w4a16_kernel, grid_of(blocks), dim3(256), 0, s, a);
    return check_hip(hipGetLastError(), "w4a16_lookup launch");
}

}  // namespace basq
