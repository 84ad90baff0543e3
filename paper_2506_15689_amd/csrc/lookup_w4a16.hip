// Rows of a 4-bit matrix with group scales, in bf16: the embeddings of tokens, from the matrix that is the output head's too or
// from one of their own.  Y[t,k] = bf16(scale * (sw (q - zp))), row ids[t]; an id that is no row (padding) gives zeros.
//
// Bound by memory: K/2 bytes of codes and 4 K/G of scales in, 2 K out.  A workgroup takes a token (a piece of a long one where there are
// few), a thread 8 channels at a time, so that 64 lanes write 1 KB side by side; all of a thread's reads are under way before
// it takes any up.  In the streaming layout a row lies in pieces of 16 bytes, 256 bytes apart, and a cache line of 128 bytes comes with
// each: a row costs eight times its codes (4096 rows of 8192 channels 32 us, 136 MB in and 67 out, 6.3 TB/s).
#include "basq_internal.h"

namespace basq {

namespace {

typedef float f2 __attribute__((ext_vector_type(2)));
typedef __bf16 b2 __attribute__((ext_vector_type(2)));

constexpr int THREADS = 256;

// AT_ONCE: pieces of 8 channels of a thread
template <int AT_ONCE>
__global__ __launch_bounds__(THREADS) void lookup_w4a16_kernel(LookupArgs a) {
    const int64_t t = (int64_t)blockIdx.y * gridDim.z + blockIdx.z;
    if (t >= a.T) return;
    const int id = a.ids[t], pieces = a.K / 8, p0 = blockIdx.x * (THREADS * AT_ONCE) + threadIdx.x;
    const bool there = id >= 0 && id < a.N;
    const int n = there ? id : 0;
    const int64_t KB = a.K / 2;
    const bool streamed = a.w_layout == BASQ_W_DECODE16;
    const uint8_t* row = a.Wq + (streamed ? (n & ~15) * KB + (n & 15) * 16 : n * KB);
    const uint16_t *scale = a.w_scale + (int64_t)n * a.groups, *zero = a.w_zero + (int64_t)n * a.groups;
    unsigned q[AT_ONCE];
    uint16_t s[AT_ONCE], z[AT_ONCE];
#pragma unroll
    for (int i = 0; i < AT_ONCE; ++i) {
        const int p = p0 + i * THREADS < pieces ? p0 + i * THREADS : pieces - 1;
        const unsigned unit = (unsigned)p / 4;                                 // of 32 channels
        q[i] = *reinterpret_cast<const unsigned*>(row + (streamed ? unit * 256 + 4 * (p & 3) : 4 * p));
        const unsigned g = a.per_group ? __umulhi(unit, a.per_group) : unit;
        s[i] = scale[g];
        z[i] = zero[g];
    }
#pragma unroll
    for (int i = 0; i < AT_ONCE; ++i) {
        const int p = p0 + i * THREADS;
        if (p >= pieces) break;
        const float sw = bf16_to_f32(s[i]), zp = bf16_to_f32(z[i]);
        auto two = [&](int e) {
            const f2 v = {a.scale * (sw * ((float)(q[i] >> (4 * e) & 15) - zp)), a.scale * (sw * ((float)(q[i] >> (4 * e + 4) & 15) - zp))};
            return __builtin_bit_cast(unsigned, __builtin_convertvector(v, b2));                // round-to-nearest-even
        };
        const uint4 out = there ? make_uint4(two(0), two(2), two(4), two(6)) : make_uint4(0, 0, 0, 0);
        nt_store16(a.Y + t * a.ldy + 8 * p, out);
    }
}

}  // namespace

int launch_lookup_w4a16(LookupArgs a, hipStream_t s) {
    a.groups = a.K / a.group;
    const unsigned units = (unsigned)(a.group / 32);                           // (as in launch_gemm_w4a16)
    a.per_group = units > 1 ? (unsigned)((1ull << 32) / units + 1) : 0;
    const int pieces = a.K / 8;
    // rows of tokens in two dimensions of the grid
    const unsigned z = (unsigned)(a.T < 32768 ? a.T : 32768), y = (unsigned)((a.T + z - 1) / z);
    // few tokens: a piece a thread, more workgroups (512 tokens of 4096 channels 4.5 us either way, a call's; 1024 5.3 with one, 5.0 with four)
    if (a.T * ((pieces + 4 * THREADS - 1) / (4 * THREADS)) < 1024) {
        hipLaunchKernelGGL(lookup_w4a16_kernel<1>, dim3((pieces + THREADS - 1) / THREADS, y, z), dim3(THREADS), 0, s, a);
    } else {
        hipLaunchKernelGGL(lookup_w4a16_kernel<4>, dim3((pieces + 4 * THREADS - 1) / (4 * THREADS), y, z), dim3(THREADS), 0, s, a);
    }
    return check_hip(hipGetLastError(), "w4a16_lookup launch");
}

}  // namespace basq
