// Root-mean-square norm with the residual's addition (the step in front of every W4A4 linear layer of a transformer block):
//
//     h = bf16(x + residual),   y = (h * rstd) * w,   rstd = 1 / sqrt(mean_k h_k^2 + eps)
//
// with y in bf16 and / or in e4m3 with one scale per token, s = max_k |y_k| / 448.  h is rounded before the norm, so that the norm
// is that of the stored stream; sums, rstd and y are fp32.
//
// Bound by memory: 8 bytes a channel with everything in bf16 and about ten vector instructions.  A token stays in registers from
// its only read to its only write: a workgroup holds it in 16-byte pieces, thread t those of number t, t + THREADS, ...  4096 tokens of
// 8192 channels, 268 MB: 41.5 us, 6.5 TB/s (a large copy reaches 4.8).  Eight pieces a thread 50 us, four 43.5; without the
// non-temporal hint on what is read and on h 47.4; with it on y too, which the next kernel reads, 46; with the weight read behind the sum
// and sums through LDS 42.1, 61 tokens 4.2 instead of 3.8.  One token: 1.8 us, of which the launch is most.
#include "basq_internal.h"

namespace basq {

namespace {

typedef __bf16 v2bf __attribute__((ext_vector_type(2)));
typedef float v2f __attribute__((ext_vector_type(2)));

// two fp32 -> two bf16 in one register, round-half-to-even
__device__ __forceinline__ uint32_t pack_bf16(float a, float b) {
    return __builtin_bit_cast(uint32_t, __builtin_convertvector((v2f){a, b}, v2bf));
}
__device__ __forceinline__ float low_f32(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float high_f32(uint32_t w) { return __uint_as_float(w & 0xFFFF0000u); }

template <int CTRL>
__device__ __forceinline__ float dpp(float v) {
    return __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(v), CTRL, 0xF, 0xF, true));
}
template <int THREADS, class Op>
__device__ __forceinline__ float across(float v, float* scratch, Op op) {
    v = op(v, dpp<0xB1>(v));                                     // the lane beside, the pair beside, both halves of eight, of sixteen
    v = op(v, dpp<0x4E>(v));
    v = op(v, dpp<0x141>(v));
    v = op(v, dpp<0x140>(v));
    v = across_rows(v, op);
    if constexpr (THREADS > 64) {
        if ((threadIdx.x & 63) == 0) scratch[threadIdx.x >> 6] = v;
        __syncthreads();
        v = scratch[0];
#pragma unroll
        for (int w = 1; w < THREADS / 64; ++w) v = op(v, scratch[w]);
    }
    return v;
}

template <int THREADS, int PIECES, bool RES>
__global__ __launch_bounds__(THREADS) void add_rms_norm_kernel(RmsNormArgs a) {
    __shared__ float scratch[2][THREADS / 64];
    const int64_t m = workgroup_of_grid();
    if (m >= a.M) return;
    const int tid = threadIdx.x, pieces = a.K / 8;
    const uint4* x = reinterpret_cast<const uint4*>(a.X + m * a.ldx);
    const uint4* r = reinterpret_cast<const uint4*>(RES ? a.residual + m * a.ldr : nullptr);
    const uint4* w = reinterpret_cast<const uint4*>(a.weight);
    uint4 h[PIECES], g[PIECES], weight[PIECES];
#pragma unroll
    for (int i = 0; i < PIECES; ++i) {
        const int p = tid + i * THREADS;
        h[i] = make_uint4(0, 0, 0, 0);
        g[i] = make_uint4(0, 0, 0, 0);
        if (p < pieces) {
            h[i] = nt_load16(x + p);
            if (RES) g[i] = nt_load16(r + p);
        }
    }
    // (before anything is stored: a wait for them would be for the stores too)
#pragma unroll
    for (int i = 0; i < PIECES; ++i) {
        const int p = tid + i * THREADS;
        weight[i] = make_uint4(0, 0, 0, 0);
        if (p < pieces) weight[i] = w[p];
    }
    float sum = 0.0f;
#pragma unroll
    for (int i = 0; i < PIECES; ++i) {
        uint32_t* hw = reinterpret_cast<uint32_t*>(&h[i]);
        const uint32_t* gw = reinterpret_cast<const uint32_t*>(&g[i]);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            if (RES) hw[j] = pack_bf16(low_f32(hw[j]) + low_f32(gw[j]), high_f32(hw[j]) + high_f32(gw[j]));
            sum = fmaf(low_f32(hw[j]), low_f32(hw[j]), sum);
            sum = fmaf(high_f32(hw[j]), high_f32(hw[j]), sum);
        }
        const int p = tid + i * THREADS;
        if (a.res_out && p < pieces) nt_store16(reinterpret_cast<uint4*>(a.res_out + m * a.ldro) + p, h[i]);
    }
    sum = across<THREADS>(sum, scratch[0], [](float u, float v) { return u + v; });
    const float rstd = rsqrtf(sum / (float)a.K + a.eps);

    float top = 0.0f;
#pragma unroll
    for (int i = 0; i < PIECES; ++i) {
        const int p = tid + i * THREADS;
        const uint32_t* hw = reinterpret_cast<const uint32_t*>(&h[i]);
        const uint32_t* ww = reinterpret_cast<const uint32_t*>(&weight[i]);
        uint4 out;
        uint32_t* ow = reinterpret_cast<uint32_t*>(&out);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const float u = low_f32(hw[j]) * rstd * low_f32(ww[j]), v = high_f32(hw[j]) * rstd * high_f32(ww[j]);
            ow[j] = pack_bf16(u, v);
            top = fmaxf(top, fmaxf(fabsf(u), fabsf(v)));
        }
        if (a.Y && p < pieces) reinterpret_cast<uint4*>(a.Y + m * a.ldy)[p] = out;
    }
    if (!a.Y8) return;
    top = across<THREADS>(top, scratch[1], [](float u, float v) { return fmaxf(u, v); });
    float scale = __fdiv_rn(top, 448.0f);
    if (!(scale > 0.0f && scale < INFINITY)) scale = 1.0f;
    if (tid == 0) a.y8_scale[m] = scale;
    // Quotients by s: the product with 1 / s, and what it leaves over (exact by fused multiply-add) times 1 / s once more, which is y / s to
    // 2^-47 before its one rounding.  (The product alone is rounded twice, which moves a code now and then.)  Where that remainder could
    // be subnormal, 1 / s infinite, or y infinite, a division: 4096 tokens of 8192 channels take 40.0 us if all divide, 61 tokens 4.3.
    auto store = [&](auto over_scale) {
#pragma unroll
        for (int i = 0; i < PIECES; ++i) {
            const int p = tid + i * THREADS;
            if (p >= pieces) break;
            const uint32_t* hw = reinterpret_cast<const uint32_t*>(&h[i]);
            const uint32_t* ww = reinterpret_cast<const uint32_t*>(&weight[i]);
            uint32_t c[2];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                float u = over_scale(low_f32(hw[j]) * rstd * low_f32(ww[j])), v = over_scale(high_f32(hw[j]) * rstd * high_f32(ww[j]));
                // (over the largest number by one rounding, or further where s is subnormal; NaN stays NaN)
                if (fabsf(u) > 448.0f) u = copysignf(448.0f, u);
                if (fabsf(v) > 448.0f) v = copysignf(448.0f, v);
                c[j / 2] = j % 2 ? __builtin_amdgcn_cvt_pk_fp8_f32(u, v, c[j / 2], true) : __builtin_amdgcn_cvt_pk_fp8_f32(u, v, 0, false);
            }
            reinterpret_cast<uint2*>(a.Y8 + m * a.ldy8)[p] = make_uint2(c[0], c[1]);
        }
    };
    // Quotients by s: the product with 1 / s, and what it leaves over (exact by fused multiply-add) times 1 / s once more, which is y / s to
    // 2^-47 before its one rounding.  (The product alone is rounded twice, which moves a code now and then.)  Where what is left over could be
    // subnormal, 1 / s infinite, or y infinite, divisions.  4096 tokens of 8192 channels, e4m3 alone: 39.1 us, 40.0 if all divide; 61: 3.9, 4.3.
    if (scale >= 0x1p-80f && top < INFINITY) {
        const float inv = __fdiv_rn(1.0f, scale);
        store([&](float y) {
            const float q = y * inv;
            return fmaf(fmaf(-q, scale, y), inv, q);
        });
    } else {
        store([&](float y) { return __fdiv_rn(y, scale); });
    }
}

template <int THREADS, int PIECES>
void launch(const RmsNormArgs& a, hipStream_t s) {
    if (a.residual) hipLaunchKernelGGL((add_rms_norm_kernel<THREADS, PIECES, true>), grid_of(a.M), dim3(THREADS), 0, s, a);
    else hipLaunchKernelGGL((add_rms_norm_kernel<THREADS, PIECES, false>), grid_of(a.M), dim3(THREADS), 0, s, a);
}

}  // namespace

int launch_add_rms_norm(const RmsNormArgs& a, hipStream_t s) {
    if (a.M == 0) return BASQ_OK;
    const int pieces = a.K / 8;
    // two pieces a thread; up to 1024 channels one wavefront does, without a barrier
    if (pieces <= 128) launch<64, 2>(a, s);
    else if (pieces <= 256) launch<128, 2>(a, s);
    else if (pieces <= 512) launch<256, 2>(a, s);
    else if (pieces <= 1024) launch<512, 2>(a, s);
    else if (pieces <= 2048) launch<1024, 2>(a, s);
    else launch<1024, 4>(a, s);
    return check_hip(hipGetLastError(), "add_rms_norm launch");
}

}  // namespace basq
