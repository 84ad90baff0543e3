// Few tokens in bf16 times 4-bit weights with a scale and a zero point for each group of channels (an output head, a layer whose
// activations are not quantised):
//
//     Y[m,n] = sum_g sw[n,g] * ( sum_{k in g} (16 + q[n,k]) x[m,k]  -  (16 + zp[n,g]) sum_{k in g} x[m,k] )  + bias[n]
//
// which is the definition's sum of sw (q - zp) x: 16 + q is a bf16 number whose four mantissa bits are the code, so a code becomes
// an operand by a shift and an and-or, exactly; products and sums are the matrix cores' fp32, and scales stay out of them.  (Weights
// rounded to bf16 would put 2^-9 on each; with 128 + q, the next such form, eight times as much cancels in the difference.)  The
// sums of x over a group are one more product, with ones.
//
// One pass over the weights, which bound it: each lane requests its batch of 16-byte pieces before it takes any up.  A workgroup
// owns TILES tiles of 16 weight rows, its waves share K in chunks of 128 channels; D = x (rows) times weights (columns), so a
// lane's results belong to one weight row and take one scale.
//
// A 16-byte piece is 32 channels of one row, and an instruction takes the 8 channels of one dword from each of a row's four pieces
// of a chunk: where groups are whole chunks, any split of the chunk over the four instructions will do.  Where groups are smaller
// (32 or 64 channels, say) the dwords are transposed over the wave's rows first (four swaps), and each instruction takes one piece.
#include "basq_internal.h"

namespace basq {

namespace {

typedef float v4f __attribute__((ext_vector_type(4)));
typedef unsigned v4u __attribute__((ext_vector_type(4)));
typedef __bf16 v8b __attribute__((ext_vector_type(8)));

constexpr int TILE = 16;

// 8 codes -> 16 + code in bf16: pairs (0,4) (1,5) (2,6) (3,7) of the dword's channels
__device__ __forceinline__ v8b widen(unsigned v) {
    constexpr unsigned mask = 0x00780078u, base = 0x41804180u;
    const v4u r = {(v << 3 & mask) | base, (v >> 1 & mask) | base, (v >> 5 & mask) | base, (v >> 9 & mask) | base};
    return __builtin_bit_cast(v8b, r);
}
// 8 channels of a token in the same order
__device__ __forceinline__ v8b in_pairs(v4u d) {
    const v4u r = {__builtin_amdgcn_perm(d.z, d.x, 0x05040100u), __builtin_amdgcn_perm(d.z, d.x, 0x07060302u),
                   __builtin_amdgcn_perm(d.w, d.y, 0x05040100u), __builtin_amdgcn_perm(d.w, d.y, 0x07060302u)};
    return __builtin_bit_cast(v8b, r);
}
// dword i of row j of the wave <-> dword j of row i
__device__ __forceinline__ v4u transposed(v4u r) {
    const auto a = __builtin_amdgcn_permlane32_swap(r.x, r.z, false, false);
    const auto b = __builtin_amdgcn_permlane32_swap(r.y, r.w, false, false);
    const auto c = __builtin_amdgcn_permlane16_swap(a[0], b[0], false, false);
    const auto d = __builtin_amdgcn_permlane16_swap(a[1], b[1], false, false);
    return v4u{c[0], c[1], d[0], d[1]};
}

// UNIT: channels that certainly share a group: 128, 64 or 32.   TT: tiles of 16 tokens.   STEPS: chunks that a lane holds at once.
template <bool STREAM_LAYOUT, int WAVES, int STEPS, int TILES, int TT, int UNIT>
__global__ __launch_bounds__(WAVES * 64) void gemm_w4a16_kernel(W4A16Args a) {
    constexpr int UNITS = 128 / UNIT;                                          // of a chunk
    constexpr int NT = TILES * TT;
    __shared__ v4f part[WAVES * NT * 64];

    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int row = lane & 15, sub = lane >> 4;
    const int n0 = blockIdx.x * (TILE * TILES), m0 = blockIdx.y * (TILE * TT);
    const int KB = a.K / 2, chunks = (a.K + 127) / 128;
    const int M = (int)(a.M - m0 < TILE * TT ? a.M - m0 : TILE * TT);
    const int groups = a.groups;

    const uint8_t* wrow[TILES];
    const uint16_t *srow[TILES], *zrow[TILES];
#pragma unroll
    for (int t = 0; t < TILES; ++t) {
        const int nt0 = n0 + TILE * t < a.N ? n0 + TILE * t : n0;              // (a tile past the last: the first again, not stored)
        const int n = nt0 + row < a.N ? nt0 + row : a.N - 1;
        wrow[t] = STREAM_LAYOUT ? a.Wq + (int64_t)nt0 * KB + lane * 16 : a.Wq + (int64_t)n * KB + sub * 16;
        srow[t] = a.w_scale + (int64_t)n * groups;
        zrow[t] = a.w_zero + (int64_t)n * groups;
    }
    const uint16_t* xrow[TT];
#pragma unroll
    for (int tt = 0; tt < TT; ++tt) {
        const int m = TILE * tt + row < M ? TILE * tt + row : M - 1;           // (rows past the last: the last again, not stored)
        xrow[tt] = a.X + (m0 + m) * a.ldx + (UNIT == 128 ? 32 * sub : 8 * sub);
    }
    constexpr int WSTEP = STREAM_LAYOUT ? 1024 : 64;
    constexpr int XPIECE = UNIT == 128 ? 8 : 32;                               // channels from one instruction's operand to the next's
    const int within = UNIT == 128 ? 32 * sub : 8 * sub;

    const v4f zero = {0.f, 0.f, 0.f, 0.f};
    const v4u ones_bits = {0x3F803F80u, 0x3F803F80u, 0x3F803F80u, 0x3F803F80u};
    const v8b ones = __builtin_bit_cast(v8b, ones_bits);
    v4f acc[NT];
#pragma unroll
    for (int i = 0; i < NT; ++i) acc[i] = zero;

    for (int c0 = wave; c0 < chunks; c0 += WAVES * STEPS) {
        v4u w[TILES][STEPS], x[TT][STEPS][4];
        uint16_t sw[TILES][STEPS][UNITS], zp[TILES][STEPS][UNITS];
#pragma unroll
        for (int i = 0; i < STEPS; ++i) {
            const int c = c0 + i * WAVES;
            const bool ok = c < chunks;
            const bool piece = ok && (STREAM_LAYOUT || 128 * c + 32 * sub < a.K);          // (K need not be whole chunks)
#pragma unroll
            for (int t = 0; t < TILES; ++t)
                w[t][i] = piece ? __builtin_nontemporal_load(reinterpret_cast<const v4u*>(wrow[t] + (int64_t)c * WSTEP)) : v4u{0, 0, 0, 0};
#pragma unroll
            for (int u = 0; u < UNITS; ++u) {
                const unsigned unit = (unsigned)(UNITS * (ok ? c : 0) + u);
                int g = (int)(a.per_group ? __umulhi(unit, a.per_group) : unit);
                g = g < groups ? g : groups - 1;                               // (a last chunk's units past K)
#pragma unroll
                for (int t = 0; t < TILES; ++t) { sw[t][i][u] = srow[t][g]; zp[t][i][u] = zrow[t][g]; }
            }
#pragma unroll
            for (int tt = 0; tt < TT; ++tt)
#pragma unroll
                for (int p = 0; p < 4; ++p)
                    x[tt][i][p] = ok && (STREAM_LAYOUT || 128 * c + within + XPIECE * p < a.K) ? *reinterpret_cast<const v4u*>(xrow[tt] + 128 * c + XPIECE * p) : v4u{0, 0, 0, 0};
        }
#pragma unroll
        for (int i = 0; i < STEPS; ++i) {
            if (c0 + i * WAVES >= chunks) break;
#pragma unroll
            for (int tt = 0; tt < TT; ++tt)
#pragma unroll
                for (int p = 0; p < 4; ++p) x[tt][i][p] = __builtin_bit_cast(v4u, in_pairs(x[tt][i][p]));
            v4f sums[TT][UNITS];
#pragma unroll
            for (int tt = 0; tt < TT; ++tt)
#pragma unroll
                for (int u = 0; u < UNITS; ++u) {
                    sums[tt][u] = zero;
#pragma unroll
                    for (int p = u * 4 / UNITS; p < (u + 1) * 4 / UNITS; ++p)
                        sums[tt][u] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(v8b, x[tt][i][p]), ones, sums[tt][u], 0, 0, 0);
                }
#pragma unroll
            for (int t = 0; t < TILES; ++t) {
                const v4u d = UNIT == 128 ? w[t][i] : transposed(w[t][i]);
#pragma unroll
                for (int u = 0; u < UNITS; ++u) {
                    const float s = bf16_to_f32(sw[t][i][u]), z = 16.0f + bf16_to_f32(zp[t][i][u]);
                    v4f r[TT];
#pragma unroll
                    for (int tt = 0; tt < TT; ++tt) r[tt] = zero;
#pragma unroll
                    for (int p = u * 4 / UNITS; p < (u + 1) * 4 / UNITS; ++p) {
                        const v8b q = widen(d[p]);
#pragma unroll
                        for (int tt = 0; tt < TT; ++tt) r[tt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(v8b, x[tt][i][p]), q, r[tt], 0, 0, 0);
                    }
#pragma unroll
                    for (int tt = 0; tt < TT; ++tt)
#pragma unroll
                        for (int e = 0; e < 4; ++e) acc[t * TT + tt][e] = fmaf(s, fmaf(-z, sums[tt][u][e], r[tt][e]), acc[t * TT + tt][e]);
                }
            }
        }
    }
    // the waves' sums meet in a fixed order; element e of lane l is token 4 (l/16) + e, row l % 16 of its tiles
#pragma unroll
    for (int i = 0; i < NT; ++i) part[(wave * NT + i) * 64 + lane] = acc[i];
    __syncthreads();
    for (int i = wave; i < NT; i += WAVES) {
        const int t = i / TT, tt = i % TT, n = n0 + TILE * t + row;
        v4f v = part[i * 64 + lane];
#pragma unroll
        for (int w = 1; w < WAVES; ++w) v += part[(w * NT + i) * 64 + lane];
        if (n >= a.N) continue;
        const float b = a.bias ? a.bias[n] : 0.0f;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const int m = TILE * tt + 4 * sub + e;
            if (m >= M) continue;
            const int64_t at = (m0 + m) * a.ldy + n;
            if (a.y_f32) static_cast<float*>(a.Y)[at] = v[e] + b;
            else static_cast<uint16_t*>(a.Y)[at] = f32_to_bf16(v[e] + b);
        }
    }
}

template <bool SL, int WAVES, int STEPS, int TILES, int TT, int UNIT>
void launch_shape(const W4A16Args& a, hipStream_t s) {
    const unsigned x = (unsigned)((a.N + TILE * TILES - 1) / (TILE * TILES)), y = (unsigned)((a.M + TILE * TT - 1) / (TILE * TT));
    hipLaunchKernelGGL((gemm_w4a16_kernel<SL, WAVES, STEPS, TILES, TT, UNIT>), dim3(x, y), dim3(WAVES * 64), 0, s, a);
}

template <bool SL, int UNIT>
void launch_unit(const W4A16Args& a, hipStream_t s) {
    if (a.M <= 16) launch_shape<SL, 4, 4, 1, 1, UNIT>(a, s);
    else if (a.M <= 32) launch_shape<SL, 4, 2, 1, 2, UNIT>(a, s);
    else launch_shape<SL, 4, 1, 2, 4, UNIT>(a, s);
}

template <bool SL>
void launch_layout(const W4A16Args& a, hipStream_t s) {
    if (a.unit == 128) launch_unit<SL, 128>(a, s);
    else if (a.unit == 64) launch_unit<SL, 64>(a, s);
    else launch_unit<SL, 32>(a, s);
}

}  // namespace

int launch_gemm_w4a16(W4A16Args a, hipStream_t s) {
    a.unit = a.group % 128 == 0 ? 128 : a.group % 64 == 0 ? 64 : 32;
    a.groups = a.K / a.group;
    // group of unit u, in `units` to a group: the upper half of u (2^32 / units + 1), exact as there are fewer than 2^16 units; 0: u
    const unsigned units = (unsigned)(a.group / a.unit);
    a.per_group = units > 1 ? (unsigned)((1ull << 32) / units + 1) : 0;
    if (a.w_layout == BASQ_W_DECODE16) launch_layout<true>(a, s);
    else launch_layout<false>(a, s);
    return check_hip(hipGetLastError(), "w4a16_gemm launch");
}

}  // namespace basq
