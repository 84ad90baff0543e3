// Rotary positions, online per-head Hadamard rotation and INT4 quantisation of a token's heads on their way into the paged
// cache (paper Sec. 4 "online rotations" of q and k; Sec. 5 "Deployment Details": per-head asymmetric INT4 of the cache):
//
//     q' = H_D rope(q) / sqrt(D),  k' = H_D rope(k) / sqrt(D)        (either step optional)
//     k', v -> lo = clip_lo min, hi = clip_hi max, s = (hi - lo) / 15, q = rint(clamp((x - lo) / s, 0, 15))
//
// Every step is one fp32 operation in the order given in basq.h, so codes and ranges are the same bits whatever the call's size.
//
// A head of D channels lies on D/8 lanes, eight neighbouring channels (16 bytes) each, so a wavefront takes 512 channels (four
// or eight heads) per step.  The pair of a channel under rope is in the lane itself (interleaved) or rot/16 lanes away (halves);
// the transform's stages over channel bits 0-2 are in the lane, the others are DPP moves; the range is a DPP reduction over the
// head's lanes.  Nothing goes through LDS memory, and a token's cosines and sines stay in registers for all its heads.
#include "basq_internal.h"

namespace basq {

namespace {

typedef __bf16 v2bf __attribute__((ext_vector_type(2)));
typedef float v2f __attribute__((ext_vector_type(2)));

constexpr int RA_WAVES = 4, AHEAD = 2;                           // steps of a wave under way

template <int CTRL>
__device__ __forceinline__ float dpp(float v) {
    return __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(v), CTRL, 0xF, 0xF, true));
}
constexpr int XOR1 = 0xB1, XOR2 = 0x4E, XOR3 = 0x1B, HALF_MIRROR = 0x141, MIRROR = 0x140, XOR8 = 0x128;

// the value of the lane whose number differs in bit BIT (0..3)
template <int BIT>
__device__ __forceinline__ float neighbour(float v) {
    if constexpr (BIT == 0) return dpp<XOR1>(v);
    else if constexpr (BIT == 1) return dpp<XOR2>(v);
    else if constexpr (BIT == 2) return dpp<HALF_MIRROR>(dpp<XOR3>(v));        // 7 ^ 3
    else return dpp<XOR8>(v);                                                  // a rotation by half a row
}

template <int BIT>
__device__ __forceinline__ void stage(float (&x)[8], int lane) {
    const uint32_t sign = (uint32_t)((lane >> BIT) & 1) << 31;
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = neighbour<BIT>(x[i]) + __uint_as_float(__float_as_uint(x[i]) ^ sign);
}

template <int D>
__device__ __forceinline__ void hadamard(float (&x)[8], int lane, float norm) {
#pragma unroll
    for (int step = 1; step < 8; step *= 2)
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (!(i & step)) {
                const float a = x[i], b = x[i + step];
                x[i] = a + b;
                x[i + step] = a - b;
            }
    stage<0>(x, lane);
    stage<1>(x, lane);
    stage<2>(x, lane);
    if constexpr (D == 128) stage<3>(x, lane);
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] *= norm;
}

template <int D, class Op>
__device__ __forceinline__ float over_head(const float (&x)[8], Op op) {
    float v = op(op(op(x[0], x[1]), op(x[2], x[3])), op(op(x[4], x[5]), op(x[6], x[7])));
    v = op(v, dpp<XOR1>(v));
    v = op(v, dpp<XOR2>(v));
    v = op(v, dpp<HALF_MIRROR>(v));
    if constexpr (D == 128) v = op(v, dpp<MIRROR>(v));
    return v;
}

__device__ __forceinline__ void widen(const uint4& w, float (&x)[8]) {
    const uint32_t* u = reinterpret_cast<const uint32_t*>(&w);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        x[2 * i] = __uint_as_float(u[i] << 16);
        x[2 * i + 1] = __uint_as_float(u[i] & 0xFFFF0000u);
    }
}
__device__ __forceinline__ uint4 narrow(const float (&x)[8]) {
    uint4 w;
    uint32_t* u = reinterpret_cast<uint32_t*>(&w);
#pragma unroll
    for (int i = 0; i < 4; ++i)
        u[i] = __builtin_bit_cast(uint32_t, __builtin_convertvector((v2f){x[2 * i], x[2 * i + 1]}, v2bf));
    return w;
}

// A wave takes `per` consecutive steps of one token; the steps of a token are its q heads, its k heads and its v heads, each
// rounded up to whole steps.
template <int D, bool INTERLEAVED>
__global__ __launch_bounds__(RA_WAVES * 64) void rope_append_kernel(RopeAppendArgs a, int parts, int per) {
    constexpr int LANES = D / 8, HEADS = 64 / LANES;             // lanes of a head, heads of a step
    const int lane = threadIdx.x & 63;
    const uint32_t wave = blockIdx.x * (uint32_t)RA_WAVES + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int64_t t = wave / (uint32_t)parts;
    if (t >= a.T) return;
    const int part = (int)(wave - (uint32_t)t * (uint32_t)parts);
    const int sub = lane % LANES, in_step = lane / LANES, c0 = 8 * sub;
    const int q_steps = (a.heads + HEADS - 1) / HEADS, kv_steps = (a.kv_heads + HEADS - 1) / HEADS;
    const int end = min(q_steps + 2 * kv_steps, (part + 1) * per);

    int position = 0;
    if (a.cos_sin) {
        position = a.positions[t];
        if (position < 0 || position >= a.table_rows) return;   // padding
    }
    const int slot = a.slots && a.kv_heads ? a.slots[t] : -1;

    // out = x * co + pair * si
    float co[8], si[8];
    const bool turned = a.cos_sin != nullptr && c0 < a.rot;
    const int half = a.rot / 2;
    const bool second = !INTERLEAVED && c0 >= half;
    // the lane that holds the pairs of this one's channels (itself where they are not turned)
    const int pair_lane = INTERLEAVED || !turned ? lane : second ? lane - half / 8 : lane + half / 8;
    if (turned) {
        const float* row = a.cos_sin + (int64_t)position * a.rot;
        if (INTERLEAVED) {
            const float4 c = *reinterpret_cast<const float4*>(row + c0 / 2), s = *reinterpret_cast<const float4*>(row + half + c0 / 2);
            co[0] = co[1] = c.x; co[2] = co[3] = c.y; co[4] = co[5] = c.z; co[6] = co[7] = c.w;
            si[0] = -s.x; si[1] = s.x; si[2] = -s.y; si[3] = s.y; si[4] = -s.z; si[5] = s.z; si[6] = -s.w; si[7] = s.w;
        } else {
            const int j = second ? c0 - half : c0;
            const float4 c = *reinterpret_cast<const float4*>(row + j), d = *reinterpret_cast<const float4*>(row + j + 4);
            const float4 s = *reinterpret_cast<const float4*>(row + half + j), u = *reinterpret_cast<const float4*>(row + half + j + 4);
            co[0] = c.x; co[1] = c.y; co[2] = c.z; co[3] = c.w; co[4] = d.x; co[5] = d.y; co[6] = d.z; co[7] = d.w;
            si[0] = s.x; si[1] = s.y; si[2] = s.z; si[3] = s.w; si[4] = u.x; si[5] = u.y; si[6] = u.z; si[7] = u.w;
            if (!second)
#pragma unroll
                for (int i = 0; i < 8; ++i) si[i] = -si[i];
        }
    }

    auto head_of = [&](int step, int& kind) {
        kind = step < q_steps ? 0 : step < q_steps + kv_steps ? 1 : 2;
        return (step - (kind == 0 ? 0 : kind == 1 ? q_steps : q_steps + kv_steps)) * HEADS + in_step;
    };
    auto request = [&](int step) {
        int kind;
        const int head = head_of(step, kind);
        uint4 w = make_uint4(0, 0, 0, 0);
        const uint16_t* x = kind == 0 ? a.q + t * a.ldq : kind == 1 ? a.k + t * a.ldk : a.v + t * a.ldv;
        if (head < (kind == 0 ? a.heads : a.kv_heads)) w = nt_load16(x + head * D + c0);
        return w;
    };

    uint4 next[AHEAD];
#pragma unroll
    for (int i = 0; i < AHEAD; ++i) next[i] = part * per + i < end ? request(part * per + i) : make_uint4(0, 0, 0, 0);
    for (int step = part * per; step < end; ++step) {
        const uint4 w = next[0];
#pragma unroll
        for (int i = 0; i + 1 < AHEAD; ++i) next[i] = next[i + 1];
        if (step + AHEAD < end) next[AHEAD - 1] = request(step + AHEAD);
        int kind;
        const int head = head_of(step, kind);
        float x[8];
        widen(w, x);
        if (kind < 2) {
            if (a.cos_sin) {
                float p[8];
                if (INTERLEAVED) {
#pragma unroll
                    for (int i = 0; i < 8; ++i) p[i] = x[i ^ 1];
                } else {
                    uint4 other;
                    other.x = __shfl(w.x, pair_lane, 64);
                    other.y = __shfl(w.y, pair_lane, 64);
                    other.z = __shfl(w.z, pair_lane, 64);
                    other.w = __shfl(w.w, pair_lane, 64);
                    widen(other, p);
                }
                if (turned)
#pragma unroll
                    for (int i = 0; i < 8; ++i) x[i] = x[i] * co[i] + p[i] * si[i];
            }
            if (a.rotate) hadamard<D>(x, lane, a.norm);
        }
        if (kind == 0) {
            if (head < a.heads) nt_store16(a.q_out + t * a.ldqo + head * D + c0, narrow(x));
            continue;
        }
        const float lo = a.clip_lo * over_head<D>(x, [](float u, float v) { return fminf(u, v); });
        const float hi = a.clip_hi * over_head<D>(x, [](float u, float v) { return fmaxf(u, v); });
        float s = __fdiv_rn(hi - lo, 15.0f);
        if (!(s > 0.0f && s < INFINITY)) s = 1.0f;
        const float inv = __fdiv_rn(1.0f, s);
        const float nlo = -(lo * inv);
        uint32_t even = 0, odd = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            x[2 * i] = __builtin_amdgcn_fmed3f(fmaf(x[2 * i], inv, nlo), 0.0f, 15.0f);
            x[2 * i + 1] = __builtin_amdgcn_fmed3f(fmaf(x[2 * i + 1], inv, nlo), 0.0f, 15.0f);
            even = __builtin_amdgcn_cvt_pk_u8_f32(x[2 * i], i, even);          // round-half-to-even, NaN -> 0
            odd = __builtin_amdgcn_cvt_pk_u8_f32(x[2 * i + 1], i, odd);
        }
        if (head >= a.kv_heads) continue;
        const int page = slot >> a.page_log2, at = slot & ((1 << a.page_log2) - 1);
        if (slot >= 0 && page < a.num_pages) {
            const int P = 1 << a.page_log2, which = kind - 1;
            uint8_t* mine = a.cache + ((int64_t)page * a.kv_heads + head) * ((int64_t)P * (D + 16));
            *reinterpret_cast<uint32_t*>(mine + (int64_t)(which * P + at) * (D / 2) + 4 * sub) = even | (odd << 4);
            if (sub == 0) *reinterpret_cast<float2*>(mine + (int64_t)P * D + (which * P + at) * 8) = make_float2(s, lo);
        }
        uint16_t* hat = kind == 1 ? a.k_hat : a.v_hat;
        if (hat) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                x[2 * i] = fmaf(s, (float)((even >> (8 * i)) & 255u), lo);
                x[2 * i + 1] = fmaf(s, (float)((odd >> (8 * i)) & 255u), lo);
            }
            nt_store16(hat + t * a.ldh + head * D + c0, narrow(x));
        }
    }
}

template <int D>
int launch(const RopeAppendArgs& a, hipStream_t s) {
    constexpr int HEADS = 512 / D;
    const int steps = (a.heads + HEADS - 1) / HEADS + 2 * ((a.kv_heads + HEADS - 1) / HEADS);
    // eight thousand waves while a token has steps for several of them (32 a compute unit; 4096 tokens of 64 and 8 heads: 41.8 us with half
    // as many and one step under way, 37.4 with twice as many, as built 35.4 .. 36.9), and one to a token from there on
    int64_t parts = (8192 + a.T - 1) / a.T;
    if (parts > steps) parts = steps;
    const int per = (int)((steps + parts - 1) / parts);
    parts = (steps + per - 1) / per;
    const int64_t blocks = (a.T * parts + RA_WAVES - 1) / RA_WAVES;
    if (blocks * RA_WAVES > 0xFFFFFFFFll) return fail(BASQ_EUNSUPPORTED, "rope_append: too many tokens");
    if (a.interleaved) hipLaunchKernelGGL((rope_append_kernel<D, true>), dim3((unsigned)blocks), dim3(RA_WAVES * 64), 0, s, a, (int)parts, per);
    else hipLaunchKernelGGL((rope_append_kernel<D, false>), dim3((unsigned)blocks), dim3(RA_WAVES * 64), 0, s, a, (int)parts, per);
    return check_hip(hipGetLastError(), "rope_append launch");
}

__global__ __launch_bounds__(256) void rope_table_kernel(float* out, int64_t rows, int rot, RopeScaling k) {
    const int half = rot / 2;
    const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (i >= rows * half) return;
    const int64_t row = i / half;
    const int j = (int)(i - row * half);
    constexpr double TWO_PI = 6.283185307179586476925286766559;
    double f = pow(k.base, -2.0 * j / rot);
    double amplitude = 1.0;
    if (k.kind == BASQ_ROPE_LINEAR) {
        f /= k.factor;
    } else if (k.kind == BASQ_ROPE_BANDS) {
        // turns that the pair makes over the original length: few -> interpolated, many -> kept, linear in between
        const double turns = k.original_len * f / TWO_PI;
        const double keep = fmin(fmax((turns - k.low) / (k.high - k.low), 0.0), 1.0);
        f = (1.0 - keep) * f / k.factor + keep * f;
    } else if (k.kind == BASQ_ROPE_YARN) {
        // the same, linear in the pair's number between the numbers at which a pair makes `high` and `low` turns
        auto pair_of = [&](double turns) { return rot * log(k.original_len / (turns * TWO_PI)) / (2.0 * log(k.base)); };
        const double from = fmax(floor(pair_of(k.high)), 0.0), to = fmin(ceil(pair_of(k.low)), (double)rot - 1.0);
        const double ramp = fmin(fmax((j - from) / fmax(to - from, 0.001), 0.0), 1.0);
        f = f / k.factor * ramp + f * (1.0 - ramp);
        amplitude = k.factor > 1.0 ? 0.1 * log(k.factor) + 1.0 : 1.0;
    }
    double s, c;
    sincos((double)row * f, &s, &c);
    out[row * rot + j] = (float)(amplitude * c);
    out[row * rot + half + j] = (float)(amplitude * s);
}

}  // namespace

int launch_rope_append(const RopeAppendArgs& a, hipStream_t s) {
    if (a.T == 0) return BASQ_OK;
    return a.D == 64 ? launch<64>(a, s) : launch<128>(a, s);
}

int launch_rope_table(float* out, int64_t rows, int32_t rot, const RopeScaling& k, hipStream_t s) {
    if (rows == 0) return BASQ_OK;
    const int64_t blocks = (rows * (rot / 2) + 255) / 256;
    if (blocks > 0x7FFFFFFFll) return fail(BASQ_EUNSUPPORTED, "rope_table: too many positions");
    hipLaunchKernelGGL(rope_table_kernel, dim3((unsigned)blocks), dim3(256), 0, s, out, rows, rot, k);
    return check_hip(hipGetLastError(), "rope_table launch");
}

}  // namespace basq
