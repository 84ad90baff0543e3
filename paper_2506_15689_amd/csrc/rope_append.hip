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
// the transform's stages over channel bits 0-2 are in the lane, the others are DPP operands; the range is a DPP reduction over the
// head's lanes; only the pairs rot/16 lanes away change lanes by the LDS unit, four instructions a step (no LDS memory).  A token's cosines
// and sines stay in registers for all its heads.  A zero out of the transform is positive.
//
// Bound by memory, with vector instructions not far behind (about 150 for a step of queries).  4096 tokens of 64 and 8 heads of 128 channels
// move 173 MB in 33.4 us, 5.2 TB/s, 32768 tokens in 246 us, 5.6 (a large copy reaches 4.8).  With the lanes' butterflies as two or three
// instructions each and branches around loads and stores 35.4 .. 36.5, and 17.9 instead of 15.7 for 1946 tokens of 40 and 40 heads of 64
// channels.  (The first heads are requested once the token's position is known: requested beside it, 1 .. 2 % less, but padding's would be read.)
// Sixteen tokens: 3.6 us, the launch and four loads, one after the other.
#include "basq_internal.h"

namespace basq {

namespace {

typedef __bf16 v2bf __attribute__((ext_vector_type(2)));
typedef float v2f __attribute__((ext_vector_type(2)));
typedef uint32_t basq_v2u __attribute__((ext_vector_type(2)));

constexpr int RA_WAVES = 4;
constexpr int NT = 2;                                            // non-temporal
constexpr int BEYOND = 0x7FFFFFF0;                               // behind the end of any buffer here

__device__ __forceinline__ __amdgpu_buffer_rsrc_t buffer(const void* p, int bytes) {
    return __builtin_amdgcn_make_buffer_rsrc(const_cast<void*>(p), 0, bytes, 0x00020000);
}

template <int CTRL>
__device__ __forceinline__ float dpp(float v) {
    return __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(v), CTRL, 0xF, 0xF, true));
}
constexpr int XOR1 = 0xB1, XOR2 = 0x4E, HALF_MIRROR = 0x141, MIRROR = 0x140;

// The piece of eight channels that is on a head's lane (and the lane that a piece is on): pieces 4 .. 7 of eight lie backwards, so that the
// mirror of eight lanes exchanges pieces whose numbers differ in bit 2 alone.
__device__ __forceinline__ int piece_of(int lane) { return lane ^ (lane & 4 ? 3 : 0); }

// Butterflies over lanes, a + b where the piece's bit is clear and a - b where it is set, one instruction each: the latter lane's sum is kept
// with the other sign (x - neighbour), as the lanes that it meets in later stages keep theirs.  (What an instruction writes may be another
// lane's operand two instructions later: a s_nop in front, the eight values in turn behind it.)
#define RA_STAGE(x, sign, CTRL)                                                                                                        \
    asm("s_nop 1\n\t"                                                                                                                  \
        "v_fmac_f32_dpp %0, %0, %8 " CTRL " row_mask:0xf bank_mask:0xf\n\t"                                                            \
        "v_fmac_f32_dpp %1, %1, %8 " CTRL " row_mask:0xf bank_mask:0xf\n\t"                                                            \
        "v_fmac_f32_dpp %2, %2, %8 " CTRL " row_mask:0xf bank_mask:0xf\n\t"                                                            \
        "v_fmac_f32_dpp %3, %3, %8 " CTRL " row_mask:0xf bank_mask:0xf\n\t"                                                            \
        "v_fmac_f32_dpp %4, %4, %8 " CTRL " row_mask:0xf bank_mask:0xf\n\t"                                                            \
        "v_fmac_f32_dpp %5, %5, %8 " CTRL " row_mask:0xf bank_mask:0xf\n\t"                                                            \
        "v_fmac_f32_dpp %6, %6, %8 " CTRL " row_mask:0xf bank_mask:0xf\n\t"                                                            \
        "v_fmac_f32_dpp %7, %7, %8 " CTRL " row_mask:0xf bank_mask:0xf"                                                                \
        : "+v"(x[0]), "+v"(x[1]), "+v"(x[2]), "+v"(x[3]), "+v"(x[4]), "+v"(x[5]), "+v"(x[6]), "+v"(x[7])                               \
        : "v"(sign))

// norm: with the sign of a lane's sums (see above), signs[b]: -1 where the piece's bit b is set, else 1
template <int D>
__device__ __forceinline__ void hadamard(float (&x)[8], const float (&signs)[4], float norm) {
#pragma unroll
    for (int step = 1; step < 8; step *= 2)
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (!(i & step)) {
                const float a = x[i], b = x[i + step];
                x[i] = a + b;
                x[i + step] = a - b;
            }
    RA_STAGE(x, signs[0], "quad_perm:[1,0,3,2]");
    RA_STAGE(x, signs[1], "quad_perm:[2,3,0,1]");
    RA_STAGE(x, signs[2], "row_half_mirror");
    if constexpr (D == 128) RA_STAGE(x, signs[3], "row_ror:8");
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = fmaf(x[i], norm, 0.0f);                 // (+ 0: a zero is positive, with either sign of norm)
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

__device__ __forceinline__ void widen(const basq_v4u& w, float (&x)[8]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        x[2 * i] = __uint_as_float(w[i] << 16);
        x[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
    }
}
__device__ __forceinline__ basq_v4u narrow(const float (&x)[8]) {
    basq_v4u w;
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = __builtin_bit_cast(uint32_t, __builtin_convertvector((v2f){x[2 * i], x[2 * i + 1]}, v2bf));
    return w;
}

// A wave takes `per` consecutive steps of one token; the steps of a token are its q heads, its k heads and its v heads, each
// rounded up to whole steps.
template <int D, bool INTERLEAVED>
__global__ __launch_bounds__(RA_WAVES * 64, 8) void rope_append_kernel(RopeAppendArgs a, int parts, int per) {
    constexpr int LANES = D / 8, HEADS = 64 / LANES;             // lanes of a head, heads of a step
    const int lane = threadIdx.x & 63;
    const uint32_t wave = (uint32_t)workgroup_of_grid() * RA_WAVES + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int64_t t = (uint32_t)__builtin_amdgcn_readfirstlane(wave / (uint32_t)parts);
    if (t >= a.T) return;
    const int part = (int)(wave - (uint32_t)t * (uint32_t)parts);
    const int sub = lane % LANES, in_step = lane / LANES, piece = piece_of(sub), c0 = 8 * piece;
    const int q_steps = (a.heads + HEADS - 1) / HEADS, kv_steps = (a.kv_heads + HEADS - 1) / HEADS;
    const int end = min(q_steps + 2 * kv_steps, (part + 1) * per);

    // Loads and stores go through buffer descriptors that end with the heads there are: what lies behind them, and steps behind the last one,
    // moves nothing, without a branch, so that a wait is for the one load it needs.
    const uint32_t mine = 2 * (in_step * D + c0);
    auto first_head = [&](int step) { return (step < q_steps ? step : step < q_steps + kv_steps ? step - q_steps : step - q_steps - kv_steps) * HEADS; };
    auto request = [&](int step) {
        const int first = first_head(step);
        const uint16_t* row = step < q_steps ? a.q + t * a.ldq : step < q_steps + kv_steps ? a.k + t * a.ldk : a.v + t * a.ldv;
        return __builtin_amdgcn_raw_buffer_load_b128(buffer(row + first * D, step < end ? ((step < q_steps ? a.heads : a.kv_heads) - first) * D * 2 : 0), mine, 0, NT);
    };

    // where the token stands and goes (scalar loads: a vector load's wait would be for the heads too); of padding no head is read
    const int slot = a.slots && a.kv_heads ? ((const __attribute__((address_space(4))) int32_t*)a.slots)[t] : -1;
    int position = 0;
    if (a.cos_sin) {
        position = ((const __attribute__((address_space(4))) int32_t*)a.positions)[t];
        if (position < 0 || position >= a.table_rows) return;
    }
    basq_v4u even_step = request(part * per), odd_step = request(part * per + 1);

    // out = x * co + pair * si
    float co[8], si[8];
    const bool turned = a.cos_sin != nullptr && c0 < a.rot;
    const int half = a.rot / 2;
    const bool second = !INTERLEAVED && c0 >= half;
    // the lane that holds the pairs of this one's channels (itself where they are not turned)
    const int pair_lane = INTERLEAVED || !turned ? lane : lane - sub + piece_of(second ? piece - half / 8 : piece + half / 8);
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

    float signs[4], norm = a.norm;
#pragma unroll
    for (int b = 0; b < 4; ++b) {
        signs[b] = (piece >> b) & 1 ? -1.0f : 1.0f;
        norm *= signs[b];
    }

    auto turn = [&](const basq_v4u& w, float (&x)[8]) {
        if (a.cos_sin) {
            float p[8];
            if (INTERLEAVED) {
#pragma unroll
                for (int i = 0; i < 8; ++i) p[i] = x[i ^ 1];
            } else {
                basq_v4u other;
#pragma unroll
                for (int i = 0; i < 4; ++i) other[i] = __shfl(w[i], pair_lane, 64);
                widen(other, p);
            }
            if (turned)
#pragma unroll
                for (int i = 0; i < 8; ++i) x[i] = x[i] * co[i] + p[i] * si[i];
        }
        if (a.rotate) hadamard<D>(x, signs, norm);
    };
    auto query = [&](int step, const basq_v4u& w) {
        float x[8];
        widen(w, x);
        turn(w, x);
        const int first = step * HEADS;
        __builtin_amdgcn_raw_buffer_store_b128(narrow(x), buffer(a.q_out + t * a.ldqo + first * D, (a.heads - first) * D * 2), mine, 0, NT);
    };
    const int P = 1 << a.page_log2, page = slot >> a.page_log2, at = slot & (P - 1), pitch = P * (D + 16);
    const bool stored = slot >= 0 && page < a.num_pages;
    auto key_or_value = [&](int step, const basq_v4u& w) {
        const bool value = step >= q_steps + kv_steps;
        float x[8];
        widen(w, x);
        if (!value) turn(w, x);
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
        const int first = first_head(step), row = value ? P + at : at;
        const auto blocks = buffer(a.cache + ((int64_t)page * a.kv_heads + first) * pitch, stored ? min(a.kv_heads - first, HEADS) * pitch : 0);
        __builtin_amdgcn_raw_buffer_store_b32(even | (odd << 4), blocks, in_step * pitch + row * (D / 2) + 4 * piece, 0, 0);
        const basq_v2u range = {__float_as_uint(s), __float_as_uint(lo)};
        __builtin_amdgcn_raw_buffer_store_b64(range, blocks, sub == 0 ? in_step * pitch + P * D + row * 8 : BEYOND, 0, 0);
        uint16_t* hat = value ? a.v_hat : a.k_hat;
        if (hat) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                x[2 * i] = fmaf(s, (float)((even >> (8 * i)) & 255u), lo);
                x[2 * i + 1] = fmaf(s, (float)((odd >> (8 * i)) & 255u), lo);
            }
            __builtin_amdgcn_raw_buffer_store_b128(narrow(x), buffer(hat + t * a.ldh + first * D, (a.kv_heads - first) * D * 2), mine, 0, NT);
        }
    };

    int step = part * per;
    for (const int last = min(end, q_steps) - 1; step < last; step += 2) {
        basq_v4u w = even_step;
        even_step = request(step + 2);
        query(step, w);
        w = odd_step;
        odd_step = request(step + 3);
        query(step + 1, w);
    }
    auto any = [&](int step, const basq_v4u& w) {
        if (step < q_steps) query(step, w);
        else key_or_value(step, w);
    };
    for (; step < end; step += 2) {
        basq_v4u w = even_step;
        even_step = request(step + 2);
        any(step, w);
        if (step + 1 == end) break;
        w = odd_step;
        odd_step = request(step + 3);
        any(step + 1, w);
    }
}

template <int D>
int launch(const RopeAppendArgs& a, hipStream_t s) {
    constexpr int HEADS = 512 / D;
    const int steps = (a.heads + HEADS - 1) / HEADS + 2 * ((a.kv_heads + HEADS - 1) / HEADS);
    if (a.T > 0x7FFFFFFFll) return fail(BASQ_EUNSUPPORTED, "rope_append: too many tokens");
    // eight thousand waves, as many as the chip holds, while a token has steps for several of them, and one to a token from there on (half as
    // many, as built, twice as many: 4096 tokens of 64 and 8 heads 35.0, 33.6, 33.0 us; 1946 of 40 and 40 heads of 64 channels 15.4, 15.7,
    // 16.3; 668 of 64 and 8 8.2, 8.4, 10.0; 7081 of 28 and 4 15.5, 15.8, 18.5)
    int64_t parts = (8192 + a.T - 1) / a.T;
    if (parts > steps) parts = steps;
    const int per = (int)((steps + parts - 1) / parts);
    parts = (steps + per - 1) / per;
    const int64_t blocks = (a.T * parts + RA_WAVES - 1) / RA_WAVES;
    if (blocks * RA_WAVES > 0x7FFFFFFFll) return fail(BASQ_EUNSUPPORTED, "rope_append: too many tokens");
    if (a.interleaved) hipLaunchKernelGGL((rope_append_kernel<D, true>), grid_of(blocks), dim3(RA_WAVES * 64), 0, s, a, (int)parts, per);
    else hipLaunchKernelGGL((rope_append_kernel<D, false>), grid_of(blocks), dim3(RA_WAVES * 64), 0, s, a, (int)parts, per);
    return check_hip(hipGetLastError(), "rope_append launch");
}

__global__ __launch_bounds__(256) void rope_table_kernel(float* out, int64_t rows, int rot, RopeScaling k) {
    const int half = rot / 2;
    const int64_t i = workgroup_of_grid() * 256 + threadIdx.x;
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
    if (rows > 0x7FFFFFFFll * 256 / (rot / 2)) return fail(BASQ_EUNSUPPORTED, "rope_table: too many positions");
    const int64_t blocks = (rows * (rot / 2) + 255) / 256;
    hipLaunchKernelGGL(rope_table_kernel, grid_of(blocks), dim3(256), 0, s, out, rows, rot, k);
    return check_hip(hipGetLastError(), "rope_table launch");
}

}  // namespace basq
