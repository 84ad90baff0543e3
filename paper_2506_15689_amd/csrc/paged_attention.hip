// Attention of a sequence's newest tokens over its paged INT4 cache (paper Sec. 5: per-head asymmetric INT4 of the cache; the
// decode step between the qkv and the output projection).  With k_t = ks_t c_t + kl_t and v_t = vs_t d_t + vl_t, c and d codes:
//
//     s_t = scale (ks_t (q . c_t) + kl_t sum(q)),   p_t = 2^(log2(e) s_t - M),   l = sum_t p_t
//     out = ( sum_t (p_t vs_t) d_t + sum_t p_t vl_t ) / l
//
// so the codes go into the matrix cores as they are, and ranges into the scores and the weights: one pass over the cache, with the
// running reference M of the softmax.
//
// Bound by reading the cache, D + 16 bytes a token and kv head.  A wavefront takes 32 tokens of one kv head at a time on 16 x 16 x 32
// MFMAs whose 16 columns are the query rows that share the kv head (its heads, times the new tokens): tokens x channels of the keys
// times channels x rows gives scores with the row on lane % 16, four tokens to a quarter of the wave and block of 16; these are, as
// they lie, the weights' operand of channels x tokens of the values times tokens x rows, whose results keep the row on lane % 16.  So
// no value changes lanes between the two products, and M, l and the rescaling are per lane.  The step's loads (codes and ranges) are
// requested while the step before is worked on.
//
// A code's bit pattern, taken for an fp16 number, is the code times 2^-24 (and the code in the next nibble, left in place, 16 times
// that): exact, two codes to an instruction, and no conversion.  Query rows are brought to fp16 times a power of two of their own
// (a bf16 value fits it exactly while it is within 2^-30 of the row's largest); weights p_t vs_t are rounded to fp16 (2^-12
// relative, against 2^-9 of the bf16 output) near 2^5 of their running maximum, far from either end of fp16.  l, M and both sums are
// fp32.
#include "basq_internal.h"

#include <type_traits>

namespace basq {

namespace {

typedef _Float16 v8h __attribute__((ext_vector_type(8)));
typedef float v4f __attribute__((ext_vector_type(4)));
typedef uint32_t v4u __attribute__((ext_vector_type(4)));
typedef __bf16 v2bf __attribute__((ext_vector_type(2)));
typedef float v2f __attribute__((ext_vector_type(2)));

constexpr int PA_WAVES = 4, PA_STEP = 32;                        // tokens of a wave's step
constexpr float UNSET = -1e30f;                                  // M before the first token that counts
constexpr float LOG2E = 1.4426950408889634f, LN2 = 0.6931471805599453f;

// eight codes (one dword, low nibble first) as fp16: codes 0, 4, 2, 6 times 2^-24 and 1, 5, 3, 7 times 2^-20, in the order
// 0 4 | 1 5 | 2 6 | 3 7
__device__ __forceinline__ v8h spread(uint32_t x) {
    const v4u w = {x & 0x000F000Fu, x & 0x00F000F0u, (x >> 8) & 0x000F000Fu, (x >> 8) & 0x00F000F0u};
    return __builtin_bit_cast(v8h, w);
}
__device__ __forceinline__ float quarters_max(float v) {
    v = fmaxf(v, __shfl_xor(v, 16, 64));
    return fmaxf(v, __shfl_xor(v, 32, 64));
}
__device__ __forceinline__ float quarters_sum(float v) {
    v += __shfl_xor(v, 16, 64);
    return v + __shfl_xor(v, 32, 64);
}

// What a step reads: for block j of 16 tokens the keys of token lane % 16 (channels D/4 * (lane / 16) ..), and for the four tokens
// 4 * (lane / 16) .. the values of channels D/16 * (lane % 16) .. and both ranges.
template <int D>
struct Step {
    typedef typename std::conditional<D == 128, uint4, uint2>::type Keys;
    typedef typename std::conditional<D == 128, uint32_t, uint16_t>::type Values;
    Keys k[2];
    Values v[2][4];
    float4 kr[2][2], vr[2][2];                                   // (scale, lo) of two tokens each
};

template <int D, bool CAP>
__global__ __launch_bounds__(PA_WAVES * 64, 2) void paged_attention_kernel(PagedAttentionArgs a) {
    constexpr int TILES = D / 16;                                // channel tiles of the second product: channel TILES * n + c
    constexpr int KS = D / 32;                                   // 32-channel steps of the first
    __shared__ float lds_o[PA_WAVES][16][D + 4];
    __shared__ float lds_ml[PA_WAVES][2][16];

    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int col = lane & 15, quarter = lane >> 4;
    const int group = a.heads / a.kv_heads, rows = group * a.q_len, row_tiles = (rows + 15) / 16;
    int id = blockIdx.x;
    const int split = id % a.splits;
    id /= a.splits;
    const int row_tile = id % row_tiles;
    id /= row_tiles;
    const int kv_head = id % a.kv_heads, b = id / a.kv_heads;

    const int len = min(max(a.lengths[b], 0), a.max_len);
    // this lane's query row: new token j, head, and the tokens [begin, end) that it sees
    const int row = row_tile * 16 + col, j = min(row, rows - 1) / group, head = kv_head * group + min(row, rows - 1) - j * group;
    const int end = len - (a.q_len - 1) + j, begin = a.window > 0 ? max(end - a.window, 0) : 0;
    // the tokens of all rows of the tile, in whole blocks from the first's, and this workgroup's part of them
    const int j_first = row_tile * 16 / group, j_last = min(row_tile * 16 + 15, rows - 1) / group;
    const int all_end = len - (a.q_len - 1) + j_last, all_begin = a.window > 0 ? max(len - (a.q_len - 1) + j_first - a.window, 0) & ~15 : 0;
    const int from = all_begin + split * a.chunk, to = min(all_end, from + a.chunk);
    if (split > 0 && from >= to) return;                          // (the first part of an empty row writes its zeros)

    const int P = 1 << a.page_log2;
    const int64_t head_bytes = (int64_t)P * (D + 16);
    const int32_t* pages = a.page_table + (int64_t)b * a.table_stride;

    // query rows
    v8h q[KS];
    float c1, qs;
    {
        const uint16_t* src = a.q + ((int64_t)b * a.q_len + j) * a.ldq + (int64_t)head * D + quarter * (D / 4);
        float x[D / 4], top = 0.0f, sum = 0.0f;
#pragma unroll
        for (int i = 0; i < D / 4; i += 8) {
            const uint4 w = *reinterpret_cast<const uint4*>(src + i);
            const uint32_t* u = reinterpret_cast<const uint32_t*>(&w);
#pragma unroll
            for (int h = 0; h < 4; ++h) {
                x[i + 2 * h] = __uint_as_float(u[h] << 16);
                x[i + 2 * h + 1] = __uint_as_float(u[h] & 0xFFFF0000u);
            }
        }
#pragma unroll
        for (int i = 0; i < D / 4; ++i) {
            top = fmaxf(top, fabsf(x[i]));
            sum += x[i];
        }
        top = quarters_max(top);
        sum = quarters_sum(sum);
        // the largest becomes 2^14 .. 2^15 (exponent field of top, 127 = 2^0)
        const int e = min(max(141 - (int)(__float_as_uint(top) >> 23), -100), 100);
        const float up = __uint_as_float((uint32_t)(127 + e) << 23);
        c1 = a.scale * LOG2E * __uint_as_float((uint32_t)(127 - e) << 23) * 0x1p24f;
        qs = a.scale * LOG2E * sum;
#pragma unroll
        for (int s = 0; s < KS; ++s) {
            const float* y = x + 8 * s;
            const float odd = up * 0.0625f;
            q[s] = (v8h){(_Float16)(y[0] * up), (_Float16)(y[4] * up), (_Float16)(y[1] * odd), (_Float16)(y[5] * odd),
                         (_Float16)(y[2] * up), (_Float16)(y[6] * up), (_Float16)(y[3] * odd), (_Float16)(y[7] * odd)};
        }
    }

    v4f o[TILES];
#pragma unroll
    for (int c = 0; c < TILES; ++c) o[c] = (v4f){0.f, 0.f, 0.f, 0.f};
    float M = UNSET, l = 0.0f, lows = 0.0f;                       // l and lows: this lane's tokens

    // byte offsets of the lane's pieces inside one head of one page
    const uint32_t k_at = col * (D / 2) + quarter * (D / 8);
    const uint32_t v_at = P * (D / 2) + 4 * quarter * (D / 2) + col * (D / 32);
    const uint32_t r_at = P * D + 4 * quarter * 8;

    // Page ids of this wave's next 32 steps, block 2i + h of them on lane 2i + h; -1 for blocks past the end and for no page.
    int ids = 0;
    const int first = from + wave * PA_STEP;
    auto fetch_ids = [&](int t0) {
        const int t = t0 + (lane >> 1) * (PA_WAVES * PA_STEP) + (lane & 1) * 16;
        int id = -1;
        if (t < to) id = pages[t >> a.page_log2];
        ids = id >= 0 && id < a.num_pages ? id : -1;
    };
    auto load = [&](int i, int t, Step<D>& s) {                   // step i of the fetched ids, tokens t ..
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int id = max(__builtin_amdgcn_readlane(ids, 2 * i + h), 0);
            const uint8_t* base = a.cache + ((int64_t)id * a.kv_heads + kv_head) * head_bytes;
            const int at = (t + 16 * h) & (P - 1);
            const uint8_t* codes = base + at * (D / 2);
            s.k[h] = *reinterpret_cast<const typename Step<D>::Keys*>(codes + k_at);
#pragma unroll
            for (int r = 0; r < 4; ++r) s.v[h][r] = *reinterpret_cast<const typename Step<D>::Values*>(codes + v_at + r * (D / 2));
            const float4* kr = reinterpret_cast<const float4*>(base + at * 8 + r_at);
            const float4* vr = reinterpret_cast<const float4*>(base + at * 8 + r_at + 8 * P);
            s.kr[h][0] = kr[0]; s.kr[h][1] = kr[1];
            s.vr[h][0] = vr[0]; s.vr[h][1] = vr[1];
        }
    };
    // whether no row of the tile masks any token of the step
    const int inner_begin = a.window > 0 ? max(len - (a.q_len - 1) + j_last - a.window, 0) : 0, inner_end = len - (a.q_len - 1) + j_first;

    auto work = [&](int i, int t, const Step<D>& s) {
        float sc[8], vs[8], vl[8];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            v4f acc = {0.f, 0.f, 0.f, 0.f};
            const uint32_t* kw = reinterpret_cast<const uint32_t*>(&s.k[h]);
#pragma unroll
            for (int n = 0; n < KS; ++n) acc = __builtin_amdgcn_mfma_f32_16x16x32_f16(spread(kw[n]), q[n], acc, 0, 0, 0);
            const float* kr = reinterpret_cast<const float*>(&s.kr[h]);
            const float* vr = reinterpret_cast<const float*>(&s.vr[h]);
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                float x = fmaf(kr[2 * r], acc[r] * c1, kr[2 * r + 1] * qs);
                if (CAP) {
                    // log2(e) cap tanh(y), y = x / (log2(e) cap): tanh(y) = 1 - 2 / (e^2y + 1), whose rounding near 0 is that of 1,
                    // and there its series, below 2^-23 of the value off up to 1/4
                    const float y = x * a.inv_cap, y2 = y * y;
                    const float far = 1.0f - 2.0f * __builtin_amdgcn_rcpf(__builtin_amdgcn_exp2f(y * (2.0f * LOG2E)) + 1.0f);
                    const float near = y * fmaf(y2, fmaf(y2, fmaf(y2, fmaf(y2, 62.0f / 2835, -17.0f / 315), 2.0f / 15), -1.0f / 3), 1.0f);
                    x = a.cap_log2e * (fabsf(y) < 0.25f ? near : far);
                }
                sc[4 * h + r] = x;
                vs[4 * h + r] = vr[2 * r];
                vl[4 * h + r] = vr[2 * r + 1];
            }
        }
        const int id0 = __builtin_amdgcn_readlane(ids, 2 * i), id1 = __builtin_amdgcn_readlane(ids, 2 * i + 1);
        if ((id0 | id1) < 0 || t < inner_begin || t + PA_STEP > inner_end) {
            // what is masked may hold anything, also ranges that are no numbers
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    const int at = t + 16 * h + 4 * quarter + r;
                    const bool seen = at >= begin && at < end && (h ? id1 : id0) >= 0;
                    sc[4 * h + r] = seen ? sc[4 * h + r] : -INFINITY;
                    vs[4 * h + r] = seen ? vs[4 * h + r] : 0.0f;
                    vl[4 * h + r] = seen ? vl[4 * h + r] : 0.0f;
                }
        }
        float p[8], w[8], top = 0.0f;
        auto weigh = [&]() {
            top = 0.0f;
#pragma unroll
            for (int r = 0; r < 8; ++r) {
                p[r] = __builtin_amdgcn_exp2f(sc[r] - M);
                w[r] = p[r] * vs[r];
            }
            // (a token whose scale is 0 has no w: its p counts once it nears the end of fp32)
#pragma unroll
            for (int r = 0; r < 8; ++r) top = fmaxf(top, fabsf(w[r]));
            float most = p[0];
#pragma unroll
            for (int r = 1; r < 8; ++r) most = fmaxf(most, p[r]);
            top = fmaxf(top, most * 0x1p-60f);
        };
        weigh();
        // A row whose weights leave fp16's range (its first token does) gets a new reference: its largest weight becomes 2^5.
        if (__any(top > 0x1p15f)) {
            float best = -INFINITY;
#pragma unroll
            for (int r = 0; r < 8; ++r) best = fmaxf(best, sc[r] + fmaxf(__builtin_amdgcn_logf(vs[r]), -60.0f));
            const bool mine = quarters_max(top) > 0x1p15f;
            const float next = mine ? quarters_max(best) - 5.0f : M;
            const float f = __builtin_amdgcn_exp2f(M - next);
            M = next;
            l *= f;
            lows *= f;
#pragma unroll
            for (int c = 0; c < TILES; ++c) o[c] *= f;
            weigh();
        }
#pragma unroll
        for (int r = 0; r < 8; ++r) {
            l += p[r];
            lows = fmaf(p[r], vl[r], lows);
        }
        const v8h pw = {(_Float16)w[0], (_Float16)w[1], (_Float16)w[2], (_Float16)w[3], (_Float16)w[4], (_Float16)w[5], (_Float16)w[6], (_Float16)w[7]};
        // channels x tokens of the values: pairs of tokens side by side, then a code of both per instruction
        constexpr int HALVES = D == 128 ? 2 : 1;
#pragma unroll
        for (int half = 0; half < HALVES; ++half) {
            uint32_t x[4];
#pragma unroll
            for (int i2 = 0; i2 < 4; ++i2)
                x[i2] = __builtin_amdgcn_perm((uint32_t)s.v[i2 / 2][2 * (i2 % 2) + 1], (uint32_t)s.v[i2 / 2][2 * (i2 % 2)],
                                              half ? 0x07060302u : 0x05040100u);
#pragma unroll
            for (int c = 0; c < 4; ++c) {
                const uint32_t mask = c & 1 ? 0x00F000F0u : 0x000F000Fu;
                const int down = c & 2 ? 8 : 0;
                const v4u f = {(x[0] >> down) & mask, (x[1] >> down) & mask, (x[2] >> down) & mask, (x[3] >> down) & mask};
                o[4 * half + c] = __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(v8h, f), pw, o[4 * half + c], 0, 0, 0);
            }
        }
    };

    constexpr int STRIDE = PA_WAVES * PA_STEP;
    for (int t0 = first; t0 < to; t0 += 32 * STRIDE) {
        fetch_ids(t0);
        const int steps = min(32, (to - t0 + STRIDE - 1) / STRIDE);
        Step<D> s[2];
        load(0, t0, s[0]);
        for (int i = 0; i < steps; i += 2) {
            if (i + 1 < steps) load(i + 1, t0 + (i + 1) * STRIDE, s[1]);
            work(i, t0 + i * STRIDE, s[0]);
            if (i + 1 >= steps) break;
            if (i + 2 < steps) load(i + 2, t0 + (i + 2) * STRIDE, s[0]);
            work(i + 1, t0 + (i + 1) * STRIDE, s[1]);
        }
    }

    // join the four waves: sums brought to the largest reference
    l = quarters_sum(l);
    lows = quarters_sum(lows);
    if (quarter == 0) {
        lds_ml[wave][0][col] = M;
        lds_ml[wave][1][col] = l;
    }
    __syncthreads();
    float best = UNSET;
#pragma unroll
    for (int w = 0; w < PA_WAVES; ++w) best = fmaxf(best, lds_ml[w][0][col]);
    const float f = __builtin_amdgcn_exp2f(M - best);
#pragma unroll
    for (int r = 0; r < 4; ++r)
#pragma unroll
        for (int c = 0; c < TILES; ++c)
            lds_o[wave][col][TILES * (4 * quarter + r) + c] = f * fmaf(o[c][r], c & 1 ? 0x1p20f : 0x1p24f, lows);
    __syncthreads();
    // sixteen threads to a row, D/16 neighbouring channels each
    const int out_col = threadIdx.x / 16, piece = threadIdx.x % 16, out_row = row_tile * 16 + out_col;
    if (out_row >= rows) return;
    float x[TILES], total = 0.0f;
    best = UNSET;
#pragma unroll
    for (int w = 0; w < PA_WAVES; ++w) best = fmaxf(best, lds_ml[w][0][out_col]);
#pragma unroll
    for (int c = 0; c < TILES; ++c) x[c] = 0.0f;
#pragma unroll
    for (int w = 0; w < PA_WAVES; ++w) {
        total = fmaf(lds_ml[w][1][out_col], __builtin_amdgcn_exp2f(lds_ml[w][0][out_col] - best), total);
#pragma unroll
        for (int c = 0; c < TILES; ++c) x[c] += lds_o[w][out_col][TILES * piece + c];
    }
    const int out_j = out_row / group, out_head = kv_head * group + out_row - out_j * group;
    const int64_t token = (int64_t)b * a.q_len + out_j;
    if (a.splits > 1) {
        const int64_t at = (token * a.heads + out_head) * a.splits + split;
#pragma unroll
        for (int c = 0; c < TILES; c += 4)
            *reinterpret_cast<float4*>(a.part_o + at * D + TILES * piece + c) = make_float4(x[c], x[c + 1], x[c + 2], x[c + 3]);
        if (piece == 0) a.part_ml[at] = make_float2(best, total);
        return;
    }
    const float inv = total > 0.0f ? __fdiv_rn(1.0f, total) : total == 0.0f ? 0.0f : total;      // (NaN stays)
    uint32_t y[TILES / 2];
#pragma unroll
    for (int c = 0; c < TILES; c += 2) y[c / 2] = __builtin_bit_cast(uint32_t, __builtin_convertvector((v2f){x[c] * inv, x[c + 1] * inv}, v2bf));
    uint16_t* dst = a.out + token * a.ldo + out_head * D + TILES * piece;
    if constexpr (TILES == 8) *reinterpret_cast<uint4*>(dst) = make_uint4(y[0], y[1], y[2], y[3]);
    else *reinterpret_cast<uint2*>(dst) = make_uint2(y[0], y[1]);
    if (a.lse && piece == 0) a.lse[token * a.heads + out_head] = total == 0.0f ? -INFINITY : (best + __log2f(total)) * LN2;
}

// Joins the parts of a row: one wavefront to a row.
template <int D>
__global__ __launch_bounds__(256) void paged_attention_join_kernel(PagedAttentionArgs a) {
    constexpr int PER = D / 64;
    const int lane = threadIdx.x & 63;
    const int64_t row = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
    if (row >= (int64_t)a.B * a.q_len * a.heads) return;
    const int64_t token = row / a.heads;
    const int head = (int)(row - token * a.heads), b = (int)(token / a.q_len), j = (int)(token - (int64_t)b * a.q_len);
    const int group = a.heads / a.kv_heads, rows = group * a.q_len;
    const int row_tile = (j * group + head % group) / 16;
    const int j_first = row_tile * 16 / group, j_last = min(row_tile * 16 + 15, rows - 1) / group;
    const int len = min(max(a.lengths[b], 0), a.max_len);
    const int all_end = len - (a.q_len - 1) + j_last, all_begin = a.window > 0 ? max(len - (a.q_len - 1) + j_first - a.window, 0) & ~15 : 0;
    const int parts = max(1, (all_end - all_begin + a.chunk - 1) / a.chunk);     // those that have tokens, and the first
    const float2* ml = a.part_ml + row * a.splits;
    const float* po = a.part_o + row * a.splits * D + PER * lane;
    float best = UNSET;
    for (int s = lane; s < parts; s += 64) best = fmaxf(best, ml[s].x);
#pragma unroll
    for (int off = 32; off >= 1; off >>= 1) best = fmaxf(best, __shfl_xor(best, off, 64));
    float total = 0.0f, x[PER] = {};
    for (int s = 0; s < parts; ++s) {
        const float2 m = ml[s];
        const float f = __builtin_amdgcn_exp2f(m.x - best);
        total = fmaf(m.y, f, total);
#pragma unroll
        for (int c = 0; c < PER; ++c) x[c] = fmaf(po[(int64_t)s * D + c], f, x[c]);
    }
    const float inv = total > 0.0f ? __fdiv_rn(1.0f, total) : total == 0.0f ? 0.0f : total;
    uint16_t* dst = a.out + token * a.ldo + head * D + PER * lane;
#pragma unroll
    for (int c = 0; c < PER; ++c) dst[c] = f32_to_bf16(x[c] * inv);
    if (a.lse && lane == 0) a.lse[row] = total == 0.0f ? -INFINITY : (best + __log2f(total)) * LN2;
}

template <int D>
int launch(const PagedAttentionArgs& a, hipStream_t s) {
    const int rows = a.heads / a.kv_heads * a.q_len;
    const int64_t blocks = (int64_t)a.B * a.kv_heads * ((rows + 15) / 16) * a.splits;
    if (blocks > 0x7FFFFFFFll) return fail(BASQ_EUNSUPPORTED, "paged_attention: too many rows");
    if (a.softcap > 0.0f) hipLaunchKernelGGL((paged_attention_kernel<D, true>), dim3((unsigned)blocks), dim3(PA_WAVES * 64), 0, s, a);
    else hipLaunchKernelGGL((paged_attention_kernel<D, false>), dim3((unsigned)blocks), dim3(PA_WAVES * 64), 0, s, a);
    int rc = check_hip(hipGetLastError(), "paged_attention launch");
    if (rc != BASQ_OK || a.splits == 1) return rc;
    const int64_t joins = ((int64_t)a.B * a.q_len * a.heads + 3) / 4;
    hipLaunchKernelGGL((paged_attention_join_kernel<D>), dim3((unsigned)joins), dim3(256), 0, s, a);
    return check_hip(hipGetLastError(), "paged_attention join launch");
}

}  // namespace

// How the contexts are split: enough workgroups to fill the chip four times over, and no part shorter than 128 tokens, a step of
// each of a workgroup's waves.
void paged_attention_split(int32_t B, int32_t q_len, int32_t heads, int32_t kv_heads, int32_t max_len, int32_t window,
                           int32_t* splits, int32_t* chunk) {
    const int64_t base = (int64_t)B * kv_heads * (((int64_t)(heads / kv_heads) * q_len + 15) / 16);
    // (a window is cut to whole blocks of 16 at its begin, and the rows of a tile have windows up to q_len - 1 tokens apart)
    const int64_t range = window > 0 && window + (int64_t)q_len + 15 < max_len ? window + (int64_t)q_len + 15 : max_len;
    constexpr int64_t PART = 128;
    const int64_t most = (range + PART - 1) / PART, want = base > 0 ? (1024 + base - 1) / base : 1;
    int64_t n = want < most ? want : most;
    if (n < 1) n = 1;
    int64_t each = ((range + n - 1) / n + PART - 1) / PART * PART;
    if (each < PART) each = PART;
    *chunk = (int32_t)each;
    *splits = (int32_t)((range + each - 1) / each > 1 ? (range + each - 1) / each : 1);
}

int launch_paged_attention(PagedAttentionArgs a, hipStream_t s) {
    if (a.B == 0) return BASQ_OK;
    a.cap_log2e = a.softcap * LOG2E;
    a.inv_cap = a.softcap > 0.0f ? 1.0f / a.cap_log2e : 0.0f;
    return a.D == 64 ? launch<64>(a, s) : launch<128>(a, s);
}

}  // namespace basq
