// Attention of a sequence's newest tokens over its paged INT4 cache (paper Sec. 5: per-head asymmetric INT4 of the cache; the
// decode step between the qkv and the output projection).  With k_t = ks_t c_t + kl_t and v_t = vs_t d_t + vl_t, c and d codes:
//
//     s_t = scale (ks_t (q . c_t) + kl_t sum(q)),   p_t = 2^(log2(e) s_t - M),   l = sum_t p_t
//     out = ( sum_t (p_t vs_t) d_t + sum_t p_t vl_t ) / l
//
// so the codes go into the matrix cores as they are, and ranges into the scores and the weights: one pass over the cache, with the
// running reference M of the softmax.
//
// A wavefront takes 32 tokens of one kv head at a time on 16 x 16 x 32 MFMAs whose 16 columns are the query rows that share the kv head
// (its heads, times the new tokens): tokens x channels of the keys times channels x rows gives scores with the row on lane % 16, four
// tokens to a quarter of the wave and block of 16; these are, as they lie, the weights' operand of channels x tokens of the values
// times tokens x rows, whose results keep the row on lane % 16.  So no value changes lanes between the two products, and M, l and the
// rescaling are per lane.  Of up to eight rows, half the columns would be empty: there the rows stand twice, and a lane does one
// block's softmax instead of two (166 vector instructions a step instead of 227).
//
// Codes become fp16 numbers without a conversion, two to an instruction, by masks: a bit pattern of 0 .. 15, taken for an fp16 number,
// is the code times 2^-24, and the code in the next nibble, left in place, 16 times that.  The matrix cores drop low bits of products
// with subnormal operands, the more the smaller they are: with patterns of 0 .. 15 scores are 2.4e-6 off, with 16 times that 3.5e-7
// (q of standard deviation 1.8, D = 128; fp32 arithmetic 2.5e-7), so the keys' codes are all brought to the second nibble; the values',
// whose products end in bf16, are not.  Query rows are brought to fp16 times a power of two of their own (a bf16 value fits it exactly
// while it is within 2^-30 of the row's largest); weights p_t vs_t are rounded to fp16 near 2^5 of their running maximum: 2^-11 of each
// (against 2^-8 of the bf16 output), and of those under 2^-19 of the largest, 2^-30 of that.  Vectors without codes, those of zeros, do not
// count as largest.  l, M and both sums are fp32.
//
// Codes and ranges come by direct loads into a ring of LDS stages that the wave has to itself, a step ahead of the one that is
// worked on: registers hold none of it, and three workgroups of four waves fit a compute unit (loads into registers and two workgroups took
// a quarter longer; three or four stages and two workgroups, or four workgroups, gain nothing).  The loads carry the non-temporal hint:
// nothing is read twice (without it a sixth longer).  With two steps under way, the second requested once the first is in registers, calls
// take 1 .. 3 % longer.
//
// Bound: reading the cache, D + 16 bytes a token and kv head, and not far behind the vector instructions.  64 contexts of 4340 tokens on
// average, 64 heads over 8, are 327 MB and take 61 us, 5.4 TB/s: 56 .. 57 of this kernel and 4.7 of the join; from a cache of one page, so without
// the memory, 53; a kernel that only reads as many bytes takes 49.  What is left is the start of a workgroup (5 us until its first loads are
// in: lengths, page ids, codes, one after the other), its end, where the three workgroups of a compute unit are done one after the other,
// and the join.  16 contexts of 2600 on average, 32 heads over 8: 15.4 us; one of 131072: 32.7.  A call with little to read is the start: 6 us.
#include "basq_internal.h"

#include <type_traits>

namespace basq {

namespace {

typedef _Float16 v8h __attribute__((ext_vector_type(8)));
typedef float v4f __attribute__((ext_vector_type(4)));
typedef uint32_t v4u __attribute__((ext_vector_type(4)));
typedef int v4i __attribute__((ext_vector_type(4)));
typedef __bf16 v2bf __attribute__((ext_vector_type(2)));
typedef float v2f __attribute__((ext_vector_type(2)));
typedef _Float16 v2h __attribute__((ext_vector_type(2)));

constexpr int PA_STEP = 32;                                      // tokens of a wave's step
constexpr int PA_UNIT = 4 * PA_STEP;                             // a step of each of four waves: what work is counted in
constexpr int PA_START = 2;                                       // what the start and the end of a part cost, in units
constexpr int PA_BRIEF = 4;                                      // contexts of that many units are short: never shared
constexpr int PA_STAGES = 2;                                      // steps of a wave in LDS
constexpr float UNSET = -1e30f;                                  // M of a row that has seen no token
constexpr float LOG2E = 1.4426950408889634f, LN2 = 0.6931471805599453f;

// eight codes (one dword, low nibble first) as fp16 numbers 2^-20 times the code, in the order 0 4 | 1 5 | 2 6 | 3 7
__device__ __forceinline__ v8h spread(uint32_t x) {
    constexpr uint32_t MASK = 0x00F000F0u;
    const v4u w = {(x << 4) & MASK, x & MASK, (x >> 4) & MASK, (x >> 8) & MASK};
    return __builtin_bit_cast(v8h, w);
}
__device__ __forceinline__ float quarters_max(float v) {
    return across_rows(v, [](float a, float b) { return fmaxf(a, b); });
}
__device__ __forceinline__ float quarters_sum(float v) {
    return across_rows(v, [](float a, float b) { return a + b; });
}
// the value of lane ^ 8
__device__ __forceinline__ float half_row_on(float v) { return __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(v), 0x128, 0xF, 0xF, true)); }

#define PA_LDS_PTR(p) ((__attribute__((address_space(3))) void*)(p))

// A block of 16 tokens in LDS: its keys, its values, its ranges (4 KB would be the next power of two; blocks lie end to end).
template <int D>
struct Block {
    static constexpr int V_AT = 8 * D, R_AT = 16 * D, BYTES = 16 * D + 256;
    static constexpr int LOADS = D == 128 ? 3 : 2;               // direct loads that bring it
};

// N neighbouring values (2, 4 or 8) in one go
template <int N>
__device__ __forceinline__ void store(float* to, const float (&x)[N]) {
    if constexpr (N == 2) *reinterpret_cast<float2*>(to) = make_float2(x[0], x[1]);
    else
#pragma unroll
        for (int c = 0; c < N; c += 4) *reinterpret_cast<float4*>(to + c) = make_float4(x[c], x[c + 1], x[c + 2], x[c + 3]);
}

// N neighbouring channels of a row's result, from its sums at reference M: out = x / l (0 where no token counted), lse.
template <int N>
__device__ __forceinline__ void finish(const PagedAttentionArgs& a, int64_t token, int head, int D, int channel, const float (&x)[N], float M, float l) {
    const float inv = l > 0.0f ? __fdiv_rn(1.0f, l) : l;         // (0 and NaN stay)
    uint32_t y[N / 2];
#pragma unroll
    for (int c = 0; c < N; c += 2) y[c / 2] = __builtin_bit_cast(uint32_t, __builtin_convertvector((v2f){x[c] * inv, x[c + 1] * inv}, v2bf));
    uint16_t* dst = a.out + token * a.ldo + head * D + channel;
    if constexpr (N == 8) *reinterpret_cast<uint4*>(dst) = make_uint4(y[0], y[1], y[2], y[3]);
    else if constexpr (N == 4) *reinterpret_cast<uint2*>(dst) = make_uint2(y[0], y[1]);
    else *reinterpret_cast<uint32_t*>(dst) = y[0];
    if (a.lse && channel == 0) a.lse[token * a.heads + head] = l == 0.0f ? -INFINITY : (M + __log2f(l)) * LN2;
}

// the length of a sequence that is the same for the whole wave (a scalar load: a vector load's wait would be for all direct loads too)
__device__ __forceinline__ int clamped(const PagedAttentionArgs& a, int len) { return min(max(len, 0), a.max_len); }
__device__ __forceinline__ int length_of(const PagedAttentionArgs& a, int b) {
    return clamped(a, ((const __attribute__((address_space(4))) int32_t*)a.lengths)[b]);
}
// the first token that a new token sees, in whole blocks, when it sees those before `end`
__device__ __forceinline__ int first_token(const PagedAttentionArgs& a, int end) { return a.window > 0 ? max(end - a.window, 0) & ~15 : 0; }
// units of PA_UNIT tokens that any new token of a sequence sees, the same for all its segments; at least one, whose taker also writes
// the zeros of rows that see nothing
__device__ __forceinline__ int units_of(const PagedAttentionArgs& a, int len) {
    return max((len - first_token(a, len - (a.q_len - 1)) + PA_UNIT - 1) / PA_UNIT, 1);
}

// ROWS query rows at most in a tile.  LDS is allocated in steps of 1280 bytes: D = 128 with 8 rows takes 42 of the 128, three workgroups
// to a compute unit.
template <int D, int WAVES, int ROWS>
struct Shared {
    uint8_t ring[WAVES][PA_STAGES][2][Block<D>::BYTES];
    int o[WAVES][ROWS][D];                                    // fp32 (integers for the compiler, see below), groups of 4 in another order in each row
    int ml[WAVES][3][ROWS];                                    // M, l, lows of each wave
};

static_assert(sizeof(Shared<128, 4, 8>) <= 42 * 1280, "three workgroups to a compute unit");

template <int N>
__device__ __forceinline__ void wait_loads() {
    asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory");
}
// (the compiler's own barrier waits for every load that is under way)
__device__ __forceinline__ void lds_barrier() { asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory"); }
__device__ __forceinline__ int same(int v) { return __builtin_amdgcn_readfirstlane(v); }

// Some units of a segment, one kv head and tile of query rows of sequence b: `taken` of its `units`, from number `unit` on.
struct Part {
    int b, len, segment, unit, taken, units;
    int kv_head, row_tile;
    int from, to;                                                // the tokens of it that any row of the tile sees
    int j_first;                                                 // the first row's new token
    int inner_begin, inner_end;                                  // between these, all rows see all tokens
};

// Work is a row of units: sequence by sequence, in it segment by segment (kv head by kv head, row tile by row tile), in it token by
// token; in front of each segment stand PA_START units that are no tokens, for what a part costs besides its tokens.  With a.workers > 0
// that many workgroups take equal shares of it, whatever the lengths are: a share begins and ends inside segments, whose parts the
// second kernel joins.  Otherwise a workgroup takes whole segments, every gridDim.x-th.
//
// FOLD: tiles of at most eight rows, which stand in columns 0 .. 7 and again in 8 .. 15; a lane works on the first block's scores, or
// on the second's, instead of on both.
template <int D, int WAVES, bool CAP, bool FOLD>
__global__ __launch_bounds__(WAVES * 64, WAVES == 8 || (D == 128 && !FOLD) ? 2 : 3) void paged_attention_kernel(PagedAttentionArgs a) {
#if defined(__HIP_DEVICE_COMPILE__)   // buffer resources are a device-only type; the host pass only needs the stub
    constexpr int TILES = D / 16;                                // channel tiles of the second product: channel TILES * n + c
    constexpr int KS = D / 32;                                   // 32-channel steps of the first
    constexpr int MINE = FOLD ? 4 : 8;                           // tokens of a lane in a step
    constexpr int ROWS = FOLD ? 8 : 16;
    constexpr int STRIDE = WAVES * PA_STEP;
    __shared__ __attribute__((aligned(256))) Shared<D, WAVES, ROWS> lds;
    const int lane = threadIdx.x & 63, wave = same(threadIdx.x >> 6);
    const int col = lane & 15, quarter = lane >> 4;
    const int group = a.group, rows = group * a.q_len, row_tiles = a.row_tiles;
    const int segments = a.kv_heads * row_tiles;                 // of a sequence
    const int P = 1 << a.page_log2;
    const int64_t head_bytes = (int64_t)P * (D + 16);

    // ---- this workgroup's first part, and the units that it has to take
    int b = 0, len, segment, unit = 0, units, left, share = 1;   // left: with PA_START units for each segment that begins
    if (a.workers == 0) {
        b = blockIdx.x / segments;
        segment = blockIdx.x - b * segments;
        len = length_of(a, b);
        units = units_of(a, len);
        left = units + PA_START;
    } else {
        int mine = 0, u = 0, sum = 0;                            // of sequence base + lane: length, units, units of all up to it
        auto scan = [&](int base) {
            mine = base + lane < a.B ? clamped(a, a.lengths[base + lane]) : 0;
            u = base + lane < a.B ? units_of(a, mine) + PA_START : 0;
            sum = u;
            sum += __builtin_amdgcn_update_dpp(0, sum, 0x111, 0xF, 0xF, true);       // rows of 16 lanes: shifts by 1, 2, 4, 8
            sum += __builtin_amdgcn_update_dpp(0, sum, 0x112, 0xF, 0xF, true);
            sum += __builtin_amdgcn_update_dpp(0, sum, 0x114, 0xF, 0xF, true);
            sum += __builtin_amdgcn_update_dpp(0, sum, 0x118, 0xF, 0xF, true);
            sum += __builtin_amdgcn_update_dpp(0, sum, 0x142, 0xA, 0xF, false);      // lane 15 into the second row, 47 into the fourth
            sum += __builtin_amdgcn_update_dpp(0, sum, 0x143, 0xC, 0xF, false);      // lane 31 into the upper half
            return __builtin_amdgcn_readlane(sum, 63);
        };
        int total = 0, last_round = 0;
        for (int base = 0; base < a.B; base += 64) {
            total += scan(base);
            last_round = base;
        }
        total *= segments;
        share = same((total + a.workers - 1) / a.workers);
        const int first = blockIdx.x * share;
        left = min(share, total - first);                        // (not above 0 behind the last)
        if (left <= 0) return;
        int before = 0;                                          // units of the sequences before b, that of unit `first`
        for (;;) {
            const int these = last_round > 0 ? scan(b) : __builtin_amdgcn_readlane(sum, 63);
            const uint64_t behind = __ballot((before + sum) * segments > first);
            if (behind != 0) {                                   // (it is in one of the rounds: first < total)
                const int n = __builtin_ctzll(behind);
                before += __builtin_amdgcn_readlane(sum - u, n);
                units = __builtin_amdgcn_readlane(u, n) - PA_START;
                len = __builtin_amdgcn_readlane(mine, n);
                b += n;
                break;
            }
            before += these;
            b += 64;
        }
        segment = (first - before * segments) / (units + PA_START);
        unit = first - before * segments - segment * (units + PA_START) - PA_START;
        if (unit < 0) {                                          // some of the start is this share's
            left += unit + PA_START;
            unit = 0;
        } else {
            left += PA_START;
        }
        if (left <= PA_START) return;
    }

    auto describe = [&](int b, int len, int segment, int unit, int units, int left) {
        Part p;
        p.b = b; p.len = len; p.segment = segment; p.unit = unit; p.units = units;
        p.taken = min(units - unit, left - PA_START);
        p.kv_head = row_tiles == 1 ? segment : same(segment / row_tiles);
        p.row_tile = segment - p.kv_head * row_tiles;
        const int seen = len - (a.q_len - 1);                     // tokens that the first new token sees
        const int j_first = row_tiles == 1 ? 0 : same(p.row_tile * 16 / group);
        const int j_last = row_tiles == 1 ? a.q_len - 1 : same(min(p.row_tile * 16 + 15, rows - 1) / group);
        const int begin = first_token(a, seen);
        p.from = max(begin + unit * PA_UNIT, first_token(a, seen + j_first));
        p.to = min(begin + (unit + p.taken) * PA_UNIT, seen + j_last);
        p.inner_begin = a.window > 0 ? max(seen + j_last - a.window, 0) : 0;
        p.inner_end = seen + j_first;
        p.j_first = j_first;
        return p;
    };
    // the lane's query row in a part's tile; the new token of a row
    auto new_token = [&](int row) { return a.q_len == 1 ? 0 : row / group; };
    auto row_of = [&](const Part& p) { return min(p.row_tile * 16 + (FOLD ? col & 7 : col), rows - 1); };

    // ---- what a lane requests, as byte offsets into one head of one page, and where it reads what it works on.  Row i of the first
    // product's results is token 4 * (i % 4) + i / 4 of a block, so quarter g of the wave works on tokens g, 4 + g, 8 + g, 12 + g:
    // for each of the four, the wave reads 256 (128) bytes of values side by side.  Keys lie in 16-byte pieces whose place
    // inside their row changes from token to token, so that 16 lanes read from all banks; ranges lie by quarter.
    uint32_t code_from[Block<D>::LOADS - 1];
    if constexpr (D == 128) {
        code_from[0] = 16 * ((lane & 60) | ((lane ^ (lane >> 4)) & 3));
        code_from[1] = P * 64 + 16 * lane;
    } else {
        code_from[0] = lane < 32 ? 16 * ((lane & 30) | ((lane ^ (lane >> 4)) & 1)) : P * 32 + 16 * (lane - 32);
    }
    const uint32_t range_from = P * D + (lane >> 5) * 8 * P + 8 * (4 * ((lane >> 1) & 3) + ((lane >> 3) & 3)) + 4 * (lane & 1);
    const int token = 4 * (col & 3) + (col >> 2);
    const int k_at = D == 128 ? token * 64 + ((quarter ^ token >> 2) & 3) * 16 : token * 32 + ((quarter >> 1) ^ (token >> 3)) * 16 + (quarter & 1) * 8;
    const int v_at = Block<D>::V_AT + quarter * (D / 2) + col * (D / 32), r_at = Block<D>::R_AT + quarter * 32 + (FOLD ? (col >> 3) * Block<D>::BYTES : 0);
    uint8_t* const ring = &lds.ring[wave][0][0][0];

    // The wave's next 32 steps: where block 2i + h of 16 tokens begins in the cache, on lane 2i + h; and whether it is there (not
    // past the end, of a page that exists; the others are read from the first page, and masked).
    int64_t place = 0;
    uint64_t there = 0;
    auto request_ids = [&](const Part& p, int t0) {
        const int t = t0 + (lane >> 1) * STRIDE + (lane & 1) * 16;
        return t < p.to ? a.page_table[(int64_t)p.b * a.table_stride + (t >> a.page_log2)] : -1;
    };
    auto take_ids = [&](const Part& p, int id) {
        const bool ok = id >= 0 && id < a.num_pages;
        there = __ballot(ok);
        place = ((int64_t)(ok ? id : 0) * a.kv_heads + p.kv_head) * head_bytes;
    };
    // requests step i, tokens t .., into a stage of the ring; nothing (which counts as loads) behind the last
    auto load = [&](int i, int last, int t, int stage) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int from_lane = (2 * i + h) & 63;
            const uint32_t low = __builtin_amdgcn_readlane((int)place, from_lane), high = __builtin_amdgcn_readlane((int)(place >> 32), from_lane);
            const __amdgpu_buffer_rsrc_t rsrc = __builtin_amdgcn_make_buffer_rsrc(const_cast<uint8_t*>(a.cache) + (int64_t)((uint64_t)high << 32 | low), 0,
                                                                                  i <= last ? (int)head_bytes : 0, 0x00020000);
            const int at = (t + 16 * h) & (P - 1);
            uint8_t* dst = ring + (stage * 2 + h) * Block<D>::BYTES;
#pragma unroll
            for (int n = 0; n < Block<D>::LOADS - 1; ++n)
                __builtin_amdgcn_raw_ptr_buffer_load_lds(rsrc, PA_LDS_PTR(dst + 1024 * n), 16, (int)code_from[n], at * (D / 2), 0, 2);
            __builtin_amdgcn_raw_ptr_buffer_load_lds(rsrc, PA_LDS_PTR(dst + Block<D>::R_AT), 4, (int)range_from, at * 8, 0, 2);
        }
    };
    auto last_step = [&](const Part& p, int t0) { return t0 < p.to ? min(32, (p.to - t0 + STRIDE - 1) / STRIDE) - 1 : -1; };
    auto load_first = [&](const Part& p, int t0) {
#pragma unroll
        for (int i = 0; i < PA_STAGES - 1; ++i) load(i, last_step(p, t0), t0 + i * STRIDE, i);
    };
    uint4 raw[KS];                                               // the lane's D/4 channels of its query row
    auto request_row = [&](const Part& p) {
        const int row = row_of(p), j = new_token(row), head = p.kv_head * group + row - j * group;
        const uint4* src = reinterpret_cast<const uint4*>(a.q + ((int64_t)p.b * a.q_len + j) * a.ldq + (int64_t)head * D + quarter * (D / 4));
#pragma unroll
        for (int i = 0; i < KS; ++i) raw[i] = src[i];
    };

    // ---- the state of a part
    v8h q[KS];
    float c1, qs;
    int begin, end;                                               // the tokens that the lane's row sees
    v4f o[TILES];
    float M, l, lows;                                             // l and lows: this lane's tokens
    bool set;                                                     // M is a reference: the row has seen a token
    bool fresh;                                                   // all sums are 0
    auto start = [&](const Part& p) {
        end = p.inner_end - p.j_first + new_token(row_of(p));
        begin = a.window > 0 ? max(end - a.window, 0) : 0;
        // (sums of pairs by the dot product with 1, 1)
        float x[D / 4], top = 0.0f, sum = 0.0f;
#pragma unroll
        for (int i = 0; i < D / 4; i += 2) {
            const uint32_t u = reinterpret_cast<const uint32_t*>(raw)[i / 2];
            x[i] = __uint_as_float(u << 16);
            x[i + 1] = __uint_as_float(u & 0xFFFF0000u);
            top = fmaxf(top, fmaxf(fabsf(x[i]), fabsf(x[i + 1])));
            sum = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(v2bf, u), (v2bf){(__bf16)1.0f, (__bf16)1.0f}, sum, false);
        }
        top = quarters_max(top);
        sum = quarters_sum(sum);
        qs = a.scale * LOG2E * sum;
        // The largest value is brought to 2^14 .. 2^15 (exponent field of top, 127 = 2^0).  (All rows, always: doing so where some row needs it
        // spares 0.1 us, but then the bits of one depend on the others.)
        const int e = min(max(141 - (int)(__float_as_uint(top) >> 23), -100), 100);
        const float up = __uint_as_float((uint32_t)(127 + e) << 23);
        c1 = a.scale * LOG2E * 0x1p20f * __uint_as_float((uint32_t)(127 - e) << 23);
#pragma unroll
        for (int i = 0; i < D / 4; ++i) x[i] *= up;
#pragma unroll
        for (int s = 0; s < KS; ++s) {
            constexpr int ORDER[8] = {0, 4, 1, 5, 2, 6, 3, 7};
#pragma unroll
            for (int i = 0; i < 8; ++i) q[s][i] = (_Float16)x[8 * s + ORDER[i]];
        }
#pragma unroll
        for (int c = 0; c < TILES; ++c) o[c] = (v4f){0.f, 0.f, 0.f, 0.f};
        M = l = lows = 0.0f;
        set = false;
        fresh = true;
    };

    auto row_max = [&](float v) {
        v = quarters_max(v);
        return FOLD ? fmaxf(v, half_row_on(v)) : v;
    };
    auto work = [&](const Part& part, int i, int t, int stage) {
        const uint8_t* blocks = ring + stage * 2 * Block<D>::BYTES;
        // All that the step reads from LDS, in the order of its use, before any of it is used.
        // (As integers: in front of a float-typed read of LDS the compiler waits for every direct load.)
        typedef int Keys __attribute__((ext_vector_type(KS)));
        Keys kw[2];
        v4i range[MINE / 4][4];                                   // (scale, lo) of a lane's tokens, two in each: keys', values'
        uint32_t v[8];
#pragma unroll
        for (int h = 0; h < 2; ++h) kw[h] = *reinterpret_cast<const Keys*>(blocks + h * Block<D>::BYTES + k_at);
#pragma unroll
        for (int h = 0; h < MINE / 4; ++h)
#pragma unroll
            for (int n = 0; n < 4; ++n) range[h][n] = *reinterpret_cast<const v4i*>(blocks + h * Block<D>::BYTES + r_at + 128 * (n / 2) + 16 * (n % 2));
#pragma unroll
        for (int r = 0; r < 8; ++r) {
            const uint8_t* from = blocks + (r / 4) * Block<D>::BYTES + v_at + (r % 4) * (2 * D);
            v[r] = D == 128 ? (uint32_t)*reinterpret_cast<const int*>(from) : *reinterpret_cast<const uint16_t*>(from);
        }
        __builtin_amdgcn_sched_barrier(0);
        v4f acc[2];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            acc[h] = (v4f){0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int n = 0; n < KS; ++n) acc[h] = __builtin_amdgcn_mfma_f32_16x16x32_f16(spread(kw[h][n]), q[n], acc[h], 0, 0, 0);
        }
        // folded, columns 8 .. 15 are the rows of 0 .. 7 again, for the second block
        if constexpr (FOLD)
#pragma unroll
            for (int r = 0; r < 4; ++r) acc[0][r] = col & 8 ? acc[1][r] : acc[0][r];
        float sc[MINE], vs[MINE], vl[MINE];
        float least = INFINITY;                                   // scale of a value
#pragma unroll
        for (int h = 0; h < MINE / 4; ++h) {
#pragma unroll
            for (int r = 0; r < 4; r += 2) {
                const v4f kr = __builtin_bit_cast(v4f, range[h][r / 2]), vr = __builtin_bit_cast(v4f, range[h][2 + r / 2]);
#pragma unroll
                for (int n = 0; n < 2; ++n) {
                    // less M; with a cap, M goes off behind that
                    const float x = fmaf(kr[2 * n], acc[h][r + n] * c1, CAP ? kr[2 * n + 1] * qs : fmaf(kr[2 * n + 1], qs, -M));
                    sc[4 * h + r + n] = x;
                    vs[4 * h + r + n] = vr[2 * n];
                    vl[4 * h + r + n] = vr[2 * n + 1];
                    least = fminf(least, vr[2 * n]);
                }
            }
        }
        if constexpr (CAP) {
            // log2(e) cap tanh(y), y = x / (log2(e) cap).  Up to 3/8 by its series, under 2^-24 of the value off, which is all that most
            // steps need; beyond, 1 - 2 / (e^2y + 1) by the instructions for 1 / x and 2^x, each a unit in the last place off at most: some 2^-23
            // together, as the rounding of the 1 is.
            bool far = false;
            float y[MINE];
#pragma unroll
            for (int n = 0; n < MINE; ++n) {
                y[n] = sc[n] * a.inv_cap;
                far = far || !(fabsf(y[n]) < 0.375f);
                const float y2 = y[n] * y[n];
                sc[n] = y[n] * fmaf(y2, fmaf(y2, fmaf(y2, fmaf(y2, fmaf(y2, -1382.0f / 155925, 62.0f / 2835), -17.0f / 315), 2.0f / 15), -1.0f / 3), 1.0f);
            }
            if (__any(far)) {
                asm volatile("");
#pragma unroll
                for (int n = 0; n < MINE; ++n) {
                    const float t = 1.0f - 2.0f * __builtin_amdgcn_rcpf(__builtin_amdgcn_exp2f(y[n] * (2.0f * LOG2E)) + 1.0f);
                    sc[n] = fabsf(y[n]) < 0.375f ? sc[n] : t;
                }
            }
#pragma unroll
            for (int n = 0; n < MINE; ++n) sc[n] = fmaf(sc[n], a.cap_log2e, -M);
        }
        const unsigned both = (unsigned)(there >> (2 * i)) & 3u;
        if (both != 3u || t < part.inner_begin || t + PA_STEP > part.inner_end) {
            asm volatile("");                                     // (a branch: few steps come here)
            // what is masked may hold anything, also ranges that are no numbers
#pragma unroll
            for (int n = 0; n < MINE; ++n) {
                const int h = FOLD ? col >> 3 : n / 4, at = t + 16 * h + 4 * (n % 4) + quarter;
                const bool seen = at >= begin && at < end && (both >> h & 1u);
                sc[n] = seen ? sc[n] : -INFINITY;
                vs[n] = seen ? vs[n] : 0.0f;
                vl[n] = seen ? vl[n] : 0.0f;
            }
        }
        float p[MINE], w[MINE];
        auto weigh = [&]() {
            float top = 0.0f;
#pragma unroll
            for (int r = 0; r < MINE; ++r) {
                p[r] = __builtin_amdgcn_exp2f(sc[r]);
                w[r] = p[r] * vs[r];
                top = fmaxf(top, w[r]);
            }
            return top;
        };
        float top = weigh();
        // A row's first tokens, and weights that leave fp16's range, give it a new reference: its largest weight becomes 2^5.
        // (Where a scale is next to 0, p itself counts once it nears the end of fp32.)
        if (__any(top > 0x1p15f || !set || !(least >= 0x1p-60f))) {
            asm volatile("");
            // A vector without an extent is stored with a scale of 1, and codes of 0 if it is zero: it weighs nothing, but a reference set by
            // that scale would leave the others, on whom the output depends, few bits.
            bool without_extent = false;
#pragma unroll
            for (int r = 0; r < MINE; ++r) without_extent = without_extent || vs[r] == 1.0f;
            if (__any(without_extent)) {
                asm volatile("");
#pragma unroll
                for (int r = 0; r < MINE; ++r) {
                    const uint64_t first = __ballot(v[r] != 0), second = FOLD ? __ballot(v[4 + r] != 0) : 0;
                    const uint64_t some = FOLD && col & 8 ? second : first;
                    const uint32_t of_pair = quarter & 2 ? (uint32_t)(some >> 32) : (uint32_t)some;
                    if (vs[r] == 1.0f && (of_pair & (quarter & 1 ? 0xFFFF0000u : 0xFFFFu)) == 0) vs[r] = 0.0f;
                }
            }
            float best = -INFINITY;
            top = 0.0f;
#pragma unroll
            for (int r = 0; r < MINE; ++r) {
                best = fmaxf(best, sc[r] + fmaxf(__builtin_amdgcn_logf(vs[r]), -60.0f));
                w[r] = p[r] * vs[r];
                top = fmaxf(top, fmaxf(fabsf(w[r]), p[r] * 0x1p-60f));
            }
            best = row_max(best);
            const float up = (row_max(top) > 0x1p15f || !set) && best > -INFINITY ? best - 5.0f : 0.0f;
            M += up;
#pragma unroll
            for (int r = 0; r < MINE; ++r) sc[r] -= up;
            if (!fresh) {
                const float f = set ? __builtin_amdgcn_exp2f(-up) : 0.0f;        // (the sums of a row without a reference are 0)
                l *= f;
                lows *= f;
#pragma unroll
                for (int c = 0; c < TILES; ++c) o[c] *= f;
            }
            set = set || best > -INFINITY;
            weigh();
        }
        fresh = false;
#pragma unroll
        for (int r = 0; r < MINE; ++r) {
            l += p[r];
            lows = fmaf(p[r], vl[r], lows);
        }
        v8h pw;
        if constexpr (FOLD) {
            // the second block's weights from eight lanes further on (in columns 8 .. 15, whose results nobody reads, the first's)
            v4u both_w;
#pragma unroll
            for (int n = 0; n < 2; ++n) {
                both_w[n] = __builtin_bit_cast(uint32_t, (v2h){(_Float16)w[2 * n], (_Float16)w[2 * n + 1]});
                both_w[2 + n] = (uint32_t)__builtin_amdgcn_mov_dpp((int)both_w[n], 0x128, 0xF, 0xF, true);
            }
            pw = __builtin_bit_cast(v8h, both_w);
        } else {
#pragma unroll
            for (int n = 0; n < 8; ++n) pw[n] = (_Float16)w[n];
        }
        // channels x tokens of the values: pairs of tokens side by side, then a code of both per instruction
        constexpr int HALVES = D == 128 ? 2 : 1;
#pragma unroll
        for (int half = 0; half < HALVES; ++half) {
            uint32_t x[4];
#pragma unroll
            for (int r = 0; r < 4; ++r) x[r] = __builtin_amdgcn_perm(v[2 * r + 1], v[2 * r], half ? 0x07060302u : 0x05040100u);
#pragma unroll
            for (int c = 0; c < 4; ++c) {
                const uint32_t mask = c & 1 ? 0x00F000F0u : 0x000F000Fu;
                const int down = c & 2 ? 8 : 0;
                const v4u f = {(x[0] >> down) & mask, (x[1] >> down) & mask, (x[2] >> down) & mask, (x[3] >> down) & mask};
                o[4 * half + c] = __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(v8h, f), pw, o[4 * half + c], 0, 0, 0);
            }
        }
    };

    bool joined = false;
    // ---- the four waves' sums into one: written at each wave's own reference, read at the largest
    auto finish_part = [&](const Part& p) {
        // a segment that begins here: its first part's workgroup, and how many parts it has
        if (a.workers > 0 && p.unit == 0 && threadIdx.x == 0)
            a.part_of[(int64_t)p.b * segments + p.segment] = make_int2(blockIdx.x, 1 + (p.units - p.taken + share - 1) / share);
        l = quarters_sum(l);
        lows = quarters_sum(lows);
        if constexpr (FOLD) {
            l += half_row_on(l);
            lows += half_row_on(lows);
        }
        if (joined) lds_barrier();                                // the part before is read
        joined = true;
        if (col < ROWS) {
            if (quarter == 0) {
                lds.ml[wave][0][col] = __float_as_int(set ? M : UNSET);
                lds.ml[wave][1][col] = __float_as_int(l);
                lds.ml[wave][2][col] = __float_as_int(lows);
            }
#pragma unroll
            for (int r = 0; r < 4; ++r)
#pragma unroll
                for (int c = 0; c < TILES; c += 4)
                    *reinterpret_cast<v4i*>(&lds.o[wave][col][(TILES * (4 * quarter + r) + c) ^ (col & 7) * 4]) =
                        __builtin_bit_cast(v4i, (v4f){o[c][r], o[c + 1][r], o[c + 2][r], o[c + 3][r]});
        }
        lds_barrier();
        // 16 to 64 threads to a row, 2 to 8 neighbouring channels each
        constexpr int THREADS = WAVES * 64 / ROWS < D / 2 ? WAVES * 64 / ROWS : D / 2, N = D / THREADS;
        const int r = threadIdx.x / THREADS, piece = threadIdx.x % THREADS, row = p.row_tile * 16 + r;
        if (r >= ROWS || row >= rows) return;
        float x[N] = {}, total = 0.0f, bias = 0.0f, best = UNSET;
#pragma unroll
        for (int w = 0; w < WAVES; ++w) best = fmaxf(best, __int_as_float(lds.ml[w][0][r]));
#pragma unroll
        for (int w = 0; w < WAVES; ++w) {
            const float f = __builtin_amdgcn_exp2f(__int_as_float(lds.ml[w][0][r]) - best);
            total = fmaf(__int_as_float(lds.ml[w][1][r]), f, total);
            bias = fmaf(__int_as_float(lds.ml[w][2][r]), f, bias);
#pragma unroll
            for (int c = 0; c < N; ++c) x[c] = fmaf(__int_as_float(lds.o[w][r][(N * piece + c) ^ (r & 7) * 4]), f, x[c]);
        }
        // (codes of even channels went in 2^-24 times their size, those of odd ones 2^-20)
#pragma unroll
        for (int c = 0; c < N; ++c) x[c] = fmaf(x[c], c & 1 ? 0x1p20f : 0x1p24f, bias);
        if (p.taken < p.units) {
            // the part of a workgroup that the segment began before, and the one that begins in it
            const int64_t at = (2 * (int64_t)blockIdx.x + (p.unit == 0)) * 16 + r;
            store<N>(a.part_o + at * D + N * piece, x);
            if (piece == 0) a.part_ml[at] = make_float2(best, total);
            return;
        }
        const int j = new_token(row);
        finish<N>(a, (int64_t)p.b * a.q_len + j, p.kv_head * group + row - j * group, D, N * piece, x, best, total);
    };

    // ---- part by part; the first loads of the next are under way while the sums of one are joined
    Part part = describe(same(b), same(len), same(segment), same(unit), same(units), same(left));
    take_ids(part, request_ids(part, part.from + wave * PA_STEP));
    request_row(part);
    load_first(part, part.from + wave * PA_STEP);
    left = same(left);
    uint32_t round = 1;
    for (;;) {
        left -= part.taken + PA_START;
        const bool more = a.workers > 0 ? left > PA_START : (uint32_t)blockIdx.x + round * gridDim.x < (uint32_t)(a.B * segments);
        int next_ids = -1, next_b = part.b, next_segment = part.segment + 1, next_len = 0, next_units = 0;
        if (more) {
            if (a.workers == 0) {
                const int index = blockIdx.x + round++ * gridDim.x;
                next_b = same(index / segments);
                next_segment = index - next_b * segments;
            } else if (next_segment == segments) {
                ++next_b;
                next_segment = 0;
            }
            next_len = next_b == part.b ? part.len : length_of(a, next_b);
            next_units = units_of(a, next_len);
            if (a.workers == 0) left = next_units + PA_START;
            const Part next = describe(next_b, next_len, next_segment, 0, next_units, left);
            next_ids = request_ids(next, next.from + wave * PA_STEP);
        }
        start(part);
        // PA_STAGES - 1 steps are under way while one is worked on
        for (int t0 = part.from + wave * PA_STEP; t0 < part.to; t0 += 32 * STRIDE) {
            const int last = last_step(part, t0);
            if (t0 >= part.from + 32 * STRIDE) {
                take_ids(part, request_ids(part, t0));
                load_first(part, t0);
            }
            int stage = 0;
            for (int i = 0; i <= last; ++i) {
                load(i + PA_STAGES - 1, last, t0 + (i + PA_STAGES - 1) * STRIDE, stage == 0 ? PA_STAGES - 1 : stage - 1);
                wait_loads<(PA_STAGES - 1) * 2 * Block<D>::LOADS>();
                work(part, i, t0 + i * STRIDE, stage);
                asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");    // the stage is read before it is requested anew
                stage = stage == PA_STAGES - 1 ? 0 : stage + 1;
            }
        }
        wait_loads<0>();
        if (more) {                                               // (described anew: two parts' descriptions fill the scalar registers)
            const Part next = describe(next_b, next_len, next_segment, 0, next_units, left);
            request_row(next);
            take_ids(next, next_ids);
            load_first(next, next.from + wave * PA_STEP);
        }
        finish_part(part);
        if (!more) return;
        part = describe(next_b, next_len, next_segment, 0, next_units, left);
    }
#endif
}

// Joins the parts of the segments that have several: WAVES wavefronts to a row, groups of D/4 lanes to a part, four channels each.
// It is memory latencies: where the parts are, and what they are, all of them (up to 128 of D = 128 with eight waves) at once.
template <int D, int WAVES>
__global__ __launch_bounds__(WAVES == 1 ? 256 : WAVES * 64) void paged_attention_join_kernel(PagedAttentionArgs a) {
    constexpr int LANES = D / 4, GROUPS = WAVES * 64 / LANES, AHEAD = WAVES == 1 ? 4 : 8;
    __shared__ float lds[WAVES][LANES][6];
    const int wave = same(threadIdx.x >> 6), lane = threadIdx.x & 63;
    const uint32_t row = WAVES == 1 ? blockIdx.x * 4 + wave : blockIdx.x;            // (fewer than 2^31 rows)
    if (row >= (uint32_t)a.B * a.q_len * a.heads) return;
    const uint32_t token = same(row / (uint32_t)a.heads);
    const int head = same(row - token * a.heads), kv_head = same((uint32_t)head / (uint32_t)a.group);
    const int b = a.q_len == 1 ? (int)token : same(token / (uint32_t)a.q_len), j = (int)token - b * a.q_len;
    const int in_kv = j * a.group + head - kv_head * a.group;
    const int2 where = a.part_of[((int64_t)b * a.kv_heads + kv_head) * a.row_tiles + in_kv / 16];
    const int parts = where.y;
    if (parts <= 1) return;
    const int piece = lane % LANES, group0 = (WAVES == 1 ? 0 : wave * (64 / LANES)) + lane / LANES;
    float best = UNSET, total = 0.0f, x[4] = {};
    for (int p0 = group0; p0 < parts; p0 += AHEAD * GROUPS) {
        float2 ml[AHEAD];
        float4 o[AHEAD];
#pragma unroll
        for (int i = 0; i < AHEAD; ++i) {
            const int p = p0 + i * GROUPS;
            ml[i] = make_float2(UNSET, 0.0f);
            o[i] = make_float4(0.f, 0.f, 0.f, 0.f);
            if (p < parts) {
                const int64_t at = (2 * ((int64_t)where.x + p) + (p == 0)) * 16 + in_kv % 16;
                ml[i] = a.part_ml[at];
                o[i] = *reinterpret_cast<const float4*>(a.part_o + at * D + 4 * piece);
            }
        }
        float next = best;
#pragma unroll
        for (int i = 0; i < AHEAD; ++i) next = fmaxf(next, ml[i].x);
        const float back = __builtin_amdgcn_exp2f(best - next);
        best = next;
        total *= back;
#pragma unroll
        for (int c = 0; c < 4; ++c) x[c] *= back;
#pragma unroll
        for (int i = 0; i < AHEAD; ++i) {
            const float f = __builtin_amdgcn_exp2f(ml[i].x - best), y[4] = {o[i].x, o[i].y, o[i].z, o[i].w};
            total = fmaf(ml[i].y, f, total);
#pragma unroll
            for (int c = 0; c < 4; ++c) x[c] = fmaf(y[c], f, x[c]);
        }
    }
    // the groups of a wave, then the waves
    auto join = [&](float m, float t, const float (&y)[4]) {
        const float next = fmaxf(best, m), f = __builtin_amdgcn_exp2f(best - next), g = __builtin_amdgcn_exp2f(m - next);
        best = next;
        total = fmaf(total, f, t * g);
#pragma unroll
        for (int c = 0; c < 4; ++c) x[c] = fmaf(x[c], f, y[c] * g);
    };
#pragma unroll
    for (int off = LANES; off < 64; off <<= 1) {
        float y[4];
#pragma unroll
        for (int c = 0; c < 4; ++c) y[c] = __shfl_xor(x[c], off, 64);
        join(__shfl_xor(best, off, 64), __shfl_xor(total, off, 64), y);
    }
    if constexpr (WAVES > 1) {
        if (lane < LANES) {
            float* mine = lds[wave][lane];
            mine[0] = best; mine[1] = total;
#pragma unroll
            for (int c = 0; c < 4; ++c) mine[2 + c] = x[c];
        }
        __syncthreads();
        if (wave != 0) return;
#pragma unroll
        for (int w = 1; w < WAVES; ++w) {
            const float* theirs = lds[w][piece];
            const float y[4] = {theirs[2], theirs[3], theirs[4], theirs[5]};
            join(theirs[0], theirs[1], y);
        }
    }
    if (lane < LANES) finish<4>(a, token, head, D, 4 * piece, x, best, total);
}

// units of the longest context that there can be (a window is cut to whole blocks of 16 at its begin, and rows have windows up to
// q_len - 1 tokens apart)
int64_t longest_units(int32_t q_len, int32_t max_len, int32_t window) {
    const int64_t range = window > 0 && window + (int64_t)q_len + 15 < max_len ? window + (int64_t)q_len + 15 : max_len;
    return range > PA_UNIT ? (range + PA_UNIT - 1) / PA_UNIT : 1;
}
// workgroups that the chip holds at once, `rows` query rows to a kv head
int resident(int32_t head_dim, int64_t rows) { return head_dim == 128 && rows > 8 ? 512 : 768; }

template <int D, int WAVES>
void launch_waves(const PagedAttentionArgs& a, unsigned blocks, hipStream_t s) {
    const bool fold = a.group * a.q_len <= 8;
    auto kernel = a.softcap > 0.0f ? fold ? paged_attention_kernel<D, WAVES, true, true> : paged_attention_kernel<D, WAVES, true, false>
                                   : fold ? paged_attention_kernel<D, WAVES, false, true> : paged_attention_kernel<D, WAVES, false, false>;
    hipLaunchKernelGGL(kernel, dim3(blocks), dim3(WAVES * 64), 0, s, a);
}

template <int D>
int launch(const PagedAttentionArgs& a, hipStream_t s) {
    const int64_t segments = (int64_t)a.B * a.kv_heads * a.row_tiles;
    // Where segments go whole, each has a workgroup of its own, and the next free compute unit takes the next one; but where all are
    // short, starting is most of it, and a workgroup prepares its next segment beside the one that it works on.
    const bool brief = a.workers == 0 && longest_units(a.q_len, a.max_len, a.window) <= PA_BRIEF;
    const unsigned blocks = (unsigned)(a.workers > 0 ? a.workers : brief && segments > resident(D, a.group * a.q_len) ? resident(D, a.group * a.q_len) : segments < (1 << 20) ? segments : 1 << 20);
    if (a.waves == 8) launch_waves<D, 8>(a, blocks, s);
    else launch_waves<D, 4>(a, blocks, s);
    const int rc = check_hip(hipGetLastError(), "paged_attention launch");
    if (rc != BASQ_OK || a.workers == 0) return rc;
    // many rows have few parts each: a wavefront does
    const int64_t rows = (int64_t)a.B * a.q_len * a.heads;
    if (rows >= 512) hipLaunchKernelGGL((paged_attention_join_kernel<D, 1>), dim3((unsigned)((rows + 3) / 4)), dim3(256), 0, s, a);
    else hipLaunchKernelGGL((paged_attention_join_kernel<D, 8>), dim3((unsigned)rows), dim3(512), 0, s, a);
    return check_hip(hipGetLastError(), "paged_attention join launch");
}

}  // namespace

// Who takes the work: that many workgroups in equal shares, or (workers = 0) one to a segment, of four waves or, while there are no
// more than compute units, of eight.  workers = -1 where there are too many units to be numbered.
//
// By microseconds behind the start.  A step takes a wave 0.73 while the compute unit has four of them, 0.88 of eight, and 0.47 for each
// four that it has, where they are more; eight waves' sums are joined 0.6 later than four's; the second launch and the parts' ends are 6.  A
// context that is longer than the others keeps its workgroup alone, where shares do not mind: they are taken to have 55 % of the longest's
// work.  Measured, contexts of one length, 128-channel heads, four waves, eight waves, shares: 32 segments of 256, 512, 1024, 2048 tokens
// 6.2, 7.7, 10.6, 16.2 us; 6.7, 7.3, 9.2, 12.6; -, 10.2, 10.5, 11.4.  256 segments of 512, 1024, 2048 tokens 8.3, 11.1, 16.8; 7.9, 9.8, 15.2;
// 13.4, 15.8, 20.3.
AttentionPlan paged_attention_plan(int32_t B, int32_t q_len, int32_t heads, int32_t kv_heads, int32_t head_dim, int32_t max_len, int32_t window, bool cap) {
    const int64_t segments = (int64_t)B * kv_heads * (((int64_t)(heads / kv_heads) * q_len + 15) / 16);
    const int64_t units = longest_units(q_len, max_len, window);
    if ((int64_t)B * q_len * heads > 0x7FFFFFFFll || segments * (units + PA_START) > 0x7FFF0000ll) return {-1, 4};
    const int64_t most = resident(head_dim, heads / kv_heads * (int64_t)q_len);
    constexpr double CUS = 256, ALONE = 0.73, ALONE_EIGHT = 0.88, EACH = 0.47, END_EIGHT = 0.6, JOIN = 6.0, FILLED = 0.55;
    const double tanhs = cap ? 0.22 : 0.0;                       // of a step's scores
    auto step_us = [&](double fours, double alone) {             // fours: sets of four waves that the chip has
        const double company = (fours < (double)most ? fours : (double)most) / CUS * EACH;
        return company > alone + tanhs ? company : alone + tanhs;
    };
    const double rounds = segments > most ? (double)segments / (double)most : 1.0;
    const int64_t share = (segments * (units + PA_START) + most - 1) / most;
    const double four = (double)units * step_us((double)segments, ALONE) * rounds;
    const double eight = segments <= (int64_t)CUS ? END_EIGHT + (double)((units + 1) / 2) * step_us(2.0 * (double)segments, ALONE_EIGHT) : 2.0 * four;
    const double shared = JOIN + FILLED * (double)share * step_us((double)(segments * units), ALONE);
    // Many segments keep the chip full by themselves, the next one going to the first free place: from two rounds on, and where two to a
    // compute unit are not long (ragged contexts, whole segments and shares: 2048 segments up to 3000 tokens 85 and 95 us, up to 1000 32 and
    // 37; 800 up to 2000 26 and 30, up to 8000 88 and 81; 512 up to 4000 32 and 36, up to 8192 67 and 63).  Not where contexts can be very
    // long: one among short ones then keeps its workgroup alone, which the host cannot know (1536 segments, of which those of one sequence are
    // longest: 4096 tokens 30 and 38 us, 8192 50 and 38, 16384 89 and 39, 131072 648 and 63; all ragged up to 8192 172 and 173, up to 16384 318
    // and 308).
    const bool plenty = (segments >= 2 * most && units <= 64) || (segments >= 2 * (int64_t)CUS && units <= 32);
    if (units > PA_BRIEF && !plenty && shared < four && shared < eight) return {(int)(segments * units < most ? segments * units : most), 4};
    return {0, eight < four ? 8 : 4};
}

// The most workers of a call of this shape or of a smaller one (which may share where this one does not): each takes a unit at least, and the
// chip holds 768 where all have few rows.  -1 as above.
int paged_attention_most_workers(int32_t B, int32_t q_len, int32_t heads, int32_t kv_heads, int32_t head_dim, int32_t max_len, int32_t window) {
    if (paged_attention_plan(B, q_len, heads, kv_heads, head_dim, max_len, window, false).workers < 0) return -1;
    const int64_t segments = (int64_t)B * kv_heads * (((int64_t)(heads / kv_heads) * q_len + 15) / 16);
    const int64_t units = longest_units(q_len, max_len, window);
    if (units <= PA_BRIEF) return 0;
    const int64_t most = resident(head_dim, 1);
    return (int)(segments * units < most ? segments * units : most);
}

int launch_paged_attention(PagedAttentionArgs a, hipStream_t s) {
    if (a.B == 0) return BASQ_OK;
    a.group = a.heads / a.kv_heads;
    a.row_tiles = (a.group * a.q_len + 15) / 16;
    a.cap_log2e = a.softcap * LOG2E;
    a.inv_cap = a.softcap > 0.0f ? fminf(1.0f / a.cap_log2e, 0x1p127f) : 0.0f;
    return a.D == 64 ? launch<64>(a, s) : launch<128>(a, s);
}

}  // namespace basq
