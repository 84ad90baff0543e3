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
// One pass over the weights, which bound it where they are large (16 x 8192 x 128000, 565 MB: 117 us, 4.8 TB/s, vector instructions half of the time);
// smaller calls are bound by the waits of a step, of which each wave has few (1 x 4096 x 4096 4.2 us, 13 x 14336 x 4096 16.4, 48 x 4096 x
// 11008 17.0; their bytes 1.3, 4.9 and 4.3).  Each lane requests its batch of 16-byte pieces before it takes any up.  A workgroup
// owns TILES tiles of 16 weight rows, its waves share K in chunks of 128 channels; D = x (rows) times weights (columns), so a
// lane's results belong to one weight row and take one scale.
//
// A 16-byte piece is 32 channels of one row, and an instruction takes the 8 channels of one dword from each of a row's four pieces
// of a chunk: where groups are whole chunks, any split of the chunk over the four instructions will do.  Where groups are smaller
// (32 or 64 channels, say) the dwords are transposed over the wave's rows first (four swaps), and each instruction takes one piece.
#pragma once

#include "basq_internal.h"

namespace basq {

namespace {

typedef float v4f __attribute__((ext_vector_type(4)));
typedef unsigned v4u __attribute__((ext_vector_type(4)));
typedef __bf16 v8b __attribute__((ext_vector_type(8)));

constexpr int TILE = 16;

// 8 codes -> 16 + code in bf16: pairs (0,4) (1,5) (2,6) (3,7) of the dword's channels.  (The constants come in registers, of either kind,
// as only then they go into one and-or.)
__device__ __forceinline__ v8b widen(unsigned v, unsigned mask, unsigned base) {
    const v4u r = {(v << 3 & mask) | base, (v >> 1 & mask) | base, (v >> 5 & mask) | base, (v >> 9 & mask) | base};
    return __builtin_bit_cast(v8b, r);
}
// 8 channels of a token in the same order
__device__ __forceinline__ v4u in_pairs(v4u d) {
    return v4u{__builtin_amdgcn_perm(d.z, d.x, 0x05040100u), __builtin_amdgcn_perm(d.z, d.x, 0x07060302u),
                   __builtin_amdgcn_perm(d.w, d.y, 0x05040100u), __builtin_amdgcn_perm(d.w, d.y, 0x07060302u)};
}
// dword i of row j of the wave <-> dword j of row i
__device__ __forceinline__ v4u transposed(v4u r) {
    const auto a = __builtin_amdgcn_permlane32_swap(r.x, r.z, false, false);
    const auto b = __builtin_amdgcn_permlane32_swap(r.y, r.w, false, false);
    const auto c = __builtin_amdgcn_permlane16_swap(a[0], b[0], false, false);
    const auto d = __builtin_amdgcn_permlane16_swap(a[1], b[1], false, false);
    return v4u{c[0], c[1], d[0], d[1]};
}

// NW: waves that take different tiles and share the tokens' channels.   KW: groups of them that share K.   STEPS: chunks of a step.
// XSTEPS: chunks of which the tokens are in LDS at once.   TILES: weight tiles of a wave.   TT: tiles of 16 tokens, of which ROWS are
// there (all, but of one tile).   UNIT: channels that certainly share a group: 128, 64 or 32.   SIDE: scales of a step's chunks lie
// side by side, all of them there.
//
// Tokens go through LDS: read row by row, a row's 256 bytes of a chunk by 16 lanes, and put down in the order of the operands, in places
// that 16 rows reach without conflicts.  (Read as operands straight from memory, 16 bytes of 16 rows at a time, they cost more than the
// weights: 16 x 8192 x 128000 162 us, through LDS 129 at the time.)  A step's weights, scales and tokens are under way while the step before
// is multiplied: tokens first, which have to be in LDS first, as waits count loads in their order, and requested past the end too, where
// they come back as 0 at once, as a branch around them would make the wait behind it one for all of them (16 x 4096 x 32000 20.0 us with
// the branches, 18.3 without).
template <bool STREAM_LAYOUT, int NW, int KW, int STEPS, int XSTEPS, int TILES, int TT, int ROWS, int UNIT, bool SIDE>
__global__ __launch_bounds__(NW * KW * 64, 2) void gemm_w4a16_kernel(W4A16Args a) {
    constexpr int UNITS = 128 / UNIT;                                          // of a chunk
    constexpr int NT = TILES * TT, WG_TILES = NW * TILES;
    constexpr int BUFS = NW > 1 ? 2 : 1;                                       // (a wave by itself reads before it writes again)
    constexpr int CHUNK = (TT - 1) * 256 + ROWS * 16;                          // of 16-byte pieces: rows of 16
    constexpr int XS = BUFS * KW * XSTEPS * CHUNK, PART = KW * NW * NT * 64;
    constexpr int FOURS = CHUNK / 64;                                          // a load of a wave is 4 rows of a chunk
    constexpr int LOADS = (XSTEPS * FOURS + NW - 1) / NW;                       // pieces of tokens that a lane fetches for a step
    constexpr bool BLOCKS = SIDE && NW > 1 && KW == 1 && XSTEPS == STEPS;                 // scales by way of LDS
    static_assert(!BLOCKS || (STEPS == 4 && TILES == 1), "");
    __shared__ v4u lds[XS > PART ? XS : PART], scales[BLOCKS ? NW * KW * 64 : 1];

    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int nw = wave % NW, kw = wave / NW;
    const int row = lane & 15, sub = lane >> 4;
    const int n0 = (blockIdx.x * WG_TILES + nw * TILES) * TILE, m0 = blockIdx.y * (TILE * TT);
    const int KB = a.K / 2, chunks = (a.K + 127) / 128;
    const int M = (int)(a.M - m0 < TILE * TT ? a.M - m0 : TILE * TT);
    const int groups = a.groups;

    // Weights and tokens are read by descriptors, which give 0 past their ends: behind the last row, and where there is no tile.  What lies
    // past the last chunk, or past K in it, meets tokens of 0.
    constexpr int BEYOND = (int)0x80000000;                                    // an offset past any end
    constexpr int WSTEP = STREAM_LAYOUT ? 1024 : 64;
    const int rows_left = a.N - n0 < 0 ? 0 : a.N - n0 < TILE * TILES ? a.N - n0 : TILE * TILES;
    const __amdgpu_buffer_rsrc_t rsrc_w = __builtin_amdgcn_make_buffer_rsrc(const_cast<uint8_t*>(a.Wq) + (int64_t)n0 * KB, 0,
                                                                            (STREAM_LAYOUT ? (rows_left + TILE - 1) / TILE * TILE : rows_left) * KB, 0x00020000);
    const __amdgpu_buffer_rsrc_t rsrc_x = __builtin_amdgcn_make_buffer_rsrc(const_cast<uint16_t*>(a.X) + m0 * a.ldx, 0, (int)(((M - 1) * a.ldx + a.K) * 2), 0x00020000);
    const int w_lane = STREAM_LAYOUT ? lane * 16 : row * KB + sub * 16;
    const int x_row = (int)a.ldx * 2, x_lane = sub * x_row + row * 16;         // load at % FOURS of a chunk: 4 rows from 4 (at % FOURS) on
    // the scales of a lane's row in each tile (rows past the last: the last again, not stored)
    const uint16_t *s_base[TILES], *z_base[TILES];
    unsigned s_lane[TILES];
#pragma unroll
    for (int t = 0; t < TILES; ++t) {
        const int nt0 = n0 + TILE * t < a.N ? n0 + TILE * t : a.N - 1, n = nt0 + row < a.N ? nt0 + row : a.N - 1;
        s_base[t] = a.w_scale + (int64_t)nt0 * groups;
        z_base[t] = a.w_zero + (int64_t)nt0 * groups;
        s_lane[t] = (unsigned)(n - nt0) * (unsigned)groups;
    }

    unsigned mask = 0x00780078u, base = 0x41804180u;
    asm("" : "+s"(mask));
    asm("" : "+v"(base));
    const v4f zero = {0.f, 0.f, 0.f, 0.f};
    const v4u ones_bits = {0x3F803F80u, 0x3F803F80u, 0x3F803F80u, 0x3F803F80u};
    const v8b ones = __builtin_bit_cast(v8b, ones_bits);
    v4f acc[NT];
#pragma unroll
    for (int i = 0; i < NT; ++i) acc[i] = zero;

    constexpr int PAIRS = (STEPS * UNITS + 1) / 2;
    struct Batch {
        v4u w[TILES][STEPS];
        unsigned sw[TILES][PAIRS], zp[TILES][PAIRS];                           // two in each
    };
    // Scales in blocks of 16 groups, a lane with half of a row's scales or zero points: of 4 groups at a time, 8 bytes of 16 lines, the lines
    // came from L2 again for every step, as many bytes as the weights.  (Halves that reach past a row's end end there; 8 groups at least.)
    v4u block = {0, 0, 0, 0};
    int block_at = -1;
    auto first_of = [&](int c0) { return (c0 < chunks ? c0 : chunks - STEPS) * UNITS; };        // (past the last: the last, with tokens of 0)
    auto block_of = [&](int c0) { return first_of(c0) & ~15; };
    auto fetch = [&](Batch& to, int c0) {
#pragma unroll
        for (int i = 0; i < STEPS; ++i)
#pragma unroll
            for (int t = 0; t < TILES; ++t)
                to.w[t][i] = __builtin_bit_cast(v4u, __builtin_amdgcn_raw_buffer_load_b128(rsrc_w, w_lane + (c0 + i < chunks ? t * TILE * KB + (c0 + i) * WSTEP : BEYOND), 0, 2 /* once */));
        if constexpr (BLOCKS) {
            // (with the tokens)
        } else if constexpr (SIDE) {
            const int c = c0 < chunks ? c0 : 0;
#pragma unroll
            for (int t = 0; t < TILES; ++t) {
                __builtin_memcpy(to.sw[t], s_base[t] + c * UNITS + s_lane[t], 2 * STEPS * UNITS);
                __builtin_memcpy(to.zp[t], z_base[t] + c * UNITS + s_lane[t], 2 * STEPS * UNITS);
            }
        } else {
            auto group = [&](int u) {
                const unsigned unit = (unsigned)(UNITS * c0 + u);
                const unsigned g = a.per_group ? __umulhi(unit, a.per_group) : unit;
                return g < (unsigned)groups ? g : groups - 1u;
            };
#pragma unroll
            for (int u = 0; u < STEPS * UNITS; u += 2) {
                const unsigned g0 = group(u), g1 = group(u + 1);
#pragma unroll
                for (int t = 0; t < TILES; ++t) {
                    to.sw[t][u / 2] = s_base[t][g0 + s_lane[t]] | (unsigned)s_base[t][g1 + s_lane[t]] << 16;
                    to.zp[t][u / 2] = z_base[t][g0 + s_lane[t]] | (unsigned)z_base[t][g1 + s_lane[t]] << 16;
                }
            }
        }
    };
    v4u x_next[LOADS];
    auto fetch_tokens = [&](int c0) {
        if constexpr (BLOCKS) {
            const int from = block_of(c0);
            if (from != block_at) {
                block_at = from;
                const int half = sub & 1, start = from + 8 * half < groups - 8 ? from + 8 * half : groups - 8;
                __builtin_memcpy(&block, (sub & 2 ? z_base[0] : s_base[0]) + start + s_lane[0], 16);
            }
        }
#pragma unroll
        for (int i = 0; i < LOADS; ++i) {
            const int at = (i * NW + nw) % (XSTEPS * FOURS), c = c0 + at / FOURS;               // (past the last: the first again)
            int from = x_lane + (at % FOURS * 4 * x_row + c * 256);
            if (c >= chunks || (!STREAM_LAYOUT && 128 * c + 8 * row >= a.K)) from = BEYOND;
            x_next[i] = __builtin_bit_cast(v4u, __builtin_amdgcn_raw_buffer_load_b128(rsrc_x, from, 0, 0));
        }
        __builtin_amdgcn_sched_barrier(0);
    };
    auto put_tokens = [&](int buf) {
#pragma unroll
        for (int i = 0; i < LOADS; ++i) {
            const int at = (i * NW + nw) % (XSTEPS * FOURS), r = 4 * (at % FOURS % (ROWS / 4)) + sub;
            lds[(buf * KW + kw) * (XSTEPS * CHUNK) + at / FOURS * CHUNK + at % FOURS * 64 + sub * 16 + (row ^ r)] = in_pairs(x_next[i]);
        }
        if constexpr (BLOCKS) scales[wave * 64 + lane] = block;
        if constexpr (NW > 1) __syncthreads();
        else __builtin_amdgcn_wave_barrier();
    };
    auto number = [](const unsigned (&pairs)[PAIRS], int i) { return __uint_as_float(i & 1 ? pairs[i / 2] & 0xFFFF0000u : pairs[i / 2] << 16); };
    const int own = row & (ROWS - 1);
    auto multiply = [&](Batch& of, int c0, int i0, int buf) {
        if constexpr (BLOCKS) {
            constexpr int SPAN = STEPS * UNITS, PARTS = (SPAN + 7) / 8, EACH = SPAN / PARTS;
            const int first = first_of(c0);
#pragma unroll
            for (int h = 0; h < PARTS; ++h) {
                const int g = first + 8 * h, half = g >> 3 & 1, start = (g & ~7) < groups - 8 ? g & ~7 : groups - 8;
                const uint8_t* from = reinterpret_cast<const uint8_t*>(scales + wave * 64 + half * 16 + row) + (g - start) * 2;
                __builtin_memcpy(of.sw[0] + h * (EACH / 2), __builtin_assume_aligned(from, 8), EACH * 2);
                __builtin_memcpy(of.zp[0] + h * (EACH / 2), __builtin_assume_aligned(from + 512, 8), EACH * 2);
            }
        }
        const v4u* xs = lds + (buf * KW + kw) * (XSTEPS * CHUNK);
#pragma unroll
        for (int j = 0; j < XSTEPS; ++j) {
            const int i = i0 + j;
            v4u d[TILES];
#pragma unroll
            for (int t = 0; t < TILES; ++t) d[t] = UNIT == 128 ? of.w[t][i] : transposed(of.w[t][i]);
#pragma unroll
            for (int u = 0; u < UNITS; ++u) {
                constexpr int PARTS = 4 / UNITS;                               // instructions of a unit
                v8b x[TT][PARTS];
                v4f sums[TT];
#pragma unroll
                for (int tt = 0; tt < TT; ++tt) {
                    sums[tt] = zero;
#pragma unroll
                    for (int q = 0; q < PARTS; ++q) {
                        const int p = u * PARTS + q;
                        x[tt][q] = __builtin_bit_cast(v8b, xs[j * CHUNK + tt * 256 + own * 16 + ((UNIT == 128 ? 4 * sub + p : 4 * p + sub) ^ own)]);
                        sums[tt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(x[tt][q], ones, sums[tt], 0, 0, 0);
                    }
                }
#pragma unroll
                for (int t = 0; t < TILES; ++t) {
                    v4f r[TT];
#pragma unroll
                    for (int tt = 0; tt < TT; ++tt) r[tt] = zero;
#pragma unroll
                    for (int q = 0; q < PARTS; ++q) {
                        unsigned word = d[t][u * PARTS + q];
                        if constexpr (TT > 1) asm volatile("" : "+v"(word));
                        const v8b codes = widen(word, mask, base);
#pragma unroll
                        for (int tt = 0; tt < TT; ++tt) r[tt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(x[tt][q], codes, r[tt], 0, 0, 0);
                    }
                    const float s = number(of.sw[t], i * UNITS + u), z = 16.0f + number(of.zp[t], i * UNITS + u);
#pragma unroll
                    for (int tt = 0; tt < TT; ++tt)
#pragma unroll
                        for (int e = 0; e < 4; ++e) acc[t * TT + tt][e] = fmaf(s, fmaf(-z, sums[tt][e], r[tt][e]), acc[t * TT + tt][e]);
                }
                // (Units one after the other: the compiler would widen a batch's codes when they arrive, and take up products at the end of
                // all, and has no registers for either.)
                if constexpr (TT > 1) {
#pragma unroll
                    for (int i = 0; i < NT; ++i) asm volatile("" : "+v"(acc[i]));
                    __builtin_amdgcn_sched_barrier(0);
                }
            }
        }
    };
    // (every wave goes through as many steps: they meet at barriers)
    constexpr int NEXT = KW * STEPS;
    const int steps = (chunks + NEXT - 1) / NEXT;
    int c = kw * STEPS;
    Batch one;
    fetch_tokens(c);
    fetch(one, c);
    if constexpr (XSTEPS == STEPS) {
        Batch two;
        for (int s = 0; s < steps; s += 2) {
            put_tokens(0);
            fetch_tokens(c + NEXT);
            fetch(two, c + NEXT);
            multiply(one, c, 0, 0);
            asm volatile("" ::: "memory");                                     // (or the loads would move behind the branch)
            if (s + 1 >= steps) break;
            put_tokens(BUFS - 1);
            fetch_tokens(c + 2 * NEXT);
            fetch(one, c + 2 * NEXT);
            multiply(two, c + NEXT, 0, BUFS - 1);
            c += 2 * NEXT;
        }
    } else {
        // many tokens: registers for one batch of weights; it is long, and the tokens follow from the next cache
        for (int s = 0; s < steps; ++s) {
#pragma unroll
            for (int i = 0; i < STEPS; i += XSTEPS) {
                const int buf = i / XSTEPS & (BUFS - 1);
                put_tokens(buf);
                if (i + XSTEPS < STEPS) fetch_tokens(c + i + XSTEPS);
                multiply(one, c, i, buf);
            }
            c += NEXT;
            if (s + 1 < steps) { fetch(one, c); fetch_tokens(c); }
        }
    }
    // the sums of the waves that share K meet in a fixed order; element e of lane l is token 4 (l/16) + e, row l % 16 of its tiles
    v4f* part = reinterpret_cast<v4f*>(lds);
    __syncthreads();
#pragma unroll
    for (int i = 0; i < NT; ++i) part[((kw * NW + nw) * NT + i) * 64 + lane] = acc[i];
    __syncthreads();
    for (int i = wave; i < NW * NT; i += NW * KW) {
        const int t = i / TT, tt = i % TT, n = (blockIdx.x * WG_TILES + t) * TILE + row;
        v4f v = part[i * 64 + lane];
#pragma unroll
        for (int w = 1; w < KW; ++w) v += part[(w * NW * NT + i) * 64 + lane];
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

template <bool SL, int NW, int KW, int STEPS, int XSTEPS, int TILES, int TT, int ROWS, int UNIT, bool SIDE>
void launch_shape(const W4A16Args& a, hipStream_t s) {
    const unsigned x = (unsigned)((a.N + TILE * NW * TILES - 1) / (TILE * NW * TILES)), y = (unsigned)((a.M + TILE * TT - 1) / (TILE * TT));
    hipLaunchKernelGGL((gemm_w4a16_kernel<SL, NW, KW, STEPS, XSTEPS, TILES, TT, ROWS, UNIT, SIDE>), dim3(x, y), dim3(NW * KW * 64), 0, s, a);
}

// Up to 768 tiles a compute unit gets one workgroup, whose eight waves share K, on one to three of them; more tiles go to workgroups of
// four waves with a tile each, so that four share the tokens, twice as many to share K unless that fills the chip anyway (us;
// 1 x 8 is one wave's tiles and eight waves of K): 16 x 4096 x 4096 in groups of 128 1 x 8 6.7, 4 x 2 8.8, 4 x 1 10.3; x 12288 on three
// tiles 10.2, 4 x 2 9.6, 4 x 1 10.7; x 32000 1 x 8 26.1, 4 x 2 17.1 to 18.5, 4 x 1 16.6; x 128000 89, 64 and 57.  More tokens stay
// with 4 x 2 longer: 60 x 4096 x 32000 in groups of 128 42.3, 4 x 1 55.8; x 64000 81.4 and 69.0; x 128000 158 and 134 (in groups of 32 50.0 and
// 65.0, 96.1 and 85.8, 186 and 167); 20 x 4096 x 64000 51.4 and 46.7, x 128000 98.4 and 91.3.  33 to 48 tokens always do, which costs
// them: 40 x 4096 x 128000 176, 4 x 1 130 (in groups of 32 148 and 143).
//
// Scales that lie side by side (groups of 32, 64 or 128) are read a step at a time, so shapes with steps of four or two chunks take K of as
// many: x 32000 in groups of 128, 16 tokens, K = 4096 (32 chunks) 17.1, 2816 and 2304 (22 and 18) 22.5 and 21.6, 1024 6.4, 1152 and 896 (9
// and 7) 16.1 and 12.9.  K that ends inside a chunk has one shape in groups of 32 or 64: 16 x 2880 x 32000 74.2 and 50.7, where 2048
// takes 14.7 and 12.1.
constexpr int FEW_TILES = 768, MANY_TILES = 1500, MANY_TILES_OF_MORE = 6000;
int tiles_of(const W4A16Args& a) { return (a.N + TILE - 1) / TILE; }

// up to 16 tokens.  Steps of as many chunks as each wave has work for: K = 1024 3.3 us with one, 4.1 with two; K = 4096 6.3 with four, 7.1
// with two; but K = 14336 18.4 with four, 16.4 with two.
template <bool SL, int UNIT, bool SIDE, int ROWS>
void launch_16(const W4A16Args& a, hipStream_t s) {
    const int tiles = tiles_of(a), chunks = (a.K + 127) / 128;
    const bool fours = !SIDE || chunks % 4 == 0;                               // (scales side by side need whole steps)
    const bool blocks = fours && (!SIDE || a.groups >= 8);
    if (tiles > MANY_TILES && blocks) launch_shape<SL, 4, 1, 4, 4, 1, 1, ROWS, UNIT, SIDE>(a, s);
    else if (tiles > FEW_TILES && fours) launch_shape<SL, 4, 2, 4, 4, 1, 1, ROWS, UNIT, SIDE>(a, s);
    else if (chunks < 16 || (SIDE && chunks % 2 != 0)) launch_shape<SL, 1, 8, 1, 1, 1, 1, ROWS, UNIT, SIDE>(a, s);
    else if (ROWS < 16 || tiles <= 256) {
        if (chunks >= 32 && chunks <= 64 && fours) launch_shape<SL, 1, 8, 4, 4, 1, 1, ROWS, UNIT, SIDE>(a, s);
        else launch_shape<SL, 1, 8, 2, 2, 1, 1, ROWS, UNIT, SIDE>(a, s);
    } else if constexpr (ROWS == 16) {
        if (tiles <= 512) launch_shape<SL, 1, 8, 2, 2, 2, 1, ROWS, UNIT, SIDE>(a, s);
        else launch_shape<SL, 1, 8, 2, 2, 3, 1, ROWS, UNIT, SIDE>(a, s);
    }
}
// Up to 32, 48 or 64 tokens: their operands and sums take the registers of a second batch of weights, so a batch is long instead and the
// tokens go through LDS chunk by chunk (48 x 4096 x 11008 in groups of 32 18.6 us then, in batches of one chunk 21.6; 64 x 4096 x 32000
// on two tiles a wave 43.4, on one 51).
template <bool SL, int UNIT, bool SIDE, int TT>
void launch_64(const W4A16Args& a, hipStream_t s) {
    const int tiles = tiles_of(a), chunks = (a.K + 127) / 128;
    constexpr int T = TT == 4 ? 2 : 1;
    if (SIDE && chunks % 2 != 0) launch_shape<SL, 1, 8, 1, 1, 1, TT, 16, UNIT, SIDE>(a, s);
    else if (tiles > MANY_TILES_OF_MORE && TT != 3) launch_shape<SL, 4, 1, 2, 1, T, TT, 16, UNIT, SIDE>(a, s);
    else if (tiles > FEW_TILES) launch_shape<SL, 4, 2, 2, 1, T, TT, 16, UNIT, SIDE>(a, s);
    else if (tiles <= 256) launch_shape<SL, 1, 8, 2, 1, 1, TT, 16, UNIT, SIDE>(a, s);
    else if (tiles <= 512) launch_shape<SL, 1, 8, 2, 1, 2, TT, 16, UNIT, SIDE>(a, s);
    else if constexpr (TT == 4) launch_shape<SL, 2, 4, 2, 1, 2, TT, 16, UNIT, SIDE>(a, s);
    else launch_shape<SL, 1, 8, 2, 1, 3, TT, 16, UNIT, SIDE>(a, s);
}

// Groups that are not 32, 64 or 128 channels: scales one by one.  (Of 32 or 64 channels that share a group for certain, odd sizes: one shape.)
template <bool SL, int UNIT>
void launch_few(const W4A16Args& a, hipStream_t s) {
    if (a.group == UNIT && a.K % 128 == 0) {
        if (a.M <= 4) launch_16<SL, UNIT, true, 4>(a, s); else launch_16<SL, UNIT, true, 16>(a, s);
    } else if constexpr (UNIT == 128) {
        if (a.M <= 4) launch_16<SL, UNIT, false, 4>(a, s); else launch_16<SL, UNIT, false, 16>(a, s);
    } else {
        launch_shape<SL, 1, 8, 2, 2, 1, 1, 16, UNIT, false>(a, s);
    }
}
template <bool SL, int UNIT, bool SIDE>
void launch_tokens(const W4A16Args& a, hipStream_t s) {
    if (a.M <= 32) launch_64<SL, UNIT, SIDE, 2>(a, s);
    else if (a.M <= 48) launch_64<SL, UNIT, SIDE, 3>(a, s);
    else launch_64<SL, UNIT, SIDE, 4>(a, s);
}
template <bool SL, int UNIT>
void launch_many(const W4A16Args& a, hipStream_t s) {
    if (a.group == UNIT && a.K % 128 == 0) launch_tokens<SL, UNIT, true>(a, s);
    else if constexpr (UNIT == 128) launch_tokens<SL, UNIT, false>(a, s);
    else launch_shape<SL, 1, 8, 2, 1, 1, 4, 16, UNIT, false>(a, s);
}

}  // namespace
}  // namespace basq
