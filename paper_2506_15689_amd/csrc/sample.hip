// A token for each row of logits, with temperature, top-k, top-p and min-p, from given random numbers; the definition is beside
// basq_sample in basq.h.
//
// The tokens' order is that of their logits, so nothing is sorted but what lies next to a cut: a cut, and the draw itself, is the
// first place of that order at which a running count or a running mass reaches a target.  Three ways lead to such places, by what the
// row is like (all see the same masses, the second to 2^-36 and its cells' roundings):
//     bf16                       how often each of the 65536 numbers occurs, one workgroup and launch a row
//     fp32                       cells of a grid, then the few tokens in the cells of the cuts; rows of up to 32768 in one launch, longer ones in two
//     long rows, and those that  digits of the logits' bits, with a histogram of counts and masses over one digit at a time: any
//     defeat the other two       row, at some ten passes over it
// Equal logits share a place; which of them it is follows from arithmetic, and only the drawn one's index is looked for.
//
// Bound by latency: a row is read in full once or twice (256 rows of 128000 bf16 logits, 65.5 MB, would take 9.5 us at the rate of a
// large read), but one row is a chain of some ten steps that a workgroup's waves wait for together: scan, find, scan, find.  One row of
// 32000 bf16 logits 16 us; 256 rows of 128000 32; 64 rows of 128000 fp32 logits with top-k, top-p and min-p 46.
//
// Masses are whole numbers: a token's weight e^((z - top) / T), computed in fp64, times 2^bits, rounded once.  Sums of them are exact
// in any order, so LDS atomics give the same token every time, equal logits weigh the same, and the running mass at the last place
// is the total.  (bits: 2^bits times the tokens of a row stays below 2^62; 45 for 128000 tokens, whose roundings, half a step each, come to
// about 2^-37 of the mass, and to 2^-29 if all had one sign.  Sums in fp32 would move the draw of one row in forty to a neighbour, by
// their 2^-23.)
#include "basq_internal.h"
#include "lane_ops.h"

#include <type_traits>

namespace basq {

namespace {

constexpr int THREADS = 1024, WAVES = THREADS / 64;
constexpr unsigned LOWEST = 0x007FFFFFu;                 // the key of -inf

// a logit's bits as a number whose order is that of the logits; NaN is -inf, -0 is 0
__device__ __forceinline__ unsigned key_of(float z) {
    z = z != z ? -__builtin_inff() : z + 0.0f;
    const unsigned u = __float_as_uint(z);
    return u ^ ((unsigned)((int)u >> 31) | 0x80000000u);
}
__device__ __forceinline__ float logit_of(unsigned key) {
    return __uint_as_float(key & 0x80000000u ? key ^ 0x80000000u : ~key);
}

// The weights of a row: e^((z - top) / T) = 2^(n + r), n whole and |r| <= 1/2.
struct Weights {
    float top;
    double per;                                           // log2(e) / T
    int bits;
    // 2^(lift + n + r); 2^r by its series, ln(2)^k / k!, the first term left out under 2^-47.  (lift: from 0 to 51)
    __device__ __forceinline__ double scaled(float z, int lift) const {
        constexpr double magic = 6755399441055744.0;      // 1.5 * 2^52: adding it rounds to whole numbers, which are the low bits
        double y = ((double)z - (double)top) * per;
        y = z == top ? 0.0 : fmax(y, -1000.0);            // (-inf and NaN, of infinities, become -1000: less than any step)
        const double t = y + magic, r = y - (t - magic);
        double s = 4.44553827187081e-10;
        s = fma(s, r, 7.054911620801121e-09);
        s = fma(s, r, 1.0178086009239696e-07);
        s = fma(s, r, 1.3215486790144305e-06);
        s = fma(s, r, 1.5252733804059838e-05);
        s = fma(s, r, 1.5403530393381606e-04);
        s = fma(s, r, 1.3333558146428441e-03);
        s = fma(s, r, 9.618129107628477e-03);
        s = fma(s, r, 5.5504108664821576e-02);
        s = fma(s, r, 2.402265069591007e-01);
        s = fma(s, r, 6.931471805599453e-01);
        s = fma(s, r, 1.0);
        return __hiloint2double(__double2hiint(s) + (__double2loint(t) + lift) * (1 << 20), __double2loint(s));
    }
    // in steps of 2^-bits: adding 2^52 rounds, and the sum's low 52 bits are the number
    __device__ __forceinline__ uint64_t mass(float z) const { return (uint64_t)__double_as_longlong(scaled(z, bits) + 4503599627370496.0) - 0x4330000000000000ull; }
};

// f(index, logit) for every token of the row, by the workgroup
template <bool F32, class F>
__device__ __forceinline__ void for_each(const void* row, int V, F f) {
    if constexpr (F32) {
        const float* p = static_cast<const float*>(row);
        for (int i = threadIdx.x; i < V; i += THREADS) f(i, p[i]);
    } else {
        const uint16_t* p = static_cast<const uint16_t*>(row);
        for (int i = threadIdx.x; i < V; i += THREADS) f(i, bf16_to_f32(p[i]));
    }
}

// the largest of all lanes, in lane 63
__device__ __forceinline__ unsigned wave_most(unsigned v) {
    auto take = [&](unsigned o) { v = o > v ? o : v; };
    take(moved<0x111>(0u, v)); take(moved<0x112>(0u, v)); take(moved<0x114>(0u, v)); take(moved<0x118>(0u, v));
    take(moved<0x142, 0xA>(0u, v)); take(moved<0x143, 0xC>(0u, v));
    return v;
}
// the value of lane ^ J
template <int J>
__device__ __forceinline__ uint64_t across(uint64_t v) {
    if constexpr (J == 1) return moved<0xB1>(0, v);        // (quad_perm 1 0 3 2)
    else if constexpr (J == 2) return moved<0x4E>(0, v);   // (quad_perm 2 3 0 1)
    else if constexpr (J == 4) return moved<0x114, 0xF, 0xA>(moved<0x104, 0xF, 0x5>(0, v), v);
    else if constexpr (J == 8) return moved<0x128>(0, v);  // (row_ror 8)
    else {
        const bool upper = threadIdx.x & J;
        unsigned w[2] = {(unsigned)v, (unsigned)(v >> 32)};
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const auto p = J == 16 ? __builtin_amdgcn_permlane16_swap(w[i], w[i], false, false) : __builtin_amdgcn_permlane32_swap(w[i], w[i], false, false);
            w[i] = upper ? p[0] : p[1];
        }
        return (uint64_t)w[1] << 32 | w[0];
    }
}
__device__ __forceinline__ uint64_t wave_max(uint64_t v) {
    auto take = [&](uint64_t o) { v = o > v ? o : v; };
    take(across<1>(v)); take(across<2>(v)); take(across<4>(v)); take(across<8>(v)); take(across<16>(v)); take(across<32>(v));
    return v;
}

enum Goal { BY_COUNT, BY_MASS, BY_KEY };
// a place of the order: `nth` of the `equal` tokens with this key, behind `count` tokens of mass `mass`
struct Place {
    unsigned key;
    int count, equal, nth;
    uint64_t mass, each;
    __device__ __forceinline__ int tokens() const { return count + nth; }
    __device__ __forceinline__ uint64_t total() const { return mass + (uint64_t)nth * each; }
};

constexpr int DIGITS = 2048;                              // 11 bits, then 11, then the last 10 (and the one above once more)
struct Histogram {
    int count[DIGITS];
    unsigned long long mass[DIGITS];
};
struct Shared {
    Histogram first, next;
    uint64_t wave_counts[WAVES], wave_masses[WAVES], top;
    int found_digit;
    uint64_t found_count, found_mass;
};

__device__ __forceinline__ int shift_of(int level) { return level == 0 ? 21 : level == 1 ? 10 : 0; }

template <bool F32>
__device__ __forceinline__ void fill(Histogram& h, const void* row, int V, const Weights& w, int level, unsigned prefix) {
    for (int i = threadIdx.x; i < DIGITS; i += THREADS) { h.count[i] = 0; h.mass[i] = 0; }
    __syncthreads();
    const int shift = shift_of(level), above = level == 0 ? 32 : shift_of(level - 1);
    for_each<F32>(row, V, [&](int, float z) {
        const unsigned key = key_of(z);
        if (key <= LOWEST || (above < 32 && key >> above != prefix >> above)) return;
        const unsigned digit = key >> shift & (DIGITS - 1);
        atomicAdd(&h.count[digit], 1);
        atomicAdd(&h.mass[digit], (unsigned long long)w.mass(z));
    });
    __syncthreads();
}

// The digit, counted from the highest, in which the goal is reached; behind[] get what lies in front of it.
__device__ __forceinline__ int descend(Shared& s, const Histogram& h, Goal goal, uint64_t target, int key_digit, uint64_t& count, uint64_t& mass) {
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int hi = DIGITS - 1 - 2 * tid, lo = hi - 1;      // this thread's digits
    const uint64_t c0 = h.count[hi], c1 = h.count[lo], m0 = h.mass[hi], m1 = h.mass[lo];
    const uint64_t c = wave_scan(c0 + c1), m = wave_scan(m0 + m1);
    if (lane == 63) { s.wave_counts[wave] = c; s.wave_masses[wave] = m; }
    if (tid == 0) s.found_digit = -1;
    __syncthreads();
    uint64_t cb = count + c - c0 - c1, mb = mass + m - m0 - m1;
    for (int i = 0; i < wave; ++i) { cb += s.wave_counts[i]; mb += s.wave_masses[i]; }
    auto here = [&](int digit, uint64_t cf, uint64_t mf, uint64_t cd, uint64_t md) {
        const bool hit = goal == BY_KEY ? digit == key_digit : goal == BY_COUNT ? cf < target && target <= cf + cd : mf < target && target <= mf + md;
        if (hit) { s.found_digit = digit; s.found_count = cf; s.found_mass = mf; }
    };
    here(hi, cb, mb, c0, m0);
    here(lo, cb + c0, mb + m0, c1, m1);
    __syncthreads();
    count = s.found_count;
    mass = s.found_mass;
    const int digit = s.found_digit & (DIGITS - 1);        // (one is found: targets are reached)
    __syncthreads();
    return digit;
}

// target: at least 1, and reached.  BY_KEY: all tokens whose key is `key` or higher.
template <bool F32>
__device__ __forceinline__ Place find(Shared& s, const void* row, int V, const Weights& w, Goal goal, uint64_t target, unsigned key = 0) {
    uint64_t count = 0, mass = 0;
    unsigned prefix = 0;
    int digit = 0;
    constexpr int LEVELS = F32 ? 3 : 2;                   // (16 bits end in the second digit)
    for (int level = 0; level < LEVELS; ++level) {
        const int shift = shift_of(level);
        if (level > 0) fill<F32>(s.next, row, V, w, level, prefix);
        digit = descend(s, level == 0 ? s.first : s.next, goal, target, (int)(key >> shift & (DIGITS - 1)), count, mass);
        prefix |= (unsigned)digit << shift;
    }
    Place p;
    p.key = F32 ? prefix : prefix & 0x80000000u ? prefix : prefix | 0x3FFu;
    p.count = (int)count;
    p.mass = mass;
    p.equal = s.next.count[digit];
    p.each = w.mass(logit_of(p.key));
    __syncthreads();
    if (goal == BY_KEY) p.nth = p.equal;
    else if (goal == BY_COUNT) p.nth = (int)(target - count);
    else p.nth = (int)((target - mass + p.each - 1) / p.each);
    return p;
}

// what a request chose
struct Choices {
    float heat, p, least;
    int k;
    __device__ __forceinline__ Choices(const SampleArgs& a, int b) {
        heat = a.temperature ? a.temperature[b] : 1.0f;
        k = a.top_k ? a.top_k[b] : 0;
        p = a.top_p ? a.top_p[b] : 1.0f;
        least = a.min_p ? a.min_p[b] : 0.0f;
    }
    __device__ __forceinline__ bool greedy() const { return !(heat > 0.0f); }
    __device__ __forceinline__ double enough() const { return least < 1.0f ? (double)least : 1.0; }
};
// the running mass that top-p cuts at, of a mass that there is
__device__ __forceinline__ uint64_t cut_target(float p, uint64_t mass) {
    const double t = __builtin_ceil((double)p * (double)mass);
    const uint64_t target = t >= 1.0 ? (uint64_t)t : 1;
    return target < mass ? target : mass;
}
// the running mass that the draw reaches: the first beyond u * mass
__device__ __forceinline__ uint64_t draw_target(double u, uint64_t mass) {
    const double t = u > 0.0 ? u * (double)mass : 0.0;
    const uint64_t target = t < 9.0e18 ? (uint64_t)t + 1 : mass;
    return target < mass ? target : mass;
}
__device__ __forceinline__ void put(const SampleArgs& a, int b, int token, float logprob, int kept) {
    a.token[b] = token;
    if (a.logprob) a.logprob[b] = logprob;
    if (a.kept) a.kept[b] = kept;
}
// ln of a token's share of the kept mass
__device__ __forceinline__ float share(const Weights& w, float heat, float z, uint64_t mass) {
    const double d = z == w.top ? 0.0 : ((double)z - (double)w.top) / (double)heat;
    return (float)(d - log((double)mass * __hiloint2double((1023 - w.bits) << 20, 0)));
}
__device__ __forceinline__ const void* row_of(const SampleArgs& a, int b) {
    return static_cast<const uint8_t*>(a.logits) + (int64_t)b * a.ldl * (a.f32 ? 4 : 2);
}

// A row by digits, whatever its logits are.  best: its likeliest token, (key, ~index).
template <bool F32>
__device__ __forceinline__ void by_digits(const SampleArgs& a, int b, uint64_t best, Shared& s) {
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, V = a.V;
    const void* row = row_of(a, b);
    const Choices c(a, b);
    const unsigned top_key = (unsigned)(best >> 32);
    Weights w;
    w.top = logit_of(top_key);
    w.per = 1.4426950408889634 / (double)c.heat;
    w.bits = a.bits;
    fill<F32>(s.first, row, V, w, 0, 0);
    uint64_t kept = 0, mass = 0;
    {
        uint64_t n = 0, m = 0;
        for (int i = tid; i < DIGITS; i += THREADS) { n += s.first.count[i]; m += s.first.mass[i]; }
        n = wave_scan(n); m = wave_scan(m);
        if (lane == 63) { s.wave_counts[wave] = n; s.wave_masses[wave] = m; }
        __syncthreads();
        for (int i = 0; i < WAVES; ++i) { kept += s.wave_counts[i]; mass += s.wave_masses[i]; }
        __syncthreads();
    }
    if (c.k > 0 && (uint64_t)c.k < kept) {
        const Place at = find<F32>(s, row, V, w, BY_COUNT, (uint64_t)c.k);
        kept = at.tokens();
        mass = at.total();
    }
    if (c.p < 1.0f) {
        const Place at = find<F32>(s, row, V, w, BY_MASS, cut_target(c.p, mass));
        if ((uint64_t)at.tokens() < kept) { kept = at.tokens(); mass = at.total(); }
    }
    if (c.least > 0.0f) {
        // the lowest key whose weight is enough, by bisection: weights rise with keys
        unsigned lo = LOWEST, hi = top_key;                // (hi is enough; lo is not, or is no token)
        while (hi - lo > 1) {
            const unsigned mid = lo + (hi - lo) / 2;
            if (w.scaled(logit_of(mid), 0) >= c.enough()) hi = mid; else lo = mid;
        }
        if (!F32) hi = hi & 0x80000000u ? (hi + 0xFFFFu) & 0xFFFF0000u : hi | 0xFFFFu;          // (the next bf16 number)
        const Place at = find<F32>(s, row, V, w, BY_KEY, 0, hi);
        if ((uint64_t)at.tokens() < kept) { kept = at.tokens(); mass = at.total(); }
    }
    const Place at = find<F32>(s, row, V, w, BY_MASS, draw_target(a.u[b], mass));
    // the nth token with that key: the part of the row that holds it, then the token
    const int part = (V + DIGITS - 1) / DIGITS;
    for (int i = tid; i < DIGITS; i += THREADS) { s.next.count[i] = 0; s.next.mass[i] = 0; }
    __syncthreads();
    for_each<F32>(row, V, [&](int i, float z) { if (key_of(z) == at.key) atomicAdd(&s.next.count[DIGITS - 1 - i / part], 1); });
    __syncthreads();
    uint64_t before = 0, none = 0;
    const int in = DIGITS - 1 - descend(s, s.next, BY_COUNT, (uint64_t)at.nth, 0, before, none);
    if (wave == 0) {
        int seen = (int)before, token = -1;
        for (int i0 = in * part; i0 < (in + 1) * part && token < 0; i0 += 64) {
            const int i = i0 + lane;
            bool mine = false;
            if (i < (in + 1) * part && i < V) {
                const float z = F32 ? static_cast<const float*>(row)[i] : bf16_to_f32(static_cast<const uint16_t*>(row)[i]);
                mine = key_of(z) == at.key;
            }
            const uint64_t who = __ballot(mine);
            const int rank = seen + __popcll(who & ((1ull << lane) - 1)) + 1;
            const uint64_t hit = __ballot(mine && rank == at.nth);
            if (hit) token = i0 + __builtin_ctzll(hit);
            seen += __popcll(who);
        }
        if (lane == 0) put(a, b, token, share(w, c.heat, logit_of(at.key), mass), (int)kept);
    }
}

template <bool F32>
__global__ __launch_bounds__(THREADS) void sample_long_kernel(SampleArgs a) {
    __shared__ Shared s;
    const int b = blockIdx.x, tid = threadIdx.x;
    uint64_t best = 0;
    for_each<F32>(row_of(a, b), a.V, [&](int i, float z) {
        const uint64_t v = (uint64_t)key_of(z) << 32 | (unsigned)~i;
        best = v > best ? v : best;
    });
    if (tid == 0) s.top = 0;
    __syncthreads();
    atomicMax((unsigned long long*)&s.top, (unsigned long long)best);
    __syncthreads();
    best = s.top;
    const bool none = (unsigned)(best >> 32) <= LOWEST;
    if (none || Choices(a, b).greedy()) {
        if (tid == 0) put(a, b, none ? -1 : (int)~(unsigned)best, none ? -__builtin_inff() : 0.0f, none ? 0 : 1);
        return;
    }
    by_digits<F32>(a, b, best, s);
}

// ---- bf16: by the numbers themselves -------------------------------------------------------------------------------------------
//
// There are 65536 of them: a workgroup counts how often each occurs in its row, in LDS, two counters of 16 bits to a word, and needs
// no weight but one for each number that occurs, some thousand of 128000.  Counts and masses of 64 numbers at a time are summed and scanned
// over the workgroup; a place is found among the 1024 sums and then among the 64 numbers of one.  (With cells as for fp32, below, for which
// every token is weighed, 256 rows of 128000 logits took 63 us.)  A counter that overflows, of a number that more than 65535 tokens
// have, shows in the sum of all: such rows go by digits.
//
// The row stays in registers for the last step, the index of the token that is the nth with the number found.

typedef unsigned v4u __attribute__((ext_vector_type(4)));

// a piece of 16 bytes of a row: its logits
template <bool F32>
struct Piece {
    static constexpr int N = F32 ? 4 : 8;
    v4u v;
    __device__ __forceinline__ float operator[](int e) const {
        if constexpr (F32) return __uint_as_float(v[e]);
        else return __uint_as_float(e & 1 ? v[e / 2] & 0xFFFF0000u : v[e / 2] << 16);
    }
};
// A row in aligned pieces, element e of piece p token head + N p + e, and what lies in front of the first and behind the last of them,
// which a thread takes one each of.  Loads of pieces have no branch around them, which would wait for each in turn: pieces past the
// last are the last again, and made -inf where a block reaches past it.
template <bool F32>
struct Pieces {
    static constexpr int N = Piece<F32>::N;
    const void* row;
    const v4u* first;
    int V, head, count;
    __device__ __forceinline__ Pieces(const void* logits, int tokens) : row(logits), V(tokens) {
        head = (int)(-(intptr_t)(uintptr_t)logits & 15) / (F32 ? 4 : 2);
        head = head < V ? head : V;
        count = (V - head) / N;
        first = reinterpret_cast<const v4u*>(static_cast<const uint8_t*>(logits) + head * (F32 ? 4 : 2));
    }
    __device__ __forceinline__ int token(int p, int e) const { return head + N * p + e; }
    // pieces p0 + tid + THREADS r
    __device__ __forceinline__ void load_one(Piece<F32>& held, int p) const { held.v = first[p < count ? p : count - 1]; }
    template <int R>
    __device__ __forceinline__ void load(Piece<F32> (&held)[R], int p0) const {
        constexpr unsigned none = F32 ? 0xFF800000u : 0xFF80FF80u;
        if (p0 < count) {
#pragma unroll
            for (int r = 0; r < R; ++r) {
                const int p = p0 + r * THREADS + (int)threadIdx.x;
                held[r].v = first[p < count ? p : count - 1];
            }
        }
        if (p0 + R * THREADS <= count) return;
#pragma unroll
        for (int r = 0; r < R; ++r)
            if (p0 + r * THREADS + (int)threadIdx.x >= count) held[r].v = v4u{none, none, none, none};
    }
    // this thread's token outside the pieces; -1: none
    __device__ __forceinline__ int edge() const {
        const int tail = V - head - N * count, tid = threadIdx.x;
        return tid < head ? tid : tid < head + tail ? V - tail + tid - head : -1;
    }
    __device__ __forceinline__ float at(int i) const {
        if (i < 0) return -__builtin_inff();
        return F32 ? static_cast<const float*>(row)[i] : bf16_to_f32(static_cast<const uint16_t*>(row)[i]);
    }
};

typedef unsigned short us2 __attribute__((ext_vector_type(2)));

// Numbers from the largest on: +inf is 0; what is no token, -inf and NaN, comes from NONE on.  Two in a word.
constexpr unsigned NONE = 0xFF01u, ZERO = 0x7F80u;         // (ZERO + 1 is -0)
__device__ __forceinline__ us2 numbers_of(unsigned two) {
    const unsigned negative = two >> 15 & 0x00010001u;
    return __builtin_bit_cast(us2, two ^ (0x7FFF7FFFu & ~(negative * 0xFFFFu))) - us2{0x7F, 0x7F};
}
__device__ __forceinline__ float logit_of_number(unsigned n) {
    n += 0x7Fu;
    return __uint_as_float((n < 0x8000u ? n ^ 0x7FFFu : n) << 16);
}

struct Numbers {
    unsigned counters[32768];
    int count[1024];                                       // of 64 numbers and all in front
    uint64_t mass[1024];
    uint64_t wave_counts[WAVES], wave_masses[WAVES];
    int top, last, tokens, zeros, found, before, token;
    int parts[1024];
    __device__ __forceinline__ unsigned occurs(unsigned n) const { return counters[n >> 1] >> (n & 1 ? 16 : 0) & 0xFFFFu; }
};
union NumbersShared {
    Numbers numbers;
    Shared digits;
};

// f(piece, its number) for what a thread holds of a row, or, R = 0, reads again
template <int R, class F, class G>
__device__ __forceinline__ void each_piece(const Pieces<false>& row, Piece<false> (&held)[R ? R : 1], F f, G before) {
    if constexpr (R > 0) {
#pragma unroll
        for (int r = 0; r < R; ++r) {
            before(r);
            Piece<false> piece = held[r];
            asm volatile("" : "+v"(piece.v));              // (one after the other, in the registers of one)
            if (r * THREADS + (int)threadIdx.x < row.count) f(piece, r * THREADS + (int)threadIdx.x);
        }
    } else {
        Piece<false> some[4];
        for (int p0 = 0; p0 < row.count; p0 += 4 * THREADS) {
            row.load(some, p0);
#pragma unroll
            for (int r = 0; r < 4; ++r)
                if (p0 + r * THREADS + (int)threadIdx.x < row.count) f(some[r], p0 + r * THREADS + (int)threadIdx.x);
        }
    }
}

template <int R>
__global__ __launch_bounds__(THREADS) void sample_numbers_kernel(SampleArgs a) {
    __shared__ NumbersShared shared;
    Numbers& s = shared.numbers;
    const int b = blockIdx.x, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const Pieces<false> row(row_of(a, b), a.V);
    const Choices c(a, b);
#pragma unroll
    for (int i = 0; i < 32768; i += 4 * THREADS) *reinterpret_cast<uint4*>(&s.counters[i + 4 * tid]) = make_uint4(0, 0, 0, 0);
    s.count[tid] = 0;
    s.mass[tid] = 0;
    if (tid == 0) { s.top = NONE; s.last = 0; s.tokens = 0; }
    __syncthreads();
    // (Behind the barrier, which waits for loads; the edge first, as they are waited for in their order: pieces are counted as they arrive.)
    const int edge_token = row.edge();
    const float edge_logit = row.at(edge_token);
    Piece<false> held[R ? R : 1];
    // (a wave's loads are issued one by one as there is room for them: the first are counted before the last are asked for)
    constexpr int AHEAD = R < 6 ? R : 6;
    if (R > 0 && row.count > 0)
#pragma unroll
        for (int r = 0; r < AHEAD; ++r) row.load_one(held[r], r * THREADS + tid);
    // how often each number occurs; the largest logit; the tokens
    us2 least = {0xFFFF, 0xFFFF}, most = {0, 0};
    int tokens = 0;
    auto count = [&](unsigned n) {
        if (n < NONE) {                                    // (thousands of forbidden tokens would wait for one another at one counter)
            atomicAdd(&s.counters[n >> 1], n & 1 ? 0x10000u : 1u);
            ++tokens;
        }
    };
    each_piece<R>(row, held, [&](const Piece<false>& piece, int) {
#pragma unroll
        for (int w = 0; w < 4; ++w) {
            const us2 two = numbers_of(piece.v[w]);
            least = __builtin_elementwise_min(least, two);
            most = __builtin_elementwise_max(most, two);
            count(two.x);
            count(two.y);
        }
    }, [&](int r) {
        if (r + AHEAD < R && (r + AHEAD) * THREADS < row.count) row.load_one(held[r + AHEAD < R ? r + AHEAD : 0], (r + AHEAD) * THREADS + tid);
        __builtin_amdgcn_sched_barrier(0);
    });
    if (edge_token >= 0) {
        const us2 edge = numbers_of(__float_as_uint(edge_logit) >> 16 | 0xFF800000u);          // (and -inf)
        least = __builtin_elementwise_min(least, edge);
        most = __builtin_elementwise_max(most, edge);
        count(edge.x);
    }
    {
        const unsigned best = wave_most(0xFFFFu - (least.x < least.y ? least.x : least.y)), far = wave_most(most.x > most.y ? most.x : most.y);
        const unsigned in = wave_scan((unsigned)tokens);
        if (lane == 63) { atomicMin(&s.top, 0xFFFF - (int)best); atomicMax(&s.last, (int)far); atomicAdd(&s.tokens, (int)in); }
    }
    __syncthreads();
    const unsigned top = (unsigned)s.top;
    const int all = s.tokens;
    if (all == 0) {
        if (tid == 0) put(a, b, -1, -__builtin_inff(), 0);
        return;
    }
    if (tid == 0) {                                        // zeros are equal
        const unsigned two = s.counters[ZERO >> 1];
        s.zeros = (int)((two & 0xFFFFu) + (two >> 16));
        s.counters[ZERO >> 1] = (unsigned)s.zeros & 0xFFFFu;
    }
    Weights w;
    w.top = logit_of_number(top);
    w.per = 1.4426950408889634 / (double)c.heat;
    w.bits = a.bits;
    uint64_t kept = 1, mass = 0;
    unsigned number = top;
    int nth = 1;
    __syncthreads();
    if (!c.greedy()) {
        // 64 numbers at a time: half a wave's words, from the largest number's on
        const int end = (s.last < (int)NONE ? s.last : (int)NONE - 1) >> 1;
        constexpr int AT_ONCE = 4;
        for (int i0 = (int)(top >> 1) & ~(THREADS - 1); i0 <= end; i0 += AT_ONCE * THREADS) {
            unsigned two[AT_ONCE];
#pragma unroll
            for (int e = 0; e < AT_ONCE; ++e) two[e] = i0 + e * THREADS + tid < 32768 ? s.counters[i0 + e * THREADS + tid] : 0;
#pragma unroll
            for (int e = 0; e < AT_ONCE; ++e) {
                if (__ballot(two[e] != 0) == 0) continue;
                const int i = i0 + e * THREADS + tid;
                const unsigned n0 = two[e] & 0xFFFFu, n1 = two[e] >> 16;
                // (weights of both, whether they occur or not: one after the other they would be waited for)
                const unsigned n = half_scan(n0 + n1);
                const uint64_t m = half_scan(n0 * w.mass(logit_of_number(2 * i)) + n1 * w.mass(logit_of_number(2 * i + 1)));
                if ((lane & 31) == 31) { s.count[i >> 5] = (int)n; s.mass[i >> 5] = m; }
            }
        }
        __syncthreads();
        const uint64_t own_n = (unsigned)s.count[tid], own_m = s.mass[tid];
        uint64_t n = wave_scan((unsigned)own_n), m = wave_scan(own_m);
        if (lane == 63) { s.wave_counts[wave] = n; s.wave_masses[wave] = m; }
        if (tid == 0) s.found = 0;
        __syncthreads();
#pragma unroll
        for (int i = 0; i < WAVES; ++i) {
            n += i < wave ? s.wave_counts[i] : 0;
            m += i < wave ? s.wave_masses[i] : 0;
        }
        s.count[tid] = (int)n;
        s.mass[tid] = m;
        __syncthreads();
        if (s.count[1023] != all || s.zeros > 0xFFFF) {    // (a counter was too small)
            __syncthreads();
            by_digits<false>(a, b, (uint64_t)key_of(w.top) << 32, shared.digits);
            return;
        }
        mass = s.mass[1023];
        kept = (uint64_t)all;
        // the place at which the count, or the mass, reaches a target: the 64 numbers, then the number and which of its tokens
        struct Found { unsigned number; int nth; uint64_t count, mass; };
        auto reach = [&](bool by_mass, uint64_t target) {
            const uint64_t to = by_mass ? m : n, from = to - (by_mass ? own_m : own_n);
            if (from < target && target <= to) s.found = tid;
            __syncthreads();
            const int at = s.found;
            const unsigned x = 64u * at + lane;
            const uint64_t times = s.occurs(x), each = x < NONE ? w.mass(logit_of_number(x)) : 0;
            const uint64_t n_in = wave_scan((unsigned)times) + (at ? (unsigned)s.count[at - 1] : 0), m_in = wave_scan(times * each) + (at ? s.mass[at - 1] : 0);
            const uint64_t end = by_mass ? m_in : n_in, begin = end - (by_mass ? times * each : times);
            const uint64_t hit = __ballot(begin < target && target <= end);
            const int l = hit ? __builtin_ctzll(hit) : 0;
            auto of = [&](uint64_t v) { return (uint64_t)__shfl((unsigned long long)v, l); };
            const uint64_t each_l = of(each), begin_l = of(begin);
            Found f;
            f.number = 64u * at + l;
            const uint64_t beyond = target - begin_l;
            if (by_mass) {
                // beyond / each, rounded up: below 2^16, so a quotient of doubles is off by one at most
                f.nth = (int)__builtin_ceil((double)beyond / (double)each_l);
                if ((uint64_t)(f.nth - 1) * each_l >= beyond) --f.nth;
                if ((uint64_t)f.nth * each_l < beyond) ++f.nth;
            } else {
                f.nth = (int)beyond;
            }
            f.count = of(n_in - times) + f.nth;
            f.mass = of(m_in - times * each) + f.nth * each_l;
            __syncthreads();
            return f;
        };
        if (c.k > 0 && (uint64_t)c.k < kept) {
            const Found f = reach(false, (uint64_t)c.k);
            kept = f.count;
            mass = f.mass;
        }
        if (c.p < 1.0f) {
            const Found f = reach(true, cut_target(c.p, mass));
            if (f.count < kept) { kept = f.count; mass = f.mass; }
        }
        if (c.least > 0.0f) {
            // weights fall with numbers: the last 64 whose first weighs enough, then all in front and those of them that do
            auto enough = [&](unsigned x) { return x <= top || (x < NONE && w.scaled(logit_of_number(x), 0) >= c.enough()); };
            if (tid == 0) s.found = 0;
            __syncthreads();
            const uint64_t yes = __ballot(enough(64u * tid));
            if (lane == 0 && yes) atomicMax(&s.found, 64 * wave + 63 - __builtin_clzll(yes));
            __syncthreads();
            const int at = s.found;
            const unsigned x = 64u * at + lane;
            const uint64_t times = enough(x) ? s.occurs(x) : 0, each = times ? w.mass(logit_of_number(x)) : 0;
            const uint64_t n_in = __shfl((unsigned long long)wave_scan(times), 63) + (at ? (unsigned)s.count[at - 1] : 0);
            const uint64_t m_in = __shfl((unsigned long long)wave_scan(times * each), 63) + (at ? s.mass[at - 1] : 0);
            if (n_in < kept) { kept = n_in; mass = m_in; }
            __syncthreads();
        }
        const Found f = reach(true, draw_target(a.u[b], mass));
        number = f.number;
        nth = f.nth;
    }
    // the nth token with that number: the part of the row that holds it, then the token.  (Parts of 2^log2 tokens, 1024 at most.  The first of all,
    // where the likeliest is wanted, does not need its counter, which may have been too small.)
    const unsigned thousands = (unsigned)(a.V - 1) >> 10;
    const int log2 = thousands ? 32 - __builtin_clz(thousands) : 0;
    s.parts[tid] = 0;
    if (tid == 0) { s.found = 0; s.before = 0; s.token = 0x7FFFFFFF; }
    __syncthreads();
    // The number's bits, in both halves of a word; a half that differs from them in nothing is found by what it borrows.  (The upper one's
    // borrow may be the lower one's: each is looked at before it counts.)
    const unsigned bits = __float_as_uint(logit_of_number(number)) >> 16, both = bits | bits << 16, relevant = number == ZERO ? 0x7FFF7FFFu : 0xFFFFFFFFu;
    const bool first = nth == 1 && c.greedy();
    const bool only = !first && s.occurs(number) == 1;
    auto mark = [&](unsigned differs, int token) {
        if (differs) return;
        if (first) atomicMin(&s.token, token);
        else if (only) s.token = token;
        else atomicAdd(&s.parts[token >> log2], 1);
    };
    // (Sixteen pieces and what stands between have not the registers: the last four are read again, from the cache.  256 rows of 128000 logits
    // 34.2 us, with some 5 MB of spilled registers, with all of them kept, and some 20 MB, 37.2.)
    constexpr int KEPT = R > 12 ? 12 : R;
#pragma unroll
    for (int r = KEPT; r < R; ++r) row.load_one(held[r], r * THREADS + tid);
    each_piece<R>(row, held, [&](const Piece<false>& piece, int p) {
        unsigned x[4], zeros = 0;
#pragma unroll
        for (int w = 0; w < 4; ++w) {
            x[w] = (piece.v[w] ^ both) & relevant;
            zeros |= (x[w] - 0x00010001u) & ~x[w];
        }
        if ((zeros & 0x80008000u) == 0) return;
#pragma unroll
        for (int w = 0; w < 4; ++w) {
            mark(x[w] & 0xFFFFu, row.token(p, 2 * w));
            mark(x[w] >> 16, row.token(p, 2 * w + 1));
        }
    }, [](int) {});
    if (edge_token >= 0) mark((__float_as_uint(edge_logit) >> 16 ^ bits) & relevant & 0xFFFFu, edge_token);
    __syncthreads();
    if (!first && !only) {
        const uint64_t own = (unsigned)s.parts[tid];
        uint64_t n = wave_scan((unsigned)own);
        if (lane == 63) s.wave_counts[wave] = n;
        __syncthreads();
#pragma unroll
        for (int i = 0; i < WAVES; ++i) n += i < wave ? s.wave_counts[i] : 0;
        if (n - own < (uint64_t)nth && (uint64_t)nth <= n) { s.found = tid; s.before = (int)(n - own); }
        __syncthreads();
        if (wave == 0) {
            int seen = s.before, token = -1;
            const int from = s.found << log2, to = from + (1 << log2) < a.V ? from + (1 << log2) : a.V;
            for (int i0 = from; i0 < to && token < 0; i0 += 64) {
                const int i = i0 + lane < to ? i0 + lane : to - 1;
                const bool mine = i0 + lane < to && ((static_cast<const uint16_t*>(row.row)[i] ^ bits) & relevant & 0xFFFFu) == 0;
                const uint64_t who = __ballot(mine);
                const int rank = seen + __popcll(who & ((1ull << lane) - 1)) + 1;
                const uint64_t hit = __ballot(mine && rank == nth);
                if (hit) token = i0 + __builtin_ctzll(hit);
                seen += __popcll(who);
            }
            if (lane == 0) s.token = token;
        }
        __syncthreads();
    }
    if (tid == 0) put(a, b, s.token, c.greedy() ? 0.0f : share(w, c.heat, logit_of_number(number), mass), (int)kept);
}

// ---- fp32: cells ------------------------------------------------------------------------------------------------------------
//
// A logit's cell is its place on a grid of step 2^e between 36/2048 and 72/2048 of the temperature, so that 2047 cells cover all that has
// weight.  Cells are counted from the highest logit's, the last holds whatever lies below; the grid is the temperature's, not the
// row's, so it is the same for all slices of a row before they know of each other.  A row of up to 32768 logits stays in the registers of one
// workgroup; longer ones take two launches.  The first reads the logits once: a slice stays in registers while its maximum is found, then
// its histogram is.  The second joins a row's histograms, finds the cells in which the cuts and the draw may lie -- one or two each,
// mostly -- and reads the row again for the tokens in them, some hundred, which are sorted and settle everything exactly.  Rows whose cells hold more tokens than are sorted (nearly equal logits, thousands of
// equal ones, a high temperature) go by digits.
//
// A token's weight is the weight at its cell's lower edge times e^x, x = (z - edge) / T below 0.0352: the histogram sums e^x - 1, and
// one exponential for each cell follows in the second launch.  e^x - 1 is five terms of its series in fp64, times 2^36, in the lower
// 48 bits of a cell's 64, the number of tokens in the upper 16: one LDS atomic a token.  (With an exponential and two atomics for each
// token, 256 rows of 128000 logits, then in bf16, took this launch 67 us and took it 38 so, LDS and the vector units at their limits in turn.)  The series and the
// rounding are good for 2^-36 of a token's weight (2^-37 the rounding, 2^-38.5 the first term left out); a cell's sum is rounded to whole
// steps once, not token by token.  Of logits on the grid, as coarse ones are, e^x - 1 is 0.

constexpr int CELLS = SAMPLE_CELLS, SORTED = 4096;
// the grid of a temperature
struct Grid {
    float per_unit, step;
    __device__ __forceinline__ explicit Grid(float heat) {
        int e = (int)(__float_as_uint(36.0f / CELLS * heat) >> 23) - 126;                       // 2^e: the next power of two
        e = e < -120 ? -120 : e > 120 ? 120 : e;
        per_unit = __uint_as_float((unsigned)(127 - e) << 23);
        step = __uint_as_float((unsigned)(127 + e) << 23);
    }
    __device__ __forceinline__ int cell(float z) const { return (int)__builtin_floorf(z * per_unit); }       // (saturates)
    // The lowest logit of a cell.  That of cell 0 is not 0 where the step is 2 or more: the products of logits just below it, down to
    // -2^-150 step, round to -0.  (2^-150 is half of the least number, a tie that goes to 0; for a smaller step this is -0.)
    __device__ __forceinline__ float edge(int cell) const { return cell ? (float)cell * step : step * -0x1p-75f * 0x1p-75f; }
    // Cells next to this logit are numbers of 24 bits, edges are exact; and a cell is no wider than 72/2048 temperatures, as its sums need (one of
    // 2^-120 is, for temperatures below 2.1e-35).
    __device__ __forceinline__ bool fine(float z, float heat) const { return fabsf(z * per_unit) < 4194304.0f && step <= 72.0f / CELLS * heat; }
};
__device__ __forceinline__ int below(int top, int cell) {
    const unsigned d = (unsigned)top - (unsigned)cell;
    return d < CELLS - 1 ? (int)d : CELLS - 1;
}
constexpr int COUNT_AT = 48;
constexpr double PARTS = 68719476736.0;                   // 2^36
// Few tokens are kept: they are weighed when they are known, and need no masses of cells.
__device__ __forceinline__ bool few(const Choices& c) { return c.k > 0 && c.k <= SAMPLE_FEW; }

// The likeliest of the logits that a workgroup holds, (key, ~index), and their cells, counted from its.  Cells are not made where only the
// likeliest is wanted, or there is none.  R: pieces that a thread holds; 2^15 logits of a workgroup at most, which a cell's 48 bits hold.
struct Tally {
    unsigned long long cells[CELLS + 1];                   // (the last takes what is no token)
    uint64_t tops[WAVES];
};
template <int R>
__device__ __forceinline__ uint64_t tally(Tally& s, const Pieces<true>& row, const Piece<true> (&held)[R], int p0, int edge_token, const Choices& c) {
    static_assert(THREADS * R * Piece<true>::N <= 32768, "and a few at the row's ends");
    const int tid = threadIdx.x;
    auto& cells = s.cells;
    auto& tops = s.tops;
    const float edge_logit = row.at(edge_token);
#pragma unroll
    for (int i = 0; i < CELLS; i += THREADS) cells[i + tid] = 0;
    float top = -__builtin_inff();
    int at = -1;
#pragma unroll
    for (int r = 0; r < R; ++r)
#pragma unroll
        for (int e = 0; e < Piece<true>::N; ++e) {
            const float z = held[r][e];
            if (z > top) { top = z; at = row.token(p0 + r * THREADS + tid, e); }
        }
    const uint64_t own = (uint64_t)key_of(top) << 32 | (unsigned)~at, at_edge = (uint64_t)key_of(edge_logit) << 32 | (unsigned)~edge_token;
    uint64_t best = wave_max(own > at_edge ? own : at_edge);
    if ((tid & 63) == 0) tops[tid >> 6] = best;
    __syncthreads();
    best = tops[0];
#pragma unroll
    for (int i = 1; i < WAVES; ++i) best = tops[i] > best ? tops[i] : best;
    if (c.greedy() || (unsigned)(best >> 32) <= LOWEST) return best;
    const Grid grid(c.heat);
    const int top_cell = grid.cell(logit_of((unsigned)(best >> 32)));
    if (few(c)) {
        auto add = [&](float z) {
            if (z > -__builtin_inff()) atomicAdd(&cells[below(top_cell, grid.cell(z))], 1ull << COUNT_AT);
        };
        add(edge_logit);
#pragma unroll
        for (int r = 0; r < R; ++r)
#pragma unroll
            for (int e = 0; e < Piece<true>::N; ++e) add(held[r][e]);
    } else {
        // x = d g, d the place in the cell; coefficients g^k / k!
        const double g = (double)grid.step / (double)c.heat;
        const double c1 = PARTS * g, c2 = c1 * g * (1.0 / 2), c3 = c2 * g * (1.0 / 3), c4 = c3 * g * (1.0 / 4), c5 = c4 * g * (1.0 / 5);
        auto add = [&](float z) {
            const float y = z * grid.per_unit, edge = __builtin_floorf(y);
            const double d = (double)(y - edge);
            const double v = fma(fma(fma(fma(fma(c5, d, c4), d, c3), d, c2), d, c1), d, 4503599627370496.0);
            const int j = z > -__builtin_inff() ? below(top_cell, (int)edge) : CELLS;
            const unsigned hi = ((unsigned)__double2hiint(v) & 0xFFFFu) | 1u << (COUNT_AT - 32);
            atomicAdd(&cells[j], (unsigned long long)hi << 32 | (unsigned)__double2loint(v));
        };
        if (edge_token >= 0) add(edge_logit);
#pragma unroll
        for (int r = 0; r < R; ++r)
#pragma unroll
            for (int e = 0; e < Piece<true>::N; ++e) add(held[r][e]);
    }
    __syncthreads();
    return best;
}

template <int R>
__global__ __launch_bounds__(THREADS) void sample_slice_kernel(SampleArgs a) {
    __shared__ Tally s;
    const int slice = blockIdx.x, b = blockIdx.y, tid = threadIdx.x;
    const Pieces<true> row(row_of(a, b), a.V);
    const Choices c(a, b);
    const int p0 = slice * (THREADS * R);
    Piece<true> held[R];
    row.load(held, p0);
    const uint64_t best = tally<R>(s, row, held, p0, slice == 0 ? row.edge() : -1, c);
    SampleSlice& out = a.slices[(int64_t)b * a.slices_of_row + slice];
    if (tid == 0) out.best = best;
    if (c.greedy() || (unsigned)(best >> 32) <= LOWEST) return;
#pragma unroll
    for (int i = 0; i < CELLS; i += THREADS) out.cells[i + tid] = s.cells[i + tid];
}

struct Cells {
    uint64_t mass[CELLS];                                  // of the cells up to and with this one, from the highest
    int count[CELLS];
    uint64_t key[SORTED], running[SORTED];
    uint64_t wave_counts[WAVES], wave_masses[WAVES];
    int first, last, places[4], n;
    int found_rank;
    uint64_t found_mass, found_key;
    int most_rank;
};
union RowShared {
    Cells cells;
    Shared digits;
};

// Sorts key[0 .. n) from the highest, n <= SORTED, by a bitonic network: E keys of a thread, i = tid + 1024 e; `down` where a run of k
// keys is to fall.  Partners are a thread's own, another wave's, through LDS, or another lane's.
__device__ __forceinline__ uint64_t chosen(uint64_t v, uint64_t o, bool larger) { return (v > o) == larger ? v : o; }
template <int E, int J>
__device__ __forceinline__ void sort_in_wave(uint64_t (&v)[E], int k) {
#pragma unroll
    for (int e = 0; e < E; ++e) {
        const int i = threadIdx.x + THREADS * e;
        v[e] = chosen(v[e], across<J>(v[e]), ((i & k) == 0) == ((i & J) == 0));
    }
    if constexpr (J > 1) sort_in_wave<E, J / 2>(v, k);
}
template <int E>
__device__ void sort_keys(uint64_t* key, int n) {
    const int tid = threadIdx.x;
    uint64_t v[E];
#pragma unroll
    for (int e = 0; e < E; ++e) v[e] = tid + THREADS * e < n ? key[tid + THREADS * e] : 0;
    sort_in_wave<E, 1>(v, 2);
    sort_in_wave<E, 2>(v, 4);
    sort_in_wave<E, 4>(v, 8);
    sort_in_wave<E, 8>(v, 16);
    sort_in_wave<E, 16>(v, 32);
    sort_in_wave<E, 32>(v, 64);
    for (int k = 128; k < 2 * n; k *= 2) {
        for (int j = k / 2; j >= 64; j /= 2) {
            if (j >= THREADS) {
#pragma unroll
                for (int e = 0; e < E; ++e) {
                    const int f = e | (j / THREADS);
                    if (f == e || f >= E) continue;
                    const bool larger = ((tid + THREADS * e) & k) == 0;
                    const uint64_t x = v[e], y = v[f];
                    v[e] = chosen(x, y, larger);
                    v[f] = chosen(y, x, !larger);
                }
            } else {
                __syncthreads();
#pragma unroll
                for (int e = 0; e < E; ++e) key[tid + THREADS * e] = v[e];
                __syncthreads();
#pragma unroll
                for (int e = 0; e < E; ++e) {
                    const int i = tid + THREADS * e;
                    v[e] = chosen(v[e], key[i ^ j], ((i & k) == 0) == ((i & j) == 0));
                }
            }
        }
        sort_in_wave<E, 32>(v, k);
    }
    __syncthreads();
#pragma unroll
    for (int e = 0; e < E; ++e) key[tid + THREADS * e] = v[e];
    __syncthreads();
}

// The tokens of the row in Q stretches of cells, into key[], in any order.  A lane tests a block of its logits by three vector instructions
// each (the middle of logit and bounds; is it the logit; a bit more of a mask), the next block under way meanwhile; hits
// leave their index only, and the logits of all of them are fetched at the end.  (Tests by masks of the wave, or hits one by one in
// between, are chains of latencies: 13 .. 28 us for 128000 logits.)
template <int Q, int HELD>
__device__ __forceinline__ void collect(Cells& s, const Pieces<true>& row, const Piece<true> (&have)[HELD ? HELD : 1], const int (&from)[3], const int (&to)[3], int top_cell, const Grid& grid) {
    constexpr int R = 8, N = Piece<true>::N;
    static_assert(HELD == 0 || HELD == R, "");
    static_assert(R * N <= 32, "a mask");
    const int tid = threadIdx.x;
    float lo[Q], hi[Q];                                    // of a stretch, both within
#pragma unroll
    for (int q = 0; q < Q; ++q) {
        const int end = __float_as_int(grid.edge(top_cell - from[q] + 1));                      // the first beyond
        lo[q] = to[q] == CELLS - 1 ? -3.402823466e38f : grid.edge(top_cell - to[q]);
        hi[q] = __int_as_float(end > 0 ? end - 1 : end + 1);
    }
    auto wanted = [&](float z) {
        bool in = __builtin_amdgcn_fmed3f(z, lo[0], hi[0]) == z;
#pragma unroll
        for (int q = 1; q < Q; ++q) in |= __builtin_amdgcn_fmed3f(z, lo[q], hi[q]) == z;
        return in;
    };
    auto keep = [&](int token) {
        const int at = atomicAdd(&s.n, 1);
        if (at < SORTED) s.key[at] = (unsigned)token;
    };
    const int edge = row.edge();
    if (edge >= 0 && wanted(row.at(edge))) keep(edge);
    auto block = [&](const Piece<true> (&held)[R], int p0) {
        unsigned hits = 0;
#pragma unroll
        for (int r = 0; r < R; ++r)
#pragma unroll
            for (int e = 0; e < N; ++e) hits = hits + hits + (wanted(held[r][e]) ? 1u : 0u);
        while (hits) {
            const int i = R * N - 1 - __builtin_ctz(hits);
            hits &= hits - 1;
            keep(row.token(p0 + i / N * THREADS + tid, i % N));
        }
    };
    if constexpr (HELD) {
        block(have, 0);
    } else {
        Piece<true> held[R], next[R];
        row.load(next, 0);
        for (int p0 = 0; p0 < row.count; p0 += R * THREADS) {
#pragma unroll
            for (int r = 0; r < R; ++r) held[r] = next[r];
            row.load(next, p0 + R * THREADS);
            block(held, p0);
        }
    }
    __syncthreads();
    const int n = s.n < SORTED ? s.n : SORTED;
    for (int i = tid; i < n; i += THREADS) {
        const int token = (int)s.key[i];
        s.key[i] = (uint64_t)key_of(row.at(token)) << 32 | (unsigned)~token;
    }
}

// HELD: the row is that many pieces of each thread, and no slices were made of it; 0: it is joined from slices.
template <int HELD>
__global__ __launch_bounds__(THREADS) void sample_row_kernel(SampleArgs a) {
    __shared__ RowShared shared;
    __shared__ typename std::conditional<(HELD > 0), Tally, int>::type fresh;
    Cells& s = shared.cells;
    const int b = blockIdx.x, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, S = a.slices_of_row;
    const SampleSlice* slices = a.slices + (int64_t)b * S;
    const Choices c(a, b);
    const Pieces<true> row(row_of(a, b), a.V);
    Piece<true> held[HELD ? HELD : 1];
    uint64_t best = 0;
    if constexpr (HELD > 0) {
        row.load(held, 0);
        best = tally<HELD>(fresh, row, held, 0, row.edge(), c);
    } else {
        for (int i = 0; i < S; ++i) best = slices[i].best > best ? slices[i].best : best;
    }
    const bool none = (unsigned)(best >> 32) <= LOWEST;
    if (none || c.greedy()) {
        if (tid == 0) put(a, b, none ? -1 : (int)~(unsigned)best, none ? -__builtin_inff() : 0.0f, none ? 0 : 1);
        return;
    }
    Weights w;
    w.top = logit_of((unsigned)(best >> 32));
    w.per = 1.4426950408889634 / (double)c.heat;
    w.bits = a.bits;
    const Grid grid(c.heat);
    if (!grid.fine(w.top, c.heat)) {
        by_digits<true>(a, b, best, shared.digits);
        return;
    }
    const int top_cell = grid.cell(w.top);

    // the row's histogram: a slice's cells, as far below the row's as its maximum is
    static_assert(CELLS == 2 * THREADS, "two cells to a thread");
    s.count[tid] = s.count[tid + THREADS] = 0;
    s.mass[tid] = s.mass[tid + THREADS] = 0;
    if (tid == 0) s.n = 0;
    if (tid < 4) s.places[tid] = CELLS - 1;
    __syncthreads();
    if constexpr (HELD > 0) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const uint64_t cell = fresh.cells[tid + h * THREADS];
            s.count[tid + h * THREADS] = (int)(cell >> COUNT_AT);
            s.mass[tid + h * THREADS] = cell & ((1ull << COUNT_AT) - 1);
        }
    }
    constexpr int AT_ONCE = 4;
    for (int i0 = 0; HELD == 0 && i0 < S; i0 += AT_ONCE) {
        uint64_t cell[AT_ONCE][2];
        unsigned key[AT_ONCE];
#pragma unroll
        for (int i = 0; i < AT_ONCE; ++i) {
            const int at = i0 + i < S ? i0 + i : S - 1;
            key[i] = i0 + i < S ? (unsigned)(slices[at].best >> 32) : 0;
#pragma unroll
            for (int h = 0; h < 2; ++h) cell[i][h] = slices[at].cells[tid + h * THREADS];          // (of a slice without tokens: whatever is there)
        }
#pragma unroll
        for (int i = 0; i < AT_ONCE; ++i) {
            if (key[i] <= LOWEST) continue;
            const unsigned down = (unsigned)top_cell - (unsigned)grid.cell(logit_of(key[i]));
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int n = (int)(cell[i][h] >> COUNT_AT), own = tid + h * THREADS;
                if (n == 0) continue;
                const int j = down < CELLS && down + own < CELLS - 1 && own < CELLS - 1 ? (int)down + own : CELLS - 1;
                atomicAdd(&s.count[j], n);
                atomicAdd((unsigned long long*)&s.mass[j], cell[i][h] & ((1ull << COUNT_AT) - 1));
            }
        }
    }
    __syncthreads();
    // this thread's two cells, and what lies in front of them
    int count_to[3];
    uint64_t mass_to[3];
    {
        uint64_t n[2], m[2] = {0, 0};
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int j = 2 * tid + h;
            n[h] = (unsigned)s.count[j];
            if (!few(c) && n[h] && j < CELLS - 1) {
                const double edge = (double)(top_cell - j) * (double)grid.step, sum = (double)(int)n[h] + (double)s.mass[j] * (1.0 / PARTS);
                m[h] = (uint64_t)__builtin_rint(sum * w.scaled((float)edge, w.bits));
            }
        }
        const uint64_t n_in = wave_scan((unsigned)(n[0] + n[1])), m_in = wave_scan(m[0] + m[1]);
        if (lane == 63) { s.wave_counts[wave] = n_in; s.wave_masses[wave] = m_in; }
        __syncthreads();
        uint64_t nb = n_in - n[0] - n[1], mb = m_in - m[0] - m[1];
#pragma unroll
        for (int i = 0; i < WAVES; ++i) {
            nb += i < wave ? s.wave_counts[i] : 0;
            mb += i < wave ? s.wave_masses[i] : 0;
        }
        count_to[0] = (int)nb; count_to[1] = (int)(nb + n[0]); count_to[2] = (int)(nb + n[0] + n[1]);
        mass_to[0] = mb; mass_to[1] = mb + m[0]; mass_to[2] = mb + m[0] + m[1];
#pragma unroll
        for (int h = 0; h < 2; ++h) { s.count[2 * tid + h] = count_to[h + 1]; s.mass[2 * tid + h] = mass_to[h + 1]; }
    }
    __syncthreads();
    const int all = s.count[CELLS - 1];
    // few tokens are kept, or there are: all that matter are weighed one by one
    const bool weighed = !few(c) && all > SORTED;
    const uint64_t all_mass = s.mass[CELLS - 1];
    // the first cell with so many tokens, or so much mass, up to its end: one thread finds it
    auto cell_by_count = [&](int64_t n, int slot) {
#pragma unroll
        for (int h = 0; h < 2; ++h)
            if (count_to[h] < n && n <= count_to[h + 1]) s.places[slot] = 2 * tid + h;
    };
    auto cell_by_mass = [&](double m, int slot) {
#pragma unroll
        for (int h = 0; h < 2; ++h)
            if ((double)mass_to[h] < m && m <= (double)mass_to[h + 1]) s.places[slot] = 2 * tid + h;
    };
    auto cells_found = [&](int* to, int n) {
        __syncthreads();
        for (int i = 0; i < n; ++i) to[i] = s.places[i];
        __syncthreads();
        if (tid < 4) s.places[tid] = CELLS - 1;
        __syncthreads();
    };
    const bool by_k = c.k > 0 && c.k < all, by_p = c.p < 1.0f, by_least = c.least > 0.0f;
    // Up to three stretches of cells, one below the other, whose tokens have to be known: [from, to].  Sums by cell and sums by token
    // differ by 2^-36 of them, and by half a step a token: a target that is not among the tokens found for it sends the row to the digits.
    constexpr double under = 1.0 - 0x1p-35, over = 1.0 + 0x1p-35;
    int from[3] = {0, 0, 0}, to[3] = {-1, -1, -1};
    int least_cell = CELLS, found[4];                      // (the first cell in which a weight may be too small)
    bool least_ends = false;                               // (all cells in which some may be are among those stretches)
    if (!weighed) {
        cell_by_count(by_k ? c.k : all, 0);
        cells_found(found, 1);
        to[0] = found[0];
    } else {
        int k_cell = CELLS, cut_lo = CELLS, cut_hi = CELLS;
        double k_lo = (double)all_mass, k_hi = k_lo;
        if (by_k) {
            cell_by_count(c.k, 0);
            cells_found(found, 1);
            k_cell = cut_lo = cut_hi = found[0];
            k_lo = k_cell ? (double)s.mass[k_cell - 1] : 0.0;
            k_hi = (double)s.mass[k_cell];
        }
        if (by_p) {
            const double t1 = fmin(fmax((double)c.p * k_hi * over, 1.0), k_hi), t0 = fmin(fmax((double)c.p * k_lo * under, 1.0), t1);
            cell_by_mass(t0, 0);
            cell_by_mass(t1, 1);
            cells_found(found, 2);
            cut_lo = found[0] < cut_lo ? found[0] : cut_lo;
            cut_hi = found[1] < cut_hi ? found[1] : cut_hi;
        }
        if (by_least) {
            // the logit of a weight of min-p, give or take what its computation may be off
            const double z = (double)w.top + (double)c.heat * log(c.enough()), off = 1e-9 * (1.0 + fabs(z) + fabs((double)w.top));
            const double hi = fmin(__builtin_floor((z + off) * (double)grid.per_unit), 2147483647.0), lo = fmax(__builtin_floor((z - off) * (double)grid.per_unit), -2147483648.0);
            least_cell = hi >= (double)top_cell ? 0 : below(top_cell, (int)hi);
            const int least_end = lo >= (double)top_cell ? 0 : below(top_cell, (int)lo);
            cut_lo = least_cell < cut_lo ? least_cell : cut_lo;
            cut_hi = least_end < cut_hi ? least_end : cut_hi;
            least_ends = least_end <= cut_hi;
        }
        const double u = a.u[b];
        const double share = u > 0.0 ? (u < 1.0 ? u : 1.0) : 0.0;
        const bool cut = cut_lo < CELLS;
        const double lo = cut ? (cut_lo ? (double)s.mass[cut_lo - 1] : 0.0) : (double)all_mass, hi = cut ? (double)s.mass[cut_hi] : (double)all_mass;
        cell_by_mass(fmax(share * lo * under, 1.0), 0);
        cell_by_mass(fmin(fmax(share * hi * over + 1.0, 1.0), hi), 1);
        cells_found(found, 2);
        from[0] = found[0];
        to[0] = found[1];
        if (cut) {
            // the cuts' cells; top-k's, for what is top-p's share, also where it is not the first cut.  (Cells without mass add nothing to it.)
            from[1] = cut_lo;
            to[1] = cut_hi;
            if (by_k && by_p && k_hi > k_lo && k_cell > cut_hi) from[2] = to[2] = k_cell;
            if (from[1] <= to[0] + 1) {                    // one stretch
                from[0] = from[1] < from[0] ? from[1] : from[0];
                to[0] = to[1] > to[0] ? to[1] : to[0];
                from[1] = from[2];
                to[1] = to[2];
                to[2] = -1;
            }
        }
    }
    int base_count[3], tokens[3];
#pragma unroll
    for (int q = 0; q < 3; ++q) {
        const bool there = to[q] >= from[q];
        base_count[q] = there && from[q] ? s.count[from[q] - 1] : 0;
        tokens[q] = there ? s.count[to[q]] - base_count[q] : 0;
    }
    const int n = tokens[0] + tokens[1] + tokens[2];
    if (n > SORTED || (by_least && c.least < 1e-12f)) {    // (uniform: every thread has the same numbers)
        __syncthreads();
        by_digits<true>(a, b, best, shared.digits);
        return;
    }
    // the tokens of those cells, as (key, ~index)
    if (to[1] < from[1]) collect<1, HELD>(s, row, held, from, to, top_cell, grid);
    else if (to[2] < from[2]) collect<2, HELD>(s, row, held, from, to, top_cell, grid);
    else collect<3, HELD>(s, row, held, from, to, top_cell, grid);
    __syncthreads();
    if (n <= THREADS) sort_keys<1>(s.key, n);
    else if (n <= 2 * THREADS) sort_keys<2>(s.key, n);
    else sort_keys<4>(s.key, n);

    // their running masses: E tokens of a thread, side by side
    constexpr int E = SORTED / THREADS;
    uint64_t each[E], run[E];
    int rank[E];                                           // -1: none
    const int per_thread = n <= THREADS ? 1 : E;
    {
        uint64_t sum = 0;
#pragma unroll
        for (int e = 0; e < E; ++e) {
            const int i = tid * per_thread + e;
            const bool there = e < per_thread && i < n;
            each[e] = there ? w.mass(logit_of((unsigned)(s.key[i] >> 32))) : 0;
            sum += each[e];
            run[e] = sum;
            rank[e] = -1;
        }
        const uint64_t in = wave_scan(sum);
        if (lane == 63) s.wave_masses[wave] = in;
        __syncthreads();
        uint64_t front = in - sum;
#pragma unroll
        for (int i = 0; i < WAVES; ++i) front += i < wave ? s.wave_masses[i] : 0;
#pragma unroll
        for (int e = 0; e < E; ++e) {
            const int i = tid * per_thread + e;
            run[e] += front;
            if (e < per_thread && i < n) s.running[i] = run[e];
        }
    }
    __syncthreads();
    {
        // places in the whole order: behind a stretch lies what is between it and the next, which has the mass from its cells' on, so none of
        // its tokens' goes beyond
        int start = 0;
#pragma unroll
        for (int q = 0; q < 3; ++q) {
            if (tokens[q] == 0) continue;
            const uint64_t shift = (weighed && from[q] ? s.mass[from[q] - 1] : 0) - (start ? s.running[start - 1] : 0);
            const uint64_t end = weighed ? s.mass[to[q]] : ~0ull;
#pragma unroll
            for (int e = 0; e < E; ++e) {
                const int i = tid * per_thread + e;
                if (e >= per_thread || i < start || i >= start + tokens[q]) continue;
                rank[e] = base_count[q] + i - start;
                run[e] += shift;
                const uint64_t in_front = run[e] - each[e];
                run[e] = run[e] < end ? run[e] : end;
                each[e] = run[e] - (in_front < end ? in_front : end);
            }
            start += tokens[q];
        }
    }
    // the first of them whose running mass reaches the target
    auto reach = [&](uint64_t target) {
        __syncthreads();
        if (tid == 0) s.found_rank = -1;
        __syncthreads();
#pragma unroll
        for (int e = 0; e < E; ++e)
            if (rank[e] >= 0 && run[e] >= target && run[e] - each[e] < target) {
                s.found_rank = rank[e];
                s.found_mass = run[e];
                s.found_key = s.key[tid * per_thread + e];
            }
        __syncthreads();
        return s.found_rank;
    };
    int kept = all;
    uint64_t mass = all_mass;
    // (a target between the tokens' sums and the cells', or keys that were counted and not collected, which are not there: next to never)
    bool lost = s.n != n;
    uint64_t p_target = 0;
    bool p_found = true;
    if (by_k) {
        if (tid == 0) s.found_rank = -1;
        __syncthreads();
#pragma unroll
        for (int e = 0; e < E; ++e)
            if (rank[e] == c.k - 1) { s.found_rank = rank[e]; s.found_mass = run[e]; }
        __syncthreads();
        kept = c.k;
        if (s.found_rank >= 0) {
            mass = s.found_mass;
        } else {
            // not among them: another cut comes first, or its cell has no mass
            int j = 0;                                     // (the cell that reaches it)
            for (int step = CELLS / 2; step; step /= 2) if (s.count[j + step - 1] < c.k) j += step;
            mass = s.mass[j];
        }
    } else if (!weighed) {
        mass = n > 0 ? s.running[n - 1] : 0;
    }
    if (by_p) {
        p_target = cut_target(c.p, mass);
        const int r = reach(p_target);
        const uint64_t m = s.found_mass;
        p_found = r >= 0;
        if (p_found && r + 1 < kept) { kept = r + 1; mass = m; }
    }
    if (by_least) {
        // the last that weighs enough; where none of them does, the cells in front hold it
        __syncthreads();
        if (tid == 0) s.most_rank = -1;
        __syncthreads();
        int most = -1;
#pragma unroll
        for (int e = 0; e < E; ++e)
            if (rank[e] >= 0 && w.scaled(logit_of((unsigned)(s.key[tid * per_thread + e] >> 32)), 0) >= c.enough()) most = rank[e];
        most = (int)wave_max((uint64_t)(most + 1)) - 1;
        if (lane == 0 && most >= 0) atomicMax(&s.most_rank, most);
        __syncthreads();
        most = s.most_rank;
        if (tid == 0) s.found_rank = -1;
        __syncthreads();
#pragma unroll
        for (int e = 0; e < E; ++e)
            if (most >= 0 && rank[e] == most) { s.found_rank = most; s.found_mass = run[e]; }
        __syncthreads();
        int m_kept = most + 1;
        uint64_t m_mass = most >= 0 ? s.found_mass : 0;
        const int whole = weighed && least_cell > 0 ? s.count[least_cell - 1] : 0;          // (cells that weigh enough altogether)
        if (whole > m_kept) { m_kept = whole; m_mass = s.mass[least_cell - 1]; }
        // (min-p cuts in front of it)
        if (!p_found && least_ends && m_mass < p_target) p_found = true;
        if (m_kept < kept) { kept = m_kept; mass = m_mass; }
    }
    if (!p_found) lost = true;
    if (reach(draw_target(a.u[b], mass)) < 0) lost = true;
    if (lost) {
        __syncthreads();
        by_digits<true>(a, b, best, shared.digits);
        return;
    }
    if (tid == 0) put(a, b, (int)~(unsigned)s.found_key, share(w, c.heat, logit_of((unsigned)(s.found_key >> 32)), mass), kept);
}

// Slices of a row: as many pieces of a thread as it holds in registers, or two where those are 256 workgroups at most.  (Eight, four:
// 64 rows of 128000 logits 14.4 us the slices and 29.2 the rows, 15.5 and 31.2.  Eight, two, the whole with top-p: 8 rows of 40000 47.8 us
// and 28.6, 50 rows 50.1 and 31.6, but also 80 rows 50.5 and 34.0; 4 rows of 128000 39.9 and 43.3, 48 rows 47.2 and 59.1.)
constexpr int FEW_PIECES = 2, MANY_PIECES = 8;
static_assert(SAMPLE_SHORT == THREADS * MANY_PIECES * Piece<true>::N, "a row that a workgroup holds");
int slices_of(int32_t V, int r) { return (V / 4 + 1 + THREADS * r - 1) / (THREADS * r); }

}  // namespace

// A workspace holds the slices of 2048 / (slices of a row) rows; a call of more runs in parts, one after the other.  So does one of more
// rows than a launch has workgroups (2^32 threads).
constexpr int64_t SLICES_AT_ONCE = 2048;
constexpr int32_t ROWS_AT_ONCE = 1 << 21;

size_t sample_workspace_bytes(int32_t B, int32_t V) {
    if (V <= SAMPLE_SHORT) return 0;
    if (V > SAMPLE_LONG) V = SAMPLE_LONG;                  // (rows by digits need none, but what does for a call does for smaller ones)
    const int64_t row = slices_of(V, MANY_PIECES), most = row > SLICES_AT_ONCE ? row : SLICES_AT_ONCE;
    const int64_t many = row * B < most ? row * B : most, few_rows = 256 + slices_of(V, FEW_PIECES);
    return (size_t)(many > few_rows ? many : few_rows) * sizeof(SampleSlice);
}

namespace {

// the rows of a part
void launch_rows(const SampleArgs& a, bool few_rows, hipStream_t s) {
    const dim3 rows(a.B), block(THREADS);
    constexpr int WORD = THREADS * 8;                      // logits of a piece of each thread
    if (a.V > SAMPLE_LONG) {
        if (a.f32) hipLaunchKernelGGL(sample_long_kernel<true>, rows, block, 0, s, a);
        else hipLaunchKernelGGL(sample_long_kernel<false>, rows, block, 0, s, a);
    } else if (!a.f32) {
        if (a.V <= 4 * WORD) hipLaunchKernelGGL(sample_numbers_kernel<4>, rows, block, 0, s, a);
        else if (a.V <= 16 * WORD) hipLaunchKernelGGL(sample_numbers_kernel<16>, rows, block, 0, s, a);
        else hipLaunchKernelGGL(sample_numbers_kernel<0>, rows, block, 0, s, a);
    } else if (a.slices_of_row == 0) {
        hipLaunchKernelGGL(sample_row_kernel<MANY_PIECES>, rows, block, 0, s, a);
    } else {
        const dim3 grid(a.slices_of_row, a.B);
        if (few_rows) hipLaunchKernelGGL(sample_slice_kernel<FEW_PIECES>, grid, block, 0, s, a);
        else hipLaunchKernelGGL(sample_slice_kernel<MANY_PIECES>, grid, block, 0, s, a);
        hipLaunchKernelGGL(sample_row_kernel<0>, rows, block, 0, s, a);
    }
}

}  // namespace

int launch_sample(SampleArgs a, hipStream_t s) {
    int log2 = 0;
    while ((1ll << log2) < a.V) ++log2;
    a.bits = 62 - log2 < 50 ? 62 - log2 : 50;
    bool few_rows = false;
    int32_t at_once = ROWS_AT_ONCE;
    a.slices_of_row = 0;
    if (a.f32 && a.V > SAMPLE_SHORT && a.V <= SAMPLE_LONG) {
        a.slices = reinterpret_cast<SampleSlice*>(a.workspace);
        const int fine = slices_of(a.V, FEW_PIECES);
        few_rows = (int64_t)fine * a.B <= 256;
        a.slices_of_row = few_rows ? fine : slices_of(a.V, MANY_PIECES);
        at_once = a.slices_of_row < SLICES_AT_ONCE ? (int32_t)(SLICES_AT_ONCE / a.slices_of_row) : 1;
    }
    for (int64_t b0 = 0; b0 < a.B; b0 += at_once) {
        SampleArgs p = a;
        p.B = a.B - b0 < at_once ? (int32_t)(a.B - b0) : at_once;
        p.logits = static_cast<const uint8_t*>(a.logits) + b0 * a.ldl * (a.f32 ? 4 : 2);
        if (p.temperature) p.temperature += b0;
        if (p.top_k) p.top_k += b0;
        if (p.top_p) p.top_p += b0;
        if (p.min_p) p.min_p += b0;
        p.u += b0;
        p.token += b0;
        if (p.logprob) p.logprob += b0;
        if (p.kept) p.kept += b0;
        launch_rows(p, few_rows, s);
    }
    return check_hip(hipGetLastError(), "sample launch");
}

}  // namespace basq
