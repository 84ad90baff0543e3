// A token for each row of logits, with temperature, top-k, top-p and min-p, from given random numbers; the definition is beside
// basq_sample in basq.h.
//
// The tokens' order is that of their logits, so nothing is sorted: a cut, and the draw itself, is the first place of that order at
// which a running count or a running mass reaches a target, and such a place is found digit by digit of the logits' bits, with a
// histogram of counts and masses over one digit at a time.  Equal logits share a place; which of them it is follows from
// arithmetic, and only the drawn one's index is looked for.
//
// Masses are whole numbers: a token's weight e^((z - top) / T), computed in fp64, times 2^bits, rounded once.  Sums of them are exact
// in any order, so LDS atomics give the same token every time, equal logits weigh the same, and the running mass at the last place
// is the total.  (bits: 2^bits times the tokens of a row stays below 2^62; 45 for 128000 tokens, whose roundings together are about
// 2^-37 of the mass at most.  Sums in fp32 would move the draw of one row in forty to a neighbour, by their 2^-23.)
#include "basq_internal.h"

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

// The weights of a row: 2^bits e^((z - top) / T) = 2^(bits + n + r), n whole and |r| <= 1/2.
struct Weights {
    double top, per;                                      // per = log2(e) / T
    unsigned top_key;
    int bits;
    // 2^r by its series, ln(2)^k / k!, the first term left out under 2^-47
    __device__ __forceinline__ double scaled(unsigned key, int lift) const {
        if (key == top_key) return ldexp(1.0, lift);
        constexpr double magic = 6755399441055744.0;      // 1.5 * 2^52: adding it rounds to whole numbers
        double y = ((double)logit_of(key) - top) * per;
        y = fmax(y, -1020.0);                             // (-inf too, and NaN of two infinities)
        const double n = (y + magic) - magic, r = y - n;
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
        return ldexp(s, (int)n + lift);
    }
    __device__ __forceinline__ uint64_t mass(unsigned key) const { return (uint64_t)__builtin_rint(scaled(key, bits)); }
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

// sums over the lanes in front of this one, and this one
__device__ __forceinline__ uint64_t wave_scan(uint64_t v, int lane) {
#pragma unroll
    for (int d = 1; d < 64; d *= 2) {
        const uint64_t o = __shfl_up(v, d);
        if (lane >= d) v += o;
    }
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
__device__ void fill(Histogram& h, const void* row, int V, const Weights& w, int level, unsigned prefix) {
    for (int i = threadIdx.x; i < DIGITS; i += THREADS) { h.count[i] = 0; h.mass[i] = 0; }
    __syncthreads();
    const int shift = shift_of(level), above = level == 0 ? 32 : shift_of(level - 1);
    for_each<F32>(row, V, [&](int, float z) {
        const unsigned key = key_of(z);
        if (key <= LOWEST || (above < 32 && key >> above != prefix >> above)) return;
        const unsigned digit = key >> shift & (DIGITS - 1);
        atomicAdd(&h.count[digit], 1);
        atomicAdd(&h.mass[digit], (unsigned long long)w.mass(key));
    });
    __syncthreads();
}

// The digit, counted from the highest, in which the goal is reached; behind[] get what lies in front of it.
__device__ int descend(Shared& s, const Histogram& h, Goal goal, uint64_t target, int key_digit, uint64_t& count, uint64_t& mass) {
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int hi = DIGITS - 1 - 2 * tid, lo = hi - 1;      // this thread's digits
    const uint64_t c0 = h.count[hi], c1 = h.count[lo], m0 = h.mass[hi], m1 = h.mass[lo];
    const uint64_t c = wave_scan(c0 + c1, lane), m = wave_scan(m0 + m1, lane);
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
__device__ Place find(Shared& s, const void* row, int V, const Weights& w, Goal goal, uint64_t target, unsigned key = 0) {
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
    p.each = w.mass(p.key);
    __syncthreads();
    if (goal == BY_KEY) p.nth = p.equal;
    else if (goal == BY_COUNT) p.nth = (int)(target - count);
    else p.nth = (int)((target - mass + p.each - 1) / p.each);
    return p;
}

template <bool F32>
__global__ __launch_bounds__(THREADS) void sample_row_kernel(SampleArgs a) {
    __shared__ Shared s;
    const int b = blockIdx.x, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, V = a.V;
    const void* row = F32 ? (const void*)(static_cast<const float*>(a.logits) + b * a.ldl) : (const void*)(static_cast<const uint16_t*>(a.logits) + b * a.ldl);
    // the likeliest token: the highest key, of equal ones the lowest index
    uint64_t best = 0;
    for_each<F32>(row, V, [&](int i, float z) {
        const uint64_t v = (uint64_t)key_of(z) << 32 | (unsigned)~i;
        best = v > best ? v : best;
    });
    if (tid == 0) s.top = 0;
    __syncthreads();
    atomicMax((unsigned long long*)&s.top, (unsigned long long)best);
    __syncthreads();
    best = s.top;
    const float T = a.temperature ? a.temperature[b] : 1.0f;
    const unsigned top_key = (unsigned)(best >> 32);
    if (top_key <= LOWEST || !(T > 0.0f)) {                // no token at all, or the likeliest
        if (tid == 0) {
            const bool none = top_key <= LOWEST;
            a.token[b] = none ? -1 : (int)~(unsigned)best;
            if (a.logprob) a.logprob[b] = none ? -__builtin_inff() : 0.0f;
            if (a.kept) a.kept[b] = none ? 0 : 1;
        }
        return;
    }
    Weights w;
    w.top = (double)logit_of(top_key);
    w.per = 1.4426950408889634 / (double)T;
    w.top_key = top_key;
    w.bits = a.bits;
    fill<F32>(s.first, row, V, w, 0, 0);
    uint64_t all_count = 0, all_mass = 0;
    {
        uint64_t c = 0, m = 0;
        for (int i = tid; i < DIGITS; i += THREADS) { c += s.first.count[i]; m += s.first.mass[i]; }
        c = wave_scan(c, lane); m = wave_scan(m, lane);
        if (lane == 63) { s.wave_counts[wave] = c; s.wave_masses[wave] = m; }
        __syncthreads();
        for (int i = 0; i < WAVES; ++i) { all_count += s.wave_counts[i]; all_mass += s.wave_masses[i]; }
        __syncthreads();
    }
    uint64_t kept = all_count, mass = all_mass;
    const int k = a.top_k ? a.top_k[b] : 0;
    const float p = a.top_p ? a.top_p[b] : 1.0f, least = a.min_p ? a.min_p[b] : 0.0f;
    if (k > 0 && (uint64_t)k < kept) {
        const Place at = find<F32>(s, row, V, w, BY_COUNT, (uint64_t)k);
        kept = at.tokens();
        mass = at.total();
    }
    if (p < 1.0f) {
        const double t = __builtin_ceil((double)p * (double)mass);
        uint64_t target = t >= 1.0 ? (uint64_t)t : 1;
        target = target < mass ? target : mass;
        const Place at = find<F32>(s, row, V, w, BY_MASS, target);
        if ((uint64_t)at.tokens() < kept) { kept = at.tokens(); mass = at.total(); }
    }
    if (least > 0.0f) {
        // the lowest key whose weight is enough, by bisection: weights rise with keys
        const double enough = least < 1.0f ? (double)least : 1.0;
        unsigned lo = LOWEST, hi = top_key;                // (hi is enough; lo is not, or is no token)
        while (hi - lo > 1) {
            const unsigned mid = lo + (hi - lo) / 2;
            if (w.scaled(mid, 0) >= enough) hi = mid; else lo = mid;
        }
        if (!F32) hi = hi & 0x80000000u ? (hi + 0xFFFFu) & 0xFFFF0000u : hi | 0xFFFFu;          // (the next bf16 number)
        const Place at = find<F32>(s, row, V, w, BY_KEY, 0, hi);
        if ((uint64_t)at.tokens() < kept) { kept = at.tokens(); mass = at.total(); }
    }
    const double u = a.u[b];
    const double t = u > 0.0 ? u * (double)mass : 0.0;
    uint64_t target = t < 9.0e18 ? (uint64_t)t + 1 : mass;
    target = target < mass ? target : mass;
    const Place at = find<F32>(s, row, V, w, BY_MASS, target);
    // the nth token with that key: the part of the row that holds it, then the token
    const int part = (V + DIGITS - 1) / DIGITS;
    for (int i = tid; i < DIGITS; i += THREADS) s.next.count[i] = 0;
    __syncthreads();
    for_each<F32>(row, V, [&](int i, float z) { if (key_of(z) == at.key) atomicAdd(&s.next.count[DIGITS - 1 - i / part], 1); });
    for (int i = tid; i < DIGITS; i += THREADS) s.next.mass[i] = 0;
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
        if (lane == 0) {
            a.token[b] = token;
            if (a.logprob) {
                const double d = at.key == top_key ? 0.0 : (w.top - (double)logit_of(at.key)) / (double)T;
                a.logprob[b] = (float)(-d - log(ldexp((double)mass, -w.bits)));
            }
            if (a.kept) a.kept[b] = (int)kept;
        }
    }
}

}  // namespace

size_t sample_workspace_bytes(int32_t, int32_t) { return 0; }

int launch_sample(SampleArgs a, hipStream_t s) {
    int log2 = 0;
    while ((1ll << log2) < a.V) ++log2;
    a.bits = 62 - log2 < 50 ? 62 - log2 : 50;
    if (a.f32) hipLaunchKernelGGL(sample_row_kernel<true>, dim3(a.B), dim3(THREADS), 0, s, a);
    else hipLaunchKernelGGL(sample_row_kernel<false>, dim3(a.B), dim3(THREADS), 0, s, a);
    return check_hip(hipGetLastError(), "sample launch");
}

}  // namespace basq
