// The books of a paged cache, kept on the GPU: pages for new tokens, the pages of tokens that go, and with them the places that
// append and attention take -- so that a step needs no copy from the host and one captured graph serves all of them.  Whole
// numbers only; the definition is beside basq_kv_extend in basq.h.
//
// A thread to a sequence looks it over, and one scan over the workgroup of the pages that are wanted, that go back and of the new
// tokens gives each its place in all three.  The order is fixed: pages that go back lie on the free ones in the order of the
// sequences, then pages are taken from the end in the order of the sequences; so the books do not depend on how threads run.  Either
// all of it is done or, with a status, nothing.
//
// Bound by the latency of a chain: what is known of a sequence, its page, its token.  Few tokens are placed by the same workgroup
// (64 sequences, one token each: 5.0 us); many, or many sequences, by a second launch that fills the chip (48 packed prompts of up to 4096
// tokens on pages of 16: 3.4 + 6.0).
#include "basq_internal.h"
#include "lane_ops.h"

namespace basq {

namespace {

constexpr int THREADS = 1024, WAVES = THREADS / 64;
constexpr int HASH = 2 * KV_MAX_SEQUENCES;

// one sequence of the plan
struct Seq {
    int row;                  // of the pool
    int before, plus;         // tokens in front of the new ones, new ones
    int start;                // packed: the first of them
    int had, need;            // pages
    int taken, back;          // pages that sequences in front of this one take, and give back
};
static_assert(sizeof(Seq) == KV_PLAN_BYTES, "");

__device__ __forceinline__ int pages_of(int64_t tokens, int log2) { return (int)((tokens + (1ll << log2) - 1) >> log2); }

// The page of column c of a sequence: one that it had, or from the end of the `top` free ones (with those that go back).  Not by way of the
// table, which a neighbour may not have written yet.
__device__ __forceinline__ int page_at(const KvExtendArgs& a, const Seq& p, int c, int top) {
    return c < p.had ? a.pool_table[p.row * a.pool_stride + c] : a.free_pages[top - 1 - (p.taken + c - p.had)];
}
// token t: its position and slot
__device__ __forceinline__ void place(const KvExtendArgs& a, const Seq* plan, int64_t t, bool good, int top) {
    int position = -1, slot = -1;
    if (good && a.B > 0) {
        int b, i;
        if (a.q_len > 0) {
            b = (int)(t / a.q_len);
            i = (int)(t - (int64_t)b * a.q_len) - (a.q_len - plan[b].plus);
        } else {
            // the last sequence that starts at t or in front of it: sequences without new tokens start where the next one does
            int lo = 0, hi = a.B;
            while (hi - lo > 1) {
                const int mid = (lo + hi) >> 1;
                if (plan[mid].start <= t) lo = mid; else hi = mid;
            }
            b = lo;
            i = (int)t - plan[b].start;
        }
        const Seq p = plan[b];
        if (i >= 0 && i < p.plus) {
            position = p.before + i;
            const int64_t page = page_at(a, p, position >> a.page_log2, top);
            const int64_t s = (page << a.page_log2) + (position & ((1 << a.page_log2) - 1));
            slot = page >= 0 && s <= 0x7FFFFFFFll ? (int)s : -1;
        }
    }
    a.positions[t] = position;
    a.slots[t] = slot;
}
// row b of the pool's table, and of the batch's, by one wave
__device__ __forceinline__ void write_row(const KvExtendArgs& a, const Seq& p, int b, int lane, int top) {
    int32_t *own = a.pool_table + p.row * a.pool_stride, *to = a.batch_table ? a.batch_table + b * a.batch_stride : nullptr;
    for (int c = (to ? 0 : p.had) + lane; c < p.need; c += 64) {
        const int page = page_at(a, p, c, top);
        if (c >= p.had) own[c] = page;
        if (to) to[c] = page;
    }
}

__global__ __launch_bounds__(THREADS) void kv_plan_kernel(KvExtendArgs a) {
    __shared__ Seq plan[KV_MAX_SEQUENCES];
    __shared__ int hash[HASH], first[HASH];              // rows, and which sequence of the batch names each first
    __shared__ uint64_t pages_at[WAVES], tokens_at[WAVES];
    __shared__ int fault;
    const int b = threadIdx.x, lane = b & 63, wave = b >> 6;
    constexpr int NONE = 0x7FFFFFFF;
    const int64_t most = (int64_t)a.columns << a.page_log2;
    int row = -1, fresh = 0, before = 0, had = 0, need = 0, wrong = 0;
    const int count = a.free_count[0];
    if (b < a.B) {
        row = a.seqs ? a.seqs[b] : b;
        fresh = a.new_tokens ? a.new_tokens[b] : a.q_len;
        if (row >= 0 && row < a.rows) before = a.lengths[row];
    }
    for (int i = b; i < HASH; i += THREADS) { hash[i] = -1; first[i] = NONE; }
    if (b == 0) fault = NONE;
    __syncthreads();

    uint64_t pages = 0, tokens = 0;                      // (more pages low, pages back high)
    unsigned entry = HASH;
    if (b < a.B) {
        if (row < 0 || row >= a.rows) {
            wrong = BASQ_KV_SEQUENCE;
        } else {
            const int64_t after = (int64_t)before + fresh;
            if (before < 0 || before > most || after < 0 || after > most || (a.q_len > 0 && fresh > a.q_len)) wrong = BASQ_KV_LENGTH;
            // at most B entries of twice as many places: a free one is found
            for (entry = (unsigned)row * 2654435761u % HASH;; entry = (entry + 1) % HASH) {
                const int seen = atomicCAS(&hash[entry], -1, row);
                if (seen == -1 || seen == row) break;
            }
            atomicMin(&first[entry], b);
            if (!wrong) {
                had = pages_of(before, a.page_log2);
                need = pages_of(after, a.page_log2);
                pages = need > had ? (uint64_t)(need - had) : (uint64_t)(had - need) << 32;
                tokens = fresh > 0 ? (uint64_t)fresh : 0;
            }
        }
    }
    __syncthreads();
    if (entry < HASH && first[entry] != b) wrong = BASQ_KV_SEQUENCE;           // (named twice)
    if (wrong) atomicMin(&fault, b * 8 + wrong);
    const uint64_t pages_in = wave_scan(pages), tokens_in = wave_scan(tokens);
    if (lane == 63) { pages_at[wave] = pages_in; tokens_at[wave] = tokens_in; }
    __syncthreads();
    uint64_t pages_before = 0, tokens_before = 0, pages_all = 0, tokens_all = 0;
    const int waves = (a.B + 63) / 64;
    for (int w = 0; w < waves; ++w) {
        const uint64_t p = pages_at[w], t = tokens_at[w];
        if (w < wave) { pages_before += p; tokens_before += t; }
        pages_all += p;
        tokens_all += t;
    }
    const int64_t more = (int64_t)(pages_all & 0xFFFFFFFFull), less = (int64_t)(pages_all >> 32);
    int code = 0, detail = 0;
    if (fault != NONE) { code = fault & 7; detail = fault >> 3; }
    else if (count < 0 || count + less > a.capacity) { code = BASQ_KV_FREE; detail = count; }
    else if (more > count + less) { code = BASQ_KV_PAGES; detail = (int)(more - count - less); }
    else if (a.q_len == 0 && (int64_t)tokens_all > a.T) { code = BASQ_KV_TOKENS; detail = (int)((int64_t)tokens_all - a.T > NONE ? NONE : (int64_t)tokens_all - a.T); }
    const bool good = code == 0;
    if (b < a.B) {
        const uint64_t p = pages_before + pages_in - pages, t = tokens_before + tokens_in - tokens;
        plan[b] = Seq{row, before, (int)tokens, (int)t, had, good ? need : 0, (int)(p & 0xFFFFFFFFull), (int)(p >> 32)};
        if (a.plan) reinterpret_cast<Seq*>(a.plan + 64)[b] = plan[b];
        if (good) a.lengths_out[row] = before + fresh;
        if (a.batch_lengths) a.batch_lengths[b] = good ? before + fresh : 0;
        if (a.starts) a.starts[b + 1] = good ? (int)(t + tokens) : 0;
    }
    if (b == 0) {
        if (a.starts) a.starts[0] = 0;
        a.status[0] = code;
        a.status[1] = detail;
        a.free_out[0] = good ? (int)(count + less - more) : count;
        if (a.plan) *reinterpret_cast<int2*>(a.plan) = make_int2(good, (int)(count + less));
    }
    __syncthreads();
    const int top = (int)(count + less);
    if (good && less > 0) {
        for (int i = wave; i < a.B; i += WAVES) {
            const Seq& p = plan[i];
            for (int c = p.need + lane; c < p.had; c += 64) a.free_pages[count + p.back + c - p.need] = a.pool_table[p.row * a.pool_stride + c];
        }
        __syncthreads();
    }
    if (a.plan) return;                                  // (the rest in a launch of its own)
    for (int64_t t = b; t < a.T; t += THREADS) place(a, plan, t, good, top);
    if (good)
        for (int i = wave; i < a.B; i += WAVES) write_row(a, plan[i], i, lane, top);
}

// a workgroup to 256 tokens, then a wave to a row of the table
__global__ __launch_bounds__(256) void kv_place_kernel(KvExtendArgs a, int token_blocks) {
    __shared__ Seq plan[KV_MAX_SEQUENCES];
    const int2 known = *reinterpret_cast<const int2*>(a.plan);
    const bool good = known.x != 0;
    const Seq* kept = reinterpret_cast<const Seq*>(a.plan + 64);
    const int lane = threadIdx.x & 63;
    if ((int)blockIdx.x >= token_blocks) {
        const int b = ((int)blockIdx.x - token_blocks) * 4 + (threadIdx.x >> 6);
        if (good && b < a.B) write_row(a, kept[b], b, lane, known.y);
        return;
    }
    for (int i = threadIdx.x; i < a.B; i += 256) plan[i] = kept[i];
    __syncthreads();
    const int64_t t = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (t < a.T) place(a, plan, t, good, known.y);
}

}  // namespace

int launch_kv_extend(KvExtendArgs a, hipStream_t s) {
    uint8_t* books = a.plan;
    // (one launch, two: one token of 128 sequences 6.5 us and 8.1, of 200 8.6 and 8.0; some 4000 packed tokens of 16 sequences 6.4 and 8.0, 8000 9.0
    // and 8.0)
    const bool one = a.T <= 4096 && a.B <= 128;
    a.plan = one ? nullptr : books;
    hipLaunchKernelGGL(kv_plan_kernel, dim3(1), dim3(THREADS), 0, s, a);
    if (!one) {
        const int token_blocks = (int)((a.T + 255) / 256), row_blocks = (a.B + 3) / 4;
        if (token_blocks + row_blocks > 0) hipLaunchKernelGGL(kv_place_kernel, dim3(token_blocks + row_blocks), dim3(256), 0, s, a, token_blocks);
    }
    return check_hip(hipGetLastError(), "kv_extend launch");
}

}  // namespace basq
