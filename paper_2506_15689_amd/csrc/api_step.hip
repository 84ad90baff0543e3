// C-ABI layer of the ends of a step: products and lookups of 4-bit weights with group scales, sampled tokens, the books of the
// paged cache.  Argument validation, error text, dispatch; no arithmetic.
#include "basq_internal.h"

#include <math.h>

namespace basq {
namespace {

bool aligned(const void* p, uintptr_t to) { return (reinterpret_cast<uintptr_t>(p) & (to - 1)) == 0; }

int check_matrix(const uint8_t* Wq, int32_t N, int32_t K, int32_t w_layout, const void* w_scale, const void* w_zero, int32_t* group) {
    if (N < 1) return fail(BASQ_EINVAL, "N must be >= 1 (got %d)", N);
    if (K < 32 || K % 32 != 0) return fail(BASQ_EINVAL, "K must be a positive multiple of 32 (got %d)", K);
    if (K > 1 << 20) return fail(BASQ_EUNSUPPORTED, "K up to 2^20 is supported (got %d)", K);
    if (N > 1 << 28) return fail(BASQ_EUNSUPPORTED, "N up to 2^28 is supported (got %d)", N);
    if (w_layout != BASQ_W_CANONICAL && w_layout != BASQ_W_DECODE16) return fail(BASQ_EINVAL, "unknown w_layout %d", w_layout);
    if (w_layout == BASQ_W_DECODE16 && K % 128 != 0) return fail(BASQ_EINVAL, "the streaming layout needs K %% 128 == 0 (got %d)", K);
    if (*group == 0) *group = K;
    if (*group < 32 || *group % 32 != 0 || K % *group != 0) return fail(BASQ_EINVAL, "group_size must be a multiple of 32 that divides K = %d (got %d)", K, *group);
    if (!Wq || !aligned(Wq, 16)) return fail(BASQ_EINVAL, "Wq is null or not 16-byte aligned");
    if (!w_scale || !w_zero || !aligned(w_scale, 2) || !aligned(w_zero, 2)) return fail(BASQ_EINVAL, "w_scale and w_zero must be given, 2-byte aligned");
    return BASQ_OK;
}

int check_ints(const char* name, const void* p, bool needed) {
    if (!p && needed) return fail(BASQ_EINVAL, "%s is null", name);
    if (!aligned(p, 4)) return fail(BASQ_EINVAL, "%s must be 4-byte aligned", name);
    return BASQ_OK;
}

}  // namespace
}  // namespace basq

using namespace basq;

extern "C" {

int basq_w4a16_gemm(const void* X, int64_t M, int32_t K, int64_t ldx, const uint8_t* Wq, int32_t N, int32_t w_layout,
                    const void* w_scale, const void* w_zero, int32_t group_size, const float* bias, void* Y, int64_t ldy,
                    int32_t y_f32, void* stream) {
    if (M < 0) return fail(BASQ_EINVAL, "M must be >= 0 (got %lld)", (long long)M);
    if (M > W4A16_MAX_TOKENS) return fail(BASQ_EUNSUPPORTED, "M up to %lld is supported (got %lld)", (long long)W4A16_MAX_TOKENS, (long long)M);
    const int rc = check_matrix(Wq, N, K, w_layout, w_scale, w_zero, &group_size);
    if (rc != BASQ_OK) return rc;
    if (!aligned(bias, 4)) return fail(BASQ_EINVAL, "bias must be 4-byte aligned");
    if (M == 0) return BASQ_OK;
    if (!X || !aligned(X, 16)) return fail(BASQ_EINVAL, "X is null or not 16-byte aligned");
    if (ldx < K || ldx % 8 != 0) return fail(BASQ_EINVAL, "ldx must be >= K and a multiple of 8 (got %lld)", (long long)ldx);
    if (ldx > 1 << 23) return fail(BASQ_EUNSUPPORTED, "ldx up to 2^23 is supported (got %lld)", (long long)ldx);
    if (!Y || !aligned(Y, y_f32 ? 4 : 2)) return fail(BASQ_EINVAL, "Y is null or not aligned as its type is");
    if (ldy < N) return fail(BASQ_EINVAL, "ldy must be >= N (got %lld)", (long long)ldy);
    W4A16Args a{};
    a.X = static_cast<const uint16_t*>(X); a.M = M; a.ldx = ldx; a.K = K; a.N = N;
    a.Wq = Wq; a.w_layout = w_layout;
    a.w_scale = static_cast<const uint16_t*>(w_scale); a.w_zero = static_cast<const uint16_t*>(w_zero);
    a.group = group_size; a.bias = bias;
    a.Y = Y; a.ldy = ldy; a.y_f32 = y_f32 != 0;
    return launch_gemm_w4a16(a, static_cast<hipStream_t>(stream));
}

int basq_w4a16_lookup(const int32_t* ids, int64_t T, const uint8_t* Wq, int32_t N, int32_t K, int32_t w_layout, const void* w_scale,
                      const void* w_zero, int32_t group_size, float scale, void* Y, int64_t ldy, void* stream) {
    if (T < 0 || T > 0x7FFFFFFFll) return fail(BASQ_EINVAL, "T must be 0 .. 2^31 - 1 (got %lld)", (long long)T);
    if (T > 1 << 30) return fail(BASQ_EUNSUPPORTED, "T up to 2^30 is supported (got %lld)", (long long)T);
    int rc = check_matrix(Wq, N, K, w_layout, w_scale, w_zero, &group_size);
    if (rc != BASQ_OK) return rc;
    if (!isfinite(scale)) return fail(BASQ_EINVAL, "scale must be finite (got %g)", (double)scale);
    if (T == 0) return BASQ_OK;
    rc = check_ints("ids", ids, true);
    if (rc != BASQ_OK) return rc;
    if (!Y || !aligned(Y, 16)) return fail(BASQ_EINVAL, "Y is null or not 16-byte aligned");
    if (ldy < K || ldy % 8 != 0) return fail(BASQ_EINVAL, "ldy must be >= K and a multiple of 8 (got %lld)", (long long)ldy);
    LookupArgs a{};
    a.ids = ids; a.T = T; a.Wq = Wq; a.N = N; a.K = K; a.w_layout = w_layout;
    a.w_scale = static_cast<const uint16_t*>(w_scale); a.w_zero = static_cast<const uint16_t*>(w_zero);
    a.group = group_size; a.scale = scale;
    a.Y = static_cast<uint16_t*>(Y); a.ldy = ldy;
    return launch_lookup_w4a16(a, static_cast<hipStream_t>(stream));
}

size_t basq_sample_workspace_bytes(int32_t B, int32_t V) {
    return B < 1 || V < 1 || V > SAMPLE_MAX_TOKENS ? 0 : sample_workspace_bytes(B, V);
}

int basq_sample(const void* logits, int64_t ldl, int32_t B, int32_t V, int32_t f32, const float* temperature, const int32_t* top_k,
                const float* top_p, const float* min_p, const double* u, int32_t* token, float* logprob, int32_t* kept,
                void* workspace, size_t workspace_bytes, void* stream) {
    if (B < 0 || V < 1) return fail(BASQ_EINVAL, "B must be >= 0 and V >= 1 (got %d, %d)", B, V);
    if (V > SAMPLE_MAX_TOKENS) return fail(BASQ_EUNSUPPORTED, "V up to %d is supported (got %d)", SAMPLE_MAX_TOKENS, V);
    if (B == 0) return BASQ_OK;
    if (!logits || !aligned(logits, f32 ? 4 : 2)) return fail(BASQ_EINVAL, "logits are null or not aligned as their type is");
    if (ldl < V && ldl != 0) return fail(BASQ_EINVAL, "ldl must be >= V, or 0 (got %lld)", (long long)ldl);
    int rc = check_ints("temperature", temperature, false);
    if (rc == BASQ_OK) rc = check_ints("top_k", top_k, false);
    if (rc == BASQ_OK) rc = check_ints("top_p", top_p, false);
    if (rc == BASQ_OK) rc = check_ints("min_p", min_p, false);
    if (rc == BASQ_OK) rc = check_ints("token", token, true);
    if (rc == BASQ_OK) rc = check_ints("logprob", logprob, false);
    if (rc == BASQ_OK) rc = check_ints("kept", kept, false);
    if (rc != BASQ_OK) return rc;
    if (!u || !aligned(u, 8)) return fail(BASQ_EINVAL, "u is null or not 8-byte aligned");
    const size_t need = f32 ? sample_workspace_bytes(B, V) : 0;
    if (need > 0) {
        if (!workspace || !aligned(workspace, 256)) return fail(BASQ_EINVAL, "workspace is null or not 256-byte aligned");
        if (workspace_bytes < need) return fail(BASQ_EWORKSPACE, "workspace too small: %zu bytes given, %zu needed", workspace_bytes, need);
    }
    SampleArgs a{};
    a.logits = logits; a.ldl = ldl; a.B = B; a.V = V; a.f32 = f32 != 0;
    a.temperature = temperature; a.top_k = top_k; a.top_p = top_p; a.min_p = min_p; a.u = u;
    a.token = token; a.logprob = logprob; a.kept = kept;
    a.workspace = static_cast<uint8_t*>(workspace);
    return launch_sample(a, static_cast<hipStream_t>(stream));
}

size_t basq_kv_books_bytes(int32_t B) { return B < 0 || B > KV_MAX_SEQUENCES ? 0 : 64 + (size_t)KV_PLAN_BYTES * (size_t)B; }

int basq_kv_extend(const int32_t* lengths, int32_t* pool_table, int64_t pool_stride, int32_t rows, int32_t columns, int32_t page_size,
                   int32_t* free_pages, int32_t capacity, const int32_t* free_count, const int32_t* seqs, const int32_t* new_tokens,
                   int32_t B, int32_t q_len, int32_t* positions, int32_t* slots, int64_t T, int32_t* starts, int32_t* batch_table,
                   int64_t batch_stride, int32_t* batch_lengths, int32_t* lengths_out, int32_t* free_out, int32_t* status,
                   void* books, size_t books_bytes, void* stream) {
    if (B < 0 || q_len < 0 || rows < 0 || columns < 0 || capacity < 0)
        return fail(BASQ_EINVAL, "B, q_len, rows, columns and capacity must be >= 0 (got %d, %d, %d, %d, %d)", B, q_len, rows, columns, capacity);
    if (page_size < 16 || page_size > 1024 || (page_size & (page_size - 1)) != 0)
        return fail(BASQ_EUNSUPPORTED, "page_size must be a power of two from 16 to 1024 (got %d)", page_size);
    if (B > KV_MAX_SEQUENCES) return fail(BASQ_EUNSUPPORTED, "B up to %d is supported (got %d)", KV_MAX_SEQUENCES, B);
    if ((int64_t)B * columns > 0x7FFFFFFFll || (int64_t)columns * page_size > 0x7FFFFFFFll)
        return fail(BASQ_EUNSUPPORTED, "B * columns and columns * page_size below 2^31 are supported (got %d, %d, %d)", B, columns, page_size);
    if (T < 0 || T > 0x7FFFFFFFll) return fail(BASQ_EINVAL, "T must be 0 .. 2^31 - 1 (got %lld)", (long long)T);
    if (q_len > 0 && T != (int64_t)B * q_len) return fail(BASQ_EINVAL, "T must be B * q_len (got %lld, %d, %d)", (long long)T, B, q_len);
    if (q_len > 0 && starts) return fail(BASQ_EINVAL, "starts goes with packed tokens, q_len = 0");
    if (q_len == 0 && B > 0 && !new_tokens) return fail(BASQ_EINVAL, "packed tokens need new_tokens");
    if (!seqs && B > rows) return fail(BASQ_EINVAL, "without seqs, B must be at most the %d rows of the pool (got %d)", rows, B);
    int rc = check_ints("lengths", lengths, B > 0);
    if (rc == BASQ_OK) rc = check_ints("lengths_out", lengths_out, B > 0);
    if (rc == BASQ_OK) rc = check_ints("pool_table", pool_table, B > 0 && columns > 0);
    if (rc == BASQ_OK) rc = check_ints("free_pages", free_pages, capacity > 0);
    if (rc == BASQ_OK) rc = check_ints("free_count", free_count, true);
    if (rc == BASQ_OK) rc = check_ints("free_out", free_out, true);
    if (rc == BASQ_OK) rc = check_ints("status", status, true);
    if (rc == BASQ_OK) rc = check_ints("seqs", seqs, false);
    if (rc == BASQ_OK) rc = check_ints("new_tokens", new_tokens, false);
    if (rc == BASQ_OK) rc = check_ints("positions", positions, T > 0);
    if (rc == BASQ_OK) rc = check_ints("slots", slots, T > 0);
    if (rc == BASQ_OK) rc = check_ints("starts", starts, false);
    if (rc == BASQ_OK) rc = check_ints("batch_table", batch_table, false);
    if (rc == BASQ_OK) rc = check_ints("batch_lengths", batch_lengths, false);
    if (rc != BASQ_OK) return rc;
    if (rows > 1 && pool_stride < columns) return fail(BASQ_EINVAL, "pool_stride must be >= columns (got %lld)", (long long)pool_stride);
    if (batch_table && B > 1 && batch_stride < columns) return fail(BASQ_EINVAL, "batch_stride must be >= columns (got %lld)", (long long)batch_stride);
    if (!books || !aligned(books, 16)) return fail(BASQ_EINVAL, "books is null or not 16-byte aligned");
    if (books_bytes < basq_kv_books_bytes(B)) return fail(BASQ_EWORKSPACE, "books too small: %zu bytes given, %zu needed", books_bytes, basq_kv_books_bytes(B));
    KvExtendArgs a{};
    a.lengths = lengths; a.pool_table = pool_table; a.pool_stride = pool_stride;
    a.rows = rows; a.columns = columns; a.page_log2 = __builtin_ctz((unsigned)page_size);
    a.free_pages = free_pages; a.capacity = capacity; a.free_count = free_count;
    a.seqs = seqs; a.new_tokens = new_tokens; a.B = B; a.q_len = q_len;
    a.positions = positions; a.slots = slots; a.T = T; a.starts = starts;
    a.batch_table = columns > 0 ? batch_table : nullptr; a.batch_stride = batch_stride; a.batch_lengths = batch_lengths;
    a.lengths_out = lengths_out; a.free_out = free_out; a.status = status;
    a.plan = static_cast<uint8_t*>(books);
    return launch_kv_extend(a, static_cast<hipStream_t>(stream));
}

}  // extern "C"
