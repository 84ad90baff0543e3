// C-ABI layer of the operators around the linear layer of a transformer block: norm, rotary positions and cache, attention over
// it.  Argument validation, error text, dispatch; no arithmetic.
#include "basq_internal.h"

#include <math.h>

namespace basq {
namespace {

bool aligned(const void* p, uintptr_t to) { return (reinterpret_cast<uintptr_t>(p) & (to - 1)) == 0; }

int check_rows(const char* name, const void* p, int64_t ld, int64_t width) {
    if (!p) return fail(BASQ_EINVAL, "%s is null", name);
    if (!aligned(p, 16)) return fail(BASQ_EINVAL, "%s must be 16-byte aligned", name);
    if (ld < width || ld % 8 != 0) return fail(BASQ_EINVAL, "the row stride of %s must be >= %lld and a multiple of 8 (got %lld)", name, (long long)width, (long long)ld);
    return BASQ_OK;
}

int check_heads(int32_t heads, int32_t kv_heads, int32_t head_dim, bool kv_needed) {
    if (head_dim != 64 && head_dim != 128) return fail(BASQ_EUNSUPPORTED, "head_dim must be 64 or 128 (got %d)", head_dim);
    if (heads < 0 || kv_heads < 0 || heads + (int64_t)kv_heads > 65536) return fail(BASQ_EINVAL, "heads and kv_heads must be >= 0, at most 65536 together (got %d, %d)", heads, kv_heads);
    if (kv_needed && (heads < 1 || kv_heads < 1 || heads % kv_heads != 0))
        return fail(BASQ_EINVAL, "heads must be a multiple of kv_heads (got %d, %d)", heads, kv_heads);
    return BASQ_OK;
}

int check_cache(const void* cache, int32_t num_pages, int32_t page_size, int32_t* page_log2) {
    if (page_size < 16 || page_size > 1024 || (page_size & (page_size - 1)) != 0)
        return fail(BASQ_EUNSUPPORTED, "page_size must be a power of two from 16 to 1024 (got %d)", page_size);
    if (!cache) return fail(BASQ_EINVAL, "cache is null");
    if (!aligned(cache, 16)) return fail(BASQ_EINVAL, "cache must be 16-byte aligned");
    if (num_pages < 1 || (int64_t)num_pages * page_size > 0x7FFFFFFFll)
        return fail(BASQ_EINVAL, "num_pages must be >= 1, with fewer than 2^31 tokens in all pages (got %d pages of %d)", num_pages, page_size);
    *page_log2 = __builtin_ctz((unsigned)page_size);
    return BASQ_OK;
}

int64_t attention_segments(int32_t B, int32_t q_len, int32_t heads, int32_t kv_heads) {
    return (int64_t)B * kv_heads * (((int64_t)(heads / kv_heads) * q_len + 15) / 16);
}

// (the kernel counts tokens in 32 bits: a little room above the longest context, and below zero for what new tokens do not see)
bool attention_counts(int32_t q_len, int32_t heads, int32_t max_len) {
    return q_len <= 32768 && (int64_t)q_len * heads <= 0x3FFFFFFFll && max_len <= 0x7FFF0000;
}

// parts of 16 rows of D sums with their reference and sum, and a segment's place (PagedAttentionArgs)
size_t parts_bytes(int32_t workers, int32_t head_dim, int64_t segments) {
    return workers > 0 ? 2 * (size_t)workers * 16 * (4 * (size_t)head_dim + 8) + 8 * (size_t)segments : 0;
}

}  // namespace
}  // namespace basq

using namespace basq;

extern "C" {

int basq_add_rms_norm(const void* X, const void* residual, const void* weight, int64_t M, int32_t K, int64_t ldx, int64_t ldr,
                      float eps, void* res_out, int64_t ldro, void* Y, int64_t ldy, uint8_t* Y8, int64_t ldy8, float* y8_scale,
                      void* stream) {
    if (M < 0 || M > 0x7FFFFFFFll) return fail(BASQ_EINVAL, "M must be 0 .. 2^31 - 1 (got %lld)", (long long)M);
    if (K <= 0 || K % 8 != 0) return fail(BASQ_EINVAL, "K must be a positive multiple of 8 (got %d)", K);
    if (K > 32768) return fail(BASQ_EUNSUPPORTED, "K up to 32768 is supported (got %d)", K);
    if (!(eps >= 0.0f)) return fail(BASQ_EINVAL, "eps must be >= 0 (got %g)", (double)eps);
    if (M == 0) return BASQ_OK;
    int rc = check_rows("X", X, ldx, K);
    if (rc == BASQ_OK && residual) rc = check_rows("residual", residual, ldr, K);
    if (rc == BASQ_OK) rc = check_rows("weight", weight, K, K);
    if (rc == BASQ_OK && res_out) rc = check_rows("res_out", res_out, ldro, K);
    if (rc == BASQ_OK && Y) rc = check_rows("Y", Y, ldy, K);
    if (rc == BASQ_OK && Y8) {
        if (!aligned(Y8, 8)) rc = fail(BASQ_EINVAL, "Y8 must be 8-byte aligned");
        else if (ldy8 < K || ldy8 % 8 != 0) rc = fail(BASQ_EINVAL, "ldy8 must be >= K and a multiple of 8 (got %lld)", (long long)ldy8);
        else if (!y8_scale || !aligned(y8_scale, 4)) rc = fail(BASQ_EINVAL, "y8_scale is null or not 4-byte aligned");
    }
    if (rc != BASQ_OK) return rc;
    if (!Y && !Y8) return fail(BASQ_EINVAL, "Y and Y8 are both null");
    RmsNormArgs a{static_cast<const uint16_t*>(X), static_cast<const uint16_t*>(residual), static_cast<const uint16_t*>(weight),
                  static_cast<uint16_t*>(res_out), static_cast<uint16_t*>(Y), Y8, y8_scale, M, K, ldx, ldr, ldro, ldy, ldy8, eps};
    return launch_add_rms_norm(a, static_cast<hipStream_t>(stream));
}

int basq_rope_table(int32_t rot_dim, int64_t positions, double base, int32_t scaling, double factor, double low, double high,
                    double original_len, float* cos_sin, void* stream) {
    if (rot_dim < 2 || rot_dim % 2 != 0 || rot_dim > 1024) return fail(BASQ_EINVAL, "rot_dim must be even, 2 .. 1024 (got %d)", rot_dim);
    if (positions < 0) return fail(BASQ_EINVAL, "positions must be >= 0 (got %lld)", (long long)positions);
    if (!(base > 1.0) || !isfinite(base)) return fail(BASQ_EINVAL, "base must be > 1 (got %g)", base);
    if (scaling < BASQ_ROPE_PLAIN || scaling > BASQ_ROPE_YARN) return fail(BASQ_EUNSUPPORTED, "unknown scaling %d", scaling);
    if (scaling != BASQ_ROPE_PLAIN && (!(factor > 0.0) || !isfinite(factor))) return fail(BASQ_EINVAL, "factor must be > 0 (got %g)", factor);
    if (scaling >= BASQ_ROPE_BANDS && (!(low > 0.0) || !(high > low) || !isfinite(high) || !(original_len > 0.0) || !isfinite(original_len)))
        return fail(BASQ_EINVAL, "0 < low < high and original_len > 0 are needed (got %g, %g, %g)", low, high, original_len);
    if (positions > 0 && (!cos_sin || !aligned(cos_sin, 4))) return fail(BASQ_EINVAL, "cos_sin is null or not 4-byte aligned");
    return launch_rope_table(cos_sin, positions, rot_dim, RopeScaling{scaling, base, factor, low, high, original_len}, static_cast<hipStream_t>(stream));
}

size_t basq_kv_page_bytes(int32_t kv_heads, int32_t head_dim, int32_t page_size) {
    if (kv_heads < 1 || kv_heads > 65536 || (head_dim != 64 && head_dim != 128) || page_size < 16 || page_size > 1024 || (page_size & (page_size - 1)) != 0) return 0;
    return (size_t)kv_heads * (size_t)page_size * (size_t)(head_dim + 16);
}

int basq_rope_append(const void* q, int64_t ldq, const void* k, int64_t ldk, const void* v, int64_t ldv, int64_t T, int32_t heads,
                     int32_t kv_heads, int32_t head_dim, const int32_t* positions, const float* cos_sin, int64_t table_rows,
                     int32_t rot_dim, int32_t interleaved, int32_t rotate, float clip_lo, float clip_hi, int32_t bits,
                     const int32_t* slots, uint8_t* cache, int32_t num_pages, int32_t page_size, void* q_out, int64_t ldqo,
                     void* k_hat, void* v_hat, int64_t ldh, void* stream) {
    if (T < 0) return fail(BASQ_EINVAL, "T must be >= 0 (got %lld)", (long long)T);
    int rc = check_heads(heads, kv_heads, head_dim, false);
    if (rc != BASQ_OK) return rc;
    if (bits != 4) return fail(BASQ_EUNSUPPORTED, "only bits == 4 is implemented (got %d)", bits);
    if (heads == 0 && kv_heads == 0) return fail(BASQ_EINVAL, "no heads at all");
    RopeAppendArgs a{};
    a.page_log2 = 4;
    if (cos_sin) {
        if (rot_dim < 16 || rot_dim > head_dim || rot_dim % 16 != 0)
            return fail(BASQ_EUNSUPPORTED, "rot_dim must be a multiple of 16 up to head_dim (got %d)", rot_dim);
        if (!aligned(cos_sin, 16)) return fail(BASQ_EINVAL, "cos_sin must be 16-byte aligned");
        if (table_rows < 1) return fail(BASQ_EINVAL, "table_rows must be >= 1 (got %lld)", (long long)table_rows);
    }
    if (kv_heads > 0) {
        if (!(clip_lo > 0.0f) || !(clip_hi > 0.0f) || !(clip_lo <= 1.0f) || !(clip_hi <= 1.0f))
            return fail(BASQ_EINVAL, "clip ratios must be in (0, 1] (got %g, %g)", (double)clip_lo, (double)clip_hi);
        if (!cache && !k_hat && !v_hat) return fail(BASQ_EINVAL, "cache, k_hat and v_hat are all null");
        if (cache) {
            rc = check_cache(cache, num_pages, page_size, &a.page_log2);
            if (rc != BASQ_OK) return rc;
        }
    }
    if (T == 0) return BASQ_OK;
    if (cos_sin && (!positions || !aligned(positions, 4))) return fail(BASQ_EINVAL, "positions is null or not 4-byte aligned");
    if (kv_heads > 0 && cache && (!slots || !aligned(slots, 4))) return fail(BASQ_EINVAL, "slots is null or not 4-byte aligned");
    if (heads > 0) {
        rc = check_rows("q", q, ldq, (int64_t)heads * head_dim);
        if (rc == BASQ_OK) rc = check_rows("q_out", q_out, ldqo, (int64_t)heads * head_dim);
    }
    if (rc == BASQ_OK && kv_heads > 0) {
        const int64_t width = (int64_t)kv_heads * head_dim;
        rc = check_rows("k", k, ldk, width);
        if (rc == BASQ_OK) rc = check_rows("v", v, ldv, width);
        if (rc == BASQ_OK && k_hat) rc = check_rows("k_hat", k_hat, ldh, width);
        if (rc == BASQ_OK && v_hat) rc = check_rows("v_hat", v_hat, ldh, width);
    }
    if (rc != BASQ_OK) return rc;
    a.q = static_cast<const uint16_t*>(q); a.k = static_cast<const uint16_t*>(k); a.v = static_cast<const uint16_t*>(v);
    a.T = T; a.ldq = ldq; a.ldk = ldk; a.ldv = ldv;
    a.heads = heads; a.kv_heads = kv_heads; a.D = head_dim;
    a.positions = positions; a.cos_sin = cos_sin; a.table_rows = table_rows;
    a.rot = rot_dim; a.interleaved = interleaved != 0; a.rotate = rotate != 0;
    a.norm = (float)(1.0 / sqrt((double)head_dim));
    a.slots = kv_heads > 0 && cache ? slots : nullptr;
    a.cache = cache; a.num_pages = num_pages;
    a.clip_lo = clip_lo; a.clip_hi = clip_hi;
    a.q_out = static_cast<uint16_t*>(q_out); a.ldqo = ldqo;
    a.k_hat = static_cast<uint16_t*>(k_hat); a.v_hat = static_cast<uint16_t*>(v_hat); a.ldh = ldh;
    return launch_rope_append(a, static_cast<hipStream_t>(stream));
}

size_t basq_paged_attention_workspace_bytes(int32_t B, int32_t q_len, int32_t heads, int32_t kv_heads, int32_t head_dim,
                                            int32_t max_len, int32_t window) {
    if (B < 1 || q_len < 1 || heads < 1 || kv_heads < 1 || heads % kv_heads != 0 || (head_dim != 64 && head_dim != 128) || max_len < 0 || window < 0) return 0;
    if (heads + (int64_t)kv_heads > 65536 || !attention_counts(q_len, heads, max_len)) return 0;
    const int workers = paged_attention_most_workers(B, q_len, heads, kv_heads, head_dim, max_len, window);
    return parts_bytes(workers, head_dim, attention_segments(B, q_len, heads, kv_heads));
}

int basq_paged_attention(const void* q, int64_t ldq, int32_t B, int32_t q_len, int32_t heads, int32_t kv_heads, int32_t head_dim,
                         int32_t bits, const uint8_t* cache, int32_t num_pages, int32_t page_size, const int32_t* page_table,
                         int64_t table_stride, const int32_t* lengths, int32_t max_len, float scale, float softcap, int32_t window,
                         void* out, int64_t ldo, float* lse, void* workspace, size_t workspace_bytes, void* stream) {
    if (B < 0 || q_len < 1) return fail(BASQ_EINVAL, "B must be >= 0 and q_len >= 1 (got %d, %d)", B, q_len);
    int rc = check_heads(heads, kv_heads, head_dim, true);
    if (rc != BASQ_OK) return rc;
    if (!attention_counts(q_len, heads, max_len))
        return fail(BASQ_EUNSUPPORTED, "q_len up to 32768, q_len * heads < 2^30 and max_len up to 2^31 - 2^16 are supported (got %d, %d, %d)", q_len, heads, max_len);
    if (bits != 4) return fail(BASQ_EUNSUPPORTED, "only bits == 4 is implemented (got %d)", bits);
    if (max_len < 0) return fail(BASQ_EINVAL, "max_len must be >= 0 (got %d)", max_len);
    if (!isfinite(scale)) return fail(BASQ_EINVAL, "scale must be finite (got %g)", (double)scale);
    if (!(softcap >= 0.0f) || !isfinite(softcap)) return fail(BASQ_EINVAL, "softcap must be >= 0 and finite (got %g)", (double)softcap);
    if (window < 0) return fail(BASQ_EINVAL, "window must be >= 0 (got %d)", window);
    PagedAttentionArgs a{};
    rc = check_cache(cache, num_pages, page_size, &a.page_log2);
    if (rc != BASQ_OK) return rc;
    if (table_stride < 0 || (max_len + (int64_t)page_size - 1) / page_size > table_stride)
        return fail(BASQ_EINVAL, "a row of the page table holds %lld pages of %d tokens, fewer than max_len = %d", (long long)table_stride, page_size, max_len);
    if (B == 0) return BASQ_OK;
    rc = check_rows("q", q, ldq, (int64_t)heads * head_dim);
    if (rc == BASQ_OK) rc = check_rows("out", out, ldo, (int64_t)heads * head_dim);
    if (rc != BASQ_OK) return rc;
    if ((max_len > 0 && !page_table) || !lengths || !aligned(page_table, 4) || !aligned(lengths, 4) || !aligned(lse, 4))
        return fail(BASQ_EINVAL, "page_table and lengths must be given; they and lse must be 4-byte aligned");
    const AttentionPlan plan = paged_attention_plan(B, q_len, heads, kv_heads, head_dim, max_len, window, softcap > 0.0f);
    a.workers = plan.workers;
    a.waves = plan.waves;
    if (a.workers < 0) return fail(BASQ_EUNSUPPORTED, "2^31 or more parts of 128 tokens, or rows of a head");
    const size_t need = parts_bytes(a.workers, head_dim, attention_segments(B, q_len, heads, kv_heads));
    if (need > 0) {
        if (!workspace || !aligned(workspace, 256)) return fail(BASQ_EINVAL, "workspace is null or not 256-byte aligned");
        if (workspace_bytes < need) return fail(BASQ_EWORKSPACE, "workspace too small: %zu bytes given, %zu needed", workspace_bytes, need);
    }
    a.q = static_cast<const uint16_t*>(q); a.ldq = ldq;
    a.B = B; a.q_len = q_len; a.heads = heads; a.kv_heads = kv_heads; a.D = head_dim;
    a.cache = cache; a.num_pages = num_pages;
    a.page_table = page_table; a.table_stride = table_stride; a.lengths = lengths; a.max_len = max_len;
    a.scale = scale; a.softcap = softcap;
    a.window = window < max_len ? window : 0;                     // (a window of all tokens is none)
    a.out = static_cast<uint16_t*>(out); a.ldo = ldo; a.lse = lse;
    a.part_o = static_cast<float*>(workspace);
    a.part_ml = reinterpret_cast<float2*>(a.part_o + 2 * (size_t)a.workers * 16 * head_dim);
    a.part_of = reinterpret_cast<int2*>(a.part_ml + 2 * (size_t)a.workers * 16);
    return launch_paged_attention(a, static_cast<hipStream_t>(stream));
}

}  // extern "C"
