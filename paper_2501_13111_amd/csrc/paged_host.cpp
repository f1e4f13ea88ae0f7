// C entries of the paged cache and of draft verification: argument checks on the host, then one
// launch sequence on the caller's stream.  Nothing here allocates or synchronises, so every call
// may be captured into a graph.  See include/fp.h for the contracts.
#include <cmath>
#include <cstdarg>
#include <cstdio>

#include "fp_internal.h"

using namespace fpk;

namespace {

fp_status fail(fp_status s, const char* fmt, ...) {
    char buf[256];
    va_list ap;
    va_start(ap, fmt);
    vsnprintf(buf, sizeof buf, fmt, ap);
    va_end(ap);
    return report_error(s, buf);
}

bool aligned(const void* p, size_t n) { return (uintptr_t)p % n == 0; }

fp_status done(hipError_t e, const char* what) {
    return e == hipSuccess ? FP_OK : fail(FP_ERR_HIP, "%s launch failed: %s", what, hipGetErrorString(e));
}

// Kernels count positions in int32, up to a few blocks past a sequence's last.
constexpr int MAX_POSITIONS = INT32_MAX - 1023;

fp_status check_shape(const fp_paged_kv* kv, const fp_chunk* c) {
    if (!kv || !c) return fail(FP_ERR_INVALID_ARG, "kv and chunk must not be NULL");
    if (kv->format != FP_KV_BF16 && kv->format != FP_KV_INT8)
        return fail(FP_ERR_INVALID_ARG, "bad kv format %d", kv->format);
    if (kv->n_pages < 1 || kv->n_kv_heads < 1) return fail(FP_ERR_INVALID_ARG, "n_pages and n_kv_heads must be >= 1");
    if (kv->page_size < VT_BLK || kv->page_size % VT_BLK != 0)
        return fail(FP_ERR_INVALID_ARG, "page_size %d is not a positive multiple of %d", kv->page_size, VT_BLK);
    if (kv->page_size > 65536) return fail(FP_ERR_UNSUPPORTED, "page_size %d > 65536", kv->page_size);
    if (kv->head_dim != 64 && kv->head_dim != 128)
        return fail(FP_ERR_UNSUPPORTED, "head_dim %d not supported (64 or 128)", kv->head_dim);
    // block indices are int32
    if ((double)kv->n_pages * kv->n_kv_heads * (kv->page_size / VT_BLK) > 2147483647.0)
        return fail(FP_ERR_UNSUPPORTED, "the pool has 2^31 blocks or more");
    if (c->n_seqs < 1 || c->n_rows < 0 || c->max_new < 1 || c->max_len < 1 || c->table_stride < 1)
        return fail(FP_ERR_INVALID_ARG, "n_seqs, max_new, max_len and table_stride must be >= 1, n_rows >= 0");
    if (c->n_seqs > 4096) return fail(FP_ERR_UNSUPPORTED, "n_seqs %d > 4096", c->n_seqs);
    if (c->n_rows > 1 << 24) return fail(FP_ERR_UNSUPPORTED, "n_rows %d > 2^24", c->n_rows);
    if (c->max_len > (int64_t)c->table_stride * kv->page_size)
        return fail(FP_ERR_CAPACITY, "max_len %d passes the table's %d pages of %d", c->max_len, c->table_stride, kv->page_size);
    if (c->max_len > MAX_POSITIONS) return fail(FP_ERR_UNSUPPORTED, "max_len %d > %d", c->max_len, MAX_POSITIONS);
    return FP_OK;
}

}  // namespace

// The pages' and the chunk's checks, with their pointers' if `pointers`.
fp_status fpk::check_paged(const fp_paged_kv* kv, const fp_chunk* c, bool pointers) {
    if (const fp_status s = check_shape(kv, c)) return s;
    if (!pointers) return FP_OK;
    if (!kv->k || !kv->v || !aligned(kv->k, 16) || !aligned(kv->v, 16))
        return fail(FP_ERR_INVALID_ARG, "k and v pools must be 16-byte aligned device pointers");
    if (kv->format == FP_KV_INT8 && (!kv->k_scales || !kv->v_scales || !aligned(kv->k_scales, 16) || !aligned(kv->v_scales, 16)))
        return fail(FP_ERR_INVALID_ARG, "an int8 cache needs 16-byte aligned k_scales and v_scales");
    if (!c->row_start || !c->ctx_len || !c->table) return fail(FP_ERR_INVALID_ARG, "row_start, ctx_len and table must be device pointers");
    return FP_OK;
}

namespace {

fp_status check_chunk(const fp_paged_kv* kv, const fp_chunk* c) { return check_paged(kv, c, true); }

fp_status check_heads(const fp_paged_kv* kv, int n_heads) {
    if (n_heads < 1 || n_heads % kv->n_kv_heads != 0)
        return fail(FP_ERR_INVALID_ARG, "n_heads %d not a positive multiple of n_kv_heads %d", n_heads, kv->n_kv_heads);
    if (n_heads / kv->n_kv_heads > 16) return fail(FP_ERR_UNSUPPORTED, "query group size %d not supported (1 to 16)", n_heads / kv->n_kv_heads);
    return FP_OK;
}

// a row buffer of bf16: 16-byte aligned rows that hold `width` elements
fp_status check_rows(const char* name, const void* p, int64_t stride, int64_t width) {
    if (!p || !aligned(p, 16)) return fail(FP_ERR_INVALID_ARG, "%s must be a 16-byte aligned device pointer", name);
    if (stride % 8 != 0 || stride < width)
        return fail(FP_ERR_INVALID_ARG, "%s rows are %lld elements apart: a multiple of 8, at least %lld, is needed", name,
                    (long long)stride, (long long)width);
    if (stride > (int64_t)1 << 32) return fail(FP_ERR_UNSUPPORTED, "%s row stride above 2^32", name);
    return FP_OK;
}

bool overlap(const void* a, size_t na, const void* b, size_t nb) {
    return (const char*)a < (const char*)b + nb && (const char*)b < (const char*)a + na;
}

// bytes from the first element of strided rows to the last one's end
size_t rows_bytes(int64_t rows, int64_t stride, int64_t width) { return rows > 0 ? 2 * (size_t)((rows - 1) * stride + width) : 0; }

}  // namespace

extern "C" {

fp_status fp_kv_append(const fp_paged_kv* kv, const fp_chunk* chunk, const void* k, const void* v, int64_t kv_stride,
                       const void* q, int64_t q_stride, int32_t n_heads, void* q_out, const float* cos_t,
                       const float* sin_t, int32_t n_pos, void* stream) {
    fp_status s = check_chunk(kv, chunk);
    if (s) return s;
    const int64_t kw = (int64_t)kv->n_kv_heads * kv->head_dim;
    if ((s = check_rows("k", k, kv_stride, kw)) || (s = check_rows("v", v, kv_stride, kw))) return s;
    if (!cos_t != !sin_t) return fail(FP_ERR_INVALID_ARG, "cos and sin come together");
    if (cos_t && (!aligned(cos_t, 16) || !aligned(sin_t, 16))) return fail(FP_ERR_INVALID_ARG, "cos and sin must be 16-byte aligned");
    if (cos_t && n_pos < chunk->max_len) return fail(FP_ERR_CAPACITY, "%d table positions for max_len %d", n_pos, chunk->max_len);
    if (q || q_out) {
        if (!cos_t) return fail(FP_ERR_INVALID_ARG, "queries are rotated: cos and sin are needed");
        if ((s = check_heads(kv, n_heads))) return s;
        const int64_t qw = (int64_t)n_heads * kv->head_dim;
        if ((s = check_rows("q", q, q_stride, qw)) || (s = check_rows("q_out", q_out, qw, qw))) return s;
        const size_t nq = rows_bytes(chunk->n_rows, qw, qw);
        if (overlap(q, rows_bytes(chunk->n_rows, q_stride, qw), q_out, nq) ||
            overlap(k, rows_bytes(chunk->n_rows, kv_stride, kw), q_out, nq) ||
            overlap(v, rows_bytes(chunk->n_rows, kv_stride, kw), q_out, nq))
            return fail(FP_ERR_INVALID_ARG, "q_out overlaps an input");
    }
    if (chunk->n_rows == 0) return FP_OK;
    KvAppendArgs a{};
    a.kv = *kv;
    a.chunk = *chunk;
    a.k = k;
    a.v = v;
    a.q = q;
    a.kv_stride = kv_stride;
    a.q_stride = q_stride;
    a.ks = 1;
    a.n_heads = n_heads;
    a.q_out = (uint16_t*)q_out;
    a.cos_t = cos_t;
    a.sin_t = sin_t;
    return done(launch_kv_append(a, false, (hipStream_t)stream), "kv append");
}

fp_status fp_kv_read(const fp_paged_kv* kv, const fp_chunk* chunk, void* k_out, void* v_out, void* stream) {
    fp_status s = check_chunk(kv, chunk);
    if (s) return s;
    const int64_t kw = (int64_t)kv->n_kv_heads * kv->head_dim;
    if ((s = check_rows("k_out", k_out, kw, kw)) || (s = check_rows("v_out", v_out, kw, kw))) return s;
    const size_t n = rows_bytes(chunk->n_rows, kw, kw);
    if (overlap(k_out, n, v_out, n)) return fail(FP_ERR_INVALID_ARG, "k_out and v_out overlap");
    if (chunk->n_rows == 0) return FP_OK;
    KvReadArgs a{};
    a.kv = *kv;
    a.chunk = *chunk;
    a.k_out = (uint16_t*)k_out;
    a.v_out = (uint16_t*)v_out;
    return done(launch_kv_read(a, (hipStream_t)stream), "kv read");
}

fp_status fp_attn_chunk_workspace(const fp_paged_kv* kv, const fp_chunk* chunk, int32_t n_heads, size_t* bytes) {
    if (!bytes) return fail(FP_ERR_INVALID_ARG, "bytes is NULL");
    fp_status s = check_shape(kv, chunk);
    if (s || (s = check_heads(kv, n_heads))) return s;
    *bytes = attn_chunk_ws_bytes(*kv, *chunk, n_heads);
    return FP_OK;
}

fp_status fp_attn_chunk(const fp_paged_kv* kv, const fp_chunk* chunk, const void* q, int64_t q_stride, int32_t n_heads,
                        float scale, void* out, void* workspace, size_t workspace_bytes, void* stream) {
    fp_status s = check_chunk(kv, chunk);
    if (s || (s = check_heads(kv, n_heads))) return s;
    const int64_t qw = (int64_t)n_heads * kv->head_dim;
    if ((s = check_rows("q", q, q_stride, qw)) || (s = check_rows("out", out, qw, qw))) return s;
    if (overlap(q, rows_bytes(chunk->n_rows, q_stride, qw), out, rows_bytes(chunk->n_rows, qw, qw)))
        return fail(FP_ERR_INVALID_ARG, "q and out overlap");
    // times log2 e it must stay finite
    if (!(std::fabs(scale) < 0x1p127f)) return fail(FP_ERR_INVALID_ARG, "scale is not below 2^127 in magnitude");
    const size_t need = attn_chunk_ws_bytes(*kv, *chunk, n_heads);
    if (need > 0 && (!workspace || !aligned(workspace, 16))) return fail(FP_ERR_INVALID_ARG, "workspace must be a 16-byte aligned device pointer");
    if (workspace_bytes < need) return fail(FP_ERR_CAPACITY, "workspace of %zu bytes, %zu needed", workspace_bytes, need);
    if (chunk->n_rows == 0) return FP_OK;
    AttnChunkArgs a{};
    a.kv = *kv;
    a.chunk = *chunk;
    a.q = (const uint16_t*)q;
    a.q_stride = q_stride;
    a.n_heads = n_heads;
    a.scale = scale;
    a.out = (uint16_t*)out;
    a.out_fmt = ACT_BF16;
    a.ws = (float*)workspace;
    return done(launch_attn_chunk(a, (hipStream_t)stream), "chunk attention");
}

static fp_status check_verify(int32_t n_seqs, int32_t n_rows, int32_t vocab) {
    if (n_seqs < 1 || n_rows < 0 || vocab < 1) return fail(FP_ERR_INVALID_ARG, "n_seqs and vocab must be >= 1, n_rows >= 0");
    if (n_seqs > 4096 || n_rows > 65535 || vocab > 1 << 20)
        return fail(FP_ERR_UNSUPPORTED, "n_seqs %d > 4096, n_rows %d > 65535 or vocab %d > 2^20", n_seqs, n_rows, vocab);
    return FP_OK;
}

fp_status fp_verify_draft_workspace(int32_t n_seqs, int32_t n_rows, int32_t vocab, size_t* bytes) {
    if (!bytes) return fail(FP_ERR_INVALID_ARG, "bytes is NULL");
    if (const fp_status s = check_verify(n_seqs, n_rows, vocab)) return s;
    *bytes = verify_ws_bytes(n_seqs, n_rows, vocab);
    return FP_OK;
}

fp_status fp_verify_draft(const float* logits, int64_t row_stride, int32_t n_seqs, int32_t n_rows, int32_t max_rows,
                          int32_t vocab, const int32_t* row_start, const int32_t* draft_ids, const float* draft_probs,
                          int64_t draft_stride, const float* u, const float* u_last, float temperature,
                          int32_t* out_ids, int32_t* n_out, void* workspace, size_t workspace_bytes, void* stream) {
    if (const fp_status s = check_verify(n_seqs, n_rows, vocab)) return s;
    if (max_rows < 1) return fail(FP_ERR_INVALID_ARG, "max_rows must be >= 1");
    if (max_rows > 64) return fail(FP_ERR_UNSUPPORTED, "max_rows %d > 64", max_rows);
    if (!std::isfinite(temperature) || temperature < 0.f) return fail(FP_ERR_INVALID_ARG, "temperature must be finite and >= 0");
    if (!row_start || !out_ids || !n_out) return fail(FP_ERR_INVALID_ARG, "row_start, out_ids and n_out must be device pointers");
    if (n_rows > 0) {
        if (!logits || !draft_ids) return fail(FP_ERR_INVALID_ARG, "logits and draft_ids must be device pointers");
        if (row_stride < vocab) return fail(FP_ERR_INVALID_ARG, "logits rows are %lld apart, vocab is %d", (long long)row_stride, vocab);
        if (temperature > 0.f && (!u || !u_last)) return fail(FP_ERR_INVALID_ARG, "u and u_last must be device pointers");
        if (temperature > 0.f && draft_probs && draft_stride < vocab)
            return fail(FP_ERR_INVALID_ARG, "draft_probs rows are %lld apart, vocab is %d", (long long)draft_stride, vocab);
    }
    const size_t need = verify_ws_bytes(n_seqs, n_rows, vocab);
    if (!workspace || !aligned(workspace, 16)) return fail(FP_ERR_INVALID_ARG, "workspace must be a 16-byte aligned device pointer");
    if (workspace_bytes < need) return fail(FP_ERR_CAPACITY, "workspace of %zu bytes, %zu needed", workspace_bytes, need);
    VerifyArgs a{};
    a.logits = logits;
    a.row_stride = row_stride;
    a.n_seqs = n_seqs;
    a.n_rows = n_rows;
    a.max_rows = max_rows;
    a.V = vocab;
    a.row_start = row_start;
    a.draft_ids = draft_ids;
    a.draft_probs = temperature > 0.f ? draft_probs : nullptr;
    a.draft_stride = draft_stride;
    a.u = u;
    a.u_last = u_last;
    a.c = temperature > 0.f ? 1.44269504088896340736 / (double)temperature : 0.0;
    a.out_ids = out_ids;
    a.n_out = n_out;
    a.ws = workspace;
    return done(launch_verify(a, (hipStream_t)stream), "draft verification");
}

}  // extern "C"
