// C entries of the paged cache and of the log-probabilities: argument checks, workspace layout, launches.
#include "common.h"
#include "kernels.h"
#include "cache_view.h"

static bool aligned(const void* p, size_t a) { return ((uintptr_t)p & (a - 1)) == 0; }

static size_t page_ws_bytes(const CacheView& v, size_t n) { return align_up(page_ws_layout(v.n_pages, n).total * 4, 256); }

// What the calls with a list of n entries and a workspace share.
static int check_page_call(const radix_cache* cache, int32_t n, const void* ws, size_t ws_bytes, CacheView* v) {
    const int rc = cache_view(cache, v);
    if (rc != RADIX_OK) return rc;
    if (n < 0) return RADIX_ERR_BAD_SIZE;
    if (n > RADIX_CACHE_MAX_LIST) return RADIX_ERR_UNSUPPORTED;
    if (!ws) return RADIX_ERR_NULL_POINTER;
    if (!aligned(ws, 256)) return RADIX_ERR_MISALIGNED;
    if (ws_bytes < page_ws_bytes(*v, (size_t)n)) return RADIX_ERR_WORKSPACE_TOO_SMALL;
    return RADIX_OK;
}

extern "C" int radix_cache_bytes(const radix_cache* cache, size_t* bytes_out) {
    if (!cache || !bytes_out) return RADIX_ERR_NULL_POINTER;
    CacheView v;
    const int rc = cache_shape(cache, &v);
    if (rc != RADIX_OK) return rc;
    *bytes_out = (size_t)v.n_layers * v.layer_bytes;
    return RADIX_OK;
}

extern "C" int radix_cache_workspace_bytes(const radix_cache* cache, int32_t max_n, size_t* bytes_out) {
    if (!cache || !bytes_out) return RADIX_ERR_NULL_POINTER;
    if (max_n < 0) return RADIX_ERR_BAD_SIZE;
    if (max_n > RADIX_CACHE_MAX_LIST) return RADIX_ERR_UNSUPPORTED;
    CacheView v;
    const int rc = cache_shape(cache, &v);
    if (rc != RADIX_OK) return rc;
    *bytes_out = page_ws_bytes(v, (size_t)max_n);
    return RADIX_OK;
}

extern "C" int radix_cache_reset(const radix_cache* cache, void* stream) {
    CacheView v;
    const int rc = cache_view(cache, &v);
    if (rc != RADIX_OK) return rc;
    launch_cache_reset(v, (hipStream_t)stream);
    HIP_TRY(hipGetLastError());
    return RADIX_OK;
}

extern "C" int radix_cache_extend(const radix_cache* cache, const int32_t* slots, const int32_t* cu_seqlens, int32_t B, int32_t* past,
                                  void* ws, size_t ws_bytes, int32_t* status_dev, void* stream) {
    CacheView v;
    const int rc = check_page_call(cache, B, ws, ws_bytes, &v);
    if (rc != RADIX_OK) return rc;
    if (B == 0) return RADIX_OK;
    if (!cu_seqlens || !past) return RADIX_ERR_NULL_POINTER;
    if (!slots && B > v.max_seqs) return RADIX_ERR_BAD_SIZE;
    launch_cache_extend(v, slots, cu_seqlens, B, v.max_pages * v.page_size, past, (int32_t*)ws, nullptr, status_dev, (hipStream_t)stream);
    HIP_TRY(hipGetLastError());
    return RADIX_OK;
}

extern "C" int radix_cache_fork(const radix_cache* cache, const int32_t* parents, const int32_t* children, int32_t n, void* ws,
                                size_t ws_bytes, int32_t* status_dev, void* stream) {
    CacheView v;
    const int rc = check_page_call(cache, n, ws, ws_bytes, &v);
    if (rc != RADIX_OK) return rc;
    if (n == 0) return RADIX_OK;
    if (!parents || !children) return RADIX_ERR_NULL_POINTER;
    launch_cache_fork(v, parents, children, n, (int32_t*)ws, status_dev, (hipStream_t)stream);
    HIP_TRY(hipGetLastError());
    return RADIX_OK;
}

extern "C" int radix_cache_free(const radix_cache* cache, const int32_t* slots, const int32_t* keep_lens, int32_t n, int32_t* status_dev,
                                void* stream) {
    CacheView v;
    const int rc = cache_view(cache, &v);
    if (rc != RADIX_OK) return rc;
    if (n < 0) return RADIX_ERR_BAD_SIZE;
    if (n > RADIX_CACHE_MAX_LIST) return RADIX_ERR_UNSUPPORTED;
    if (n == 0) return RADIX_OK;
    if (!slots) return RADIX_ERR_NULL_POINTER;
    launch_cache_free(v, slots, keep_lens, n, status_dev, (hipStream_t)stream);
    HIP_TRY(hipGetLastError());
    return RADIX_OK;
}

extern "C" int radix_cache_compact(const radix_cache* cache, int32_t* n_used, void* ws, size_t ws_bytes, int32_t* status_dev,
                                   void* stream) {
    CacheView v;
    const int rc = check_page_call(cache, 0, ws, ws_bytes, &v);
    if (rc != RADIX_OK) return rc;
    if (!n_used) return RADIX_ERR_NULL_POINTER;
    launch_cache_compact(v, n_used, (int32_t*)ws, status_dev, (hipStream_t)stream);
    HIP_TRY(hipGetLastError());
    return RADIX_OK;
}

extern "C" int radix_cache_copy_pages(const radix_cache* cache, const int32_t* src, const int32_t* dst, int32_t n, void* ws,
                                      size_t ws_bytes, int32_t* status_dev, void* stream) {
    CacheView v;
    const int rc = check_page_call(cache, n, ws, ws_bytes, &v);
    if (rc != RADIX_OK) return rc;
    if (n == 0) return RADIX_OK;
    if (!src || !dst) return RADIX_ERR_NULL_POINTER;
    launch_cache_copy(v, src, dst, n, (int32_t*)ws, status_dev, (hipStream_t)stream);
    HIP_TRY(hipGetLastError());
    return RADIX_OK;
}

extern "C" int radix_cache_append(const radix_cache* cache, int32_t layer, const void* k, int64_t k_stride, const void* v,
                                  int64_t v_stride, const int32_t* cu_seqlens, const int32_t* past, const int32_t* slots, int32_t B,
                                  int32_t N, int32_t* status_dev, void* stream) {
    CacheView c;
    const int rc = cache_view(cache, &c);
    if (rc != RADIX_OK) return rc;
    if (layer < 0 || layer >= c.n_layers || B < 0 || N < 0) return RADIX_ERR_BAD_SIZE;
    if (B > RADIX_CACHE_MAX_LIST || N > MAX_BLOCKS) return RADIX_ERR_UNSUPPORTED;
    if (B == 0 || N == 0) return RADIX_OK;
    if (!k || !v || !cu_seqlens || !past) return RADIX_ERR_NULL_POINTER;
    const int64_t es = cache->dtype == RADIX_F32 ? 4 : 2, row = (int64_t)c.n_kv_heads * c.head_dim;
    if (k_stride < row || v_stride < row || k_stride > INT32_MAX || v_stride > INT32_MAX) return RADIX_ERR_BAD_SIZE;
    if (!aligned(k, 16) || !aligned(v, 16) || k_stride * es % 16 != 0 || v_stride * es % 16 != 0) return RADIX_ERR_MISALIGNED;
    launch_cache_append(c, layer, k, v, (size_t)(k_stride * es), (size_t)(v_stride * es), cu_seqlens, past, slots, B, N, status_dev,
                        (hipStream_t)stream);
    HIP_TRY(hipGetLastError());
    return RADIX_OK;
}

static int paged_shape(const CacheView& c, int32_t n_q_heads, int32_t B, int32_t N, int32_t max_new, int32_t find_shared, PagedShape* s) {
    if (B < 0 || N < 0 || max_new < 0 || n_q_heads <= 0 || n_q_heads % c.n_kv_heads != 0) return RADIX_ERR_BAD_SIZE;
    if (B > RADIX_CACHE_MAX_LIST || (int64_t)N * n_q_heads > INT32_MAX || (int64_t)B * n_q_heads > INT32_MAX / 4) return RADIX_ERR_UNSUPPORTED;
    *s = {n_q_heads, B, N, max_new < N ? max_new : N, find_shared != 0, 0, 0};
    return RADIX_OK;
}

extern "C" int radix_paged_attention_workspace_bytes(const radix_cache* cache, int32_t n_q_heads, int32_t max_N, int32_t max_B,
                                                     int32_t max_new, int32_t find_shared, size_t* bytes_out) {
    if (!cache || !bytes_out) return RADIX_ERR_NULL_POINTER;
    CacheView c;
    int rc = cache_shape(cache, &c);
    if (rc != RADIX_OK) return rc;
    PagedShape s;
    rc = paged_shape(c, n_q_heads, max_B, max_N, max_new, find_shared, &s);
    if (rc != RADIX_OK) return rc;
    const PagedLayout L = paged_layout(c, cache->dtype, s);
    if (L.items > MAX_BLOCKS) return RADIX_ERR_UNSUPPORTED;
    *bytes_out = L.total;
    return RADIX_OK;
}

extern "C" int radix_paged_attention(const radix_cache* cache, int32_t layer, const void* q, int64_t q_stride, int32_t n_q_heads,
                                     const int32_t* cu_seqlens, const int32_t* past, const int32_t* slots, int32_t B, int32_t N,
                                     int32_t max_new, int32_t find_shared, void* out, int64_t out_stride, void* ws, size_t ws_bytes, int32_t* status_dev,
                                     void* stream) {
    CacheView c;
    int rc = cache_view(cache, &c);
    if (rc != RADIX_OK) return rc;
    if (layer < 0 || layer >= c.n_layers) return RADIX_ERR_BAD_SIZE;
    PagedShape s;
    rc = paged_shape(c, n_q_heads, B, N, max_new, find_shared, &s);
    if (rc != RADIX_OK) return rc;
    if (B == 0 || N == 0) return RADIX_OK;
    if (max_new == 0) return RADIX_ERR_BAD_SIZE;
    if (!q || !out || !cu_seqlens || !past || !ws) return RADIX_ERR_NULL_POINTER;
    const int64_t es = cache->dtype == RADIX_F32 ? 4 : 2, row = (int64_t)n_q_heads * c.head_dim;
    if (q_stride < row || out_stride < row || q_stride > INT32_MAX || out_stride > INT32_MAX) return RADIX_ERR_BAD_SIZE;
    if (!aligned(q, 16) || !aligned(out, 16) || !aligned(ws, 256) || q_stride * es % 16 != 0 || out_stride * es % 16 != 0)
        return RADIX_ERR_MISALIGNED;
    s.q_stride = (size_t)q_stride;
    s.out_stride = (size_t)out_stride;
    const PagedLayout L = paged_layout(c, cache->dtype, s);
    if (ws_bytes < L.total) return RADIX_ERR_WORKSPACE_TOO_SMALL;
    if (L.items > MAX_BLOCKS) return RADIX_ERR_UNSUPPORTED;
    launch_paged_plan(c, s, L, cu_seqlens, past, slots, ws, status_dev, (hipStream_t)stream);
    launch_paged_attention(c, cache->dtype, layer, s, L, q, cu_seqlens, past, slots, out, ws, status_dev, (hipStream_t)stream);
    HIP_TRY(hipGetLastError());
    return RADIX_OK;
}

static int check_logprobs(int32_t n_rows, int32_t vocab, int32_t n_given, int32_t top_k) {
    if (n_rows < 0 || vocab <= 0 || n_given < 0 || top_k < 0 || top_k > vocab) return RADIX_ERR_BAD_SIZE;
    if (top_k > RADIX_MAX_TOP_K || n_rows > MAX_BLOCKS) return RADIX_ERR_UNSUPPORTED;
    return RADIX_OK;
}

extern "C" int radix_token_logprobs_workspace_bytes(int32_t max_rows, int32_t vocab, int32_t n_given, int32_t top_k, size_t* bytes_out) {
    if (!bytes_out) return RADIX_ERR_NULL_POINTER;
    const int rc = check_logprobs(max_rows, vocab, n_given, top_k);
    if (rc != RADIX_OK) return rc;
    *bytes_out = token_logprobs_ws_bytes(max_rows, top_k);
    return RADIX_OK;
}

extern "C" int radix_token_logprobs(const void* logits, int32_t dtype, int64_t row_stride, int32_t n_rows, int32_t vocab,
                                    const int32_t* given, int32_t n_given, int32_t top_k, float* logprobs, float* entropy,
                                    int32_t* top_ids, float* top_logprobs, void* ws, size_t ws_bytes, int32_t* status_dev, void* stream) {
    const int rc = check_logprobs(n_rows, vocab, n_given, top_k);
    if (rc != RADIX_OK) return rc;
    if (dtype != RADIX_F32 && dtype != RADIX_BF16 && dtype != RADIX_F16) return RADIX_ERR_UNSUPPORTED;
    if (row_stride < vocab) return RADIX_ERR_BAD_SIZE;
    if (n_rows == 0) return RADIX_OK;
    if (!logits || !ws || (n_given > 0 && (!given || !logprobs)) || (top_k > 0 && (!top_ids || !top_logprobs))) return RADIX_ERR_NULL_POINTER;
    if (!aligned(ws, 256) || !aligned(logits, dtype == RADIX_F32 ? 4 : 2)) return RADIX_ERR_MISALIGNED;
    if (ws_bytes < token_logprobs_ws_bytes(n_rows, top_k)) return RADIX_ERR_WORKSPACE_TOO_SMALL;
    launch_token_logprobs(logits, dtype, (size_t)row_stride, n_rows, vocab, given, n_given, top_k, logprobs, entropy, top_ids, top_logprobs,
                          ws, status_dev, (hipStream_t)stream);
    HIP_TRY(hipGetLastError());
    return RADIX_OK;
}
