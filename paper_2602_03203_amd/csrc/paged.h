// The paged cache of a prompt (fk_paged_*): its parameters, where a pair lies, what a query sees, and the checks of its calls.
#pragma once
#include "fk_common.h"

namespace fk {

struct PagedParams {
    const void* q;
    const void *K, *V;
    const int32_t *table, *kv_len, *q_start;
    int batch, n_kv, g, page_shift, n_pages, max_pages, n_tokens;
    int window, sink;      // window: INT_MAX without one
    float scale_log2e;     // >= 0: queries are negated as they are read where softmax_scale is negative (exact)
    bool negate;
};

// Tokens of sequence b in the packed buffers, and its pairs; whatever the arrays hold, inside the buffers.
__device__ __forceinline__ int chunk_begin(const PagedParams& P, int b) { return min(max(P.q_start[b], 0), P.n_tokens); }
__device__ __forceinline__ int chunk_end(const PagedParams& P, int b, int begin) { return min(max(P.q_start[b + 1], begin), P.n_tokens); }
__device__ __forceinline__ int pairs_of(const PagedParams& P, int b) { return min(max(P.kv_len[b], 0), P.max_pages << P.page_shift); }

__device__ __forceinline__ bool page_ok(const PagedParams& P, int page) { return (unsigned)page < (unsigned)P.n_pages; }

// The sequence that token t belongs to, -1 for none (q_start ascending: the last one that starts at or before t)
__device__ __forceinline__ int sequence_of(const PagedParams& P, int t) {
    int lo = 0, hi = P.batch;
    while (lo < hi) {
        const int mid = (lo + hi) / 2;
        if (P.q_start[mid + 1] > t) hi = mid;
        else lo = mid + 1;
    }
    return lo < P.batch && P.q_start[lo] <= t ? lo : -1;
}

__device__ __forceinline__ bool sees(const PagedParams& P, int p, int j) { return j <= p && (j > p - P.window || j < P.sink); }

// ---- host side ---------------------------------------------------------------------------------------------------
inline fk_status check_paged(const fk_paged_desc* d) {
    if (!d) return FK_ERR_INVALID_ARG;
    if (d->batch <= 0 || d->n_q_heads <= 0 || d->n_kv_heads <= 0 || d->head_dim <= 0 || d->page_size <= 0 || d->n_pages <= 0 || d->max_pages <= 0)
        return FK_ERR_INVALID_ARG;
    if (d->n_q_heads % d->n_kv_heads != 0) return FK_ERR_INVALID_ARG;
    if (d->dtype != FK_F32 && d->dtype != FK_BF16) return FK_ERR_UNSUPPORTED;
    if (d->head_dim != 64 && d->head_dim != 128) return FK_ERR_UNSUPPORTED;
    if (d->n_q_heads / d->n_kv_heads > 8) return FK_ERR_UNSUPPORTED;
    if (d->page_size < 16 || d->page_size > 1024 || (d->page_size & (d->page_size - 1))) return FK_ERR_UNSUPPORTED;
    if ((int64_t)d->max_pages * d->page_size >= (1 << 24)) return FK_ERR_UNSUPPORTED;
    if ((int64_t)d->batch * d->n_kv_heads >= (1 << 24)) return FK_ERR_UNSUPPORTED;
    return FK_OK;
}

// sizes of a call on chunks; 32-bit counts of query rows
inline fk_status check_chunks(const fk_paged_desc* d, int32_t n_tokens, int32_t max_chunk, int32_t max_len) {
    if (n_tokens < 0 || max_chunk <= 0 || max_len <= 0 || (int64_t)max_len > (int64_t)d->max_pages * d->page_size) return FK_ERR_INVALID_ARG;
    if ((int64_t)n_tokens * d->n_q_heads >= (1 << 28)) return FK_ERR_UNSUPPORTED;
    return FK_OK;
}

inline PagedParams paged_params(const fk_paged_desc* d, const int32_t* table, const int32_t* kv_len, const int32_t* q_start, int32_t n_tokens) {
    PagedParams P = {};
    P.table = table;
    P.kv_len = kv_len;
    P.q_start = q_start;
    P.batch = d->batch;
    P.n_kv = d->n_kv_heads;
    P.g = d->n_q_heads / d->n_kv_heads;
    P.page_shift = __builtin_ctz(d->page_size);
    P.n_pages = d->n_pages;
    P.max_pages = d->max_pages;
    P.n_tokens = n_tokens;
    return P;
}

}  // namespace fk
