// fk_paged_attn and fk_paged_weights: attention of chunks over the pages of a prompt, and the weights that its pairs received.
// One workgroup per (token, KV head), a thread per key: the plain form.
#include "thin.h"
#include <climits>
#include <cmath>

namespace fk {

template <typename T> __device__ __forceinline__ float load1(const T* p);
template <> __device__ __forceinline__ float load1<float>(const float* p) { return *p; }
template <> __device__ __forceinline__ float load1<bf16_t>(const bf16_t* p) { return bf16_lo(*p); }

template <typename T>
__global__ __launch_bounds__(256) void paged_weights_plain_kernel(const PagedParams P, const float2* stats, float* acc, int D) {
    const int b = blockIdx.z, h = blockIdx.y, j = blockIdx.x * 256 + threadIdx.x;
    const int begin = chunk_begin(P, b), end = chunk_end(P, b, begin), n = pairs_of(P, b), first = n - (end - begin);
    if (begin == end || j >= n) return;
    const int page = P.table[(size_t)b * P.max_pages + (j >> P.page_shift)];
    const T* kr = reinterpret_cast<const T*>(P.K) + ((((size_t)(page_ok(P, page) ? page : 0) * P.n_kv + h) << P.page_shift) + (j & ((1 << P.page_shift) - 1))) * D;
    float sum = 0.f;
    for (int t = begin; page_ok(P, page) && t < end; ++t) {
        if (!sees(P, first + t - begin, j)) continue;
        for (int k = 0; k < P.g; ++k) {
            const size_t row = ((size_t)t * P.n_kv + h) * P.g + k;
            const T* q = reinterpret_cast<const T*>(P.q) + row * D;
            float s = 0.f;
            for (int e = 0; e < D; ++e) s = fmaf(load1(q + e), load1(kr + e), s);
            const float2 st = stats[row];
            sum += exp2f(s * P.scale_log2e * (P.negate ? -1.f : 1.f) - st.x) / st.y;
        }
    }
    float* a = acc + ((size_t)b * P.n_kv + h) * ((size_t)P.max_pages << P.page_shift) + j;
    *a = (j >= first ? 0.f : *a) + sum;
}

}  // namespace fk

using namespace fk;

static fk_status check_view(const fk_paged_desc* desc, const void* q, const void* K, const int32_t* table, const int32_t* kv_len, const int32_t* q_start,
                            int32_t n_tokens, int32_t max_chunk, int32_t max_len, int32_t window, int32_t n_sink, const float* stats) {
    fk_status s = check_paged(desc);
    if (s == FK_OK) s = check_chunks(desc, n_tokens, max_chunk, max_len);
    if (s != FK_OK) return s;
    if (!q || !K || !table || !kv_len || !q_start || window < 0 || n_sink < 0) return FK_ERR_INVALID_ARG;
    if (!aligned16(q) || !aligned16(K) || (reinterpret_cast<uintptr_t>(stats) & 7)) return FK_ERR_INVALID_ARG;
    return FK_OK;
}

static PagedParams view_params(const fk_paged_desc* desc, const void* q, const void* K, const int32_t* table, const int32_t* kv_len, const int32_t* q_start,
                               int32_t n_tokens, int32_t window, int32_t n_sink, float softmax_scale) {
    PagedParams P = paged_params(desc, table, kv_len, q_start, n_tokens);
    P.q = q;
    P.K = K;
    P.window = window == 0 ? INT_MAX : window;
    P.sink = n_sink;
    P.negate = std::signbit(softmax_scale);
    P.scale_log2e = std::fabs(softmax_scale) * 1.4426950408889634f;
    return P;
}

extern "C" size_t fk_paged_attn_workspace(const fk_paged_desc* desc, int32_t n_tokens, int32_t max_chunk, int32_t max_len) {
    if (check_paged(desc) != FK_OK || check_chunks(desc, n_tokens, max_chunk, max_len) != FK_OK) return 0;
    return 16 + thin_paged_workspace(desc, tile_grid(desc, n_tokens, max_chunk, 16), max_len);
}

extern "C" fk_status fk_paged_attn(const fk_paged_desc* desc, const void* q, const void* K, const void* V, const int32_t* page_table,
                                   const int32_t* kv_len, const int32_t* q_start, int32_t n_tokens, int32_t max_chunk, int32_t max_len,
                                   int32_t window, int32_t n_sink, float softmax_scale, void* out, float* stats, void* workspace,
                                   size_t workspace_bytes, void* stream) {
    const fk_status s = check_view(desc, q, K, page_table, kv_len, q_start, n_tokens, max_chunk, max_len, window, n_sink, stats);
    if (s != FK_OK) return s;
    if (!V || !out || !aligned16(V) || !aligned16(out)) return FK_ERR_INVALID_ARG;
    if (!workspace || workspace_bytes < fk_paged_attn_workspace(desc, n_tokens, max_chunk, max_len) || !aligned16(workspace)) return FK_ERR_WORKSPACE;
    if (n_tokens == 0) return FK_OK;
    PagedParams P = view_params(desc, q, K, page_table, kv_len, q_start, n_tokens, window, n_sink, softmax_scale);
    P.V = V;
    ThinParams T = {};
    T.view = P;
    T.out = out;
    T.stats = reinterpret_cast<float2*>(stats);
    T.grid = tile_grid(desc, n_tokens, max_chunk, 16);
    return thin_paged(desc, T, max_len, workspace, (hipStream_t)stream);
}

extern "C" size_t fk_paged_weights_workspace(const fk_paged_desc* desc, int32_t n_tokens, int32_t max_chunk, int32_t max_len) {
    if (check_paged(desc) != FK_OK || check_chunks(desc, n_tokens, max_chunk, max_len) != FK_OK) return 0;
    return 16;
}

extern "C" fk_status fk_paged_weights(const fk_paged_desc* desc, const void* q, const void* K, const int32_t* page_table, const int32_t* kv_len,
                                      const int32_t* q_start, int32_t n_tokens, int32_t max_chunk, int32_t max_len, int32_t window,
                                      int32_t n_sink, float softmax_scale, const float* stats, float* acc, void* workspace,
                                      size_t workspace_bytes, void* stream) {
    const fk_status s = check_view(desc, q, K, page_table, kv_len, q_start, n_tokens, max_chunk, max_len, window, n_sink, stats);
    if (s != FK_OK) return s;
    if (!stats || !acc) return FK_ERR_INVALID_ARG;
    if (!workspace || workspace_bytes < fk_paged_weights_workspace(desc, n_tokens, max_chunk, max_len) || !aligned16(workspace)) return FK_ERR_WORKSPACE;
    if (n_tokens == 0) return FK_OK;
    const PagedParams P = view_params(desc, q, K, page_table, kv_len, q_start, n_tokens, window, n_sink, softmax_scale);
    const dim3 grid((((unsigned)desc->max_pages << P.page_shift) + 255) / 256, desc->n_kv_heads, desc->batch);
    if (desc->dtype == FK_F32) hipLaunchKernelGGL(paged_weights_plain_kernel<float>, grid, dim3(256), 0, (hipStream_t)stream, P, (const float2*)stats, acc, desc->head_dim);
    else hipLaunchKernelGGL(paged_weights_plain_kernel<bf16_t>, grid, dim3(256), 0, (hipStream_t)stream, P, (const float2*)stats, acc, desc->head_dim);
    return launch_status();
}
