// The entry points of attention over the pages of a prompt and of the weights that its pairs received: fk_paged_attn (thin.h, prompt.h),
// fk_paged_weights (weights.hip).
#include "attn_paged.h"
#include "weights.h"
#include <climits>
#include <cmath>

using namespace fk;

static fk_status check_view(const fk_paged_desc* desc, const void* q, const void* K, const int32_t* table, const int32_t* kv_len, const int32_t* q_start,
                            int32_t n_tokens, int32_t max_chunk, int32_t max_len, int32_t window, int32_t n_sink, const float* stats) {
    fk_status s = check_paged(desc);
    if (s == FK_OK) s = check_chunks(desc, n_tokens, max_chunk, max_len);
    if (s != FK_OK) return s;
    if ((!q && n_tokens > 0) || !K || !table || !kv_len || !q_start || window < 0 || n_sink < 0) return FK_ERR_INVALID_ARG;   // (no token: an empty q)
    if (!aligned16(q) || !aligned16(K) || (reinterpret_cast<uintptr_t>(stats) & 7)) return FK_ERR_INVALID_ARG;
    return FK_OK;
}

static PagedParams view_params(const fk_paged_desc* desc, const void* q, const void* K, const int32_t* table, const int32_t* kv_len, const int32_t* q_start,
                               int32_t n_tokens, int32_t window, int32_t n_sink, float softmax_scale) {
    PagedParams P = paged_params(desc, table, kv_len, q_start, n_tokens);
    P.q = q;
    P.K = K;
    P.window = window == 0 || window >= (1 << 24) ? INT_MAX : window;   // (longer than any sequence: none)
    P.sink = n_sink;
    P.negate = std::signbit(softmax_scale);
    P.scale_log2e = base2_scale(softmax_scale);
    return P;
}

// Which kernel takes a chunk goes by its query rows: up to kThinRows the one that reads every pair once for 16 of them, beyond it the one with
// tiles of 128.  A call that may hold both kinds is one launch of both kernels' tiles.  Calls whose 16-row tiles meet few
// pairs altogether are the first one's alone, however long their chunks: it spreads over more workgroups and its tiles take less time to
// set up.  Measured on either side (one kernel / the other): 4 chunks of 32..64 tokens, g 7, D 128, 512 pairs (229 thousand): 16 / 23 us; 1 chunk of
// 80 tokens, g 4, D 64, 4096 pairs (327 thousand): 15 / 22; 4 chunks of 12..24, g 7, D 128, 4096 pairs (516 thousand): 42 / 32.  In fp32, where
// a tile's products take longer than its loads: 1 chunk of 896, g 8, D 64, 896 pairs (401 thousand) 20 / 49; 2 of 30..60, 8 heads of g 4, D 128, 4096 pairs
// (737 thousand) 80 / 95; 1 of 64 of 8192 (1.05 million) 113 / 105.
static constexpr int kThinRows = 16;
static constexpr long long kThinWork = 3 << 17, kThinWorkF32 = 1 << 20;

struct AttnPlanPaged {
    bool thin, prompt;
    TileGrid thin_grid, prompt_grid;
};
static AttnPlanPaged plan_paged(const fk_paged_desc* d, int32_t n_tokens, int32_t max_chunk, int32_t max_len) {
    const int g = d->n_q_heads / d->n_kv_heads;
    AttnPlanPaged p = {};
    // what is left for the shortest chunk where all others have the bound's length (should they be longer, prompt tiles take short chunks as well)
    const long long shortest = n_tokens - (long long)(d->batch - 1) * max_chunk;
    const long long work = ((long long)n_tokens * g + 15) / 16 * d->n_kv_heads * max_len;
    p.prompt = (long long)max_chunk * g > kThinRows && work > (d->dtype == FK_F32 ? kThinWorkF32 : kThinWork);
    p.thin = !p.prompt || shortest * g <= kThinRows;
    if (p.thin) {   // (also all chunks there are, should they be longer than max_chunk says)
        p.thin_grid = tile_grid(d, n_tokens, p.prompt ? kThinRows / g : max_chunk, 16);
        if (p.prompt) p.thin_grid.most = kThinRows;
    }
    if (p.prompt) {
        p.prompt_grid = tile_grid(d, n_tokens, max_chunk, kPromptRows);
        if (p.thin) p.prompt_grid.least = kThinRows + 1;
    }
    return p;
}

extern "C" size_t fk_paged_attn_workspace(const fk_paged_desc* desc, int32_t n_tokens, int32_t max_chunk, int32_t max_len) {
    if (check_paged(desc) != FK_OK || check_chunks(desc, n_tokens, max_chunk, max_len) != FK_OK) return 0;
    const AttnPlanPaged p = plan_paged(desc, n_tokens, max_chunk, max_len);
    const size_t a = p.thin ? thin_paged_workspace(desc, p.thin_grid, max_len) : 0, b = p.prompt ? prompt_workspace(desc, p.prompt_grid, n_tokens, max_chunk, max_len) : 0;
    return 16 + up256(a) + b;
}

extern "C" fk_status fk_paged_attn(const fk_paged_desc* desc, const void* q, const void* K, const void* V, const int32_t* page_table,
                                   const int32_t* kv_len, const int32_t* q_start, int32_t n_tokens, int32_t max_chunk, int32_t max_len,
                                   int32_t window, int32_t n_sink, float softmax_scale, void* out, float* stats, void* workspace,
                                   size_t workspace_bytes, void* stream) {
    const fk_status s = check_view(desc, q, K, page_table, kv_len, q_start, n_tokens, max_chunk, max_len, window, n_sink, stats);
    if (s != FK_OK) return s;
    if (!V || (!out && n_tokens > 0) || !aligned16(V) || !aligned16(out)) return FK_ERR_INVALID_ARG;
    if (!workspace || workspace_bytes < fk_paged_attn_workspace(desc, n_tokens, max_chunk, max_len) || !aligned16(workspace)) return FK_ERR_WORKSPACE;
    if (n_tokens == 0) return FK_OK;
    PagedParams P = view_params(desc, q, K, page_table, kv_len, q_start, n_tokens, window, n_sink, softmax_scale);
    P.V = V;
    AttnPagedParams T = {};
    T.view = P;
    T.out = out;
    T.stats = reinterpret_cast<float2*>(stats);
    const AttnPlanPaged p = plan_paged(desc, n_tokens, max_chunk, max_len);
    if (!p.prompt) {
        T.grid = p.thin_grid;
        return thin_paged(desc, T, max_len, workspace, (hipStream_t)stream);
    }
    AttnPagedParams F = T;
    bool cold = false;
    char* ws = static_cast<char*>(workspace);
    if (p.thin) {
        F.grid = p.thin_grid;
        thin_prepare(desc, F, max_len, ws, cold);
        ws += up256(thin_paged_workspace(desc, p.thin_grid, max_len));
    }
    T.grid = p.prompt_grid;
    return prompt_paged(desc, T, p.thin ? &F : nullptr, cold, max_chunk, max_len, ws, (hipStream_t)stream);
}

extern "C" size_t fk_paged_weights_workspace(const fk_paged_desc* desc, int32_t n_tokens, int32_t max_chunk, int32_t max_len) {
    if (check_paged(desc) != FK_OK || check_chunks(desc, n_tokens, max_chunk, max_len) != FK_OK) return 0;
    return 16 + weights_workspace(desc, n_tokens, max_chunk, max_len);
}

extern "C" fk_status fk_paged_weights(const fk_paged_desc* desc, const void* q, const void* K, const int32_t* page_table, const int32_t* kv_len,
                                      const int32_t* q_start, int32_t n_tokens, int32_t max_chunk, int32_t max_len, int32_t window,
                                      int32_t n_sink, float softmax_scale, const float* stats, float* acc, void* workspace,
                                      size_t workspace_bytes, void* stream) {
    const fk_status s = check_view(desc, q, K, page_table, kv_len, q_start, n_tokens, max_chunk, max_len, window, n_sink, stats);
    if (s != FK_OK) return s;
    if ((!stats && n_tokens > 0) || !acc) return FK_ERR_INVALID_ARG;
    if (!workspace || workspace_bytes < fk_paged_weights_workspace(desc, n_tokens, max_chunk, max_len) || !aligned16(workspace)) return FK_ERR_WORKSPACE;
    if (n_tokens == 0) return FK_OK;
    WeightsParams P = {};
    P.view = view_params(desc, q, K, page_table, kv_len, q_start, n_tokens, window, n_sink, softmax_scale);
    P.stats = reinterpret_cast<const float2*>(stats);
    P.acc = acc;
    return weights_launch(desc, P, max_chunk, max_len, workspace, (hipStream_t)stream);
}
