// fk_tree_attn, fk_paged_tree_attn: launches and entry points of the attention of drafted trees (tree.h)
#include "tree.h"

#include <algorithm>
#include <climits>
#include <cmath>

namespace fk {

// KIND: 1, 2: tree_tile with so many 16-row blocks; 4, 8: wide_tile with so many
template <typename T, int D, int KIND> struct TreeKind {
    static constexpr bool WIDE = KIND >= 4;
    static constexpr size_t LDS = WIDE ? WideCfg<T, D, WIDE ? KIND / 4 : 1>::LDS : TreeCfg<T, D, WIDE ? 1 : KIND>::LDS;
};

template <typename T, int D, int KIND, bool ROWS>
__global__ __launch_bounds__(256, KIND == 1 && D == 64 ? 3 : 2) void tree_kernel(const TreeParams P) {
    if constexpr (KIND >= 4) wide_tile<T, D, KIND / 4, ROWS>(P, blockIdx.x, blockIdx.y);
    else tree_tile<T, D, KIND, ROWS>(P, blockIdx.x, blockIdx.y);
}

// ---- host side ---------------------------------------------------------------------------------------------------
struct TreePlan {
    int kind;                  // 16-row blocks of a tile
    TileGrid grid;
    int splits, shift;
};
static TreePlan tree_plan(const fk_paged_desc* d, int32_t n_tokens, int32_t max_tree, long long pairs) {
    const int g = d->n_q_heads / d->n_kv_heads, tree = std::min(std::min(max_tree, n_tokens), kTreeNodes), rows = tree * g;
    TreePlan p = {rows <= 16 ? 1 : rows <= 32 ? 2 : rows <= 64 ? 4 : 8, {}, 1, 0};
    p.grid = tile_grid(d, n_tokens, tree, 16 * p.kind);
    p.grid.most = kTreeNodes * g;
    const int kt_shift = (d->dtype == FK_BF16 ? 5 : 4) + (p.kind >= 4 ? 1 : 0);
    p.shift = 8 - kt_shift;
    const long long items = (long long)p.grid.places * d->n_kv_heads, fill = p.kind == 1 ? 768 : 512;
    long long s = items < fill ? fill / items : 1;
    s = std::min(std::min(s, (long long)kMostTreeSplits), (pairs + tree) >> 8);
    p.splits = items > kSplitItems ? 1 : (int)std::max(s, 1ll);
    return p;
}
// workspace: counters, the same for every call (so that calls of any sizes may take turns with one workspace) | sums and references of records | records
static constexpr size_t kCounterBytes = kSplitItems * 4 * sizeof(uint32_t);
static size_t ml_bytes(const TreePlan& p, long long items) {   // wide: 16 bytes a lane and 16 rows; 8 a row
    return p.splits > 1 ? up256((size_t)items * p.splits * 16 * p.kind * (p.kind >= 4 ? 64 : 8)) : 0;
}
static size_t tree_workspace(const fk_paged_desc* d, int32_t n_tokens, int32_t max_tree, int32_t max_len) {
    const TreePlan p = tree_plan(d, std::max(n_tokens, 1), max_tree, max_len);
    const long long items = (long long)p.grid.places * d->n_kv_heads;
    return kCounterBytes + ml_bytes(p, items) + (p.splits > 1 ? (size_t)items * p.splits * 16 * p.kind * d->head_dim * sizeof(float) : 0);
}

template <typename T, int D, int KIND, bool ROWS> static fk_status tree_start(const TreeParams& P, hipStream_t st) {
    using C = TreeKind<T, D, KIND>;
    auto kern = tree_kernel<T, D, KIND, ROWS>;
    static bool lds_ok[kMaxDevices] = {};
    if (!allow_dynamic_lds((const void*)kern, C::LDS, lds_ok)) return FK_ERR_LAUNCH;
    const int items = P.a.grid.places * P.a.view.n_kv;
    hipLaunchKernelGGL(kern, dim3((unsigned)items, (unsigned)P.a.splits), dim3(256), C::LDS, st, P);
    return launch_status();
}
template <typename T, int D, bool ROWS> static fk_status tree_rows_of(int kind, const TreeParams& P, hipStream_t st) {
    return kind == 1 ? tree_start<T, D, 1, ROWS>(P, st) : kind == 2 ? tree_start<T, D, 2, ROWS>(P, st) : kind == 4 ? tree_start<T, D, 4, ROWS>(P, st) : tree_start<T, D, 8, ROWS>(P, st);
}
template <bool ROWS> static fk_status tree_launch(const fk_paged_desc* d, const TreePlan& p, TreeParams& P, void* ws, hipStream_t st) {
    AttnPagedParams& A = P.a;
    A.grid = p.grid;
    A.splits = p.splits;
    A.split_shift = p.shift;
    P.here = static_cast<uint32_t*>(ws);
    A.rec_ml = reinterpret_cast<float2*>(static_cast<char*>(ws) + kCounterBytes);
    A.rec = reinterpret_cast<float*>(static_cast<char*>(ws) + kCounterBytes + ml_bytes(p, (long long)p.grid.places * d->n_kv_heads));
    if (d->dtype == FK_F32) return d->head_dim == 64 ? tree_rows_of<float, 64, ROWS>(p.kind, P, st) : tree_rows_of<float, 128, ROWS>(p.kind, P, st);
    return d->head_dim == 64 ? tree_rows_of<bf16_t, 64, ROWS>(p.kind, P, st) : tree_rows_of<bf16_t, 128, ROWS>(p.kind, P, st);
}

// what both entry points check beyond their descriptors
static fk_status check_trees(const fk_paged_desc* d, const void* q, const void* K, const void* V, const int32_t* len, const void* k_tree, const void* v_tree,
                             const int32_t* parent, const int32_t* q_start, int32_t n_tokens, int32_t max_tree, const void* out, const float* stats) {
    if (!K || !V || !len || !q_start) return FK_ERR_INVALID_ARG;
    if (n_tokens > 0 && (!q || !k_tree || !v_tree || !parent || !out)) return FK_ERR_INVALID_ARG;   // (no token: empty buffers)
    if (!aligned16(q) || !aligned16(K) || !aligned16(V) || !aligned16(k_tree) || !aligned16(v_tree) || !aligned16(out) || (reinterpret_cast<uintptr_t>(stats) & 7))
        return FK_ERR_INVALID_ARG;
    return FK_OK;
}
static fk_status check_tree_sizes(const fk_paged_desc* d, int32_t n_tokens, int32_t max_tree) {
    if (n_tokens < 0 || max_tree <= 0) return FK_ERR_INVALID_ARG;
    if (max_tree > kTreeNodes || d->n_kv_heads >= (1 << 16) || (int64_t)n_tokens * d->n_q_heads >= (1 << 28)) return FK_ERR_UNSUPPORTED;
    return FK_OK;
}
// the rows of a budgeted cache as far as plans and launches go: one page of `capacity` pairs each
static fk_paged_desc as_paged(const fk_cache_desc* d) {
    return {d->batch, d->n_q_heads, d->n_kv_heads, d->head_dim, 1, 1, d->capacity, d->dtype};
}
static void set_scale(PagedParams& P, float softmax_scale) {
    P.negate = std::signbit(softmax_scale);
    P.scale_log2e = base2_scale(softmax_scale);
}

}  // namespace fk

using namespace fk;

static fk_status check_rows(const fk_cache_desc* desc, int32_t n_tokens, int32_t max_tree, int32_t max_len) {
    fk_status s = check_desc(desc);
    if (s != FK_OK) return s;
    if (max_len <= 0 || max_len > desc->capacity) return FK_ERR_INVALID_ARG;
    if ((int64_t)desc->batch * desc->n_kv_heads >= (1 << 24)) return FK_ERR_UNSUPPORTED;
    const fk_paged_desc d = as_paged(desc);
    return check_tree_sizes(&d, n_tokens, max_tree);
}

extern "C" size_t fk_tree_attn_workspace(const fk_cache_desc* desc, int32_t n_tokens, int32_t max_tree, int32_t max_len) {
    if (check_rows(desc, n_tokens, max_tree, max_len) != FK_OK) return 0;
    const fk_paged_desc d = as_paged(desc);
    return tree_workspace(&d, n_tokens, max_tree, max_len);
}

extern "C" fk_status fk_tree_attn(const fk_cache_desc* desc, const void* q, const void* K, const void* V, const int32_t* len, const void* k_tree,
                                  const void* v_tree, const int32_t* parent, const int32_t* q_start, int32_t n_tokens, int32_t max_tree,
                                  int32_t max_len, float softmax_scale, void* out, float* stats, void* workspace, size_t workspace_bytes, void* stream) {
    fk_status s = check_rows(desc, n_tokens, max_tree, max_len);
    if (s != FK_OK) return s;
    const fk_paged_desc d = as_paged(desc);
    s = check_trees(&d, q, K, V, len, k_tree, v_tree, parent, q_start, n_tokens, max_tree, out, stats);
    if (s != FK_OK) return s;
    if (!workspace || workspace_bytes < fk_tree_attn_workspace(desc, n_tokens, max_tree, max_len) || !aligned16(workspace)) return FK_ERR_WORKSPACE;
    if (n_tokens == 0) return FK_OK;
    TreeParams P = {};
    P.a.view = paged_params(&d, nullptr, len, q_start, n_tokens);
    P.a.view.q = q;
    P.a.view.K = K;
    P.a.view.V = V;
    P.a.view.window = INT_MAX;
    set_scale(P.a.view, softmax_scale);
    P.a.out = out;
    P.a.stats = reinterpret_cast<float2*>(stats);
    P.a.cap = desc->capacity;
    P.parent = parent;
    P.k_tree = k_tree;
    P.v_tree = v_tree;
    return tree_launch<true>(&d, tree_plan(&d, n_tokens, max_tree, max_len), P, workspace, (hipStream_t)stream);
}

static fk_status check_pages(const fk_paged_desc* desc, int32_t n_tokens, int32_t max_tree, int32_t max_len) {
    fk_status s = check_paged(desc);
    if (s != FK_OK) return s;
    if (max_len <= 0 || (int64_t)max_len > (int64_t)desc->max_pages * desc->page_size) return FK_ERR_INVALID_ARG;
    return check_tree_sizes(desc, n_tokens, max_tree);
}

extern "C" size_t fk_paged_tree_attn_workspace(const fk_paged_desc* desc, int32_t n_tokens, int32_t max_tree, int32_t max_len) {
    if (check_pages(desc, n_tokens, max_tree, max_len) != FK_OK) return 0;
    return tree_workspace(desc, n_tokens, max_tree, max_len);
}

extern "C" fk_status fk_paged_tree_attn(const fk_paged_desc* desc, const void* q, const void* K, const void* V, const int32_t* page_table,
                                        const int32_t* kv_len, const void* k_tree, const void* v_tree, const int32_t* parent,
                                        const int32_t* q_start, int32_t n_tokens, int32_t max_tree, int32_t max_len, int32_t window,
                                        int32_t n_sink, float softmax_scale, void* out, float* stats, void* workspace, size_t workspace_bytes,
                                        void* stream) {
    fk_status s = check_pages(desc, n_tokens, max_tree, max_len);
    if (s == FK_OK) s = check_trees(desc, q, K, V, kv_len, k_tree, v_tree, parent, q_start, n_tokens, max_tree, out, stats);
    if (s != FK_OK) return s;
    if (!page_table || window < 0 || n_sink < 0) return FK_ERR_INVALID_ARG;
    if (!workspace || workspace_bytes < fk_paged_tree_attn_workspace(desc, n_tokens, max_tree, max_len) || !aligned16(workspace)) return FK_ERR_WORKSPACE;
    if (n_tokens == 0) return FK_OK;
    TreeParams P = {};
    P.a.view = paged_params(desc, page_table, kv_len, q_start, n_tokens);
    P.a.view.q = q;
    P.a.view.K = K;
    P.a.view.V = V;
    P.a.view.window = window == 0 || window >= (1 << 24) + kTreeNodes ? INT_MAX : window;   // (longer than any sequence and tree: none)
    P.a.view.sink = n_sink;
    set_scale(P.a.view, softmax_scale);
    P.a.out = out;
    P.a.stats = reinterpret_cast<float2*>(stats);
    P.parent = parent;
    P.k_tree = k_tree;
    P.v_tree = v_tree;
    return tree_launch<false>(desc, tree_plan(desc, n_tokens, max_tree, max_len), P, workspace, (hipStream_t)stream);
}
