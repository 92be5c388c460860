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

// ONCE: one tile of rows for every tree, nobody else reads its pairs
template <typename T, int D, int KIND, bool ROWS, bool ONCE>
__global__ __launch_bounds__(256, KIND == 1 && D == 64 ? 3 : 2) void tree_kernel(const TreeParams P) {
    if constexpr (KIND >= 4) wide_tile<T, D, KIND / 4, ROWS, ONCE>(P, blockIdx.x, blockIdx.y);
    else tree_tile<T, D, KIND, ROWS>(P, blockIdx.x, blockIdx.y);
}

// ---- host side ---------------------------------------------------------------------------------------------------
// Which kernel takes a call's tiles, by the query rows of its largest tree (us, in the order of the kinds 16, 32, 64, 128 rows; 16 sequences of 2112
// pairs, 8 heads of g 4, D 128 where nothing else is said): 16 rows 27.6, 28.8, 29.4, 43.0; 32 rows 33.9, 30.5, 31.9, 43.2, of one sequence 11.7, 15.0, 16.3, 25.0;
// 48 rows 51.6, 39.8, 32.9, 48.7; up to 128 rows of 4 sequences 28.4, 23.5, 21.6, 33.4; up to 182 rows of 16, 4 heads of g 7, 4160 pairs 117, 84, 57, 63; up to 256 rows of 16
// 167, 99, 73, 71; up to 96 rows of 16 in pages, 1024 to 16384 pairs 355, 221, 183, 158: beyond 64 rows by the estimate below.  fp32, where products take longer than loads:
// 4 sequences, 32 rows 21.9 and, of the third kind, 34.5; 56 rows 32.3 and 38.1; up to 128 rows 51.1 and 52.8 - the first kind, tile by tile, up to 64 rows, then the third.
struct TreePlan {
    int kind;                  // 16-row blocks of a tile
    TileGrid grid;
    int splits, shift;
};
static long long items_of(const fk_paged_desc* d, const TileGrid& G) { return (long long)G.places * d->n_kv_heads; }

// Splits of a tile's pairs, each 256 and more, where the items are few.  16 and 32 rows, bound by memory: up to 512 workgroups (16 rows, D 128: 128 items of 2112
// pairs whole 32.1, in two 28.5, four 27.7, eight 32.1; 8 items in four 14.1, eight 11.6), D 64 up to 192 (128 items whole 17.9, in two 17.8, four 16.7, eight 20.1).  Others by an
// estimate: a turn of the loop takes `turn[k]` us with k + 1 workgroups on a CU, and records go out and come back at 4 TB/s (up to 182 rows of 4160 pairs, 192
// items of 64 rows: whole 109, in two 72, three 69, four 57, six 73; up to 256 rows of 2112, 256 items of 128: 87, 71, 96, 89).  Sequences in pages differ in
// length as a rule, which only the device knows: up to twice as many splits, of 512 pairs and more, even them out (16 sequences of 1024 to 16384 pairs, 8 heads: 16 rows
// in four 126, eight 111; 32 rows 132 and 119; up to 96 rows 173 and 158).
// bound: the most splits of which rounding can make the estimate choose, for fewer pairs too (a split more costs records and saves turns: more pairs, more splits).
static int tree_splits(const fk_paged_desc* d, int kind, long long items, long long pairs, bool uneven, double& least, bool bound = false) {
    const long long most = std::min((long long)kMostTreeSplits, pairs >> (uneven ? 9 : 8)), places = uneven ? 1024 : 512;
    const bool bf16 = d->dtype == FK_BF16;
    least = 0;
    if (kind <= 2) return items > kSplitItems ? 1 : (int)std::max(1ll, std::min(most, (bf16 ? d->head_dim == 128 ? places : places * 3 / 8 : places / 2) / items));
    const double wide = kind == 8 ? 2. : 1., turn[3] = {wide, wide * 1.3, wide * 1.6};   // (of as many pairs as take 0.75 us alone with 64 rows)
    const int held = kind == 8 ? 2 : 3;   // workgroups that a CU holds
    const double turns = (double)pairs / (kind == 8 ? 64 : 32) * d->head_dim / 128 * (kind == 8 ? 1. : .75) * (bf16 ? 1. : 4.);
    auto allowed = [&](int s) { return s == 1 || (s <= most && items <= kSplitItems && items * s * kind <= 1 << 15 /* a quarter of a GiB of records */); };
    auto time_of = [&](int s) {
        const long long per_cu = (items * s + 255) / 256, rest = per_cu % held;
        const double rounds = (double)(per_cu / held) * turn[held - 1] + (rest ? turn[rest - 1] : 0.);
        return rounds * turns / s + (s == 1 ? 0. : 3 + (double)items * s * 16 * kind * d->head_dim * 8 / 4e6);
    };
    int best = 1;
    for (int s = 1; allowed(s); ++s) {
        const double time = time_of(s);
        if (s == 1 || time < least) least = time, best = s;
    }
    if (bound)
        for (int s = best + 1; allowed(s); ++s)
            if (time_of(s) <= least * (1 + 1e-9)) best = s;
    if (uneven && items <= kSplitItems / 2) best = (int)std::max((long long)best, std::min(most, places / items));
    return best;
}
// uneven: sequences in pages, several of them
static TreePlan tree_plan(const fk_paged_desc* d, int32_t n_tokens, int32_t max_tree, long long pairs, bool uneven) {
    const int g = d->n_q_heads / d->n_kv_heads, tree = std::min(std::min(max_tree, n_tokens), kTreeNodes), rows = tree * g;
    TreePlan p = {};
    double time = 0;
    auto take = [&](int kind) {   // the better one
        TreePlan x = {kind, tile_grid(d, n_tokens, tree, 16 * kind), 1, 0};
        double t;
        x.splits = tree_splits(d, kind, items_of(d, x.grid), pairs + tree, uneven, t);
        if (p.kind == 0 || t < time) p = x, time = t;
    };
    if (d->dtype == FK_F32) {
        take(rows <= 64 ? 1 : 4);
    } else {
        take(rows <= 16 ? 1 : rows <= 32 ? 2 : 4);
        if (rows > 64) take(8);
    }
    p.grid.most = kTreeNodes * g;
    const int kt = p.kind <= 2 ? (d->dtype == FK_BF16 ? 32 : 16) : d->dtype == FK_BF16 && (p.kind == 8 || d->head_dim == 64) ? 64 : d->dtype == FK_BF16 || d->head_dim == 64 ? 32 : 16;
    p.shift = (uneven ? 9 : 8) - __builtin_ctz(kt);
    return p;
}
// workspace: counters, the same for every call (so that calls of any sizes may take turns with one workspace) | sums and references of records | records
static constexpr size_t kCounterBytes = kSplitItems * 4 * sizeof(uint32_t);
static size_t ml_bytes(int kind, long long items, int splits) {   // wide: 16 bytes a lane and 16 rows; 8 a row
    return splits > 1 ? up256((size_t)items * splits * 16 * kind * (kind >= 4 ? 64 : 8)) : 0;
}
static size_t need_of(const fk_paged_desc* d, int kind, long long items, int splits) {
    return kCounterBytes + ml_bytes(kind, items, splits) + (splits > 1 ? (size_t)items * splits * 16 * kind * d->head_dim * sizeof(float) : 0);
}
static size_t need_of(const fk_paged_desc* d, const TreePlan& p) { return need_of(d, p.kind, items_of(d, p.grid), p.splits); }
// The most that a call of these sizes or smaller ones needs - fewer items are split more often, and go to other kernels: every kind and number of places that
// tree_plan and tile_grid can come to.
static size_t tree_workspace(const fk_paged_desc* d, int32_t n_tokens, int32_t max_tree, int32_t max_len, bool uneven) {
    const long long g = d->n_q_heads / d->n_kv_heads, tokens = std::max(n_tokens, 1), tree = std::min<long long>(std::min<long long>(max_tree, tokens), kTreeNodes), rows = tree * g;
    size_t most = kCounterBytes;
    auto look = [&](int kind, long long least_rows, long long most_rows) {   // the kind takes trees of more than least_rows query rows, up to most_rows
        if (rows <= least_rows) return;
        const long long tm = 16 * kind, per_seq = (std::min(rows, most_rows) + tm - 1) / tm, spread = tokens * g / tm + d->batch;
        auto with = [&](long long places) {
            double t;
            const long long items = places * d->n_kv_heads;
            most = std::max(most, need_of(d, kind, items, tree_splits(d, kind, items, max_len + tree, uneven, t, true)));
        };
        for (long long i = 1; i <= per_seq && i * d->batch <= 2 * spread && i * d->batch * d->n_kv_heads <= kSplitItems; ++i) with(i * d->batch);
        for (long long x = d->batch; x <= spread && 2 * x < per_seq * d->batch && x * d->n_kv_heads <= kSplitItems; ++x) with(x);
    };
    const long long all = kTreeNodes * g;
    if (d->dtype == FK_F32) {
        look(1, 0, 64);
        look(4, 64, all);
    } else {
        look(1, 0, 16);
        look(2, 16, 32);
        look(4, 32, all);
        look(8, 64, all);
    }
    return most;
}

template <typename T, int D, int KIND, bool ROWS, bool ONCE> static fk_status tree_start(const TreeParams& P, hipStream_t st) {
    using C = TreeKind<T, D, KIND>;
    auto kern = tree_kernel<T, D, KIND, ROWS, ONCE>;
    static bool lds_ok[kMaxDevices] = {};
    if (!allow_dynamic_lds((const void*)kern, C::LDS, lds_ok)) return FK_ERR_LAUNCH;
    const int items = P.a.grid.places * P.a.view.n_kv;
    hipLaunchKernelGGL(kern, dim3((unsigned)items, (unsigned)P.a.splits), dim3(256), C::LDS, st, P);
    return launch_status();
}
template <typename T, int D, bool ROWS> static fk_status tree_rows_of(int kind, const TreeParams& P, hipStream_t st) {
    if constexpr (sizeof(T) == 2) {
        const bool once = !P.a.grid.spread && P.a.grid.per_seq == 1;
        if (kind == 2) return tree_start<T, D, 2, ROWS, false>(P, st);
        if (kind == 8) return once ? tree_start<T, D, 8, ROWS, true>(P, st) : tree_start<T, D, 8, ROWS, false>(P, st);
        if (kind == 4 && once) return tree_start<T, D, 4, ROWS, true>(P, st);
    }
    return kind == 1 ? tree_start<T, D, 1, ROWS, false>(P, st) : tree_start<T, D, 4, ROWS, false>(P, st);
}
template <bool ROWS> static fk_status tree_launch(const fk_paged_desc* d, const TreePlan& p, TreeParams& P, void* ws, hipStream_t st) {
    AttnPagedParams& A = P.a;
    A.grid = p.grid;
    A.splits = p.splits;
    A.split_shift = p.shift;
    P.here = static_cast<uint32_t*>(ws);
    A.rec_ml = reinterpret_cast<float2*>(static_cast<char*>(ws) + kCounterBytes);
    A.rec = reinterpret_cast<float*>(static_cast<char*>(ws) + kCounterBytes + ml_bytes(p.kind, items_of(d, p.grid), p.splits));
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
    return tree_workspace(&d, n_tokens, max_tree, max_len, false);
}

extern "C" fk_status fk_tree_attn(const fk_cache_desc* desc, const void* q, const void* K, const void* V, const int32_t* len, const void* k_tree,
                                  const void* v_tree, const int32_t* parent, const int32_t* q_start, int32_t n_tokens, int32_t max_tree,
                                  int32_t max_len, float softmax_scale, void* out, float* stats, void* workspace, size_t workspace_bytes, void* stream) {
    fk_status s = check_rows(desc, n_tokens, max_tree, max_len);
    if (s != FK_OK) return s;
    const fk_paged_desc d = as_paged(desc);
    s = check_trees(&d, q, K, V, len, k_tree, v_tree, parent, q_start, n_tokens, max_tree, out, stats);
    if (s != FK_OK) return s;
    const TreePlan plan = tree_plan(&d, std::max(n_tokens, 1), max_tree, max_len, false);
    if (!workspace || workspace_bytes < need_of(&d, plan) || !aligned16(workspace)) return FK_ERR_WORKSPACE;
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
    return tree_launch<true>(&d, plan, P, workspace, (hipStream_t)stream);
}

static fk_status check_pages(const fk_paged_desc* desc, int32_t n_tokens, int32_t max_tree, int32_t max_len) {
    fk_status s = check_paged(desc);
    if (s != FK_OK) return s;
    if (max_len <= 0 || (int64_t)max_len > (int64_t)desc->max_pages * desc->page_size) return FK_ERR_INVALID_ARG;
    return check_tree_sizes(desc, n_tokens, max_tree);
}

extern "C" size_t fk_paged_tree_attn_workspace(const fk_paged_desc* desc, int32_t n_tokens, int32_t max_tree, int32_t max_len) {
    if (check_pages(desc, n_tokens, max_tree, max_len) != FK_OK) return 0;
    return tree_workspace(desc, n_tokens, max_tree, max_len, desc->batch > 1);
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
    const TreePlan plan = tree_plan(desc, std::max(n_tokens, 1), max_tree, max_len, desc->batch > 1);
    if (!workspace || workspace_bytes < need_of(desc, plan) || !aligned16(workspace)) return FK_ERR_WORKSPACE;
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
    return tree_launch<false>(desc, plan, P, workspace, (hipStream_t)stream);
}
