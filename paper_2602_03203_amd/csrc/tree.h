// Attention of trees of drafted tokens over a cache: the rows of a budgeted cache or the pages of a prompt (fk_tree_attn, fk_paged_tree_attn).
//
// The query rows of a (tree, KV head) are its nodes times the heads of the group; a workgroup takes a tile of them and a split of what they
// see: the pairs of the cache, which all nodes see (but for a window), then the pairs of the tree, a node its ancestors' and its own.
// Products and operand layouts are those of thin.h: logits K.Q^T with the keys in an order that makes a lane's probabilities an operand of V^T.P^T as
// they are.  Which ancestors a node has is a bit for every node of its tree: found once per workgroup, in LDS, by walking up from it.
#pragma once
#include "attn_paged.h"
#include "prompt.h"
#include <type_traits>

namespace fk {

static constexpr int kTreeNodes = FK_TREE_NODES;

struct TreeParams {
    AttnPagedParams a;         // view (rows of a budgeted cache: kv_len is len, [batch][n_kv]), out, stats, grid, splits, split_shift, rec, rec_ml, cap
    const int32_t* parent;
    const void *k_tree, *v_tree;
    uint32_t* here;            // [items][4] splits whose records are there; zero between calls
};
static constexpr int kMostTreeSplits = 16;
static constexpr int kSplitItems = 1024;   // a call with more items (a tile of rows, a KV head) splits none

// Records of split tiles go from workgroup to workgroup by agent-scope relaxed atomics: loads and stores that pass the caches of the XCDs, which
// costs nothing next to a fence that writes back and invalidates a whole L2.  None is needed for these words: a wavefront waits for its stores (vmcnt 0: they are where every
// XCD sees them) before its workgroup's counter goes up, and the last one sends its loads when the counter's answer is there, for none of which a cache is asked.  That is an
// order of gfx950's own, with the waits as they stand here; the language promises it for acquire and release alone.
__device__ __forceinline__ void put2(float* p, float a, float b) {
    __hip_atomic_store(reinterpret_cast<uint64_t*>(p), (uint64_t)__float_as_uint(b) << 32 | __float_as_uint(a), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
__device__ __forceinline__ float2 get2(const float* p) {
    const uint64_t x = __hip_atomic_load(reinterpret_cast<const uint64_t*>(p), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    return make_float2(__uint_as_float((uint32_t)x), __uint_as_float((uint32_t)(x >> 32)));
}
// One more split of `splits` has its record there (its stores have arrived): true for the last one, which leaves the counter at zero.  One lane's business.
__device__ __forceinline__ bool last_one(uint32_t* here, int splits) {
    const bool last = __hip_atomic_fetch_add(here, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == (uint32_t)splits - 1;
    if (last) __hip_atomic_store(here, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    return last;
}

// bf16: a weight meets V as two terms, the first cut off and the second the rest, rounded: 2^-15 of it off at most (one term is off by up to 2^-8, alike for equal weights,
// which no average takes away).  Sums of weights are those of the unrounded ones.  The rest is taken 2^-20 too large, so that both terms of a weight above 0 (from 2^-106 on) are
// above 0 and an infinity among the values stays one.  With one term and two: 4 nodes for each of 16 sequences of 2112 pairs, 8 heads of g 4, D 128, 27.4 us either way, 12 nodes 32.7
// and 33.0, 64 nodes 60 and 70, D 64 40.3 and 40.5; 26 nodes of g 7 over 4160 pairs 53 and 57.
__device__ __forceinline__ void two_terms(float a, float b, uint32_t& first, uint32_t& second) {
    first = __builtin_amdgcn_perm(__float_as_uint(b), __float_as_uint(a), 0x07060302u);
    second = pack_bf16(fmaf(a, 1.f + 0x1p-20f, -__uint_as_float(__float_as_uint(a) & 0xffff0000u)), fmaf(b, 1.f + 0x1p-20f, -__uint_as_float(__float_as_uint(b) & 0xffff0000u)));
}

// What a workgroup works on; false: nothing
struct TreeWork {
    TileOf t;
    int h, n;                  // KV head, pairs of the cache
    int r0, rows;              // query rows of the tile
    int tok_lo, tok_hi;        // nodes that they belong to
    KeyTiles old;              // tiles of the cache's pairs
    int total, splits;         // with those of the tree
};
template <bool ROWS>
__device__ __forceinline__ bool tree_work(const AttnPagedParams& P, int item, int tm, TreeWork& w) {
    const PagedParams& W = P.view;
    const int slot = scalar(divide(item, W.n_kv, W.kv_magic));
    w.h = item - slot * W.n_kv;
    if (!tile_of(W, P.grid, slot, tm, w.t)) return false;
    if constexpr (ROWS) w.t.n = scalar(min(max(load_uniform(W.kv_len, w.t.b * W.n_kv + w.h), 0), P.cap));
    w.n = w.t.n;
    return true;
}
__device__ __forceinline__ void tree_tile_of(const AttnPagedParams& P, int tm, int kt, TreeWork& w) {
    const PagedParams& W = P.view;
    w.r0 = w.t.tile * tm;
    w.rows = min(tm, w.t.nq * W.g - w.r0);
    w.tok_lo = scalar(divide(w.r0, W.g, W.g_magic));
    w.tok_hi = scalar(divide(w.r0 + w.rows - 1, W.g, W.g_magic));
    w.old = key_tiles(W, w.n, w.n - 1, kt);   // (the root, at position n, sees the most under a window)
    w.total = w.old.total + (uint32_t)(w.tok_hi + kt) / (uint32_t)kt;   // (parents come first: nobody sees a later node)
    w.splits = scalar(splits_of(w.total, w.t.one ? P.splits : 1, P.split_shift));
}

// In LDS: of a tile's nodes, counted from its first one, whom they see of their tree
template <int TM> struct Ancestors {
    int16_t parent[kTreeNodes];
    uint32_t sees[TM][kTreeNodes / 32];
    uint32_t any[kTreeNodes / 32], all[kTreeNodes / 32];   // of a run's nodes some see, all see
    int level[TM];             // under a window
};
template <int TM> __device__ __forceinline__ void find_ancestors(const TreeParams& TP, const TreeWork& w, bool windowed, Ancestors<TM>& s) {
    const PagedParams& W = TP.a.view;
    for (int i = threadIdx.x; i <= w.tok_hi; i += 256) {
        const int p = TP.parent[w.t.begin + i];
        s.parent[i] = (int16_t)(p < i ? max(p, -1) : -1);
    }
    __syncthreads();
    for (int i = threadIdx.x; i <= w.tok_hi - w.tok_lo; i += 256) {
        const int self = w.tok_lo + i;
        int level = 0;
        if (windowed) {
            for (int a = s.parent[self]; a >= 0; a = s.parent[a]) ++level;
            s.level[i] = level;
        }
#pragma unroll
        for (int x = 0; x < kTreeNodes / 32; ++x) s.sees[i][x] = 0;
        int up = 0;   // levels from the node to its ancestor
        for (int a = self; a >= 0; a = s.parent[a], ++up)
            if (!windowed || up < W.window || w.n + level - up < W.sink) s.sees[i][a / 32] |= 1u << a % 32;
    }
    __syncthreads();
}
// A run's nodes lo .. hi, counted from the tile's first: what they see together.  level_lo, level_hi: their levels, under a window
template <int TM> __device__ __forceinline__ void span_of(Ancestors<TM>& s, bool windowed, int lo, int hi, int& level_lo, int& level_hi) {
    if (threadIdx.x < kTreeNodes / 32) {
        s.any[threadIdx.x] = 0;
        s.all[threadIdx.x] = ~0u;
    }
    __syncthreads();
    constexpr int WORDS = kTreeNodes / 32;
    for (int i = lo * WORDS + threadIdx.x; i < (hi + 1) * WORDS; i += 256) {
        const uint32_t x = s.sees[i / WORDS][i % WORDS];
        atomicOr(&s.any[i % WORDS], x);
        atomicAnd(&s.all[i % WORDS], x);
    }
    level_lo = level_hi = 0;
    if (windowed) {
        level_lo = level_hi = s.level[lo];
        for (int i = lo + 1; i <= hi; ++i) {
            level_lo = min(level_lo, s.level[i]);
            level_hi = max(level_hi, s.level[i]);
        }
        level_lo = scalar(level_lo);
        level_hi = scalar(level_hi);
    }
    __syncthreads();
}

// ---------------------------------------------------------------------------------------------------------
// Up to RB * 16 query rows: the wavefronts of a workgroup take tiles of KT pairs in turn, straight from memory into registers, each with its own
// online softmax for all rows; they are merged through LDS at the end.  An operand of K or V serves a product for each 16 rows.  K and V of the next tile
// are sent off when this one's products have read theirs.  Bound by the memory system: 4 nodes for each of 16 sequences of 2112 pairs, 8 heads of g 4, D 128
// (139 MB) 27.4 us, 8 nodes 30.6; one sequence, whose splits hold 256 pairs each, by the latency of its loads and of the merge: 11.6.
// ---------------------------------------------------------------------------------------------------------
template <typename T, int D, int RB> struct TreeCfg {
    static constexpr bool BF = sizeof(T) == 2;
    static constexpr int CH = D * (int)sizeof(T) / 16;   // 16-byte chunks of a row
    static constexpr int KT = BF ? 32 : 16;
    static constexpr int NT = KT / 16;                   // 16-key products of a tile
    static constexpr int KS = CH / 4;                    // chunks of a key per lane
    static constexpr int VL = BF ? 8 : 4 * D / 64;       // V loads per lane and tile (bf16 D = 64: 8 bytes each)
    static constexpr int ET = D / 16;                    // channel tiles of the output
    static constexpr int TM = 16 * RB, WAVES = 4;
    static constexpr int PART = D + 4;                   // float stride of a row of a partial output in LDS
    // LDS: partial outputs [WAVES][TM][PART] | maxima, sums, merge weights [WAVES][TM] each | merged maxima and sums [TM] each
    static constexpr size_t LDS = sizeof(float) * ((size_t)WAVES * TM * PART + 3 * WAVES * TM + 2 * TM);
};

template <typename T, int D, int RB, bool ROWS>
__device__ __forceinline__ void tree_tile(const TreeParams& TP, int item, int split) {
    using C = TreeCfg<T, D, RB>;
    constexpr bool BF = C::BF;
    constexpr int CH = C::CH, KT = C::KT, NT = C::NT, KS = C::KS, VL = C::VL, ET = C::ET, PART = C::PART, TM = C::TM, WAVES = C::WAVES;
    const AttnPagedParams& P = TP.a;
    const PagedParams& W = P.view;
    const int tid = threadIdx.x, lane = tid & (kWave - 1), n16 = lane & 15, quad = lane >> 4;
    const int wave = scalar(tid / kWave);
    const int n_kv = W.n_kv, g = W.g;
    extern __shared__ __attribute__((aligned(16))) float smem_tree[];
    float (*s_o)[TM][PART] = reinterpret_cast<float (*)[TM][PART]>(smem_tree);
    float (*s_m)[TM] = reinterpret_cast<float (*)[TM]>(smem_tree + WAVES * TM * PART), (*s_l)[TM] = s_m + WAVES, (*s_w)[TM] = s_l + WAVES;
    float *s_M = s_w[WAVES], *s_L = s_M + TM;
    __shared__ Ancestors<TM> s_tree;
    __shared__ int s_bad;   // a value that not every row of a run sees is infinite or NaN

    TreeWork w;
    if (!tree_work<ROWS>(P, item, TM, w)) return;
    const TileOf& t = w.t;
    const int n = w.n, h = w.h;
    const bool windowed = !ROWS && W.window != 0x7fffffff;
    const size_t tree_at = ((size_t)t.begin * n_kv + h) * CH * 16;
    const int32_t* tab = ROWS ? nullptr : scalar_ptr(W.table + (size_t)t.b * W.max_pages);
    for (; w.t.tile >= 0; w.t.tile -= w.t.step) {
        tree_tile_of(P, TM, KT, w);
        if (split >= w.splits) continue;
        const int r0 = w.r0, rows = w.rows, splits = w.splits, total = w.total;
        const int per = splits == 1 ? total : scalar(divide(total + splits - 1, splits)), t_begin = min(split * per, total), t_end = min(t_begin + per, total);
        auto token_of = [&](int r) { return divide(r, g, W.g_magic); };

        T128 q[RB][KS];
#pragma unroll
        for (int rb = 0; rb < RB; ++rb) {
            const int r = r0 + min(rb * 16 + n16, rows - 1), token = token_of(r);
            const size_t q_row = ((size_t)(t.begin + token) * n_kv + h) * g + (r - token * g);
#pragma unroll
            for (int ks = 0; ks < KS; ++ks) {
                q[rb][ks].u = reinterpret_cast<const tu32x4_t*>(W.q)[q_row * CH + ks * 4 + quad];
                if (W.negate) q[rb][ks].u ^= BF ? 0x80008000u : 0x80000000u;
            }
        }
        const float scale = W.scale_log2e;

        // where a tile's pairs lie: pair u of run u / 16 at at[run] + min(u, last) * stride bytes of K and V; a bit for each run that lies nowhere
        struct Place {
            size_t at[NT];
            int stride, last, base, holes;
            bool tree;
        };
        auto place_of = [&](int i) {
            Place p;
            p.tree = i >= w.old.total;
            p.holes = 0;
            if (p.tree) {
                p.base = (i - w.old.total) * KT;
                p.stride = n_kv * CH * 16;
                p.last = t.nq - 1 - p.base;
#pragma unroll
                for (int r = 0; r < NT; ++r) p.at[r] = tree_at + (size_t)p.base * p.stride;
                return p;
            }
            p.base = w.old.at(i) * KT;
            p.stride = CH * 16;
            p.last = ROWS ? n - 1 - p.base : KT;
#pragma unroll
            for (int r = 0; r < NT; ++r) {
                if constexpr (ROWS) {
                    p.at[r] = (((size_t)t.b * n_kv + h) * P.cap + p.base) * CH * 16;
                } else {
                    const int key = p.base + r * 16, page = load_uniform(tab, min(key >> W.page_shift, W.max_pages - 1));
                    const bool ok = page_ok(W, page);
                    if (!ok) p.holes |= 1 << r;
                    p.at[r] = ((((size_t)(ok ? page : 0) * n_kv + h) << W.page_shift) + (key & ((1 << W.page_shift) - 1))) * CH * 16 - r * 16 * CH * 16;
                }
            }
            return p;
        };
        // pair u of a tile, in the first run or the second, from `lane_at` bytes on (rows: one base for all lanes and an offset of 32 bits each)
        auto pair_at = [&](const void* cache, const void* tree, const Place& p, int u, bool second, int lane_at) {
            const unsigned char* X = static_cast<const unsigned char*>(p.tree ? tree : cache);
            const uint32_t off = (uint32_t)min(u, p.last) * (uint32_t)p.stride + lane_at;
            return reinterpret_cast<const tu32x4_t*>(X + (!ROWS && NT == 2 && second ? p.at[NT - 1] : p.at[0]) + off);
        };
        T128 kr[NT][KS], vr[VL];
        auto load_k = [&](const Place& p) {
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) {
                // with this order of keys, a lane's logits are keys quad * 8 + u (fp32: quad * 4 + i)
                const tu32x4_t* x = pair_at(W.K, TP.k_tree, p, BF ? n16 / 4 * 8 + nt * 4 + n16 % 4 : n16, n16 >= 8, quad * 16);
#pragma unroll
                for (int ks = 0; ks < KS; ++ks) kr[nt][ks].u = x[ks * 4];
            }
        };
        auto load_v = [&](const Place& p) {
#pragma unroll
            for (int u = 0; u < (BF ? 8 : 4); ++u) {
                const tu32x4_t* x = pair_at(W.V, TP.v_tree, p, quad * (BF ? 8 : 4) + u, quad >= 2, n16 * (BF && D == 64 ? 8 : 16));
                if constexpr (!BF) {
#pragma unroll
                    for (int c = 0; c < D / 64; ++c) vr[u * (D / 64) + c].u = x[c * 16];
                } else if constexpr (D == 128) {
                    vr[u].u = *x;
                } else {
                    const tu32x2_t y = *reinterpret_cast<const tu32x2_t*>(x);
                    vr[u].w[0] = y.x;
                    vr[u].w[1] = y.y;
                }
            }
        };
        constexpr int VW = BF && D == 64 ? 2 : 4;   // words in use of a V load

        Place at, next;
        auto begin = [&]() {
            if (t_begin + wave >= t_end) return;
            at = place_of(t_begin + wave);
            load_k(at);
            load_v(at);
        };
        begin();   // (on their way while the ancestors are found)
        // The rows of all nodes at once.  A row gives the pairs that it does not see weight 0, which must not meet an infinity or a NaN that another row
        // sees: where there is any, the run starts over with half of its nodes.
        const int nodes = w.tok_hi - w.tok_lo + 1;
        const bool some_tree = t_end > w.old.total;
        if (windowed || some_tree) find_ancestors<TM>(TP, w, windowed, s_tree);
        for (int lo = 0, hi = nodes - 1;;) {
        int level_lo = 0, level_hi = 0;
        if (tid == 0) s_bad = 0;
        if (windowed || some_tree) span_of<TM>(s_tree, windowed, lo, hi, level_lo, level_hi);
        else __syncthreads();
        const int any_from = windowed ? n + level_lo - W.window + 1 : 0, all_from = windowed ? n + level_hi - W.window + 1 : 0;
        float m_run[RB], l_run[RB];
        tf32x4_t o[RB][ET];
#pragma unroll
        for (int rb = 0; rb < RB; ++rb) {
            m_run[rb] = -INFINITY;
            l_run[rb] = 0.f;
#pragma unroll
            for (int e = 0; e < ET; ++e) o[rb][e] = (tf32x4_t){0.f, 0.f, 0.f, 0.f};
        }
        int i = t_begin + wave;
        auto tile = [&](auto LAST) {   // (twice in the code: under a condition the next tile's loads would need registers of their own)
            tf32x4_t c[RB][NT];
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                for (int rb = 0; rb < RB; ++rb) {
                    c[rb][nt] = (tf32x4_t){0.f, 0.f, 0.f, 0.f};
#pragma unroll
                    for (int ks = 0; ks < KS; ++ks) {
                        if constexpr (BF) {
                            c[rb][nt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kr[nt][ks].v, q[rb][ks].v, c[rb][nt], 0, 0, 0);
                        } else {
#pragma unroll
                            for (int e = 0; e < 4; ++e) c[rb][nt] = __builtin_amdgcn_mfma_f32_16x16x4f32(kr[nt][ks].f[e], q[rb][ks].f[e], c[rb][nt], 0, 0, 0);
                        }
                    }
                }
            if constexpr (!LAST) {
                next = place_of(i + WAVES);
                load_k(next);
            }

            float s[RB][NT * 4];
#pragma unroll
            for (int rb = 0; rb < RB; ++rb)
#pragma unroll
                for (int j = 0; j < NT * 4; ++j) s[rb][j] = attn_logit(c[rb][j / 4][j % 4], scale);
            // everything seen by every row: no masks
            const bool whole = !at.tree && at.base + KT <= n && !at.holes && (at.base >= all_from || at.base + KT <= W.sink);
            if (!whole) {
                int me = lane;
                asm volatile("" : "+v"(me));
                const int quad = me >> 4, n16 = me & 15, k0 = quad * (NT * 4);   // first of the lane's keys in the tile
                const bool there = !(at.holes >> (NT == 2 && quad >= 2 ? 1 : 0) & 1);   // (its keys of K and of V lie in the same run)
#pragma unroll
                for (int rb = 0; rb < RB; ++rb) {
                    uint32_t sees = 0;   // a bit for each of the lane's keys
                    const int tok = token_of(r0 + min(rb * 16 + n16, rows - 1)) - w.tok_lo, from = windowed ? n + s_tree.level[tok] - W.window + 1 : 0;
                    if (at.tree) {
                        sees = s_tree.sees[tok][at.base / 32] >> (at.base % 32 + k0);
                    } else {
#pragma unroll
                        for (int j = 0; j < NT * 4; ++j) {
                            const int key = at.base + k0 + j;
                            sees |= (uint32_t)(there & (key < n) & ((key >= from) | (key < W.sink))) << j;
                        }
                    }
                    if (tok < lo || tok > hi) sees = 0;
#pragma unroll
                    for (int j = 0; j < NT * 4; ++j) s[rb][j] = sees >> j & 1 ? s[rb][j] : -INFINITY;
                }
                bool bad = false;
                uint32_t any = ~0u, all = 0;
                if (at.tree) {
                    any = s_tree.any[at.base / 32] >> (at.base % 32 + k0);
                    all = s_tree.all[at.base / 32] >> (at.base % 32 + k0);
                }
#pragma unroll
                for (int x = 0; x < VL; ++x) {
                    const int u = BF ? x : x / (D / 64), key = at.base + k0 + u;
                    const bool someone = at.tree ? any >> u & 1 : there & (key < n) & ((key >= any_from) | (key < W.sink));
                    const bool everyone = at.tree ? all >> u & 1 : (key >= all_from) | (key < W.sink);
                    const uint32_t keep = someone ? ~0u : 0u;
#pragma unroll
                    for (int k = 0; k < VW; ++k) {
                        vr[x].w[k] &= keep;
                        bad |= !everyone & word_not_finite<T>(vr[x].w[k]);
                    }
                }
                if (bad && hi > lo) s_bad = 1;
            }
            T128 pr[RB], pr2[RB];   // bf16: the probabilities' two terms
#pragma unroll
            for (int rb = 0; rb < RB; ++rb) {
                float mx = s[rb][0];
#pragma unroll
                for (int j = 1; j < NT * 4; ++j) mx = fmaxf(mx, s[rb][j]);
                const float mn = fmaxf(m_run[rb], quad_max(mx)), ref = ref_of(mn);
                const bool moved = mn > m_run[rb];
                const float corr = __builtin_amdgcn_exp2f(m_run[rb] - ref);
                m_run[rb] = mn;
                float sum = 0.f;
#pragma unroll
                for (int j = 0; j < NT * 4; ++j) {
                    s[rb][j] = __builtin_amdgcn_exp2f(s[rb][j] - ref);
                    sum += s[rb][j];
                }
                l_run[rb] = fmaf(l_run[rb], corr, sum);
                if (__any(moved)) {
#pragma unroll
                    for (int e = 0; e < ET; ++e)
#pragma unroll
                        for (int k = 0; k < 4; ++k) o[rb][e][k] *= corr;
                }
                if constexpr (BF) {
#pragma unroll
                    for (int x = 0; x < 4; ++x) two_terms(s[rb][2 * x], s[rb][2 * x + 1], pr[rb].w[x], pr2[rb].w[x]);
                }
            }
#pragma unroll
            for (int e = 0; e < ET; ++e) {   // V^T.P^T
                if constexpr (BF) {
                    const uint32_t sel = (e & 1) ? 0x07060302u : 0x05040100u;
                    T128 vb;
#pragma unroll
                    for (int x = 0; x < 4; ++x) vb.w[x] = __builtin_amdgcn_perm(vr[2 * x + 1].w[e >> 1], vr[2 * x].w[e >> 1], sel);
#pragma unroll
                    for (int rb = 0; rb < RB; ++rb) o[rb][e] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vb.v, pr[rb].v, o[rb][e], 0, 0, 0);
#pragma unroll
                    for (int rb = 0; rb < RB; ++rb) o[rb][e] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vb.v, pr2[rb].v, o[rb][e], 0, 0, 0);
                } else {
#pragma unroll
                    for (int u = 0; u < 4; ++u)
#pragma unroll
                        for (int rb = 0; rb < RB; ++rb) o[rb][e] = __builtin_amdgcn_mfma_f32_16x16x4f32(vr[u * (D / 64) + e / 4].f[e % 4], s[rb][u], o[rb][e], 0, 0, 0);
                }
            }
            if constexpr (!LAST) {
                load_v(next);
                at = next;
            }
        };
        for (; i + WAVES < t_end; i += WAVES) tile(std::false_type());
        if (i < t_end) tile(std::true_type());

        // ---- merge the wavefronts ----------------------------------------------------------------------------------
        int tid = threadIdx.x;   // (opaque: or all that the merge derives from it is kept in registers over the loop)
        asm volatile("" : "+v"(tid));
        const int n16 = tid & 15, quad = (tid & (kWave - 1)) >> 4;
#pragma unroll
        for (int rb = 0; rb < RB; ++rb) {
            const float l = quad_sum(l_run[rb]);
            const int r = rb * 16 + n16;
            if (quad == 0) {
                s_m[wave][r] = m_run[rb];
                s_l[wave][r] = l;
            }
#pragma unroll
            for (int k = 0; k < 4; ++k)
#pragma unroll
                for (int e = 0; e < ET; e += 4) {
                    const int ch = BF ? (quad * 4 + k) * ET + e : e / 4 * 64 + (quad * 4 + k) * 4;
                    *reinterpret_cast<float4*>(&s_o[wave][r][ch]) = make_float4(o[rb][e][k], o[rb][e + 1][k], o[rb][e + 2][k], o[rb][e + 3][k]);
                }
        }
        __syncthreads();
        if (scalar(s_bad)) {   // (the same for every thread)
            hi = lo + (hi - lo) / 2;
            __syncthreads();
            begin();
            continue;
        }
        if (tid < TM) {
            float M = -INFINITY, L = 0.f;
#pragma unroll
            for (int x = 0; x < WAVES; ++x) M = fmaxf(M, s_m[x][tid]);
            const float ref = ref_of(M);
#pragma unroll
            for (int x = 0; x < WAVES; ++x) {
                const float f = __builtin_amdgcn_exp2f(s_m[x][tid] - ref);
                s_w[x][tid] = f;
                L = fmaf(s_l[x][tid], f, L);
            }
            s_M[tid] = M;
            s_L[tid] = L;
        }
        __syncthreads();
        const size_t rec = ((size_t)item * P.splits + split) * TM;
        for (int x = tid; x < rows * (D / 4); x += WAVES * kWave) {
            const int r = x / (D / 4), d = x % (D / 4) * 4, token = token_of(r0 + r);
            if (token - w.tok_lo < lo || token - w.tok_lo > hi) continue;
            float a[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int y = 0; y < WAVES; ++y) {
                const float4 v = *reinterpret_cast<const float4*>(&s_o[y][r][d]);
                const float f = s_w[y][r];
                a[0] = fmaf(v.x, f, a[0]);
                a[1] = fmaf(v.y, f, a[1]);
                a[2] = fmaf(v.z, f, a[2]);
                a[3] = fmaf(v.w, f, a[3]);
            }
            if (splits > 1) {
                put2(P.rec + rec * D + x * 2, a[0], a[1]);   // (neighbouring lanes side by side: these stores are not gathered on their way)
                put2(P.rec + rec * D + TM * D / 2 + x * 2, a[2], a[3]);
                if (d == 0) put2(reinterpret_cast<float*>(P.rec_ml + rec + r), s_M[r], s_L[r]);
                continue;
            }
            store_row<T, D, false>(P, ((size_t)(t.begin + token) * n_kv + h) * g + (r0 + r - token * g), d, a, s_M[r], s_L[r]);
        }
        __syncthreads();   // the LDS is the next run's
        if (hi == nodes - 1) break;
        lo = hi + 1;
        hi = nodes - 1;
        begin();
        }
        if (splits == 1) continue;
        // the last workgroup to arrive adds the records up, in the order of the splits
        int tid = threadIdx.x;
        asm volatile("" : "+v"(tid));
        arrived();
        __syncthreads();
        if (tid == 0) s_bad = last_one(TP.here + item * 4, splits);
        __syncthreads();
        if (!scalar(s_bad)) return;   // (a split tile is its place's only one)
        // (in LDS, in the place of the wavefronts' own: every split's factor for a row)
        float (*s_f)[TM] = reinterpret_cast<float (*)[TM]>(smem_tree);
        static_assert(kMostTreeSplits <= WAVES * 16 && (size_t)kMostTreeSplits * TM <= (size_t)WAVES * TM * PART, "room for the factors");
        const size_t rec = (size_t)item * P.splits * TM;
        if (tid < rows) {
            float2 ml[kMostTreeSplits];
            float M = -INFINITY, L = 0.f;
#pragma unroll
            for (int u = 0; u < kMostTreeSplits; ++u) {
                ml[u] = get2(reinterpret_cast<const float*>(P.rec_ml + rec + min(u, splits - 1) * TM + tid));
                M = fmaxf(M, ml[u].x);   // (the copies past the end change nothing)
            }
            const float ref = ref_of(M);
#pragma unroll
            for (int u = 0; u < kMostTreeSplits; ++u) {
                const float f = __builtin_amdgcn_exp2f(ml[u].x - ref);
                s_f[u][tid] = f;
                L = u < splits ? fmaf(ml[u].y, f, L) : L;
            }
            s_M[tid] = M;
            s_L[tid] = L;
        }
        __syncthreads();
        constexpr int UNITS = TM * (D / 4) / (WAVES * kWave);   // four channels of a row, this many a thread
        float a[UNITS][4];
#pragma unroll
        for (int y = 0; y < UNITS; ++y)
#pragma unroll
            for (int k = 0; k < 4; ++k) a[y][k] = 0.f;
        for (int s0 = 0; s0 < splits; s0 += 4) {   // four records' loads in flight
            float2 v[4][UNITS][2];
#pragma unroll
            for (int u = 0; u < 4; ++u)
#pragma unroll
                for (int y = 0; y < UNITS; ++y) {
                    const float* from = P.rec + (rec + min(s0 + u, splits - 1) * TM) * D + min(tid + y * WAVES * kWave, rows * (D / 4) - 1) * 2;
                    v[u][y][0] = get2(from);
                    v[u][y][1] = get2(from + TM * D / 2);
                }
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                if (s0 + u >= splits) break;
#pragma unroll
                for (int y = 0; y < UNITS; ++y) {
                    const float f = s_f[s0 + u][min((tid + y * WAVES * kWave) / (D / 4), rows - 1)];
                    a[y][0] = fmaf(v[u][y][0].x, f, a[y][0]);
                    a[y][1] = fmaf(v[u][y][0].y, f, a[y][1]);
                    a[y][2] = fmaf(v[u][y][1].x, f, a[y][2]);
                    a[y][3] = fmaf(v[u][y][1].y, f, a[y][3]);
                }
            }
        }
#pragma unroll
        for (int y = 0; y < UNITS; ++y) {
            const int x = tid + y * WAVES * kWave, r = x / (D / 4), d = x % (D / 4) * 4;
            if (r >= rows) break;
            const int token = token_of(r0 + r);
            store_row<T, D, false>(P, ((size_t)(t.begin + token) * n_kv + h) * g + (r0 + r - token * g), d, a[y], s_M[r], s_L[r]);
        }
        return;
    }
}

// ---------------------------------------------------------------------------------------------------------
// More than 32 query rows: a wavefront owns CT * 16 of them, and the pairs pass by in tiles of KT, each read once for the four wavefronts, straight into
// LDS: three places each for K and V, so that a tile's loads have two turns to arrive, one barrier a turn.  Layouts in LDS and the order of a
// turn's steps - the next tile's logits beside this one's softmax - are those of prompt.h.
// The compiler, which sees loads into LDS and reads of it, has to be told that they are of different places (the __restrict pointers of `turn`), or it waits for
// all loads before the first read.
// Bound by a turn's chain of LDS reads, products and exponentials, with two or three wavefronts a SIMD to fill its gaps (a turn of 64 pairs for 128 rows takes
// 2.1 us with the CU to itself, 3.1 beside another workgroup; the products are 0.64): 64 nodes for each of 16 sequences of 16384 pairs, 8 heads of g 4, D 128, 417 us,
// 660 TFLOP/s.  Matrix cores are busy a third of the time, vector units as long.  Smaller calls spend as long
// on a workgroup's start and the merge: 12 nodes over 16 rows of 2112 pairs 33 us, of which the pairs' way from memory is 22.
// ---------------------------------------------------------------------------------------------------------
template <typename T, int D, int CT_> struct WideCfg {
    static constexpr bool BF = sizeof(T) == 2;
    static constexpr int CT = CT_, CH = D * (int)sizeof(T) / 16, KS = CH / 4, ET = D / 16;
    static constexpr int KT = BF && (CT == 2 || D == 64) ? 64 : 512 / CH;   // pairs of a tile
    static constexpr int PLACES = KT * CH * 16 > 8192 ? 2 : 3;              // 64 KB of LDS at most: two workgroups on a CU
    static constexpr int NT = BF ? 2 : 1, BLK = 16 * NT, NB = KT / BLK, GI = KT / 16;
    static constexpr int TM = 64 * CT;
    static constexpr int LD = KT * CH / 256, RPU = 256 / CH;   // loads of a tile per thread and tensor; rows that one load of the workgroup covers
    static constexpr int TILE_BYTES = KT * CH * 16;
    static constexpr size_t LDS = 2 * PLACES * (size_t)TILE_BYTES;
};

// load_to_lds of pairs that nobody else reads: not kept (up to 96 rows of 16 sequences of 4000 pairs in pages: 87 -> 79 us; beside a second tile of rows, which
// reads them too, 225 -> 234)
__device__ __forceinline__ void load_once_to_lds(const void* from, unsigned char* to) {
    __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)from, (__attribute__((address_space(3))) void*)to, 16, 0, 2);
}

// The wavefront's loads are there but for the latest N, and what it has read of LDS; then the workgroup's.  (__syncthreads would wait for all loads.)
template <int N> __device__ __forceinline__ void arrived_but() {
    asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"(N) : "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
}
__device__ __forceinline__ void lds_barrier() {
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
}

// a lane's share of a row: x in the layout of the products, times inv; M and L
template <typename T, int D>
__device__ __forceinline__ void store_wide(const AttnPagedParams& P, size_t row, int quad, const tf32x4_t (&x)[D / 16], float M, float L, float inv) {
#pragma unroll
    for (int e = 0; e < D / 16; e += sizeof(T) == 2 ? 1 : 4) {
        if constexpr (sizeof(T) == 2) {   // channels e * 16 + quad * 4 ..
            const tf32x4_t a = x[e] * inv;
            *reinterpret_cast<tu32x2_t*>(reinterpret_cast<bf16_t*>(P.out) + row * D + e * 16 + quad * 4) = tu32x2_t{pack_bf16(a[0], a[1]), pack_bf16(a[2], a[3])};
        } else {
#pragma unroll
            for (int k = 0; k < 4; ++k)   // e / 4 * 64 + (quad * 4 + k) * 4 ..
                *reinterpret_cast<float4*>(reinterpret_cast<float*>(P.out) + row * D + e / 4 * 64 + (quad * 4 + k) * 4) =
                    make_float4(x[e][k] * inv, x[e + 1][k] * inv, x[e + 2][k] * inv, x[e + 3][k] * inv);
        }
    }
    if (P.stats && quad == 0) P.stats[row] = make_float2(M, L);
}

template <typename T, int D, int CT, bool ROWS, bool ONCE>
__device__ __forceinline__ void wide_tile(const TreeParams& TP, int item, int split) {
    using C = WideCfg<T, D, CT>;
    constexpr bool BF = C::BF;
    constexpr int CH = C::CH, KS = C::KS, ET = C::ET, KT = C::KT, NT = C::NT, BLK = C::BLK, NB = C::NB, GI = C::GI, TM = C::TM, LD = C::LD, RPU = C::RPU;
    const AttnPagedParams& P = TP.a;
    const PagedParams& W = P.view;
    const int tid = threadIdx.x, lane = tid & (kWave - 1), n16 = lane & 15, quad = lane >> 4, wave = scalar(tid / kWave);
    const int n_kv = W.n_kv, g = W.g;
    extern __shared__ __attribute__((aligned(16))) unsigned char smem[];
    __shared__ Ancestors<TM> s_tree;
    __shared__ int s_bad;
    TreeWork w;
    if (!tree_work<ROWS>(P, item, TM, w)) return;
    const TileOf& t = w.t;
    const int n = w.n, h = w.h;
    const float scale = W.scale_log2e;
    const bool windowed = !ROWS && W.window != 0x7fffffff;
    const int32_t* tab = ROWS ? nullptr : scalar_ptr(W.table + (size_t)t.b * W.max_pages);
    const size_t tree_at = ((size_t)t.begin * n_kv + h) * CH * 16, row_at = ROWS ? ((size_t)t.b * n_kv + h) * P.cap * (CH * 16) : 0;

    int k_at[KS];   // LDS places of this lane's operands (prompt.h)
    {
        const int row = BF ? n16 / 4 * 8 + n16 % 4 : n16;
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) k_at[ks] = row * CH * 16 + ((ks * 4 + quad) ^ swizzle_k<BF, CH>(row)) * 16;
    }
    const int v_row = BF ? quad * 8 + n16 / 4 : quad * 4;
    auto v_at = [&](int e) { return v_row * CH * 16 + ((2 * e + n16 % 4 / 2) ^ swizzle_v<BF, CH>(v_row)) * 16 + n16 % 2 * 8; };
    const int st_row = tid / CH, st_ch = tid % CH;

    for (; w.t.tile >= 0; w.t.tile -= w.t.step) {
        tree_tile_of(P, TM, KT, w);
        if (split >= w.splits) continue;
        const int r0 = w.r0, rows = w.rows, splits = w.splits, total = w.total;
        const int per = splits == 1 ? total : scalar(divide(total + splits - 1, splits)), t_begin = min(split * per, total), t_end = min(t_begin + per, total);
        auto token_of = [&](int r) { return divide(r, g, W.g_magic); };
        const int w0 = r0 + wave * 16 * CT, w_rows = min(16 * CT, rows - wave * 16 * CT);   // the wavefront's rows; <= 0: none
        T128 q[CT][KS];
#pragma unroll
        for (int ct = 0; ct < CT; ++ct) {
            const int r = min(w0 + ct * 16 + n16, r0 + rows - 1), token = token_of(r);
            const size_t q_row = ((size_t)(t.begin + token) * n_kv + h) * g + (r - token * g);
#pragma unroll
            for (int ks = 0; ks < KS; ++ks) {
                q[ct][ks].u = reinterpret_cast<const tu32x4_t*>(W.q)[q_row * CH + ks * 4 + quad];
                if (W.negate) q[ct][ks].u ^= BF ? 0x80008000u : 0x80000000u;
            }
        }
        // The rows of all nodes at once.  A row gives the pairs that it does not see weight 0, which must not meet an infinity or a NaN that another row
        // sees: where there is any, the run starts over with half of its nodes.
        const int nodes = w.tok_hi - w.tok_lo + 1;
        const bool some_tree = t_end > w.old.total;
        if (windowed || some_tree) find_ancestors<TM>(TP, w, windowed, s_tree);
        for (int lo = 0, hi = nodes - 1;;) {
        int level_lo = 0, level_hi = 0;
        if (tid == 0) s_bad = 0;
        if (windowed || some_tree) span_of<TM>(s_tree, windowed, lo, hi, level_lo, level_hi);   // (otherwise no barrier here: the first tiles' is ahead of the flag's use)
        const int any_from = windowed ? n + level_lo - W.window + 1 : 0, all_from = windowed ? n + level_hi - W.window + 1 : 0;
        float m_ref[CT], m_top[CT], l_run[CT];
        tf32x4_t o[ET][CT];
#pragma unroll
        for (int ct = 0; ct < CT; ++ct) {
            m_ref[ct] = m_top[ct] = -INFINITY;
            l_run[ct] = 0.f;
#pragma unroll
            for (int e = 0; e < ET; ++e) o[e][ct] = (tf32x4_t){0.f, 0.f, 0.f, 0.f};
        }
        // Where a tile's pairs lie.  Pages: its runs of 16 pairs, counted in such runs (so that 32 bits hold any pool), and a bit for each that lies nowhere.
        struct Place {
            uint32_t run[ROWS ? 1 : GI], holes;
            int base;
            bool tree;
        };
        auto place_of = [&](int i) {   // (past the end: the last tile's)
            i = min(i, t_end - 1);
            Place p;
            p.holes = 0;
            p.tree = i >= w.old.total;
            p.base = p.tree ? (i - w.old.total) * KT : w.old.at(i) * KT;
            if constexpr (!ROWS) {
                auto find = [&](int r) {
                    const int key = p.base + r * 16, page = load_uniform(tab, min(key >> W.page_shift, W.max_pages - 1));
                    const bool ok = page_ok(W, page);
                    if (!ok) p.holes |= 1u << r;
                    return ((uint32_t)(ok ? page : 0) * n_kv + h) << (W.page_shift - 4) | (key & ((1 << W.page_shift) - 1)) >> 4;
                };
                p.run[0] = find(0);
                if (1 << W.page_shift >= KT) {   // one page
#pragma unroll
                    for (int r = 1; r < GI; ++r) p.run[r] = p.run[0] + r;
                    if (p.holes) p.holes = (1u << GI) - 1;
                } else {
#pragma unroll
                    for (int r = 1; r < GI; ++r) p.run[r] = find(r);
                }
            }
            return p;
        };
        auto run_of_load = [&](int u) { return RPU == 32 ? 2 * u + (wave >= 2 ? 1 : 0) : u * RPU / 16; };   // load u of this wavefront lies in one run
        auto send = [&](bool is_k, unsigned char* to, const Place& p) {
            const unsigned char* X = static_cast<const unsigned char*>(is_k ? W.K : W.V);
            to += wave * 64 * 16;
            const int last = p.tree ? t.nq - 1 - p.base : ROWS ? n - 1 - p.base : KT;
            if (!p.tree && (!ROWS || last >= KT - 1)) {
                if constexpr (ROWS) X += row_at + (size_t)p.base * (CH * 16);
#pragma unroll
                for (int u = 0; u < LD; ++u) {
                    const int row = st_row + u * RPU, ch = st_ch ^ (is_k ? swizzle_k<BF, CH>(row) : swizzle_v<BF, CH>(row));
                    const unsigned char* from = X + (uint32_t)((row * CH + ch) * 16);
                    if constexpr (!ROWS) {
                        const uint32_t run = RPU == 32 ? (wave >= 2 ? p.run[(2 * u + 1) % GI] : p.run[2 * u % GI]) : p.run[u * RPU / 16];
                        from = X + (size_t)run * (16 * CH * 16) + (uint32_t)((row % 16 * CH + ch) * 16);
                    }
                    if constexpr (ONCE) load_once_to_lds(from, to + u * 256 * 16);
                    else load_to_lds(from, to + u * 256 * 16);
                }
                return;
            }
            // the end of a row, or nodes: the last pair again behind the last one
            int thread = tid;   // (opaque: or all that follows from it is kept in registers over the loop)
            asm volatile("" : "+v"(thread));
            const int st_row = thread / CH, st_ch = thread % CH;
            const uint32_t stride = p.tree ? n_kv * CH * 16 : CH * 16;
            X = p.tree ? static_cast<const unsigned char*>(is_k ? TP.k_tree : TP.v_tree) + tree_at : X + row_at;
            X += (size_t)p.base * stride;
#pragma unroll
            for (int u = 0; u < LD; ++u) {
                const int row = st_row + u * RPU, ch = st_ch ^ (is_k ? swizzle_k<BF, CH>(row) : swizzle_v<BF, CH>(row));
                load_to_lds(X + (uint32_t)((uint32_t)min(row, last) * stride + ch * 16), to + u * 256 * 16);
            }
        };
        auto whole = [&](const Place& p) { return !p.tree && p.base + KT <= n && !p.holes && (p.base >= all_from || p.base + KT <= W.sink); };   // seen by every row
        // V of a tile that not every row sees: values of weight 0 must not meet the products as infinities or NaN
        auto clear_hidden = [&](unsigned char* v, const Place& p) {
            bool bad = false;
            int thread = tid;
            asm volatile("" : "+v"(thread));
            const int st_row = thread / CH;
#pragma unroll
            for (int u = 0; u < LD; ++u) {
                const int row = st_row + u * RPU, key = p.base + row;
                bool someone, everyone;   // (of those that someone sees)
                if (p.tree) {
                    someone = s_tree.any[key / 32] >> key % 32 & 1;
                    everyone = s_tree.all[key / 32] >> key % 32 & 1;
                } else {
                    someone = !(p.holes >> run_of_load(u) & 1) & (key < n) & ((key >= any_from) | (key < W.sink));
                    everyone = (key >= all_from) | (key < W.sink);
                }
                tu32x4_t* at = reinterpret_cast<tu32x4_t*>(v + (u * 256 + thread) * 16);
                if (!someone) *at = tu32x4_t{0, 0, 0, 0};
                else if (!everyone) {
                    const tu32x4_t x = *at;
#pragma unroll
                    for (int k = 0; k < 4; ++k) bad |= word_not_finite<T>(x[k]);
                }
            }
            if (bad && hi > lo) s_bad = 1;
        };
        typedef tf32x4_t Logits[GI][CT];
        auto products = [&](const unsigned char* sk, Logits& c) {
#pragma unroll
            for (int gi = 0; gi < GI; ++gi) {
#pragma unroll
                for (int ct = 0; ct < CT; ++ct) c[gi][ct] = (tf32x4_t){0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int ks = 0; ks < KS; ++ks) {
                    T128 k;
                    k.u = *reinterpret_cast<const tu32x4_t*>(sk + k_at[ks] + (gi / NT * BLK + gi % NT * 4) * CH * 16);
#pragma unroll
                    for (int ct = 0; ct < CT; ++ct) {
                        if constexpr (BF) {
                            c[gi][ct] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(k.v, q[ct][ks].v, c[gi][ct], 0, 0, 0);
                        } else {
#pragma unroll
                            for (int e = 0; e < 4; ++e) c[gi][ct] = __builtin_amdgcn_mfma_f32_16x16x4f32(k.f[e], q[ct][ks].f[e], c[gi][ct], 0, 0, 0);
                        }
                    }
                }
            }
        };
        bool need = false, large = false;
        float m_new[CT];
        auto assess = [&](const Logits& c) {   // a row's largest logit of a tile; whether its reference has to move, or differences would lose their bits
            need = large = false;
#pragma unroll
            for (int ct = 0; ct < CT; ++ct) {
                float mx = c[0][ct][0];
#pragma unroll
                for (int x = 1; x < GI * 4; ++x) mx = fmaxf(mx, c[x / 4][ct][x % 4]);
                const float m = attn_logit(quad_max(mx), scale);
                m_new[ct] = m;
                need |= m > m_ref[ct] + 8.f;
                large |= fabsf(fmaxf(m, m_ref[ct])) >= kLargeLogit;
            }
        };
        auto step = [&](const unsigned char* k_next, const unsigned char* sv, const Place& p, Logits& c, Logits& next) {
            if (!whole(p)) {
                int at = lane;
                asm volatile("" : "+v"(at));
                const int quad = at >> 4, n16 = at & 15;
#pragma unroll
                for (int ct = 0; ct < CT; ++ct) {
                    uint32_t sees = 0;   // a bit for each logit of the lane
                    const int tok = token_of(min(w0 + ct * 16 + n16, r0 + rows - 1)) - w.tok_lo;
                    const int from = windowed ? n + s_tree.level[tok] - W.window + 1 : 0;   // the row sees pairs of the cache from here on (and the sinks)
#pragma unroll
                    for (int gi = 0; gi < GI; ++gi) {
                        const int first = gi / NT * BLK + quad * (NT * 4) + gi % NT * 4;   // the lane's keys of product gi: first .. first + 3
                        if (p.tree) {
                            sees |= (s_tree.sees[tok][(p.base + first) / 32] >> (p.base + first) % 32 & 15) << gi * 4;
                        } else {
                            const bool there = !(p.holes >> (BF ? 2 * (gi / NT) + (quad >= 2) : gi) & 1);
#pragma unroll
                            for (int e = 0; e < 4; ++e) {
                                const int key = p.base + first + e;
                                sees |= (uint32_t)(there & (key < n) & ((key >= from) | (key < W.sink))) << (gi * 4 + e);
                            }
                        }
                    }
                    if (tok < lo || tok > hi) sees = 0;
#pragma unroll
                    for (int x = 0; x < GI * 4; ++x) c[x / 4][ct][x % 4] = sees >> x & 1 ? c[x / 4][ct][x % 4] : -INFINITY;
                }
                assess(c);
            }
#pragma unroll
            for (int ct = 0; ct < CT; ++ct) m_top[ct] = fmaxf(m_top[ct], m_new[ct]);
            if (__any(need)) {
#pragma unroll
                for (int ct = 0; ct < CT; ++ct) {
                    const float m = m_new[ct] > m_ref[ct] + 8.f ? m_new[ct] : m_ref[ct], corr = __builtin_amdgcn_exp2f(m_ref[ct] - ref_of(m));
                    m_ref[ct] = m;
                    l_run[ct] *= corr;
#pragma unroll
                    for (int e = 0; e < ET; ++e)
#pragma unroll
                        for (int k = 0; k < 4; ++k) o[e][ct][k] *= corr;
                }
            }
            float by = scale, less[CT];
#pragma unroll
            for (int ct = 0; ct < CT; ++ct) less[ct] = ref_of(m_ref[ct]);
            if (__any(large)) {   // rounded before the reference is subtracted; the fma below then has nothing left to do
                by = 1.f;
#pragma unroll
                for (int ct = 0; ct < CT; ++ct) {
                    less[ct] = 0.f;
#pragma unroll
                    for (int x = 0; x < GI * 4; ++x) c[x / 4][ct][x % 4] = attn_logit(c[x / 4][ct][x % 4], scale) - ref_of(m_ref[ct]);
                }
            }
            __builtin_amdgcn_s_setprio(1);
            products(k_next, next);   // (behind the last tile: of what lies there, for nobody)
#pragma unroll
            for (int ct = 0; ct < CT; ++ct) {
                float sum = 0.f;
#pragma unroll
                for (int x = 0; x < GI * 4; ++x) {
                    const float y = __builtin_amdgcn_exp2f(fmaf(c[x / 4][ct][x % 4], by, -less[ct]));
                    c[x / 4][ct][x % 4] = y;
                    sum += y;
                }
                l_run[ct] += sum;
            }
            // (products with V go ahead of another wavefront's exponentials, which fill their gaps: 64 nodes 73.4 -> 69.6 us, D 64 43.7 -> 40.1, over pages 162 -> 157)
            __builtin_amdgcn_s_setprio(2);
#pragma unroll
            for (int b = 0; b < NB; ++b) {
                if constexpr (BF) {
                    T128 pr[CT], pr2[CT];
#pragma unroll
                    for (int ct = 0; ct < CT; ++ct)
#pragma unroll
                        for (int x = 0; x < 4; ++x) two_terms(c[2 * b + x / 2][ct][x % 2 * 2], c[2 * b + x / 2][ct][x % 2 * 2 + 1], pr[ct].w[x], pr2[ct].w[x]);
                    constexpr int EE = CT == 1 ? 4 : 1;   // channel tiles at a time: no product waits for the one before it (D 64, 64 nodes 48.0 -> 43.6 us)
#pragma unroll
                    for (int e0 = 0; e0 < ET; e0 += EE) {
                        T128 v[EE];
#pragma unroll
                        for (int e = 0; e < EE; ++e) {
                            const unsigned char* at = sv + v_at(e0 + e) + b * BLK * CH * 16;
                            const tu32x2_t v0 = read_transposed(at), v1 = read_transposed(at + 4 * CH * 16);
                            v[e].u = tu32x4_t{v0.x, v0.y, v1.x, v1.y};
                        }
#pragma unroll
                        for (int k = 0; k < 2 * CT; ++k)
#pragma unroll
                            for (int e = 0; e < EE; ++e) o[e0 + e][k % CT] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v[e].v, k < CT ? pr[k % CT].v : pr2[k % CT].v, o[e0 + e][k % CT], 0, 0, 0);
                    }
                } else {
#pragma unroll
                    for (int u = 0; u < 4; ++u)
#pragma unroll
                        for (int cc = 0; cc < D / 64; ++cc) {
                            T128 v;
                            v.u = *reinterpret_cast<const tu32x4_t*>(sv + (b * BLK + v_row + u) * CH * 16 + (cc * 16 + n16) * 16);
#pragma unroll
                            for (int e = 0; e < 4; ++e)
#pragma unroll
                                for (int ct = 0; ct < CT; ++ct) o[cc * 4 + e][ct] = __builtin_amdgcn_mfma_f32_16x16x4f32(v.f[e], c[b][ct][u], o[cc * 4 + e][ct], 0, 0, 0);
                        }
                }
            }
            assess(next);
            __builtin_amdgcn_s_setprio(0);
        };

        // Tile i lies in place (i - t_begin) % PLACES.  With three its K is sent for three turns ahead (the turn before it forms its logits) and its V two, so
        // that the latest 2 * LD loads may still be under way at a turn's end; with two a turn's loads arrive by its end.  Every turn sends for
        // one of each, behind the end the last tile's again.
        constexpr bool FAR = C::PLACES == 3;
        constexpr int UNDER_WAY = FAR ? 2 * LD : 0;
        Logits ca, cb;
        if (t_begin < t_end) {
            unsigned char *const sk = smem, *const sv = smem + C::PLACES * C::TILE_BYTES;
            Place here = place_of(t_begin), next1 = place_of(t_begin + 1), next2 = place_of(t_begin + 2);
            send(true, sk, here);
            send(false, sv, here);
            send(true, sk + C::TILE_BYTES, next1);
            if constexpr (FAR) {
                send(false, sv + C::TILE_BYTES, next1);
                send(true, sk + 2 * C::TILE_BYTES, next2);
            }
            arrived_but<UNDER_WAY>();
            if (w_rows > 0) {
                products(sk, ca);
                assess(ca);
            }
            lds_barrier();
            // the places of this tile, whose K is not needed any more, of the next one and the one after it
            auto turn = [&](unsigned char* __restrict k_to, unsigned char* __restrict v_to, const unsigned char* __restrict k_from, unsigned char* __restrict v_from, int i, Logits& c,
                            Logits& next) {
                const Place next3 = FAR ? place_of(i + 3) : Place();
                send(true, k_to, FAR ? next3 : next2);
                send(false, v_to, FAR ? next2 : next1);
                if (!whole(here)) {
                    clear_hidden(v_from, here);
                    lds_barrier();
                }
                const Place after = FAR ? next3 : place_of(i + 3);
                if (w_rows > 0) step(k_from, v_from, here, c, next);
                here = next1;
                next1 = next2;
                next2 = after;
                arrived_but<UNDER_WAY>();
            };
            uint32_t at = 0, at1 = C::TILE_BYTES, at2 = FAR ? 2 * C::TILE_BYTES : 0;
            for (int i = t_begin;;) {
                turn(sk + at, sv + (FAR ? at2 : at1), sk + at1, sv + at, i, ca, cb);
                if (++i == t_end) break;
                turn(sk + at1, sv + at, sk + at2, sv + at1, i, cb, ca);
                if (++i == t_end) break;
                if constexpr (FAR) {   // two turns on
                    const uint32_t x = at2;
                    at2 = at1;
                    at1 = at;
                    at = x;
                }
            }
            arrived();   // (what is under way still for nobody)
        }
        __syncthreads();
        if (scalar(s_bad)) {   // (the same for every thread)
            hi = lo + (hi - lo) / 2;
            __syncthreads();
            continue;
        }

        // Every wavefront has its rows' own.  Records: its registers as they are.
        int lane = threadIdx.x & (kWave - 1);   // (opaque, as above)
        asm volatile("" : "+v"(lane));
        const int n16 = lane & 15, quad = lane >> 4;
        const size_t rec0 = (size_t)item * P.splits * 4 + wave;   // of split 0; 4 a split on
#pragma unroll
        for (int ct = 0; ct < CT; ++ct) {
            const float l = quad_sum(l_run[ct]);
            const int r = w0 + ct * 16 + n16, token = token_of(min(r, r0 + rows - 1));
            if (r >= r0 + rows || token - w.tok_lo < lo || token - w.tok_lo > hi) continue;
            if (splits > 1) {
                const size_t rec = rec0 + (size_t)split * 4;
                float* to = P.rec + (rec * CT + ct) * (ET * 256) + lane * 2;   // (neighbouring lanes side by side)
#pragma unroll
                for (int e = 0; e < ET; ++e) {
                    put2(to + e * 256, o[e][ct][0], o[e][ct][1]);
                    put2(to + e * 256 + 128, o[e][ct][2], o[e][ct][3]);
                }
                float* ml = reinterpret_cast<float*>(P.rec_ml) + (rec * CT + ct) * 256 + lane * 2;
                put2(ml, m_ref[ct], m_top[ct]);
                put2(ml + 128, l, 0.f);
                continue;
            }
            tf32x4_t x[ET];
#pragma unroll
            for (int e = 0; e < ET; ++e) x[e] = o[e][ct];
            store_wide<T, D>(P, ((size_t)(t.begin + token) * n_kv + h) * g + (r - token * g), quad, x, m_top[ct], l * __builtin_amdgcn_exp2f(m_ref[ct] - ref_of(m_top[ct])),
                             l == 0.f ? 0.f : 1.0f / l);
        }
        __syncthreads();   // the LDS is the next run's
        if (hi == nodes - 1) break;
        lo = hi + 1;
        hi = nodes - 1;
        }
        if (splits == 1) continue;
        // the last split's wavefront to arrive adds its rows' records up, in the order of the splits
        if (w_rows <= 0) return;   // (a split tile is its place's only one)
        int lane = threadIdx.x & (kWave - 1);   // (opaque, as above)
        asm volatile("" : "+v"(lane));
        const int n16 = lane & 15, quad = lane >> 4;
        arrived();
        int last = 0;
        if (lane == 0) last = last_one(TP.here + item * 4 + wave, splits);
        if (!scalar(__shfl(last, 0))) return;
        const size_t rec0 = (size_t)item * P.splits * 4 + wave;
        auto ml_of = [&](int s, int ct) { return reinterpret_cast<const float*>(P.rec_ml) + ((rec0 + (size_t)min(s, splits - 1) * 4) * CT + ct) * 256 + lane * 2; };
        float top[CT], ref[CT], l[CT];   // largest logits, the references that the sums belong to
        tf32x4_t x[CT][ET];
#pragma unroll
        for (int ct = 0; ct < CT; ++ct) {
            top[ct] = ref[ct] = -INFINITY;
            l[ct] = 0.f;
#pragma unroll
            for (int e = 0; e < ET; ++e) x[ct][e] = (tf32x4_t){0.f, 0.f, 0.f, 0.f};
        }
        for (int s0 = 0; s0 < splits; s0 += 8) {
            float2 m[8][CT];
#pragma unroll
            for (int u = 0; u < 8; ++u)
#pragma unroll
                for (int ct = 0; ct < CT; ++ct) m[u][ct] = get2(ml_of(s0 + u, ct));   // (the copies past the end change nothing)
#pragma unroll
            for (int u = 0; u < 8; ++u)
#pragma unroll
                for (int ct = 0; ct < CT; ++ct) {
                    ref[ct] = fmaxf(ref[ct], m[u][ct].x);
                    top[ct] = fmaxf(top[ct], m[u][ct].y);
                }
        }
        for (int s0 = 0; s0 < splits; s0 += 2) {   // two records' loads in flight
            float2 v[2][CT][ET][2], m[2][CT], sum[2][CT];
#pragma unroll
            for (int u = 0; u < 2; ++u)
#pragma unroll
                for (int ct = 0; ct < CT; ++ct) {
                    m[u][ct] = get2(ml_of(s0 + u, ct));
                    sum[u][ct] = get2(ml_of(s0 + u, ct) + 128);
                    const float* from = P.rec + ((rec0 + (size_t)min(s0 + u, splits - 1) * 4) * CT + ct) * (ET * 256) + lane * 2;
#pragma unroll
                    for (int e = 0; e < ET; ++e) {
                        v[u][ct][e][0] = get2(from + e * 256);
                        v[u][ct][e][1] = get2(from + e * 256 + 128);
                    }
                }
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                if (s0 + u >= splits) break;
#pragma unroll
                for (int ct = 0; ct < CT; ++ct) {
                    const float f = __builtin_amdgcn_exp2f(m[u][ct].x - ref_of(ref[ct]));
                    l[ct] = fmaf(sum[u][ct].x, f, l[ct]);
#pragma unroll
                    for (int e = 0; e < ET; ++e) {
                        x[ct][e][0] = fmaf(v[u][ct][e][0].x, f, x[ct][e][0]);
                        x[ct][e][1] = fmaf(v[u][ct][e][0].y, f, x[ct][e][1]);
                        x[ct][e][2] = fmaf(v[u][ct][e][1].x, f, x[ct][e][2]);
                        x[ct][e][3] = fmaf(v[u][ct][e][1].y, f, x[ct][e][3]);
                    }
                }
            }
        }
#pragma unroll
        for (int ct = 0; ct < CT; ++ct) {
            const int r = w0 + ct * 16 + n16, token = token_of(min(r, r0 + rows - 1));
            if (r < r0 + rows)
                store_wide<T, D>(P, ((size_t)(t.begin + token) * n_kv + h) * g + (r - token * g), quad, x[ct], top[ct], l[ct] * __builtin_amdgcn_exp2f(ref[ct] - ref_of(top[ct])),
                                 l[ct] == 0.f ? 0.f : 1.0f / l[ct]);
        }
        return;
    }
}

}  // namespace fk
