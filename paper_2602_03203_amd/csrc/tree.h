// Attention of trees of drafted tokens over a cache: the rows of a budgeted cache or the pages of a prompt (fk_tree_attn, fk_paged_tree_attn).
//
// The query rows of a (tree, KV head) are its nodes times the heads of the group; a workgroup takes RB * 16 of them and a split of what they
// see: the pairs of the cache, which all nodes see (but for a window), then the pairs of the tree, a node its ancestors' and its own.
// Its wavefronts take tiles of KT pairs in turn, straight from memory into registers, each with its own online softmax for all rows; they are
// merged through LDS at the end.  Products and operand layouts are those of thin.h: logits K.Q^T with the keys in an order that makes a
// lane's probabilities an operand of V^T.P^T as they are; an operand of K or V serves a product for each 16 rows.
// Which ancestors a node has is a bit for every node of its tree: found once per workgroup, in LDS, by walking up from it.
#pragma once
#include "attn_paged.h"
#include <type_traits>

namespace fk {

static constexpr int kTreeNodes = FK_TREE_NODES;

struct TreeParams {
    AttnPagedParams a;         // view (rows of a budgeted cache: kv_len is len, [batch][n_kv]), out, stats, grid, splits, split_shift, rec, rec_ml, cap
    const int32_t* parent;
    const void *k_tree, *v_tree;
};

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

// What a workgroup works on; false: nothing
struct TreeWork {
    TileOf t;
    int h, n;                  // KV head, pairs of the cache
    int r0, rows;              // query rows of the tile
    int tok_lo, tok_hi;        // nodes that they belong to
    KeyTiles old;              // tiles of the cache's pairs
    int total, splits;         // with those of the tree
};
template <bool ROWS, int TM, int KT>
__device__ __forceinline__ bool tree_work(const AttnPagedParams& P, int item, TreeWork& w) {
    const PagedParams& W = P.view;
    const int slot = scalar(divide(item, W.n_kv, W.kv_magic));
    w.h = item - slot * W.n_kv;
    if (!tile_of(W, P.grid, slot, TM, w.t)) return false;
    if constexpr (ROWS) w.t.n = scalar(min(max(load_uniform(W.kv_len, w.t.b * W.n_kv + w.h), 0), P.cap));
    w.n = w.t.n;
    return true;
}
template <int TM, int KT> __device__ __forceinline__ void tree_tile_of(const AttnPagedParams& P, TreeWork& w) {
    const PagedParams& W = P.view;
    w.r0 = w.t.tile * TM;
    w.rows = min(TM, w.t.nq * W.g - w.r0);
    w.tok_lo = scalar(divide(w.r0, W.g, W.g_magic));
    w.tok_hi = scalar(divide(w.r0 + w.rows - 1, W.g, W.g_magic));
    w.old = key_tiles(W, w.n, w.n - 1, KT);   // (the root, at position n, sees the most under a window)
    w.total = w.old.total + (uint32_t)(w.tok_hi + KT) / (uint32_t)KT;   // (parents come first: nobody sees a later node)
    w.splits = scalar(splits_of(w.total, w.t.one ? P.splits : 1, P.split_shift));
}

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
    __shared__ int16_t s_parent[kTreeNodes];
    __shared__ uint32_t s_sees[TM][kTreeNodes / 32];   // nodes that the tile's nodes see
    __shared__ int s_level[TM];

    TreeWork w;
    if (!tree_work<ROWS, TM, KT>(P, item, w)) return;
    const TileOf& t = w.t;
    const int n = w.n, h = w.h;
    const bool windowed = !ROWS && W.window != 0x7fffffff;
    const tu32x4_t *Kp = reinterpret_cast<const tu32x4_t*>(W.K), *Vp = reinterpret_cast<const tu32x4_t*>(W.V);
    const tu32x4_t* k_tree = reinterpret_cast<const tu32x4_t*>(TP.k_tree) + ((size_t)t.begin * n_kv + h) * CH;
    const tu32x4_t* v_tree = reinterpret_cast<const tu32x4_t*>(TP.v_tree) + ((size_t)t.begin * n_kv + h) * CH;
    const int32_t* tab = ROWS ? nullptr : scalar_ptr(W.table + (size_t)t.b * W.max_pages);
    for (; w.t.tile >= 0; w.t.tile -= w.t.step) {
        tree_tile_of<TM, KT>(P, w);
        if (split >= w.splits) continue;
        const int r0 = w.r0, rows = w.rows, splits = w.splits, total = w.total;
        const int per = splits == 1 ? total : scalar(divide(total + splits - 1, splits)), t_begin = min(split * per, total), t_end = min(t_begin + per, total);
        auto token_of = [&](int r) { return divide(r, g, W.g_magic); };

        T128 q[RB][KS];
        int tok[RB];   // of this lane's rows, counted from the tile's first
#pragma unroll
        for (int rb = 0; rb < RB; ++rb) {
            const int r = r0 + min(rb * 16 + n16, rows - 1), token = token_of(r);
            tok[rb] = token - w.tok_lo;
            const size_t q_row = ((size_t)(t.begin + token) * n_kv + h) * g + (r - token * g);
#pragma unroll
            for (int ks = 0; ks < KS; ++ks) {
                q[rb][ks].u = reinterpret_cast<const tu32x4_t*>(W.q)[q_row * CH + ks * 4 + quad];
                if (W.negate) q[rb][ks].u ^= BF ? 0x80008000u : 0x80000000u;
            }
        }
        const float scale = W.scale_log2e;

        // who sees whom
        if (windowed || t_end > w.old.total) {
            for (int i = tid; i <= w.tok_hi; i += WAVES * kWave) {
                const int p = TP.parent[t.begin + i];
                s_parent[i] = (int16_t)(p < i ? max(p, -1) : -1);
            }
            __syncthreads();
            for (int i = tid; i <= w.tok_hi - w.tok_lo; i += WAVES * kWave) {
                const int self = w.tok_lo + i;
                int level = 0;
                if (windowed)
                    for (int a = s_parent[self]; a >= 0; a = s_parent[a]) ++level;
#pragma unroll
                for (int x = 0; x < kTreeNodes / 32; ++x) s_sees[i][x] = 0;
                int up = 0;   // levels from the node to its ancestor
                for (int a = self; a >= 0; a = s_parent[a], ++up)
                    if (!windowed || up < W.window || n + level - up < W.sink) s_sees[i][a / 32] |= 1u << a % 32;
                s_level[i] = level;
            }
            __syncthreads();
        }
        int from[RB];   // a lane's rows see pairs of the cache from here on (and the sinks)
        int top_level = 0;
#pragma unroll
        for (int rb = 0; rb < RB; ++rb) from[rb] = windowed ? n + s_level[tok[rb]] - W.window + 1 : 0;
        if (windowed) {
#pragma unroll
            for (int rb = 0; rb < RB; ++rb) top_level = max(top_level, s_level[tok[rb]]);
#pragma unroll
            for (int off = 1; off < 16; off <<= 1) top_level = max(top_level, __shfl_xor(top_level, off));
            top_level = scalar(top_level);
        }
        const int all_from = windowed ? n + top_level - W.window + 1 : 0, any_from = windowed ? n - W.window + 1 : 0;

        // where a tile's pairs lie: pair u at the first (u < 16) or second run + min(u, last) * stride; `hole`: a bit for each run that lies nowhere
        struct Place {
            const tu32x4_t *k[NT], *v[NT];
            int stride, last, base, holes;
            bool tree;
        };
        auto place_of = [&](int i) {
            Place p;
            p.tree = i >= w.old.total;
            p.holes = 0;
            if (p.tree) {
                p.base = (i - w.old.total) * KT;
                p.stride = n_kv * CH;
                p.last = t.nq - 1 - p.base;
#pragma unroll
                for (int r = 0; r < NT; ++r) {
                    p.k[r] = k_tree + (size_t)p.base * p.stride;
                    p.v[r] = v_tree + (size_t)p.base * p.stride;
                }
                return p;
            }
            p.base = w.old.at(i) * KT;
            p.stride = CH;
            p.last = ROWS ? n - 1 - p.base : KT;
#pragma unroll
            for (int r = 0; r < NT; ++r) {
                size_t pair;
                if constexpr (ROWS) {
                    pair = ((size_t)t.b * n_kv + h) * P.cap + p.base;
                } else {
                    const int key = p.base + r * 16, page = load_uniform(tab, min(key >> W.page_shift, W.max_pages - 1));
                    const bool ok = page_ok(W, page);
                    if (!ok) p.holes |= 1 << r;
                    pair = ((((size_t)(ok ? page : 0) * n_kv + h) << W.page_shift) + (key & ((1 << W.page_shift) - 1)));
                }
                p.k[r] = Kp + pair * CH - (ROWS ? 0 : r * 16 * CH);
                p.v[r] = Vp + pair * CH - (ROWS ? 0 : r * 16 * CH);
            }
            return p;
        };
        T128 kr[NT][KS], vr[VL];
        auto load_k = [&](const Place& p) {
            const tu32x4_t* run = NT == 2 && n16 >= 8 ? p.k[NT - 1] : p.k[0];
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) {
                const int key = BF ? n16 / 4 * 8 + nt * 4 + n16 % 4 : n16;   // with this order, a lane's logits are keys quad * 8 + u (fp32: quad * 4 + i)
                const tu32x4_t* x = run + (size_t)(uint32_t)(min(key, p.last) * p.stride);
#pragma unroll
                for (int ks = 0; ks < KS; ++ks) kr[nt][ks].u = x[ks * 4 + quad];
            }
        };
        auto v_run = [&](const Place& p, int quad) { return NT == 2 && quad >= 2 ? p.v[NT - 1] : p.v[0]; };
        auto load_v = [&](const Place& p) {
            const tu32x4_t* run = v_run(p, quad);
#pragma unroll
            for (int u = 0; u < (BF ? 8 : 4); ++u) {
                const tu32x4_t* x = run + (size_t)(uint32_t)(min(quad * (BF ? 8 : 4) + u, p.last) * p.stride);
                if constexpr (!BF) {
#pragma unroll
                    for (int c = 0; c < D / 64; ++c) vr[u * (D / 64) + c].u = x[c * 16 + n16];
                } else if constexpr (D == 128) {
                    vr[u].u = x[n16];
                } else {
                    const tu32x2_t y = reinterpret_cast<const tu32x2_t*>(x)[n16];
                    vr[u].w[0] = y.x;
                    vr[u].w[1] = y.y;
                }
            }
        };
        constexpr int VW = BF && D == 64 ? 2 : 4;   // words in use of a V load

        float m_run[RB], l_run[RB];
        tf32x4_t o[RB][ET];
#pragma unroll
        for (int rb = 0; rb < RB; ++rb) {
            m_run[rb] = -INFINITY;
            l_run[rb] = 0.f;
#pragma unroll
            for (int e = 0; e < ET; ++e) o[rb][e] = (tf32x4_t){0.f, 0.f, 0.f, 0.f};
        }
        Place at, next;
        int i = t_begin + wave;
        if (i < t_end) {
            at = place_of(i);
            load_k(at);
            load_v(at);
        }
        for (; i < t_end; i += WAVES) {
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
            const bool more = i + WAVES < t_end;
            next = place_of(more ? i + WAVES : i);
            if (more) load_k(next);

            float s[RB][NT * 4];
#pragma unroll
            for (int rb = 0; rb < RB; ++rb)
#pragma unroll
                for (int j = 0; j < NT * 4; ++j) s[rb][j] = attn_logit(c[rb][j / 4][j % 4], scale);
            // everything seen by every row: no masks
            const bool whole = !at.tree && at.base + KT <= n && !at.holes && (at.base >= all_from || at.base + KT <= W.sink);
            uint32_t sees[RB];   // a bit for each of the lane's keys
            bool bad = false;    // a value that not every row sees is infinite or NaN
            if (!whole) {
                const int k0 = quad * (NT * 4);   // first of the lane's keys in the tile
                if (at.tree) {
#pragma unroll
                    for (int rb = 0; rb < RB; ++rb) sees[rb] = s_sees[tok[rb]][at.base / 32] >> (at.base % 32 + k0);
                } else {
                    const bool there = !(at.holes >> (NT == 2 && quad >= 2 ? 1 : 0) & 1);
#pragma unroll
                    for (int rb = 0; rb < RB; ++rb) {
                        sees[rb] = 0;
#pragma unroll
                        for (int j = 0; j < NT * 4; ++j) {
                            const int key = at.base + k0 + j;
                            sees[rb] |= (uint32_t)(there & (key < n) & ((key >= from[rb]) | (key < W.sink))) << j;
                        }
                    }
                }
#pragma unroll
                for (int rb = 0; rb < RB; ++rb)
#pragma unroll
                    for (int j = 0; j < NT * 4; ++j) s[rb][j] = sees[rb] >> j & 1 ? s[rb][j] : -INFINITY;
                // values of weight 0 must not meet the products as infinities or NaN: what nobody sees is cleared, of what some see the numbers stay
#pragma unroll
                for (int x = 0; x < VL; ++x) {
                    const int u = BF ? quad * 8 + x : quad * 4 + x / (D / 64), key = at.base + u;
                    const bool there = !(at.holes >> (NT == 2 && quad >= 2 ? 1 : 0) & 1);
                    const bool someone = at.tree ? u <= at.last : there & (key < n) & ((key >= any_from) | (key < W.sink));
                    const bool everyone = !at.tree & ((key >= all_from) | (key < W.sink));
#pragma unroll
                    for (int k = 0; k < VW; ++k) {
                        uint32_t& word = vr[x].w[k];
                        word = someone ? word : 0;
                        if (!everyone && word_not_finite<T>(word)) {
                            bad = true;
                            if constexpr (BF) {
                                if ((word & 0x7f80u) == 0x7f80u) word &= 0xffff0000u;
                                if ((word & 0x7f800000u) == 0x7f800000u) word &= 0xffffu;
                            } else {
                                word = 0;
                            }
                        }
                    }
                }
            }
            T128 pr[RB];   // bf16: the probabilities, each rounded by half a step of bf16 at most; sums of them unrounded
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
                    for (int x = 0; x < 4; ++x) pr[rb].w[x] = pack_bf16(s[rb][2 * x], s[rb][2 * x + 1]);
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
                } else {
#pragma unroll
                    for (int u = 0; u < 4; ++u)
#pragma unroll
                        for (int rb = 0; rb < RB; ++rb) o[rb][e] = __builtin_amdgcn_mfma_f32_16x16x4f32(vr[u * (D / 64) + e / 4].f[e % 4], s[rb][u], o[rb][e], 0, 0, 0);
                }
            }
            if (__any(bad)) {   // rare: the values taken out above, one by one, for the rows that see them
                for (int kq = 0; kq < 4; ++kq) {
                    const tu32x4_t* run = v_run(at, kq);
#pragma unroll 1
                    for (int j = 0; j < NT * 4; ++j) {
                        const int u = kq * (NT * 4) + j;
                        const T* x = reinterpret_cast<const T*>(run + (size_t)(uint32_t)(min(u, at.last) * at.stride));
                        const bool everyone = !at.tree && (at.base + u >= all_from || at.base + u < W.sink);
                        if (everyone) continue;
#pragma unroll
                        for (int rb = 0; rb < RB; ++rb) {
                            float mine = s[rb][0];
#pragma unroll
                            for (int y = 1; y < NT * 4; ++y) mine = y == j ? s[rb][y] : mine;
                            const float weight = __shfl(mine, kq * 16 + n16);
                            const bool seen = __shfl((int)sees[rb], kq * 16 + n16) >> j & 1;
#pragma unroll
                            for (int e = 0; e < ET; ++e)
#pragma unroll
                                for (int k = 0; k < 4; ++k) {
                                    const int ch = BF ? (quad * 4 + k) * ET + e : e / 4 * 64 + (quad * 4 + k) * 4 + e % 4;
                                    float v;
                                    if constexpr (BF) v = __uint_as_float((uint32_t)x[ch] << 16);
                                    else v = x[ch];
                                    if (seen && (__float_as_uint(v) & 0x7f800000u) == 0x7f800000u) o[rb][e][k] = fmaf(weight, v, o[rb][e][k]);
                                }
                        }
                    }
                }
            }
            if (more) load_v(next);
            at = next;
        }

        // ---- merge the wavefronts ----------------------------------------------------------------------------------
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
            const int r = x / (D / 4), d = x % (D / 4) * 4;
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
                *reinterpret_cast<float4*>(P.rec + (rec + r) * D + d) = make_float4(a[0], a[1], a[2], a[3]);
                if (d == 0) P.rec_ml[rec + r] = make_float2(s_M[r], s_L[r]);
                continue;
            }
            const int token = token_of(r0 + r);
            store_row<T, D, false>(P, ((size_t)(t.begin + token) * n_kv + h) * g + (r0 + r - token * g), d, a, s_M[r], s_L[r]);
        }
        __syncthreads();   // the LDS is the next tile's
    }
}

}  // namespace fk
