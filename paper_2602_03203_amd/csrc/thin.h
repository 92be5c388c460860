// Attention of up to 16 query rows (tokens x heads of a group) over many pairs: every pair is read once for all of them.
//
// A workgroup takes a split of the pairs that a tile of rows sees; its wavefronts take tiles of KT keys in turn, each with its own online softmax
// (maximum, sum, un-normalised output), merged through LDS at the end.  Logits as K.Q^T, outputs as V^T.P^T, so that a lane's results
// belong to one row and its probabilities are an operand of the second product in the registers they are in:
//   bf16  16x16x32 products, KT = 32: lane (quad, n16) loads K rows in the operand's layout, straight from the cache; logits of keys quad * 8 + u
//         (key_of_row) are its share of P.V, whose V (keys quad * 8 + u, a 16th of the row) is transposed in registers by byte permutes
//   fp32  16x16x4 products, KT = 16: a 16-byte load serves four products, the contraction over channels in an order of its own (the
//         same for q); logits of keys quad * 4 + i, one key a product of P.V, V as it was loaded
// K of the next tile is sent off when this one's logits are formed, V when its outputs are: the registers that held them are free, and loads are
// in flight all the time.  Bound by the memory system: 64 tokens that see 4096 pairs each, 8 heads of g 4, D 128: 1.02 GB in 157 us, 6.5 TB/s; traffic from
// memory is the pairs, once.
// Several splits: records in the workspace, a second launch merges them (and adds the weights).
#pragma once
#include "attn_paged.h"
#include <type_traits>

namespace fk {

template <typename T, int D> struct ThinCfg {
    static constexpr bool BF = sizeof(T) == 2;
    static constexpr int CH = D * (int)sizeof(T) / 16;   // 16-byte chunks of a row
    static constexpr int KT = BF ? 32 : 16;
    static constexpr int NT = KT / 16;                   // 16-key products of a tile
    static constexpr int KS = CH / 4;                    // chunks of a key per lane
    static constexpr int VL = BF ? 8 : 4 * D / 64;       // V loads per lane and tile (bf16 D = 64: 8 bytes each)
    static constexpr int ET = D / 16;                    // channel tiles of the output
    static constexpr int PART = D + 4;                   // float stride of a row of a partial output in LDS
    // dynamic LDS: partial outputs [WAVES][R][PART] (R rows: 16, for rows of a cache 8, the heads of a group) | maxima, sums, merge weights
    // [WAVES][16] each | merged maxima and sums [16] each | rows of a cache: logits [g][pairs]
    static constexpr int LOGITS = 9344;   // so many logits of a row fit LDS beside another workgroup's (200 rows of 2000, g 4: 34 us, through the workspace 37)
    static constexpr size_t lds(bool rows, int waves, int logits) {
        return sizeof(float) * ((size_t)waves * (rows ? 8 : 16) * PART + 3 * waves * 16 + 32 + logits);
    }
};

// channel of element i of a lane's output registers o[e]: MFMA row quad * 4 + i of channel tile e
template <typename T, int D> __device__ __forceinline__ int channel_of(int row, int e) {
    if constexpr (sizeof(T) == 2) return row * (D / 16) + e;
    else return e / 4 * 64 + row * 4 + e % 4;
}

template <typename T, int D, bool ROWS, int WAVES, bool NT_LOADS>
__device__ __forceinline__ void thin_tile(const AttnPagedParams& P, int item, int split) {
    using C = ThinCfg<T, D>;
    constexpr bool BF = C::BF;
    constexpr int CH = C::CH, KT = C::KT, NT = C::NT, KS = C::KS, VL = C::VL, ET = C::ET, PART = C::PART;
    const PagedParams& W = P.view;
    const int tid = threadIdx.x, lane = tid & (kWave - 1), n16 = lane & 15, quad = lane >> 4;
    const int wave = scalar(tid / kWave);
    const int n_kv = ROWS ? 1 : W.n_kv, slot = ROWS ? item : scalar(divide(item, n_kv, W.kv_magic)), h = ROWS ? 0 : item - slot * n_kv;
    const int g = W.g;

    constexpr int R = ROWS ? 8 : 16;
    extern __shared__ __attribute__((aligned(16))) float smem_thin[];
    float (*s_o)[R][PART] = reinterpret_cast<float (*)[R][PART]>(smem_thin);
    float (*s_m)[16] = reinterpret_cast<float (*)[16]>(smem_thin + WAVES * R * PART), (*s_l)[16] = s_m + WAVES, (*s_w)[16] = s_l + WAVES;
    float *s_M = s_w[WAVES], *s_L = s_M + 16, *s_lg = s_L + 16;
    __shared__ int s_bad;   // a value that not every row of a run sees is infinite or NaN

    TileOf t;
    int fresh = -1;   // ROWS: the new pair's slot
    if constexpr (ROWS) {
        const int old = min(max(load_uniform(P.len, slot), 0), P.cap);   // (set by this row's only workgroup, or by the second launch)
        fresh = old < P.cap ? old : -1;
        t = {slot, slot, 1, fresh >= 0 ? old + 1 : old, 0, 0, 1, true};
        t.first = t.n - 1;
    } else {
        if (!tile_of(W, P.grid, slot, 16, t)) return;
    }
    const tu32x4_t* Kp = reinterpret_cast<const tu32x4_t*>(W.K);
    const tu32x4_t* Vp = reinterpret_cast<const tu32x4_t*>(W.V);
    for (; t.tile >= 0; t.tile -= t.step) {
        const int r0 = t.tile * 16, rows = min(16, t.nq * g - r0);
        auto token_of = [&](int r) { return ROWS ? 0 : divide(r, g, W.g_magic); };
        const int tile_lo = ROWS ? t.first : scalar(t.first + token_of(r0)), tile_hi = ROWS ? t.first : scalar(t.first + token_of(r0 + rows - 1));   // positions
        const KeyTiles kt = key_tiles(W, tile_lo, tile_hi, KT);
        const int splits = scalar(splits_of(kt.total, t.one ? P.splits : 1, P.split_shift));
        if (split >= splits) continue;
        const int per = splits == 1 ? kt.total : scalar(divide(kt.total + splits - 1, splits)), t_begin = min(split * per, kt.total), t_end = min(t_begin + per, kt.total);

        // This lane's row.  Rows of a bf16 cache: the heads a second time in the upper eight columns, for the second terms of their probabilities, or of
        // which the normaliser of the outputs is kept (below).
        constexpr bool TWICE = ROWS && BF;
        const int my_row = TWICE ? min(n16 % 8, rows - 1) : r0 + min(n16, rows - 1), my_token = token_of(my_row), my_head = my_row - my_token * g;
        const size_t q_row = ((size_t)(t.begin + my_token) * n_kv + h) * g + my_head;
        const bool lg_local = ROWS && t.n <= P.logits_lds;
        const float acc_first = ROWS && splits == 1 && tid < t.n ? P.acc[(size_t)slot * P.cap + tid] : 0.f;   // (on its way over the whole loop)
        T128 q[KS];
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) {
            q[ks].u = reinterpret_cast<const tu32x4_t*>(W.q)[q_row * CH + ks * 4 + quad];
            if (W.negate) q[ks].u ^= BF ? 0x80008000u : 0x80000000u;
        }
        const float scale = W.scale_log2e;
        const tu32x4_t* k_fresh = reinterpret_cast<const tu32x4_t*>(P.k_new) + (size_t)slot * CH;
        const tu32x4_t* v_fresh = reinterpret_cast<const tu32x4_t*>(P.v_new) + (size_t)slot * CH;

        // The pages of a tile's (one or two) runs of 16 pairs: wavefront uniform.  A hole's pairs are read from page 0 and not seen.
        const int32_t* tab = ROWS ? nullptr : scalar_ptr(W.table + (size_t)t.b * W.max_pages);
        auto pages_of = [&](int base, int& a, int& b) {
            if constexpr (ROWS) {
                a = b = slot;
            } else {
                a = load_uniform(tab, min(base >> W.page_shift, W.max_pages - 1));
                b = NT == 1 ? a : load_uniform(tab, min((base + 16) >> W.page_shift, W.max_pages - 1));
            }
        };
        const int page_mask = ROWS ? 0 : (1 << W.page_shift) - 1;
        // the first pair of the run of 16 that starts at `base`: one address per run, constant offsets inside
        auto run_at = [&](const tu32x4_t* X, int page, int base) -> const tu32x4_t* {
            return X + ((((size_t)(page_ok(W, page) ? page : 0) * n_kv + h) << W.page_shift) + (base & page_mask)) * CH;
        };
        // lane's key in the tile (of its 16: in_run) -> its pair
        auto pair_at = [&](const tu32x4_t* X, const tu32x4_t* fresh_row, const tu32x4_t* run, int base, int in_tile, int u) -> const tu32x4_t* {
            if constexpr (ROWS) {
                const int key = min(base + in_tile + u, t.n - 1);
                return key == fresh ? fresh_row : X + ((size_t)slot * P.cap + key) * CH;
            } else {
                return run + (size_t)(in_tile % 16) * CH + u * CH;
            }
        };
        auto ld16 = [&](const tu32x4_t* x) { return NT_LOADS ? __builtin_nontemporal_load(x) : *x; };
        auto ld8 = [&](const tu32x2_t* x) { return NT_LOADS ? __builtin_nontemporal_load(x) : *x; };
        // the key that MFMA row r of product nt is; with these, a lane's logits are keys quad * 8 + u (bf16), quad * 4 + i (fp32)
        auto key_of_row = [](int nt, int r) { return BF ? r / 4 * 8 + nt * 4 + r % 4 : r; };
        T128 kr[NT][KS], vr[VL];
        auto load_k = [&](int base, int pa, int pb) {
            const tu32x4_t* run = nullptr;
            if constexpr (!ROWS) {
                run = run_at(Kp, pa, base);
                if constexpr (NT == 2) {
                    const tu32x4_t* second = run_at(Kp, pb, base + 16);
                    if (n16 >= 8) run = second;
                }
            }
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) {
                const tu32x4_t* x = pair_at(Kp, k_fresh, run, base, key_of_row(0, n16), nt * 4);
#pragma unroll
                for (int ks = 0; ks < KS; ++ks) kr[nt][ks].u = ld16(x + ks * 4 + quad);
            }
        };
        auto load_v = [&](int base, int pa, int pb) {
            const tu32x4_t* run = nullptr;
            if constexpr (!ROWS) {
                run = run_at(Vp, pa, base);
                if constexpr (NT == 2) {
                    const tu32x4_t* second = run_at(Vp, pb, base + 16);
                    if (quad >= 2) run = second;
                }
            }
            if constexpr (BF) {
#pragma unroll
                for (int u = 0; u < 8; ++u) {
                    const tu32x4_t* x = pair_at(Vp, v_fresh, run, base, quad * 8, u);
                    if constexpr (D == 128) {
                        vr[u].u = ld16(x + n16);
                    } else {
                        const tu32x2_t y = ld8(reinterpret_cast<const tu32x2_t*>(x) + n16);
                        vr[u].w[0] = y.x;
                        vr[u].w[1] = y.y;
                    }
                }
            } else {
#pragma unroll
                for (int u = 0; u < 4; ++u) {
                    const tu32x4_t* x = pair_at(Vp, v_fresh, run, base, quad * 4, u);
#pragma unroll
                    for (int c = 0; c < D / 64; ++c) vr[u * (D / 64) + c].u = ld16(x + c * 16 + n16);
                }
            }
        };
        constexpr int VW = BF && D == 64 ? 2 : 4;   // words in use of a V load
        auto v_key = [&](int x) { return BF ? quad * 8 + x : quad * 4 + x / (D / 64); };   // key of V load x in the tile

        // The rows of all tokens at once.  A row gives the pairs that it does not see weight 0, which must not meet an infinity or a NaN that another
        // row sees: where there is any, the run starts over with half of its tokens.
        for (int lo = tile_lo, hi = tile_hi;;) {
        if (!ROWS && tid == 0) s_bad = 0;
        if constexpr (!ROWS) __syncthreads();
        const int pos = t.first + my_token, p = TWICE || (n16 < rows && pos >= lo && pos <= hi) ? pos : -1;   // -1: sees nothing
        const int p_from = p < 0 || W.window == 0x7fffffff ? -1 : p - W.window;   // sees keys (p_from, p] and [0, min(sink, p + 1))
        const int p_sink = min(W.sink, p + 1);
        float m_run = -INFINITY, l_run = 0.f;
        tf32x4_t o[ET];
        // The step's outputs, as those of the step without accumulation, are normalised by the weights as they meet V (bf16, head_dim 128): a row of
        // ones more in the product (8 rows of 1000 pairs 10.0 us a step, with it 10.1; 128 of 2112 28.7 either way).  The accumulated weights by the
        // sum of the unrounded ones.
        constexpr bool ONES = ROWS && BF && D == 128;
        tf32x4_t o_l = (tf32x4_t){0.f, 0.f, 0.f, 0.f};
        T128 ones;
        ones.u = tu32x4_t{0x3f803f80u, 0x3f803f80u, 0x3f803f80u, 0x3f803f80u};
        // head_dim 64: a probability as three bf16 terms, all 24 bits of it, the first and the second in the lower and the upper columns, the third in a
        // product of its own.  Sums of their own, added at the end: an infinite value times a later term, which may be 0 or negative, must not meet the first's.
        // One term alone, four heads: 8 rows of 300 pairs 7.9 us a step, with three 8.4; 128 of 1000 12.8, 13.5; of 2112 19.6, 20.4; eight heads 21.3, 21.8.
        constexpr bool TERMS = ROWS && BF && D == 64;
        tf32x4_t o3[TERMS ? ET : 1];
#pragma unroll
        for (int e = 0; e < (TERMS ? ET : 1); ++e) o3[e] = (tf32x4_t){0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int e = 0; e < ET; ++e) o[e] = (tf32x4_t){0.f, 0.f, 0.f, 0.f};

        int i = t_begin + wave, pa = 0, pb = 0, base = 0;
        if (i < t_end) {
            base = kt.at(i) * KT;
            pages_of(base, pa, pb);
            load_k(base, pa, pb);
            load_v(base, pa, pb);
        }
        int na = 0, nb = 0, next = 0;
        if (i + WAVES < t_end) {
            next = kt.at(i + WAVES) * KT;
            pages_of(next, na, nb);
        }
        auto tile = [&](auto LAST) {   // (twice in the code: under a condition the next tile's loads would need registers of their own)
            tf32x4_t c[NT];
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) {
                c[nt] = (tf32x4_t){0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int ks = 0; ks < KS; ++ks) {
                    if constexpr (BF) {
                        c[nt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kr[nt][ks].v, q[ks].v, c[nt], 0, 0, 0);
                    } else {
#pragma unroll
                        for (int e = 0; e < 4; ++e) c[nt] = __builtin_amdgcn_mfma_f32_16x16x4f32(kr[nt][ks].f[e], q[ks].f[e], c[nt], 0, 0, 0);
                    }
                }
            }
            if constexpr (!LAST) load_k(next, na, nb);

            // everything seen by every row: no masks
            const bool whole = base + KT <= lo + 1 && (W.window == 0x7fffffff || base > hi - W.window || base + KT <= W.sink) && (ROWS || (page_ok(W, pa) && page_ok(W, pb)));
            float s[NT * 4];
#pragma unroll
            for (int j = 0; j < NT * 4; ++j) s[j] = attn_logit(c[j / 4][j % 4], scale);
            auto key_at = [&](int j) { return base + quad * (NT * 4) + j; };   // key of logit j
            const bool ok = NT == 2 && quad >= 2 ? page_ok(W, pb) : page_ok(W, pa);   // this lane's keys' page
            if (!whole) {
#pragma unroll
                for (int j = 0; j < NT * 4; ++j) {
                    const int key = key_at(j);
                    if (!((ROWS || ok) && key <= p && (key > p_from || key < p_sink))) s[j] = -INFINITY;
                }
            }
            if constexpr (ROWS) {   // kept: with the final maximum and sum they become weights
                auto keep = [&](float* lg) {
                    if (base + KT <= t.n) {
#pragma unroll
                        for (int j = 0; j < NT * 4; j += 4) *reinterpret_cast<float4*>(lg + j) = make_float4(s[j], s[j + 1], s[j + 2], s[j + 3]);
                    } else {
#pragma unroll
                        for (int j = 0; j < NT * 4; ++j)
                            if (key_at(j) < t.n) lg[j] = s[j];
                    }
                };
                if (n16 < g) {
                    if (lg_local) keep(s_lg + n16 * P.logits_lds + base + quad * (NT * 4));
                    else keep(P.logit + ((size_t)slot * g + n16) * P.logit_stride + base + quad * (NT * 4));
                }
            }
            float mx = s[0];
#pragma unroll
            for (int j = 1; j < NT * 4; ++j) mx = fmaxf(mx, s[j]);
            const float mn = fmaxf(m_run, quad_max(mx)), ref = ref_of(mn);
            const bool moved = mn > m_run;
            const float corr = __builtin_amdgcn_exp2f(m_run - ref);
            m_run = mn;
            float sum = 0.f;
#pragma unroll
            for (int j = 0; j < NT * 4; ++j) {
                s[j] = __builtin_amdgcn_exp2f(s[j] - ref);
                sum += s[j];
            }
            l_run = fmaf(l_run, corr, sum);
            if (__any(moved)) {
#pragma unroll
                for (int e = 0; e < ET; ++e)
#pragma unroll
                    for (int k = 0; k < 4; ++k) o[e][k] *= corr;
                if constexpr (ONES) o_l[0] *= corr;   // (all four are the same sum)
                if constexpr (TERMS) {
#pragma unroll
                    for (int e = 0; e < ET; ++e)
#pragma unroll
                        for (int k = 0; k < 4; ++k) o3[e][k] *= corr;
                }
            }
            T128 pr, p3;   // bf16: the probabilities, rounded; TERMS: of what the terms before leave
            if constexpr (TERMS) {
#pragma unroll
                for (int w = 0; w < 4; ++w) {
                    const uint32_t first = pack_bf16(s[2 * w], s[2 * w + 1]);
                    const float x = s[2 * w] - bf16_lo(first), y = s[2 * w + 1] - bf16_hi(first);
                    const uint32_t second = pack_bf16(x, y);
                    pr.w[w] = n16 < 8 ? first : second;
                    p3.w[w] = pack_bf16(x - bf16_lo(second), y - bf16_hi(second));
                }
            } else if constexpr (BF) {
#pragma unroll
                for (int w = 0; w < 4; ++w) pr.w[w] = pack_bf16(s[2 * w], s[2 * w + 1]);
                if constexpr (ONES) o_l = __builtin_amdgcn_mfma_f32_16x16x32_bf16(ones.v, pr.v, o_l, 0, 0, 0);
            }
            if (!whole) {   // values of weight 0 must not meet the products as infinities or NaN
                bool bad = false;
                const bool v_ok = BF && quad >= 2 ? page_ok(W, pb) : page_ok(W, pa);
                const int any_from = W.window == 0x7fffffff ? -1 : lo - W.window, all_from = W.window == 0x7fffffff ? -1 : hi - W.window;
#pragma unroll
                for (int x = 0; x < VL; ++x) {
                    const int key = base + v_key(x);
                    const bool someone = (ROWS || v_ok) && key <= hi && (key > any_from || key < W.sink);
                    const bool everyone = (key <= lo) & ((key > all_from) | (key < W.sink));   // of those that someone sees
                    const uint32_t keep = someone ? ~0u : 0u;   // (no branch: the registers of both ways would be kept)
#pragma unroll
                    for (int w = 0; w < VW; ++w) {
                        vr[x].w[w] &= keep;
                        if constexpr (!ROWS) bad |= !everyone & word_not_finite<T>(vr[x].w[w]);
                    }
                }
                if (!ROWS && bad && hi > lo) s_bad = 1;
            }
#pragma unroll
            for (int e = 0; e < ET; ++e) {   // V^T.P^T
                if constexpr (BF) {
                    const uint32_t sel = (e & 1) ? 0x07060302u : 0x05040100u;
                    T128 vb;
#pragma unroll
                    for (int w = 0; w < 4; ++w) vb.w[w] = __builtin_amdgcn_perm(vr[2 * w + 1].w[e >> 1], vr[2 * w].w[e >> 1], sel);
                    o[e] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vb.v, pr.v, o[e], 0, 0, 0);
                    if constexpr (TERMS) o3[e] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vb.v, p3.v, o3[e], 0, 0, 0);
                } else {
#pragma unroll
                    for (int u = 0; u < 4; ++u) o[e] = __builtin_amdgcn_mfma_f32_16x16x4f32(vr[u * (D / 64) + e / 4].f[e % 4], s[u], o[e], 0, 0, 0);
                }
            }
            if constexpr (!LAST) {
                load_v(next, na, nb);
                pa = na;
                pb = nb;
                base = next;
                next = kt.at(min(i + 2 * WAVES, t_end - 1)) * KT;
                pages_of(next, na, nb);
            }
        };
        for (; i + WAVES < t_end; i += WAVES) tile(std::false_type());
        if (i < t_end) tile(std::true_type());

        // ---- merge the wavefronts ----------------------------------------------------------------------------------
        int tid = threadIdx.x;   // (opaque: or everything that the merge derives from it is kept in registers over the loop)
        asm volatile("" : "+v"(tid));
        const int n16 = tid & 15, quad = (tid & (kWave - 1)) >> 4;
        l_run = quad_sum(l_run);
        if (quad == 0) {
            s_m[wave][n16] = m_run;
            s_l[wave][n16] = ONES && n16 >= 8 ? o_l[0] : l_run;   // TWICE: of the accumulated weights, and from 8 on the normaliser of the outputs
        }
        if constexpr (TERMS) {
#pragma unroll
            for (int e = 0; e < ET; ++e)
#pragma unroll
                for (int k = 0; k < 4; ++k) o[e][k] = add_terms(o[e][k], dpp_f<DPP_ROW_ROR8>(o[e][k]), o3[e][k]);
        }
        if (!ROWS || n16 < R)
#pragma unroll
        for (int k = 0; k < 4; ++k)
#pragma unroll
            for (int e = 0; e < ET; e += 4)
                *reinterpret_cast<float4*>(&s_o[wave][n16][channel_of<T, D>(quad * 4 + k, e)]) = make_float4(o[e][k], o[e + 1][k], o[e + 2][k], o[e + 3][k]);
        __syncthreads();
        if constexpr (!ROWS) {
            if (scalar(s_bad)) {   // (the same for every thread)
                hi = lo + (hi - lo) / 2;
                __syncthreads();
                continue;
            }
        }
        if (tid < 16) {
            float M = -INFINITY, L = 0.f;
#pragma unroll
            for (int w = 0; w < WAVES; ++w) M = fmaxf(M, s_m[w][tid]);
            const float ref = ref_of(M);
#pragma unroll
            for (int w = 0; w < WAVES; ++w) {
                const float f = __builtin_amdgcn_exp2f(s_m[w][tid] - ref);
                s_w[w][tid] = f;
                L = fmaf(s_l[w][tid], f, L);
            }
            s_M[tid] = M;
            s_L[tid] = L;
        }
        __syncthreads();
        const size_t rec = (((size_t)slot * n_kv + h) * P.splits + split) * 16;
        for (int x = tid; x < rows * (D / 4); x += WAVES * kWave) {
            const int r = x / (D / 4), d = x % (D / 4) * 4;
            const int tok = token_of(r0 + r);
            if (!ROWS && (t.first + tok < lo || t.first + tok > hi)) continue;
            float a[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int w = 0; w < WAVES; ++w) {
                const float4 v = *reinterpret_cast<const float4*>(&s_o[w][r][d]);
                const float f = s_w[w][r];
                a[0] = fmaf(v.x, f, a[0]);
                a[1] = fmaf(v.y, f, a[1]);
                a[2] = fmaf(v.z, f, a[2]);
                a[3] = fmaf(v.w, f, a[3]);
            }
            if (splits > 1) {
                *reinterpret_cast<float4*>(P.rec + (rec + r) * D + d) = make_float4(a[0], a[1], a[2], a[3]);
                if (d == 0) {
                    P.rec_ml[rec + r] = make_float2(s_M[r], s_L[r]);
                    if constexpr (ROWS) P.rec_ml[rec + 8 + r] = make_float2(s_M[r], s_L[TWICE ? 8 + r : r]);
                }
                continue;
            }
            store_row<T, D, ROWS>(P, ((size_t)(t.begin + tok) * n_kv + h) * g + (r0 + r - tok * g), d, a, s_M[r], s_L[TWICE ? 8 + r : r]);
        }
        if constexpr (ROWS) {
            // the new pair joins the cache (its slot is read by nobody in this launch)
            if (split == 0 && fresh >= 0) {
                tu32x4_t *Kw = const_cast<tu32x4_t*>(Kp) + ((size_t)slot * P.cap + fresh) * CH, *Vw = const_cast<tu32x4_t*>(Vp) + ((size_t)slot * P.cap + fresh) * CH;
                if (tid < CH) Kw[tid] = k_fresh[tid];
                else if (tid < 2 * CH) Vw[tid - CH] = v_fresh[tid - CH];
                else if (tid == 2 * CH) P.pos[(size_t)slot * P.cap + fresh] = P.pos_new[slot / P.batch_of_pos];
            }
            if (split == 0 && tid == 0 && P.splits > 1) P.info[slot] = make_int2(t.n, fresh);   // (the second launch sets the length: others read it yet)
            if (splits > 1) return;
            // one workgroup a row: the weights, from the logits that this workgroup has written (the barriers above make them visible)
            float* acc = P.acc + (size_t)slot * P.cap;
            float inv[8];
#pragma unroll
            for (int k = 0; k < 8; ++k) inv[k] = k < g ? 1.0f / s_L[k] : 0.f;
            auto add = [&](const float* lg, int stride) {
                for (int key = tid; key < t.n; key += WAVES * kWave) {
                    float x[8], w = 0.f;
#pragma unroll
                    for (int k = 0; k < 8; ++k) x[k] = lg[(size_t)min(k, g - 1) * stride + key];
#pragma unroll
                    for (int k = 0; k < 8; ++k)
                        if (k < g) w = fmaf(__builtin_amdgcn_exp2f(x[k] - ref_of(s_M[k])), inv[k], w);
                    acc[key] = (key == fresh ? 0.f : key == tid ? acc_first : acc[key]) + w;
                }
            };
            if (lg_local) add(s_lg, P.logits_lds);
            else add(P.logit + (size_t)slot * g * P.logit_stride, P.logit_stride);
            if (tid == 0 && fresh >= 0 && P.splits == 1) P.len[slot] = t.n;
            return;
        }
        __syncthreads();   // the LDS is the next run's
        if (hi == tile_hi) break;
        lo = hi + 1;
        hi = tile_hi;
        }
    }
}

}  // namespace fk
