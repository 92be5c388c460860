// Attention of prompt chunks over the pages of a prompt: tiles of 128 query rows (tokens x heads of a group) against tiles of 64 pairs (fp32: 32).
//
// A wavefront owns 32 rows: their q, online softmax and outputs stay in its registers.  The pairs pass by in tiles, each read once for
// the four wavefronts, straight into LDS (two buffers each for K and V, one barrier a tile).  While the vector units turn one tile's logits into
// probabilities, the matrix units form the next one's: with a tile's steps one after the other a wavefront alone on its SIMD took 2.2 us a tile,
// of which the products are 0.4.  Products and operand layouts are those of thin.h (logits K.Q^T with the keys in an order that makes a
// lane's probabilities an operand of V^T.P^T as they are; the same 16x16 products in the same order, so that they are the same bits
// everywhere); an operand read from LDS serves two products, one for each 16 rows.
//   in LDS a row's 16-byte chunks change places (swizzle_k, swizzle_v), so that the 16 rows of an operand lie in different banks; a load writes LDS in
//   the order of its lanes, so each lane fetches the chunk that belongs in its place
//   V, bf16: the operand is 8 keys of one channel per lane, which the transposing LDS read delivers, 4 keys at a time (ds_read_tr16_b64: lane l of
//   16 gets element l % 4 of what lanes l / 4, + 4, + 8, + 12 address); fp32: four channels a lane, each a product of its own
// References follow a row's maximum only where it has grown by more than 2^8 (probabilities up to 256, sums in fp32: nothing is lost), so that
// outputs are hardly ever rescaled.
//
// Bound by matrix and vector instructions of two wavefronts a SIMD (256 registers each): 2048 tokens of 16384 pairs, 8 heads of g 4, D 128: 517 us, 1000
// TFLOP/s, a tile of 64 pairs in 2.1 us for two workgroups of a CU; matrix cores busy 42 % of the time, no LDS conflicts, each byte read from memory
// once.  Waits for operands inside the block of instructions that needs them, orders of products and vector instructions set by hand, and operands
// read a step earlier took 509 to 582 us.
#pragma once
#include "attn_paged.h"

#include <climits>
#include <type_traits>

namespace fk {

template <typename T, int D> struct PromptCfg {
    static constexpr bool BF = sizeof(T) == 2;
    static constexpr int CH = D * (int)sizeof(T) / 16, KS = CH / 4, ET = D / 16;
    static constexpr int KT = BF ? 64 : 32;       // pairs of a tile
    static constexpr int NT = BF ? 2 : 1;         // 16-key products of a block (as many keys as a product of P.V takes)
    static constexpr int BLK = 16 * NT, NB = KT / BLK, GI = KT / 16;
    static constexpr int CT = 2;                  // 16-row tiles of a wavefront
    static constexpr int TM = kPromptRows;
    static constexpr int LD = KT * CH / 256, RPU = 256 / CH;   // loads of a tile per thread and tensor; rows that one load of the workgroup covers
    static constexpr int TILE_BYTES = KT * CH * 16;
    static constexpr size_t LDS_BYTES = 4 * (size_t)TILE_BYTES;   // K, V, two buffers
};

// 16-byte chunk of a row -> its place
template <bool BF, int CH> __device__ __forceinline__ int swizzle_k(int row) {
    if constexpr (!BF) return row & 15;
    else if constexpr (CH == 16) return (row & 3) | ((row >> 3) & 3) << 2;
    else return ((row >> 1) & 1) | ((row >> 3) & 3) << 1;
}
template <bool BF, int CH> __device__ __forceinline__ int swizzle_v(int row) {
    if constexpr (!BF) return 0;
    else if constexpr (CH == 16) return (row & 3) << 1 | ((row >> 3) & 1) << 3;
    else return ((row >> 1) & 1) << 1 | ((row >> 3) & 1) << 2;
}

typedef short ps16x4_t __attribute__((ext_vector_type(4)));
__device__ __forceinline__ tu32x2_t read_transposed(const unsigned char* p) {
    typedef __attribute__((address_space(3))) ps16x4_t lds_t;
    return __builtin_bit_cast(tu32x2_t, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_t*)p));
}

template <typename T, int D>
__device__ __forceinline__ void prompt_tile(const AttnPagedParams& P, int item, int split) {
    using C = PromptCfg<T, D>;
    constexpr bool BF = C::BF;
    constexpr int CH = C::CH, KS = C::KS, ET = C::ET, KT = C::KT, NT = C::NT, BLK = C::BLK, NB = C::NB, GI = C::GI, CT = C::CT, TM = C::TM, LD = C::LD, RPU = C::RPU;
    const PagedParams& W = P.view;
    const int tid = threadIdx.x, lane = tid & (kWave - 1), n16 = lane & 15, quad = lane >> 4, wave = scalar(tid / kWave);
    const int n_kv = W.n_kv, slot = scalar(divide(item, n_kv, W.kv_magic)), h = item - slot * n_kv, g = W.g;
    extern __shared__ __attribute__((aligned(16))) unsigned char smem[];
    __shared__ int s_bad;
    TileOf t;
    if (!tile_of(W, P.grid, slot, TM, t)) return;
    const int32_t* tab = scalar_ptr(W.table + (size_t)t.b * W.max_pages);
    const float scale = W.scale_log2e;
    const bool windowed = W.window != 0x7fffffff;

    // LDS places of this lane's operands, and of what this thread stages (rows RPU apart have the same swizzle: RPU >= 8, or bits that swizzles skip)
    int k_at[KS];
    {
        const int row = BF ? n16 / 4 * 8 + n16 % 4 : n16;   // of MFMA row n16 in the first product of a block
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) k_at[ks] = row * CH * 16 + ((ks * 4 + quad) ^ swizzle_k<BF, CH>(row)) * 16;
    }
    const int v_row = BF ? quad * 8 + n16 / 4 : quad * 4;
    auto v_at = [&](int e) {   // bf16: the lane's share of channel tile e
        return v_row * CH * 16 + ((2 * e + n16 % 4 / 2) ^ swizzle_v<BF, CH>(v_row)) * 16 + n16 % 2 * 8;
    };
    const int st_row = tid / CH, st_ch = tid % CH;

    for (; t.tile >= 0; t.tile -= t.step) {
        const int r0 = t.tile * TM, rows = min(TM, t.nq * g - r0);
        auto token_of = [&](int r) { return divide(r, g, W.g_magic); };
        const int tile_lo = scalar(t.first + token_of(r0)), tile_hi = scalar(t.first + token_of(r0 + rows - 1));
        const KeyTiles kt = key_tiles(W, tile_lo, tile_hi, KT);
        const int splits = scalar(splits_of(kt.total, t.one && item >= P.whole ? P.splits : 1, P.split_shift));
        if (split >= splits) continue;
        const int per = splits == 1 ? kt.total : scalar(divide(kt.total + splits - 1, splits)), t_begin = min(split * per, kt.total), t_end = min(t_begin + per, kt.total);

        // the wavefront's rows
        const int w0 = r0 + wave * 32, w_rows = min(32, rows - wave * 32);   // <= 0: none
        const int w_first = scalar(t.first + token_of(w0)), w_last = scalar(t.first + token_of(w0 + max(w_rows, 1) - 1));
        int pos[CT];
        T128 q[CT][KS];
#pragma unroll
        for (int ct = 0; ct < CT; ++ct) {
            const int r = w0 + ct * 16 + n16, rc = min(r, r0 + rows - 1), tok = token_of(rc);
            pos[ct] = r < r0 + rows ? t.first + tok : INT_MIN;   // (negative ones see nothing)
            const size_t q_row = ((size_t)(t.begin + tok) * n_kv + h) * g + (rc - tok * g);
#pragma unroll
            for (int ks = 0; ks < KS; ++ks) {
                q[ct][ks].u = reinterpret_cast<const tu32x4_t*>(W.q)[q_row * CH + ks * 4 + quad];
                if (W.negate) q[ct][ks].u ^= BF ? 0x80008000u : 0x80000000u;
            }
        }

        // A row gives the pairs that it does not see weight 0, which must not meet an infinity or a NaN that another row sees: where there is any, the
        // run starts over with half of its tokens.
        for (int lo = tile_lo, hi = tile_hi;;) {
            if (tid == 0) s_bad = 0;
            __syncthreads();
            const int w_lo = max(w_first, lo), w_hi = w_rows > 0 ? min(w_last, hi) : -1;
            int p[CT], p_from[CT], p_sink[CT];
            bool mine[CT];   // this run's rows
            float m_ref[CT], m_top[CT], l_run[CT];
            tf32x4_t o[ET][CT];
#pragma unroll
            for (int ct = 0; ct < CT; ++ct) {
                mine[ct] = pos[ct] >= lo && pos[ct] <= hi;
                p[ct] = mine[ct] ? pos[ct] : -1;
                p_from[ct] = p[ct] < 0 || !windowed ? -1 : p[ct] - W.window;
                p_sink[ct] = min(W.sink, p[ct] + 1);
                m_ref[ct] = m_top[ct] = -INFINITY;
                l_run[ct] = 0.f;
#pragma unroll
                for (int e = 0; e < ET; ++e) o[e][ct] = (tf32x4_t){0.f, 0.f, 0.f, 0.f};
            }
            auto base_of = [&](int i) { return kt.at(i) * KT; };
            // where a tile's runs of 16 pairs lie, counted in such runs (so that 32 bits hold any pool), and a bit for each that lies nowhere
            struct Runs {
                uint32_t at[GI], holes;
            };
            auto runs_of = [&](int i) {   // (past the end: the last tile's)
                Runs x;
                const int base = base_of(min(i, t_end - 1));
                auto find = [&](int r, uint32_t& hole) {
                    const int key = base + r * 16, page = load_uniform(tab, min(key >> W.page_shift, W.max_pages - 1));
                    hole = page_ok(W, page) ? 0 : 1;
                    return ((uint32_t)(hole ? 0 : page) * n_kv + h) << (W.page_shift - 4) | (key & ((1 << W.page_shift) - 1)) >> 4;
                };
                uint32_t hole;
                if (1 << W.page_shift >= KT) {   // one page
                    const uint32_t at = find(0, hole);
#pragma unroll
                    for (int r = 0; r < GI; ++r) x.at[r] = at + r;
                    x.holes = hole ? (1 << GI) - 1 : 0;
                } else {
                    x.holes = 0;
#pragma unroll
                    for (int r = 0; r < GI; ++r) {
                        x.at[r] = find(r, hole);
                        x.holes |= hole << r;
                    }
                }
                return x;
            };
            auto run_of_load = [&](int u) { return RPU == 32 ? 2 * u + (wave >= 2 ? 1 : 0) : u * RPU / 16; };   // load u of this wavefront lies in one run
            auto send = [&](const void* X, bool is_k, int buf, const Runs& runs) {
#pragma unroll
                for (int u = 0; u < LD; ++u) {
                    const int row = st_row + u * RPU;
                    const uint32_t run = RPU == 32 ? (wave >= 2 ? runs.at[2 * u + (RPU == 32 ? 1 : 0)] : runs.at[RPU == 32 ? 2 * u : 0]) : runs.at[u * RPU / 16];
                    const int ch = st_ch ^ (is_k ? swizzle_k<BF, CH>(row) : swizzle_v<BF, CH>(row));
                    load_to_lds(static_cast<const unsigned char*>(X) + (size_t)run * (16 * CH * 16) + (uint32_t)((row % 16 * CH + ch) * 16),
                                smem + (is_k ? 0 : 2 * C::TILE_BYTES) + buf * C::TILE_BYTES + (u * 256 + wave * 64) * 16);
                }
            };
            auto whole_for = [&](int base, int from, int to, const Runs& runs) {   // every row at positions from .. to sees all of the tile
                return base + KT <= from + 1 && (!windowed || base > to - W.window || base + KT <= W.sink) && !runs.holes;
            };
            // V of a tile that not every row sees: values of weight 0 must not meet the products as infinities or NaN
            auto clear_hidden = [&](int buf, int base, const Runs& runs) {
                const int any_from = windowed ? lo - W.window : -1, all_from = windowed ? hi - W.window : -1;
                bool bad = false;
#pragma unroll
                for (int u = 0; u < LD; ++u) {
                    const int key = base + st_row + u * RPU;
                    const bool someone = !(runs.holes >> run_of_load(u) & 1) & (key <= hi) & ((key > any_from) | (key < W.sink));
                    const bool everyone = (key <= lo) & ((key > all_from) | (key < W.sink));   // of those that someone sees
                    tu32x4_t* at = reinterpret_cast<tu32x4_t*>(smem + (2 + buf) * C::TILE_BYTES + (u * 256 + tid) * 16);
                    if (!someone) *at = tu32x4_t{0, 0, 0, 0};
                    else if (!everyone) {
                        const tu32x4_t x = *at;
#pragma unroll
                        for (int w = 0; w < 4; ++w) bad |= word_not_finite<T>(x[w]);
                    }
                }
                if (bad && hi > lo) s_bad = 1;
            };
            typedef tf32x4_t Logits[GI][CT];
            // logits of a tile, raw, and the largest of a lane's of every row
            auto products = [&](auto buf, Logits& c) {
                const unsigned char* sk = smem + buf * C::TILE_BYTES;
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
            // a row's largest logit of a tile, and whether its reference has to move or differences would lose their bits
            bool need = false, large = false;
            float m_new[CT];
            auto assess = [&](const Logits& c) {
                need = large = false;
#pragma unroll
                for (int ct = 0; ct < CT; ++ct) {
                    float mx = c[0][ct][0];
#pragma unroll
                    for (int x = 1; x < GI * 4; ++x) mx = fmaxf(mx, c[x / 4][ct][x % 4]);
                    const float m = attn_logit(quad_max(mx), scale);
                    m_new[ct] = m;
                    need |= m > m_ref[ct] + 8.f;
                    large |= fabsf(fmaxf(m, m_ref[ct])) >= kLargeLogit;   // (nothing seen: -inf as well, with nothing to lose)
                }
            };
            // One tile: its logits c become weights and meet V; the next one's are formed beside them.
            auto step = [&](auto buf, int base, const Runs& runs, Logits& c, Logits& next) {
                if (!whole_for(base, w_lo, w_hi, runs)) {
#pragma unroll
                    for (int gi = 0; gi < GI; ++gi) {
                        const int b = gi / NT;
                        const bool there = !(runs.holes >> (BF ? 2 * b + (quad >= 2) : b) & 1);
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            const int key = base + b * BLK + quad * (NT * 4) + gi % NT * 4 + e;
#pragma unroll
                            for (int ct = 0; ct < CT; ++ct) {
                                const bool seen = there & (key <= p[ct]) & ((key > p_from[ct]) | (key < p_sink[ct]));
                                c[gi][ct][e] = seen ? c[gi][ct][e] : -INFINITY;
                            }
                        }
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
                for (int ct = 0; ct < CT; ++ct) less[ct] = m_ref[ct];
                if (__any(large)) {   // rounded before the reference is subtracted; the fma below then has nothing left to do
                    by = 1.f;
#pragma unroll
                    for (int ct = 0; ct < CT; ++ct) {
                        less[ct] = 0.f;
#pragma unroll
                        for (int x = 0; x < GI * 4; ++x) c[x / 4][ct][x % 4] = attn_logit(c[x / 4][ct][x % 4], scale) - ref_of(m_ref[ct]);
                    }
                }
                __builtin_amdgcn_s_setprio(1);   // against the other workgroup's wavefront, which is then at its loads and masks (520 -> 511 us)
                products(std::integral_constant<int, (buf ^ 1)>{}, next);   // (behind the last tile: of what lies there, for nobody)
#pragma unroll
                for (int ct = 0; ct < CT; ++ct) {
                    float sum = 0.f;
#pragma unroll
                    for (int x = 0; x < GI * 4; ++x) {
                        const float w = __builtin_amdgcn_exp2f(fmaf(c[x / 4][ct][x % 4], by, -less[ct]));
                        c[x / 4][ct][x % 4] = w;
                        sum += w;
                    }
                    l_run[ct] += sum;
                }
                const unsigned char* sv = smem + (2 + buf) * C::TILE_BYTES;
#pragma unroll
                for (int b = 0; b < NB; ++b) {
                    if constexpr (BF) {
                        T128 pr[CT];   // rounded: each weight by half a step of bf16 at most, sums of them in fp32
#pragma unroll
                        for (int ct = 0; ct < CT; ++ct)
#pragma unroll
                            for (int w = 0; w < 4; ++w) pr[ct].w[w] = pack_bf16(c[2 * b + w / 2][ct][w % 2 * 2], c[2 * b + w / 2][ct][w % 2 * 2 + 1]);
#pragma unroll
                        for (int e = 0; e < ET; ++e) {
                            T128 v;
                            const unsigned char* at = sv + v_at(e) + b * BLK * CH * 16;
                            const tu32x2_t v0 = read_transposed(at), v1 = read_transposed(at + 4 * CH * 16);
                            v.u = tu32x4_t{v0.x, v0.y, v1.x, v1.y};
#pragma unroll
                            for (int ct = 0; ct < CT; ++ct) o[e][ct] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v.v, pr[ct].v, o[e][ct], 0, 0, 0);
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

            // K of tile i lies in buffer (i - t_begin) % 2 from two tiles ahead on, V from one tile ahead on.
            Logits ca, cb;
            if (t_begin < t_end) {
                Runs runs = runs_of(t_begin), runs1 = runs_of(t_begin + 1), runs2 = runs_of(t_begin + 2);
                send(W.K, true, 0, runs);
                send(W.V, false, 0, runs);
                if (t_begin + 1 < t_end) send(W.K, true, 1, runs1);
                arrived();
                __syncthreads();
                if (w_rows > 0) {
                    products(std::integral_constant<int, 0>{}, ca);
                    assess(ca);
                }
                __syncthreads();
                auto turn = [&](auto buf, int i, Logits& c, Logits& next) {
                    const int base = base_of(i);
                    if (!whole_for(base, lo, hi, runs)) {
                        clear_hidden(buf, base, runs);
                        __syncthreads();
                    }
                    if (i + 2 < t_end) send(W.K, true, buf, runs2);
                    if (i + 1 < t_end) send(W.V, false, buf ^ 1, runs1);
                    const Runs runs3 = runs_of(i + 3);
                    if (w_rows > 0) step(buf, base, runs, c, next);
                    runs = runs1;
                    runs1 = runs2;
                    runs2 = runs3;
                    arrived();
                    __syncthreads();
                };
                for (int i = t_begin;;) {
                    turn(std::integral_constant<int, 0>{}, i, ca, cb);
                    if (++i == t_end) break;
                    turn(std::integral_constant<int, 1>{}, i, cb, ca);
                    if (++i == t_end) break;
                }
            }
            if (scalar(s_bad)) {   // (the same for every thread)
                hi = lo + (hi - lo) / 2;
                __syncthreads();
                continue;
            }

            // ---- results: every wavefront has its rows' own -------------------------------------------------------------
#pragma unroll
            for (int ct = 0; ct < CT; ++ct) {
                const float l = quad_sum(l_run[ct]), f = __builtin_amdgcn_exp2f(m_ref[ct] - ref_of(m_top[ct]));
                if (!mine[ct]) continue;
                const int r = w0 + ct * 16 + n16, tok = token_of(r);
                const size_t row = ((size_t)(t.begin + tok) * n_kv + h) * g + (r - tok * g);
                const size_t rec = ((size_t)(item - P.whole) * P.splits + split) * TM + (r - r0);
                const float mul = splits > 1 ? f : l == 0.f ? 0.f : 1.0f / l;
#pragma unroll
                for (int e = 0; e < ET; e += BF ? 1 : 4) {
                    if constexpr (BF) {   // channels e * 16 + quad * 4 ..
                        const tf32x4_t a = o[e][ct] * mul;
                        const int d = e * 16 + quad * 4;
                        if (splits > 1) *reinterpret_cast<float4*>(P.rec + rec * D + d) = make_float4(a[0], a[1], a[2], a[3]);
                        else *reinterpret_cast<tu32x2_t*>(reinterpret_cast<bf16_t*>(P.out) + row * D + d) = tu32x2_t{pack_bf16(a[0], a[1]), pack_bf16(a[2], a[3])};
                    } else {
#pragma unroll
                        for (int k = 0; k < 4; ++k) {   // e / 4 * 64 + (quad * 4 + k) * 4 ..
                            const float4 a = make_float4(o[e][ct][k] * mul, o[e + 1][ct][k] * mul, o[e + 2][ct][k] * mul, o[e + 3][ct][k] * mul);
                            const int d = e / 4 * 64 + (quad * 4 + k) * 4;
                            if (splits > 1) *reinterpret_cast<float4*>(P.rec + rec * D + d) = a;
                            else *reinterpret_cast<float4*>(reinterpret_cast<float*>(P.out) + row * D + d) = a;
                        }
                    }
                }
                if (quad == 0) {
                    const float2 ml = make_float2(m_top[ct], l * f);   // nothing seen: (-inf, 0); a sum that is no number stays none, whatever the maximum is
                    if (splits > 1) P.rec_ml[rec] = ml;
                    else if (P.stats) P.stats[row] = ml;
                }
            }
            if (hi == tile_hi) break;
            lo = hi + 1;
            hi = tile_hi;
        }
        __syncthreads();   // the LDS is the next tile's
    }
}

}  // namespace fk
