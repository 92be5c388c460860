// fk_paged_weights: acc_j += sum over the chunk's queries that see pair j, over the group's heads, of 2^(s - M) / L.
//
// A wavefront owns KG * 16 keys, whose K stays in registers as matrix operands; the chunk's query rows (tokens x heads) pass by in
// tiles of 64, straight into LDS two tiles ahead, with their M and 1 / L, shared by the four wavefronts.  A product of 16 keys x 16 rows leaves a
// lane with four keys of ONE row, so M and 1 / L are one register each and a pair's weight is added by one fma; the 16 lanes of a key are
// summed once, at the end.  The order of all sums is fixed.  The products are those of the attention kernels, step by step the same ones, so that
// they are the same bits; large logits are rounded before M is subtracted, as where M was found (kLargeLogit): a query's weights add up to one.
//
// Bound by matrix and vector instructions together: per 16 x 16 logits D / 32 products and, per lane, four times an fma, an exponential and an fma.  16
// products and the vector work that goes with them, registers alone, two wavefronts to a SIMD, take 272 and 214 ns by themselves and 404 together; the
// kernel is at 1.4 times that (2048 tokens of 16384 pairs, 8 heads of g 4, D 128: 278 us, 940 TFLOP/s).  Three wavefronts to a SIMD do as well as two
// whose next logits are formed beside their exponentials (286 and 290), with half of the code.
// Few keys and many queries: the queries are split over workgroups too, partial sums meet in a second launch.
#include "weights.h"
#include "window.h"

#include <algorithm>

namespace fk {

typedef __attribute__((ext_vector_type(8))) __bf16 wbf16x8_t;
typedef __attribute__((ext_vector_type(4))) float wf32x4_t;
typedef __attribute__((ext_vector_type(4))) uint32_t wu32x4_t;
union W128 {
    wu32x4_t u;
    float f[4];
    wbf16x8_t v;
};

template <typename T, int D, bool FEW> struct WeightsCfg {   // FEW: few keys, 16 to a wavefront
    static constexpr bool BF = sizeof(T) == 2;
    static constexpr int CH = D * (int)sizeof(T) / 16, KS = CH / 4;
    static constexpr int KG = FEW ? 1 : BF || D == 64 ? 4 : 2;      // groups of 16 keys per wavefront
    static constexpr int KEYS = 4 * KG * 16;              // of a workgroup
    static constexpr int QT = BF ? 64 : 32;               // query rows of a tile
    static constexpr int NQ = QT / 16, TILE_BYTES = QT * CH * 16;
    static constexpr int LD = QT * CH / 256;              // 16-byte loads of a tile per thread
};

// Keys k0 .. k1 - 1 of a block, older than the chunk and outside of all its windows: their sums stay as they are, and splits write no partial ones
__device__ __forceinline__ bool nobody_sees(const PagedParams& W, int k0, int k1, int first) {
    return W.window != 0x7fffffff && k0 >= W.sink && k1 <= first && k1 - 1 + W.window <= first;
}

template <typename T, int D, bool FEW>
__global__ __launch_bounds__(256, 3) void weights_kernel(const WeightsParams P) {
    using C = WeightsCfg<T, D, FEW>;
    constexpr bool BF = C::BF;
    constexpr int CH = C::CH, KS = C::KS, KG = C::KG, QT = C::QT, NQ = C::NQ, LD = C::LD;
    const PagedParams& W = P.view;
    const int tid = threadIdx.x, lane = tid & (kWave - 1), n16 = lane & 15, quad = lane >> 4, wave = scalar(tid / kWave);
    const int place = scalar(divide(blockIdx.x, W.n_kv, W.kv_magic)), h = (int)blockIdx.x - place * W.n_kv, b = scalar(divide(place, P.blocks, P.blocks_magic)), split = blockIdx.y;
    const int g = W.g;
    extern __shared__ __attribute__((aligned(16))) unsigned char s_q[];   // two tiles
    __shared__ float s_m[2][QT], s_il[2][QT];

    const int begin = scalar(chunk_begin(W, b)), nq = scalar(chunk_end(W, b, begin)) - begin, n = scalar(pairs_of(W, b)), first = n - nq;
    if (nq == 0) return;
    auto token_of = [&](int row) { return divide(row, g, W.g_magic); };
    const float scale = W.scale_log2e;
    for (int k0 = (place - b * P.blocks) * C::KEYS; k0 < n; k0 += P.blocks * C::KEYS) {
        const int k1 = min(k0 + C::KEYS, n);
        if (nobody_sees(W, k0, k1, first)) continue;
        // tokens that see any of these keys: from position k0 on, and under a window up to the last key's reach
        int t0 = max(k0 - first, 0), t1 = nq;
        if (W.window != 0x7fffffff && k0 >= W.sink) t1 = min((long long)nq, max(0ll, (long long)k1 - 1 + W.window - first));
        const int row_lo = t0 * g, row_hi = max(t1, t0) * g;
        const int tiles = (row_hi - row_lo + QT - 1) / QT, per = scalar((tiles + P.splits - 1) / P.splits);
        const int i0 = min(split * per, tiles), i1 = min(i0 + per, tiles);

        const int kw = k0 + wave * (KG * 16);   // the wavefront's keys
        W128 k[KG][KS];
        bool there[KG];
        const int32_t* tab = scalar_ptr(W.table + (size_t)b * W.max_pages);
#pragma unroll
        for (int j = 0; j < KG; ++j) {
            const int key = kw + j * 16;
            const int page = key < n && i0 < i1 ? load_uniform(tab, min(key >> W.page_shift, W.max_pages - 1)) : -1;
            there[j] = page_ok(W, page);
            const wu32x4_t* run = reinterpret_cast<const wu32x4_t*>(W.K) +
                                  ((((size_t)(there[j] ? page : 0) * W.n_kv + h) << W.page_shift) + (key & ((1 << W.page_shift) - 1)) + n16) * CH;
#pragma unroll
            for (int ks = 0; ks < KS; ++ks) {
                k[j][ks].u = run[ks * 4 + quad];
                if (W.negate) k[j][ks].u ^= BF ? 0x80008000u : 0x80000000u;
            }
        }
        wf32x4_t a[KG];
#pragma unroll
        for (int j = 0; j < KG; ++j) a[j] = (wf32x4_t){0.f, 0.f, 0.f, 0.f};

        // Queries go straight into LDS, two tiles ahead.  There the 16-byte chunks of a row change places, so that 16 rows' operands lie in different
        // banks; a load writes in the order of its lanes, so each lane fetches the chunk that belongs in its place.
        constexpr int kSwap = (CH < 16 ? CH : 16) - 1;
        const uint32_t q_first = ((uint32_t)begin * W.n_kv + h) * g, q_token = (uint32_t)(W.n_kv - 1) * g;   // query row r of token t: q_first + r + t * q_token, below 2^28
        // where the rows that this thread fetches lie: a tile further they are QT rows and QT / g tokens on, or one token more (no division a tile)
        struct Place {
            uint32_t at;   // query row q_first + r + t * q_token
            int head;      // of its token's g
        };
        auto place_of = [&](int in_tile) {
            const int row = row_lo + i0 * QT + in_tile, tok = token_of(row);
            return Place{q_first + row + tok * q_token, row - tok * g};
        };
        const uint32_t last = q_first + row_hi - 1 + token_of(max(row_hi - 1, 0)) * q_token;   // (rows behind it: its copies)
        const int step_token = scalar(token_of(QT)), step_head = QT - step_token * g;
        const uint32_t step = QT + step_token * q_token;
        auto advance = [&](Place& x) {
            x.at += step;
            x.head += step_head;
            const bool over = x.head >= g;
            x.at += over ? q_token : 0;
            x.head -= over ? g : 0;
        };
        Place at_q[LD], at_st;
#pragma unroll
        for (int u = 0; u < LD; ++u) at_q[u] = place_of((tid + u * 256) / CH);
        at_st = place_of(tid % QT);
        float2 st;
        int st_row = row_lo + i0 * QT + tid % QT - QT;
        auto send = [&](int buf) {   // the next tile
#pragma unroll
            for (int u = 0; u < LD; ++u) {
                const int x = tid + u * 256;
                load_to_lds(reinterpret_cast<const wu32x4_t*>(W.q) + (size_t)min(at_q[u].at, last) * CH + (x % CH ^ (x / CH & kSwap)), s_q + buf * C::TILE_BYTES + (u * 256 + wave * 64) * 16);
                advance(at_q[u]);
            }
            if (wave * kWave < QT) st = P.stats[min(at_st.at, last)];
            st_row += QT;
            advance(at_st);
        };
        auto stage = [&](int buf) {
            if (tid < QT) {
                const bool none = st_row >= row_hi || st.y == 0.f;   // no query, or one that sees nothing: weight 0
                const float il = 1.0f / st.y;
                const bool lost = !(il < INFINITY);   // a sum that is no number: by way of M, pairs that the query does not see keep theirs
                s_m[buf][tid] = none ? 0.f : lost ? NAN : st.x;
                s_il[buf][tid] = none ? 0.f : lost ? 1.f : il;
            }
        };
        int q_at[KS];
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) q_at[ks] = (n16 * CH + ((ks * 4 + quad) ^ (n16 & kSwap))) * 16;
        if (i0 < i1) {
            send(0);
            stage(0);
            if (i0 + 1 < i1) send(1);
        }
        arrived();
        __syncthreads();
        for (int i = i0, buf = 0; i < i1; ++i, buf ^= 1) {
            const int base = row_lo + i * QT, lo = first + scalar(token_of(base)), hi = first + scalar(token_of(min(base + QT, row_hi) - 1));   // positions
            const bool whole = kw + KG * 16 <= lo + 1 && base + QT <= row_hi && (W.window == 0x7fffffff || kw > hi - W.window || kw + KG * 16 <= W.sink);
            const bool none = kw > hi || (W.window != 0x7fffffff && kw >= W.sink && kw + KG * 16 - 1 <= lo - W.window);   // of these keys any of these rows
            if (!none) {
#pragma unroll
            for (int qt = 0; qt < NQ; ++qt) {
                W128 q[KS];
#pragma unroll
                for (int ks = 0; ks < KS; ++ks) q[ks].u = *reinterpret_cast<const wu32x4_t*>(s_q + buf * C::TILE_BYTES + qt * 16 * CH * 16 + q_at[ks]);
                const float m = s_m[buf][qt * 16 + n16], il = s_il[buf][qt * 16 + n16];
                wf32x4_t c[KG];   // (side by side: a product waits for the one before it in its sum)
#pragma unroll
                for (int j = 0; j < KG; ++j) c[j] = (wf32x4_t){0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int ks = 0; ks < KS; ++ks) {
#pragma unroll
                    for (int e = 0; e < (BF ? 1 : 4); ++e) {
#pragma unroll
                        for (int j = 0; j < KG; ++j) {
                            if constexpr (BF) c[j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(k[j][ks].v, q[ks].v, c[j], 0, 0, 0);
                            else c[j] = __builtin_amdgcn_mfma_f32_16x16x4f32(k[j][ks].f[e], q[ks].f[e], c[j], 0, 0, 0);
                        }
                    }
                }
                float by = scale, less = m;
                if (__any(fabsf(m) >= kLargeLogit)) {   // rounded before the maximum is subtracted; the fma below then has nothing left to do
                    by = 1.f;
                    less = 0.f;
#pragma unroll
                    for (int j = 0; j < KG; ++j)
#pragma unroll
                        for (int e = 0; e < 4; ++e) c[j][e] = attn_logit(c[j][e], scale) - m;
                }
                if (!whole) {
                    const int row = base + qt * 16 + n16, p = row < row_hi ? first + token_of(row) : -1;
                    const int from = W.window == 0x7fffffff ? -1 : p - W.window;
#pragma unroll
                    for (int j = 0; j < KG; ++j)
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            const int key = kw + j * 16 + quad * 4 + e;
                            const bool seen = (key <= p) & ((key > from) | (key < W.sink));
                            c[j][e] = seen ? fmaf(c[j][e], by, -less) : -INFINITY;
                        }
                    by = 1.f;
                    less = 0.f;
                }
#pragma unroll
                for (int j = 0; j < KG; ++j)
#pragma unroll
                    for (int e = 0; e < 4; ++e) a[j][e] = fmaf(__builtin_amdgcn_exp2f(fmaf(c[j][e], by, -less)), il, a[j][e]);
#pragma unroll
                for (int j = 0; j < KG; ++j) asm volatile("" : "+v"(a[j]));   // here, not behind the tile's last branch
            }
            }
            stage(buf ^ 1);
            arrived();
            __syncthreads();
            if (i + 2 < i1) send(buf);
        }
        __syncthreads();   // the LDS is the next keys'
        // the 16 rows of a key, then one lane a key
        const size_t row = (size_t)b * W.n_kv + h;
#pragma unroll
        for (int j = 0; j < KG; ++j) {
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const float s = group_sum<16>(a[j][e]);
                const int key = kw + j * 16 + quad * 4 + e;
                if (n16 != e || key >= n) continue;
                const float w = there[j] ? s : 0.f;
                if (P.splits > 1) {
                    if (key < P.part_len) P.part[((size_t)split * W.batch * W.n_kv + row) * P.part_len + key] = w;
                } else {
                    float* x = P.acc + row * ((size_t)W.max_pages << W.page_shift) + key;
                    *x = (key >= first ? 0.f : *x) + w;
                }
            }
        }
    }
}

// partial sums of the splits, in their order
__global__ __launch_bounds__(256) void weights_sum_kernel(const WeightsParams P) {
    const PagedParams& W = P.view;
    const int row = blockIdx.y, b = row / W.n_kv, key = blockIdx.x * 256 + threadIdx.x;
    const int begin = chunk_begin(W, b), nq = chunk_end(W, b, begin) - begin, n = pairs_of(W, b), first = n - nq;
    if (nq == 0 || key >= n) return;
    const int k0 = key / P.keys * P.keys;
    if (nobody_sees(W, k0, min(k0 + P.keys, n), first)) return;
    const size_t stride = (size_t)W.batch * W.n_kv * P.part_len;
    const float* part = P.part + (size_t)row * P.part_len + key;
    float s = 0.f;
    for (int i = 0; i < P.splits; i += 8) {   // (eight loads in flight)
        float y[8];
#pragma unroll
        for (int u = 0; u < 8; ++u) y[u] = part[min(i + u, P.splits - 1) * stride];
#pragma unroll
        for (int u = 0; u < 8; ++u) s += i + u < P.splits ? y[u] : 0.f;
    }
    float* x = P.acc + (size_t)row * ((size_t)W.max_pages << W.page_shift) + key;
    *x = (key >= first ? 0.f : *x) + s;
}

// ---- host side ---------------------------------------------------------------------------------------------------
// Splits of the queries, whose partial sums a second launch puts together: so many that 2048 workgroups (fp32, where one has the matrix units of its CU
// busy, 512) even out what the chunk's own keys and the last turn leave idle, each with 8 tiles of queries and more.  Where that is below 512 workgroups -
// few keys, or few queries - a wavefront takes 16 keys instead of 64, each tile then costs less, and 1024 workgroups with four tiles and more are enough.
// us, by splits; 8 heads of g 4, D 128:  2048 tokens of 16384 1: 312, 2: 293, 4: 293, 8: 306;  of 20000 459, 361, 362, 377;  1024 of 9000 149, 125, 107, 109;  4096 of
// 4096 416, 223, 156, 134, 16: 136;  512 of 32768 180, 180, 197;  128 of 8192 30, 26, 32, with 16 keys a wavefront 24, 27, 33;  2048 of 2048 220, 124,
// 76, 55, with 16 keys 148, 85, 65;  two of 150 to 300 of to 4000, 2 heads, D 64: 37, 27, 19, 16, with 16 keys 20, 16, 13;  fp32, 4 heads: 1000 of 4000, D 64: 332, 175,
// 100, 88, 16: 98, with 16 keys 141, 107, 96;  64 of 10000 33, 33, 34, with 16 keys 25, 25, 28.
// Partial sums are kept up to the table's length, so that a length hint below a sequence's length loses nothing.  Under a window the pairs that count are
// those that the chunk sees (4 chunks to 1000 of 12000, 4 heads of g 7, window 4096: 150, by the whole length 186; 4 to 72 of 6000, fp32, window 24: 18 and 25).  The
// workspace, which knows no window, holds four splits where they are 64 MiB at most.
struct WeightsPlan {
    bool few;
    int keys, splits;
};
template <typename T, int D> static WeightsPlan weights_plan_of(const fk_paged_desc* d, int n_tokens, int max_chunk, long long pairs) {
    const long long rows = (long long)d->batch * d->n_kv_heads;
    auto blocks = [&](int keys) { return rows * ((pairs + keys - 1) / keys); };
    const long long queries = (long long)(max_chunk < n_tokens ? max_chunk : n_tokens) * (d->n_q_heads / d->n_kv_heads);
    const long long tiles = (queries + WeightsCfg<T, D, false>::QT - 1) / WeightsCfg<T, D, false>::QT;
    const long long space = (1ll << 26) / (rows * d->max_pages * d->page_size);   // a quarter of a GiB of partial sums
    const int most = WeightsCfg<T, D, false>::BF ? 2048 : 512;
    auto splits = [&](int keys, int workgroups, int least) {
        const long long s = std::min({workgroups / blocks(keys), tiles / least, space, 16ll});
        return s < 1 || rows > 65535 ? 1 : (int)s;
    };
    WeightsPlan p = {false, WeightsCfg<T, D, false>::KEYS, splits(WeightsCfg<T, D, false>::KEYS, most, 8)};
    if (blocks(p.keys) * p.splits < 512) p = {true, WeightsCfg<T, D, true>::KEYS, splits(WeightsCfg<T, D, true>::KEYS, 1024, 4)};
    return p;
}
static WeightsPlan weights_plan(const fk_paged_desc* d, int n_tokens, int max_chunk, long long pairs) {
    if (d->dtype == FK_F32) return d->head_dim == 64 ? weights_plan_of<float, 64>(d, n_tokens, max_chunk, pairs) : weights_plan_of<float, 128>(d, n_tokens, max_chunk, pairs);
    return d->head_dim == 64 ? weights_plan_of<bf16_t, 64>(d, n_tokens, max_chunk, pairs) : weights_plan_of<bf16_t, 128>(d, n_tokens, max_chunk, pairs);
}

static size_t part_bytes(const fk_paged_desc* d) { return (size_t)d->batch * d->n_kv_heads * d->max_pages * d->page_size * sizeof(float); }
// splits that the workspace holds
static int weights_space(const fk_paged_desc* d, int n_tokens, int max_chunk, int max_len) {
    const int s = weights_plan(d, n_tokens, max_chunk, max_len).splits;
    return s < 4 && 4 * part_bytes(d) <= ((size_t)64 << 20) ? 4 : s;
}
size_t weights_workspace(const fk_paged_desc* d, int n_tokens, int max_chunk, int max_len) {
    const int s = weights_space(d, n_tokens, max_chunk, max_len);
    return s > 1 ? s * part_bytes(d) : 0;
}

template <typename T, int D>
static fk_status weights_run(const fk_paged_desc* d, WeightsParams& P, const WeightsPlan& p, int max_len, hipStream_t st) {
    P.splits = p.splits;
    P.keys = p.keys;
    P.blocks = (int)std::min((max_len + p.keys - 1ll) / p.keys, std::max(1ll, (1ll << 23) / ((long long)d->batch * d->n_kv_heads)));   // (a workgroup goes on behind them)
    P.blocks_magic = magic_of(P.blocks);
    const dim3 grid((unsigned)(d->batch * d->n_kv_heads * (long long)P.blocks), P.splits);
    if (p.few) hipLaunchKernelGGL((weights_kernel<T, D, true>), grid, dim3(256), (2 * WeightsCfg<T, D, true>::TILE_BYTES), st, P);
    else hipLaunchKernelGGL((weights_kernel<T, D, false>), grid, dim3(256), (2 * WeightsCfg<T, D, false>::TILE_BYTES), st, P);
    if (P.splits > 1) hipLaunchKernelGGL(weights_sum_kernel, dim3((P.part_len + 255) / 256, d->batch * d->n_kv_heads), dim3(256), 0, st, P);
    return launch_status();
}

fk_status weights_launch(const fk_paged_desc* d, WeightsParams P, int max_chunk, int max_len, void* ws, hipStream_t st) {
    const long long seen = (long long)P.view.window + P.view.sink + max_chunk;
    WeightsPlan p = weights_plan(d, P.view.n_tokens, max_chunk, std::min<long long>(max_len, seen));
    p.splits = std::min(p.splits, weights_space(d, P.view.n_tokens, max_chunk, max_len));
    P.part = static_cast<float*>(ws);
    P.part_len = d->max_pages * d->page_size;
    if (d->dtype == FK_F32) return d->head_dim == 64 ? weights_run<float, 64>(d, P, p, max_len, st) : weights_run<float, 128>(d, P, p, max_len, st);
    return d->head_dim == 64 ? weights_run<bf16_t, 64>(d, P, p, max_len, st) : weights_run<bf16_t, 128>(d, P, p, max_len, st);
}

}  // namespace fk
