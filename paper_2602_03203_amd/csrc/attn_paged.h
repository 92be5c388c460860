// Attention over pages and rows: what its kernels share - few query rows over many pairs (thin.h: single tokens and short chunks over a paged cache,
// the decode step that accumulates its weights over the rows of a budgeted cache) and many query rows (prompt.h) - and the merge of split tiles.
#pragma once
#include "paged.h"
#include "window.h"

namespace fk {

typedef __attribute__((ext_vector_type(8))) __bf16 tbf16x8_t;
typedef __attribute__((ext_vector_type(4))) float tf32x4_t;
typedef __attribute__((ext_vector_type(4))) uint32_t tu32x4_t;
typedef __attribute__((ext_vector_type(2))) uint32_t tu32x2_t;
union T128 {
    tu32x4_t u;
    uint32_t w[4];
    float f[4];
    tbf16x8_t v;
};

__device__ __forceinline__ float quad_max(float v) {   // over the four lanes of a row (lane % 16)
    auto a = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    v = fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1]));
    auto b = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return fmaxf(__uint_as_float(b[0]), __uint_as_float(b[1]));
}
__device__ __forceinline__ float quad_sum(float v) {
    auto a = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    v = __uint_as_float(a[0]) + __uint_as_float(a[1]);
    auto b = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return __uint_as_float(b[0]) + __uint_as_float(b[1]);
}

// 0 where nothing has been seen: what an exponent is taken against
__device__ __forceinline__ float ref_of(float m) { return m == -INFINITY ? 0.f : m; }

template <typename T> __device__ __forceinline__ bool word_not_finite(uint32_t w) {
    if constexpr (sizeof(T) == 2) return ((w & 0x7f80u) == 0x7f80u) | ((w & 0x7f800000u) == 0x7f800000u);   // (no branch)
    else return (w & 0x7f800000u) == 0x7f800000u;
}

static constexpr int kMostSplits = 64;   // of a tile's pairs

struct AttnPagedParams {
    PagedParams view;          // rows of a budgeted cache: q, K, V, batch = rows, n_kv = 1, g, scale alone
    void* out;
    float2* stats;             // [tokens][heads] or null
    TileGrid grid;
    int whole;                 // items (slot, head) before this one are not split
    int splits;                // of a tile's pairs, at most
    int split_shift;           // key tiles of a split, at least 2^split_shift
    float* rec;                // [item - whole][split][rows of a tile][D], with more than one split
    float2* rec_ml;            // [item - whole][split][rows of a tile]; rows of a cache: eight heads, then the same with the outputs' normaliser
    // rows of a budgeted cache
    int cap;
    int32_t *pos, *len;
    const int32_t* pos_new;
    const void *k_new, *v_new;
    int batch_of_pos;          // KV heads: row r belongs to sequence r / batch_of_pos
    float* acc;                // [rows][cap]
    float* logit;              // [rows][g][logit_stride] scratch
    int logits_lds;            // unsplit rows of up to so many pairs (whole tiles) keep them in LDS
    int logit_stride;          // cap, rounded up to whole 16-byte groups
    int2* info;                // [rows] (pairs, the new pair's slot or -1): for the second launch
};

// Splits of a tile of `total` key tiles: as many as leave 2^shift to each
__host__ __device__ inline int splits_of(int total, int splits, int shift) {
    const int s = total >> shift;
    return s < 1 ? 1 : s < splits ? s : splits;
}

// ---------------------------------------------------------------------------------------------------------
// The second launch, where tiles may have been split: out = sum_s o_s 2^(m_s - M) / sum_s l_s 2^(m_s - M), eight records' loads in flight.
// ---------------------------------------------------------------------------------------------------------
template <int D> struct Merged {
    float M, L, a[4];
};
template <int D>
__device__ __forceinline__ Merged<D> merge_records(const AttnPagedParams& P, size_t rec /* the row in the first split's record */, int tm, int splits, int d,
                                                   int ml_row = 0 /* rows from there to its (M, L) */) {
    Merged<D> o = {-INFINITY, 0.f, {0.f, 0.f, 0.f, 0.f}};
    for (int s0 = 0; s0 < splits; s0 += 8) {
        float2 ml[8];
        float4 v[8];
#pragma unroll
        for (int u = 0; u < 8; ++u) {
            const size_t r = rec + (size_t)min(s0 + u, splits - 1) * tm;
            ml[u] = P.rec_ml[r + ml_row];
            v[u] = *reinterpret_cast<const float4*>(P.rec + r * D + d);
        }
        float m = o.M;
#pragma unroll
        for (int u = 0; u < 8; ++u) m = fmaxf(m, ml[u].x);   // (the copies past the end change nothing)
        const float ref = ref_of(m), c0 = __builtin_amdgcn_exp2f(o.M - ref);
        o.M = m;
        o.L *= c0;
#pragma unroll
        for (int i = 0; i < 4; ++i) o.a[i] *= c0;
#pragma unroll
        for (int u = 0; u < 8; ++u) {
            if (s0 + u >= splits) break;
            const float f = __builtin_amdgcn_exp2f(ml[u].x - ref);
            o.L = fmaf(ml[u].y, f, o.L);
            o.a[0] = fmaf(v[u].x, f, o.a[0]);
            o.a[1] = fmaf(v[u].y, f, o.a[1]);
            o.a[2] = fmaf(v[u].z, f, o.a[2]);
            o.a[3] = fmaf(v[u].w, f, o.a[3]);
        }
    }
    return o;
}

// four channels of a row from the sum of its weighted values and of its weights; 0 where nothing has been seen (a row of a budgeted cache has its new
// pair at least: where all its logits are -inf it is 0 / 0, as in the step without accumulation, and as its weights are)
template <typename T, int D, bool ROWS>
__device__ __forceinline__ void store_row(const AttnPagedParams& P, size_t row, int d, const float (&a)[4], float M, float L) {
    const float inv = !ROWS && L == 0.f ? 0.f : 1.0f / L;
    if constexpr (sizeof(T) == 2) {
        const tu32x2_t y = {pack_bf16(a[0] * inv, a[1] * inv), pack_bf16(a[2] * inv, a[3] * inv)};
        *reinterpret_cast<tu32x2_t*>(reinterpret_cast<bf16_t*>(P.out) + row * D + d) = y;
    } else {
        *reinterpret_cast<float4*>(reinterpret_cast<float*>(P.out) + row * D + d) = make_float4(a[0] * inv, a[1] * inv, a[2] * inv, a[3] * inv);
    }
    if (P.stats && d == 0) P.stats[row] = make_float2(M, L);
}

template <typename T, int D, int TM, int KT>
__device__ __forceinline__ void merge_tile(const AttnPagedParams& P, int item, int part) {   // part: 16 of a tile's rows
    const PagedParams& W = P.view;
    const int tid = threadIdx.x, n_kv = W.n_kv, slot = scalar(divide(item, n_kv, W.kv_magic)), h = item - slot * n_kv, g = W.g, sub = part * 16;
    TileOf t;
    if (!tile_of(W, P.grid, slot, TM, t) || !t.one) return;   // (places that take several tiles do not split them)
    const int tile_rows = min(TM, t.nq * g - t.tile * TM), rows = min(16, tile_rows - sub), r0 = t.tile * TM + sub;
    const int lo = t.first + divide(t.tile * TM, g, W.g_magic), hi = t.first + divide(t.tile * TM + tile_rows - 1, g, W.g_magic);
    const int splits = splits_of(key_tiles(W, lo, hi, KT).total, P.splits, P.split_shift);
    if (rows <= 0 || splits == 1) return;
    const size_t rec = (size_t)(item - P.whole) * P.splits * TM + sub;
    for (int x = tid; x < rows * (D / 4); x += 256) {
        const int r = x / (D / 4), d = x % (D / 4) * 4;
        const Merged<D> o = merge_records<D>(P, rec + r, TM, splits, d);
        const int tok = divide(r0 + r, g, W.g_magic);
        store_row<T, D, false>(P, ((size_t)(t.begin + tok) * n_kv + h) * g + (r0 + r - tok * g), d, o.a, o.M, o.L);
    }
}

// Rows of a budgeted cache: the last workgroup of a row merges its outputs - threads beyond a row's channels take a share of its splits - and sets its
// length, the others add its pairs' weights, a pair per thread, whose logits are on their way while the splits' maxima and sums are put together, 32 lanes
// a head.
template <typename T, int D, int KT>
__global__ __launch_bounds__(256) void merge_rows_kernel(const AttnPagedParams P) {
    const int tid = threadIdx.x, slot = blockIdx.x, g = P.view.g;
    __shared__ float s_M[8], s_inv[8];
    const int n = load_uniform(&P.info[slot].x, 0), fresh = load_uniform(&P.info[slot].y, 0);
    const int splits = splits_of(key_tiles(P.view, n - 1, n - 1, KT).total, P.splits, P.split_shift);
    const size_t rec = (size_t)slot * P.splits * 16;
    if (blockIdx.y == gridDim.y - 1) {
        __shared__ Merged<D> s_part[256];
        if (tid == 0 && fresh >= 0) P.len[slot] = n;
        if (splits == 1) return;
        const int units = g * (D / 4), shares = 256 / units, share = tid / units, unit = tid - share * units;
        const int per = (splits + shares - 1) / shares, s0 = min(share * per, splits), count = min(per, splits - s0);
        const int r = unit / (D / 4), d = unit % (D / 4) * 4;
        Merged<D> o = {-INFINITY, 0.f, {0.f, 0.f, 0.f, 0.f}};
        if (share < shares && count > 0) o = merge_records<D>(P, rec + (size_t)s0 * 16 + r, 16, count, d, 8);
        if (share > 0) s_part[tid] = o;
        __syncthreads();
        if (share > 0) return;
        for (int i = 1; i < shares; ++i) {
            const Merged<D> x = s_part[tid + i * units];
            const float m = fmaxf(o.M, x.M), ref = ref_of(m), fo = __builtin_amdgcn_exp2f(o.M - ref), fx = __builtin_amdgcn_exp2f(x.M - ref);
            o.M = m;
            o.L = o.L * fo + x.L * fx;
#pragma unroll
            for (int k = 0; k < 4; ++k) o.a[k] = o.a[k] * fo + x.a[k] * fx;
        }
        store_row<T, D, true>(P, (size_t)slot * g + r, d, o.a, o.M, o.L);
        return;
    }
    if (splits == 1) return;   // all done
    float* acc = P.acc + (size_t)slot * P.cap;
    const float* lg = P.logit + (size_t)slot * g * P.logit_stride;
    int key = blockIdx.y * 256 + tid;
    float x[8], before = 0.f;
    auto fetch = [&]() {
        const int kc = min(key, n - 1);
        before = acc[kc];
#pragma unroll
        for (int k = 0; k < 8; ++k) x[k] = lg[(size_t)min(k, g - 1) * P.logit_stride + kc];
    };
    fetch();
    {
        const int head = tid / 32, s = tid % 32;
        float2 ml[kMostSplits / 32];
        float M = -INFINITY, L = 0.f;
#pragma unroll
        for (int u = 0; u < kMostSplits / 32; ++u) {
            ml[u] = P.rec_ml[rec + (size_t)min(s + u * 32, splits - 1) * 16 + head];
            M = fmaxf(M, ml[u].x);
        }
#pragma unroll
        for (int off = 16; off > 0; off >>= 1) M = fmaxf(M, __shfl_xor(M, off));
        M = ref_of(M);
#pragma unroll
        for (int u = 0; u < kMostSplits / 32; ++u)
            if (s + u * 32 < splits) L = fmaf(ml[u].y, __builtin_amdgcn_exp2f(ml[u].x - M), L);
#pragma unroll
        for (int off = 16; off > 0; off >>= 1) L += __shfl_xor(L, off);
        if (s == 0 && head < g) {
            s_M[head] = M;
            s_inv[head] = 1.0f / L;
        }
    }
    __syncthreads();
    while (key < n) {
        float w = 0.f;
#pragma unroll
        for (int k = 0; k < 8; ++k)
            if (k < g) w = fmaf(__builtin_amdgcn_exp2f(x[k] - s_M[k]), s_inv[k], w);
        acc[key] = (key == fresh ? 0.f : before) + w;
        key += (gridDim.y - 1) * 256;
        if (key < n) fetch();
    }
}

// ---- host side ---------------------------------------------------------------------------------------------------
inline size_t up256(size_t n) { return (n + 255) / 256 * 256; }

inline size_t record_bytes(long long items, int splits, int tm, int D) {
    return splits > 1 ? up256((size_t)items * splits * tm * sizeof(float2)) + (size_t)items * splits * tm * D * sizeof(float) : 0;
}

size_t thin_paged_workspace(const fk_paged_desc* d, const TileGrid& G, int max_len);
void thin_prepare(const fk_paged_desc* d, AttnPagedParams& P, int max_len, void* workspace, bool& cold);   // splits and records
fk_status thin_paged(const fk_paged_desc* d, AttnPagedParams P, int max_len, void* workspace, hipStream_t st);
fk_status thin_rows(const fk_cache_desc* d, AttnPagedParams P, int max_len, void* workspace, hipStream_t st);
size_t thin_rows_workspace(const fk_cache_desc* d);

static constexpr int kPromptRows = 128;   // query rows of a tile of prompt.h
size_t prompt_workspace(const fk_paged_desc* d, const TileGrid& G, int n_tokens, int max_chunk, int max_len);
// thin: the call's chunks of few rows, prepared, or null
fk_status prompt_paged(const fk_paged_desc* d, AttnPagedParams P, const AttnPagedParams* thin, bool cold, int max_chunk, int max_len, void* workspace, hipStream_t st);

}  // namespace fk
