// Attention over pages and rows: what its kernels share - few query rows over many pairs (thin.hip: single tokens and short chunks over a paged cache,
// the decode step that accumulates its weights over the rows of a budgeted cache) and many query rows (prompt.hip) - and the merge of split tiles.
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
    int splits;                // of a tile's pairs, at most
    int split_tiles;           // key tiles of a split, at least
    float* rec;                // [slot][head][split][16][D], with more than one split
    float2* rec_ml;            // [slot][head][split][16]
    // rows of a budgeted cache
    int cap;
    int32_t *pos, *len;
    const int32_t* pos_new;
    const void *k_new, *v_new;
    int batch_of_pos;          // KV heads: row r belongs to sequence r / batch_of_pos
    float* acc;                // [rows][cap]
    float* logit;              // [rows][g][cap] scratch
    int2* info;                // [rows] (pairs, the new pair's slot or -1): for the second launch
};

// Splits of a tile of `total` key tiles: as many as leave `least` to each
__host__ __device__ inline int splits_of(int total, int splits, int least) {
    const int s = total / least;
    return s < 1 ? 1 : s < splits ? s : splits;
}

// ---------------------------------------------------------------------------------------------------------
// The second launch, where tiles may have been split: out = sum_s o_s 2^(m_s - M) / sum_s l_s 2^(m_s - M).
// ROWS: also the weights of the row's pairs, a stretch of them per workgroup, and its length.
// ---------------------------------------------------------------------------------------------------------
template <typename T, int D, int TM, int KT, bool ROWS>
__global__ __launch_bounds__(256) void merge_kernel(const AttnPagedParams P) {
    const PagedParams& W = P.view;
    const int tid = threadIdx.x, n_kv = ROWS ? 1 : W.n_kv, slot = ROWS ? (int)blockIdx.x : scalar(blockIdx.x / n_kv), h = ROWS ? 0 : (int)blockIdx.x - slot * n_kv, g = W.g;
    const int sub = ROWS ? 0 : (int)blockIdx.y * 16;   // the workgroup's 16 rows of the tile
    __shared__ float s_w[16][kMostSplits], s_M[16], s_L[16];
    TileOf t;
    int fresh = -1;
    if constexpr (ROWS) {
        const int2 info = P.info[slot];
        fresh = info.y;
        if (blockIdx.y == 0 && tid == 0 && fresh >= 0) P.len[slot] = info.x;
        t = {slot, slot, 1, info.x, info.x - 1, 0, 1, true};
    } else {
        if (!tile_of(W, P.grid, slot, TM, t)) return;
    }
    for (; t.tile >= 0; t.tile -= t.step) {
        const int tile_rows = min(TM, t.nq * g - t.tile * TM), rows = min(16, tile_rows - sub), r0 = t.tile * TM + sub;
        if (rows <= 0) continue;
        const int lo = t.first + t.tile * TM / g, hi = t.first + (t.tile * TM + tile_rows - 1) / g;
        const int splits = splits_of(key_tiles(W, lo, hi, KT).total, t.one ? P.splits : 1, P.split_tiles);
        if (splits == 1) continue;
        const size_t rec = ((size_t)slot * n_kv + h) * P.splits * TM + sub;
        if (tid < rows) {
            float M = -INFINITY, L = 0.f;
            for (int s = 0; s < splits; ++s) M = fmaxf(M, P.rec_ml[rec + s * TM + tid].x);
            const float ref = ref_of(M);
            for (int s = 0; s < splits; ++s) {
                const float2 ml = P.rec_ml[rec + s * TM + tid];
                const float f = __builtin_amdgcn_exp2f(ml.x - ref);
                s_w[tid][s] = f;
                L = fmaf(ml.y, f, L);
            }
            s_M[tid] = M;
            s_L[tid] = L;
        }
        __syncthreads();
        if (!ROWS || blockIdx.y == 0) {
            for (int x = tid; x < rows * (D / 4); x += 256) {
                const int r = x / (D / 4), d = x % (D / 4) * 4;
                float a[4] = {0.f, 0.f, 0.f, 0.f};
                for (int s = 0; s < splits; ++s) {
                    const float4 v = *reinterpret_cast<const float4*>(P.rec + (rec + s * TM + r) * D + d);
                    const float f = s_w[r][s];
                    a[0] = fmaf(v.x, f, a[0]);
                    a[1] = fmaf(v.y, f, a[1]);
                    a[2] = fmaf(v.z, f, a[2]);
                    a[3] = fmaf(v.w, f, a[3]);
                }
                const float L = s_L[r];
                const size_t row = ((size_t)(t.begin + (r0 + r) / g) * n_kv + h) * g + (r0 + r) % g;
                if (L == 0.f) a[0] = a[1] = a[2] = a[3] = 0.f;
                const float inv = L == 0.f ? 1.f : L;
                if constexpr (sizeof(T) == 2) {
                    const tu32x2_t y = {pack_bf16(a[0] / inv, a[1] / inv), pack_bf16(a[2] / inv, a[3] / inv)};
                    *reinterpret_cast<tu32x2_t*>(reinterpret_cast<bf16_t*>(P.out) + row * D + d) = y;
                } else {
                    *reinterpret_cast<float4*>(reinterpret_cast<float*>(P.out) + row * D + d) = make_float4(a[0] / inv, a[1] / inv, a[2] / inv, a[3] / inv);
                }
                if (P.stats && d == 0) P.stats[row] = make_float2(s_M[r], L);
            }
        }
        if constexpr (ROWS) {
            float* acc = P.acc + (size_t)slot * P.cap;
            for (int key = blockIdx.y * 256 + tid; key < t.n; key += gridDim.y * 256) {
                float w = 0.f;
                for (int k = 0; k < g; ++k) w += __builtin_amdgcn_exp2f(P.logit[((size_t)slot * g + k) * P.cap + key] - ref_of(s_M[k])) / s_L[k];
                acc[key] = (key == fresh ? 0.f : acc[key]) + w;
            }
            return;
        }
        __syncthreads();
    }
}

// ---- host side ---------------------------------------------------------------------------------------------------
inline size_t up256(size_t n) { return (n + 255) / 256 * 256; }

inline size_t record_bytes(long long items, int splits, int tm, int D) {
    return splits > 1 ? up256((size_t)items * splits * tm * sizeof(float2)) + (size_t)items * splits * tm * D * sizeof(float) : 0;
}

size_t thin_paged_workspace(const fk_paged_desc* d, const TileGrid& G, int max_len);
fk_status thin_paged(const fk_paged_desc* d, AttnPagedParams P, int max_len, void* workspace, hipStream_t st);
fk_status thin_rows(const fk_cache_desc* d, AttnPagedParams P, int max_len, void* workspace, hipStream_t st);
size_t thin_rows_workspace(const fk_cache_desc* d);

static constexpr int kPromptRows = 128;   // query rows of a tile of prompt.hip
size_t prompt_workspace(const fk_paged_desc* d, const TileGrid& G, int max_len);
fk_status prompt_paged(const fk_paged_desc* d, AttnPagedParams P, int max_len, void* workspace, hipStream_t st);

}  // namespace fk
