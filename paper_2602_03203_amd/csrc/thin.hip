// fk_paged_attn: its launch for chunks of few query rows, and fk_decode_step_acc
#include "thin.h"

#include <algorithm>

namespace fk {

template <typename T, int D, bool ROWS, int WAVES, bool NT_LOADS>
__global__ __launch_bounds__(WAVES * kWave, WAVES == 4 ? 3 : WAVES / 4) void thin_kernel(const AttnPagedParams P) {
    thin_tile<T, D, ROWS, WAVES, NT_LOADS>(P, blockIdx.x, blockIdx.y);
}

template <typename T, int D>
__global__ __launch_bounds__(256) void thin_merge_kernel(const AttnPagedParams P) { merge_tile<T, D, 16, ThinCfg<T, D>::KT>(P, blockIdx.x, 0); }

// ---- host side ---------------------------------------------------------------------------------------------------
// Splits of a tile's pairs, by the tiles of the launch and by the pairs that one may see.  us, splits at most and pairs of one at least:
//   few tiles    8 of 32768 pairs 4 splits 78, 8 45, 16 31, 32 35;  32 of 4000 4 18.8, 8 18.3, 16 20.9;  8 of 1000 unsplit 14.5, 3 10.5;  64 of 3000
//                (D = 64) unsplit 21.8, 2 17.1, 4 16.0, 8 16.9: up to 256 workgroups, up to sixteen splits
//   128 and more, which fill the memory system by themselves, unsplit where they are short (128 of 2048 24.7, 2 27.1).  Long ones differ in length as a rule,
//                and only the device knows: splits of 1024 pairs and more even them out (512 of 1024 to 32768 pairs unsplit 947, so 840; 128 of 1024 to
//                8192 118 and 69) and cost equal ones little (512 of 4096 163 and 170, 128 of 8192 in two 86, so 89).  Chunks of several tiles beside
//                single tokens leave places empty: splits of 512 pairs (19 sequences, 3 with 8 to 15 tokens, g 2, 2315 to 3761 pairs: unsplit 69, so 53)
struct ThinPlan {
    int splits, shift;
};
static ThinPlan thin_plan(const fk_paged_desc* d, const TileGrid& G, long long pairs) {
    const long long items = (long long)G.places * d->n_kv_heads;
    const int kt_shift = d->dtype == FK_BF16 ? 5 : 4;
    const bool uneven = G.spread || G.per_seq > 1;
    ThinPlan p = {1, (items < 128 ? 8 : pairs >= 6144 ? 10 : 9) - kt_shift};
    long long s = 1;
    if (items < 128) s = 256 / items;
    else if (pairs >= 6144 || uneven) s = 16;
    if (s > 16) s = 16;
    if (s > (1 << 16) / items) s = (1 << 16) / items;   // (half a GiB of records; so many items even out by themselves)
    if (s > pairs >> (p.shift + kt_shift)) s = pairs >> (p.shift + kt_shift);
    if (s > 1) p.splits = (int)s;
    return p;
}
// the pairs that a query of the call may see
static long long most_pairs(const PagedParams& P, int max_len) {
    return P.window == 0x7fffffff || (long long)P.window + P.sink > max_len ? max_len : (long long)P.window + P.sink;
}

size_t thin_paged_workspace(const fk_paged_desc* d, const TileGrid& G, int max_len) {
    return record_bytes((long long)G.places * d->n_kv_heads, thin_plan(d, G, max_len).splits, 16, d->head_dim);
}

template <typename T, int D, bool ROWS, int WAVES, bool NT_LOADS>
static fk_status thin_start(const AttnPagedParams& P, dim3 grid, hipStream_t st) {
    auto kern = thin_kernel<T, D, ROWS, WAVES, NT_LOADS>;
    constexpr size_t most = ThinCfg<T, D>::lds(ROWS, WAVES, ROWS ? ThinCfg<T, D>::LOGITS : 0);
    const size_t lds = ThinCfg<T, D>::lds(ROWS, WAVES, P.logits_lds * P.view.g);
    static bool lds_ok[kMaxDevices] = {};
    if (most > 48 * 1024 && !allow_dynamic_lds((const void*)kern, most, lds_ok)) return FK_ERR_LAUNCH;
    hipLaunchKernelGGL(kern, grid, dim3(WAVES * kWave), lds, st, P);
    return launch_status();
}

template <typename T, int D>
static fk_status thin_paged_launch(const fk_paged_desc* d, AttnPagedParams& P, bool cold, hipStream_t st) {
    const dim3 grid(P.grid.places * d->n_kv_heads, P.splits);
    const fk_status s = cold ? thin_start<T, D, false, 4, true>(P, grid, st) : thin_start<T, D, false, 4, false>(P, grid, st);
    if (s != FK_OK) return s;
    if (P.splits > 1) hipLaunchKernelGGL((thin_merge_kernel<T, D>), dim3(grid.x), dim3(256), 0, st, P);
    return launch_status();
}

void thin_prepare(const fk_paged_desc* d, AttnPagedParams& P, int max_len, void* ws, bool& cold) {
    const long long items = (long long)P.grid.places * d->n_kv_heads;
    const ThinPlan p = thin_plan(d, P.grid, most_pairs(P.view, max_len));
    P.splits = std::min(p.splits, thin_plan(d, P.grid, max_len).splits);   // (what the workspace is for)
    P.split_shift = p.shift;
    P.rec_ml = reinterpret_cast<float2*>(ws);
    P.rec = reinterpret_cast<float*>(static_cast<char*>(ws) + up256((size_t)items * P.splits * 16 * sizeof(float2)));
    cold = (size_t)d->batch * d->n_kv_heads * max_len * d->head_dim * (d->dtype == FK_F32 ? 8 : 4) >= ((size_t)352 << 20);
}

fk_status thin_paged(const fk_paged_desc* d, AttnPagedParams P, int max_len, void* ws, hipStream_t st) {
    bool cold;
    thin_prepare(d, P, max_len, ws, cold);
    if (d->dtype == FK_F32) return d->head_dim == 64 ? thin_paged_launch<float, 64>(d, P, cold, st) : thin_paged_launch<float, 128>(d, P, cold, st);
    return d->head_dim == 64 ? thin_paged_launch<bf16_t, 64>(d, P, cold, st) : thin_paged_launch<bf16_t, 128>(d, P, cold, st);
}

// workspace of the accumulating step: info [rows] | logits [rows][g][cap rounded up] | records
struct RowsPlan {
    int waves, splits, shift;
};
// Short rows, and as many rows as CUs, take a workgroup of eight wavefronts each, which adds the weights itself; others are split over 256 workgroups of
// four, each with a tile for every wavefront or more, and the second launch, 3 us, adds them.  us a step, a row to a workgroup and split:
//   bf16 D = 128, g = 4   8 rows of 300 8.0 and 8.9, of 1000 14.6 and 8.3; 32 of 500 9.9 and 8.3; 128 of 300 8.2 and 9.3, of 1000 16.9 and 16.8, of 2112
//                         28 and 28; 256 of 600 16.4 and 21; D = 64 (in a graph, where a step takes 1 us more)  8 of 300 8.4 and 9.4, 32 of 500 9.2 and 9.6, 128
//                         of 300 8.6 and 9.8, of 1000 13.4 and 13.4, of 2112 21.6 and 20.4
//   fp32 D = 64           2 of 144 6.4 and 7.5, 8 of 300 8.2 and 7.9, 128 of 300 8.7 and 9.2, of 1000 20 and 18;  D = 128  2 of 144 9.0 and 9.2, 8 of 300
//                         12.8 and 9.8, 128 of 300 14.1 and 14.3, of 1000 34 and 27
// Between 128 rows and 256, us of eight wavefronts and of three splits: 152 of 2112 bf16 D = 128 29.6 and 30.7, D = 64 21.8 and 21.9, fp32 D = 64 36 and 31, 128 70
// and 70; of 1000 fp32 D = 64 20.2 and 20.0, 128 34 and 31; 200 of 2112 bf16 36 and 41, 24 and 28, fp32 37 and 44, 82 and 92.
// Splits: 8 rows of 4000 pairs, bf16, 8: 11.2, 16: 10.0, 32: 11.6; 32 of 2000 4: 13.4, 8: 11.8, 16: 14.1.  From 512 rows on, and fp32 with D = 128, four
// wavefronts a row: 512 rows of 1000 43.5, eight 44.4 (fp32 87 and 92; bf16 D = 64, since a probability is three terms there, 26.6 and 25.4, 1024 of 150 12.5 and 16.5).
static RowsPlan rows_plan(const fk_cache_desc* d, int max_len) {
    const int rows = d->batch * d->n_kv_heads;
    const bool bf16 = d->dtype == FK_BF16;
    RowsPlan p = {8, 1, 2};
    const int alone = bf16 ? (rows < 128 ? 384 : 1024) : d->head_dim == 64 ? (rows < 128 ? 224 : 512) : rows < 128 ? 160 : 256;
    if (rows >= 256) {
        if (rows >= 512 || (!bf16 && d->head_dim == 128)) p.waves = 4;
        return p;
    }
    if (max_len <= alone || (rows > 128 && (bf16 || rows > 160 || max_len <= 1024))) return p;
    p.waves = 4;
    p.splits = max_len / ((bf16 ? 32 : 16) << p.shift);
    const int most = rows > 128 ? 3 : 256 / rows;
    if (p.splits > most) p.splits = most;
    if (p.splits > kMostSplits) p.splits = kMostSplits;
    if (p.splits < 1) p.splits = 1;
    return p;
}
static int logit_stride(const fk_cache_desc* d) { return (d->capacity + 3) / 4 * 4; }
static size_t rows_logit_bytes(const fk_cache_desc* d) { return up256((size_t)d->batch * d->n_q_heads * logit_stride(d) * sizeof(float)); }

size_t thin_rows_workspace(const fk_cache_desc* d) {
    const size_t rows = (size_t)d->batch * d->n_kv_heads;
    return up256(rows * sizeof(int2)) + rows_logit_bytes(d) + record_bytes(rows, rows_plan(d, d->capacity).splits, 16, d->head_dim);   // (longer rows have no fewer splits)
}

template <typename T, int D>
static fk_status thin_rows_launch(AttnPagedParams& P, const RowsPlan& p, int max_len, bool cold, hipStream_t st) {
    const dim3 grid(P.view.batch, P.splits);
    fk_status s;
    if (p.waves == 4) s = cold ? thin_start<T, D, true, 4, true>(P, grid, st) : thin_start<T, D, true, 4, false>(P, grid, st);
    else s = cold ? thin_start<T, D, true, 8, true>(P, grid, st) : thin_start<T, D, true, 8, false>(P, grid, st);
    if (s != FK_OK) return s;
    if (P.splits > 1) {
        const int parts = max_len < 4096 * 256 ? (max_len + 255) / 256 : 4096;
        hipLaunchKernelGGL((merge_rows_kernel<T, D, ThinCfg<T, D>::KT>), dim3(grid.x, parts + 1), dim3(256), 0, st, P);
    }
    return launch_status();
}

fk_status thin_rows(const fk_cache_desc* d, AttnPagedParams P, int max_len, void* ws, hipStream_t st) {
    const size_t rows = (size_t)d->batch * d->n_kv_heads;
    const RowsPlan p = rows_plan(d, max_len);
    P.splits = p.splits;
    P.split_shift = p.shift;
    const int whole = (max_len + 31) / 32 * 32;
    P.logits_lds = p.splits == 1 && (long long)whole * P.view.g <= ThinCfg<float, 64>::LOGITS ? whole : 0;
    char* at = static_cast<char*>(ws);
    P.info = reinterpret_cast<int2*>(at);
    at += up256(rows * sizeof(int2));
    P.logit = reinterpret_cast<float*>(at);
    P.logit_stride = logit_stride(d);
    at += rows_logit_bytes(d);
    P.rec_ml = reinterpret_cast<float2*>(at);
    P.rec = reinterpret_cast<float*>(at + up256(rows * P.splits * 16 * sizeof(float2)));
    const bool cold = (d->flags & FK_CACHE_COLD) || rows * max_len * d->head_dim * (d->dtype == FK_F32 ? 8 : 4) >= ((size_t)352 << 20);
    if (d->dtype == FK_F32) return d->head_dim == 64 ? thin_rows_launch<float, 64>(P, p, max_len, cold, st) : thin_rows_launch<float, 128>(P, p, max_len, cold, st);
    return d->head_dim == 64 ? thin_rows_launch<bf16_t, 64>(P, p, max_len, cold, st) : thin_rows_launch<bf16_t, 128>(P, p, max_len, cold, st);
}

}  // namespace fk
