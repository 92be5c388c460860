// fk_paged_attn: its launches with chunks of many query rows, alone or with chunks of few beside them
#include "prompt.h"
#include "thin.h"

#include <algorithm>

namespace fk {

template <typename T, int D>
__global__ __launch_bounds__(256, 2) void prompt_kernel(const AttnPagedParams P) { prompt_tile<T, D>(P, blockIdx.x, blockIdx.y); }

template <typename T, int D>
__global__ __launch_bounds__(256) void prompt_merge_kernel(const AttnPagedParams P) { merge_tile<T, D, kPromptRows, PromptCfg<T, D>::KT>(P, blockIdx.x, blockIdx.y); }

// Both kinds of chunks in one launch, the long tiles first: one kind's products run beside the other's loads.  A small model's batch of four prompt chunks
// and twenty single tokens, with the append before it: 53 us in two launches and two merges, 38 in one and one.
struct MixedParams {
    AttnPagedParams prompt, thin;
    int items, merge;         // of the prompt tiles; parts of them that the second launch has
    uint32_t items_magic;
};
template <typename T, int D, bool NT_LOADS>
__global__ __launch_bounds__(256, 2) void mixed_kernel(const MixedParams P) {
    const int many = P.items * P.prompt.splits, x = blockIdx.x;
    if (x < many) {
        const int split = scalar(divide(x, P.items, P.items_magic));
        prompt_tile<T, D>(P.prompt, x - split * P.items, split);
    } else {
        const int items = P.thin.grid.places * P.thin.view.n_kv, split = scalar(divide(x - many, items));
        thin_tile<T, D, false, 4, NT_LOADS>(P.thin, x - many - split * items, split);
    }
}
template <typename T, int D>
__global__ __launch_bounds__(256) void mixed_merge_kernel(const MixedParams P) {
    const int x = blockIdx.x;
    if (x < P.merge) merge_tile<T, D, kPromptRows, PromptCfg<T, D>::KT>(P.prompt, x / (kPromptRows / 16), x % (kPromptRows / 16));
    else merge_tile<T, D, 16, ThinCfg<T, D>::KT>(P.thin, x - P.merge, 0);
}

// ---- host side ---------------------------------------------------------------------------------------------------
// Over how many workgroups the pairs of an item (a tile of rows, a kv head) are split.  256 CUs hold two workgroups each: items beyond a multiple of
// 512 cost another turn, five sixths of one where there are at most 256 of them (a workgroup alone on its CU is a little faster).  Splits make turns
// shorter and cost a second launch and their records' way to memory and back.  In microseconds, with 2.1 for 64 pairs of bf16 and D = 128, 6 for the
// launch and 4 TB/s for the records; in fp32 one workgroup has the matrix units of its CU busy, 9.4 for 64 pairs.  Whole / 2 / 3 / 4 / 8 splits measured for 8 heads of g 4, D 128: 512 tokens of 8192: 216 / 123 /
// 104 / 93 / 101; 1024 of 8192: 222 / 160 / 175 / 166 / 186; 4 chunks to 300 of 2048: 70 / 80 / 72 / 73 / 70.  How many chunks there are that are not single
// tokens the host does not know: as many as would have the longest one's length.
static int prompt_splits(const fk_paged_desc* d, const TileGrid& G, int n_tokens, int max_chunk, long long pairs, int& shift) {
    shift = d->dtype == FK_BF16 ? 3 : 4;   // 512 pairs and more each
    const long long g = d->n_q_heads / d->n_kv_heads, chunk = max_chunk < n_tokens ? max_chunk : n_tokens, rest = n_tokens - d->batch;
    const long long chunks = chunk > 1 && rest > 0 ? (rest + chunk - 2) / (chunk - 1) : 1;
    const long long items = (n_tokens * g + chunks * (kPromptRows - 1)) / kPromptRows * d->n_kv_heads;
    const double whole = (double)pairs / 64 * d->head_dim / 128 * (d->dtype == FK_BF16 ? 2.1 : 9.4);
    int best = 1;
    double least = 0;
    for (int s = 1; s <= 16 && (s == 1 || (pairs / s >= 512 && (long long)G.places * d->n_kv_heads * s <= 4096 /* a quarter of a GiB of records */)); ++s) {
        const long long all = items * s, over = all % 512;
        const double turns = d->dtype == FK_F32 ? std::max(1., (double)all / 256) : (double)(all / 512) + (over == 0 ? 0. : over <= 256 ? 5. / 6 : 1.);
        const double time = turns * whole / s + (s == 1 ? 0. : 6 + (double)all * kPromptRows * d->head_dim * 8 / 4e6);
        if (s == 1 || time < least) least = time, best = s;
    }
    return best;
}
size_t prompt_workspace(const fk_paged_desc* d, const TileGrid& G, int n_tokens, int max_chunk, int max_len) {
    int shift;
    return record_bytes((long long)G.places * d->n_kv_heads, prompt_splits(d, G, n_tokens, max_chunk, max_len, shift), kPromptRows, d->head_dim);
}

template <typename T, int D, bool NT_LOADS> static fk_status mixed_launch(const MixedParams& P, hipStream_t st) {
    auto kern = mixed_kernel<T, D, NT_LOADS>;
    constexpr size_t lds = std::max(PromptCfg<T, D>::LDS_BYTES, ThinCfg<T, D>::lds(false, 4, false));
    static bool lds_ok[kMaxDevices] = {};
    if (!allow_dynamic_lds((const void*)kern, lds, lds_ok)) return FK_ERR_LAUNCH;
    const int thin = P.thin.grid.places * P.thin.view.n_kv;
    hipLaunchKernelGGL(kern, dim3((unsigned)(P.items * P.prompt.splits + thin * P.thin.splits)), dim3(256), lds, st, P);
    const int parts = P.merge + (P.thin.splits > 1 ? thin : 0);
    if (parts > 0) hipLaunchKernelGGL((mixed_merge_kernel<T, D>), dim3((unsigned)parts), dim3(256), 0, st, P);
    return launch_status();
}

template <typename T, int D>
static fk_status prompt_launch(const fk_paged_desc* d, AttnPagedParams& P, const AttnPagedParams* thin, bool cold, int max_chunk, int max_len, void* ws, hipStream_t st) {
    using C = PromptCfg<T, D>;
    const long long items = (long long)P.grid.places * d->n_kv_heads;
    P.splits = prompt_splits(d, P.grid, P.view.n_tokens, max_chunk, max_len, P.split_shift);   // (what the workspace is for)
    const long long seen = (long long)P.view.window + P.view.sink + kPromptRows;
    if (seen < max_len) P.splits = std::min(P.splits, prompt_splits(d, P.grid, P.view.n_tokens, max_chunk, seen, P.split_shift));
    P.rec_ml = reinterpret_cast<float2*>(ws);
    P.rec = reinterpret_cast<float*>(static_cast<char*>(ws) + up256((size_t)items * P.splits * kPromptRows * sizeof(float2)));
    if (thin) {
        const MixedParams M = {P, *thin, (int)items, P.splits > 1 ? (int)items * (kPromptRows / 16) : 0, magic_of((int)items)};
        return cold ? mixed_launch<T, D, true>(M, st) : mixed_launch<T, D, false>(M, st);
    }
    auto kern = prompt_kernel<T, D>;
    static bool lds_ok[kMaxDevices] = {};
    if (!allow_dynamic_lds((const void*)kern, C::LDS_BYTES, lds_ok)) return FK_ERR_LAUNCH;
    hipLaunchKernelGGL(kern, dim3((unsigned)items, P.splits), dim3(256), C::LDS_BYTES, st, P);
    if (P.splits > 1) hipLaunchKernelGGL((prompt_merge_kernel<T, D>), dim3((unsigned)items, kPromptRows / 16), dim3(256), 0, st, P);
    return launch_status();
}

fk_status prompt_paged(const fk_paged_desc* d, AttnPagedParams P, const AttnPagedParams* thin, bool cold, int max_chunk, int max_len, void* ws, hipStream_t st) {
    if (d->dtype == FK_F32)
        return d->head_dim == 64 ? prompt_launch<float, 64>(d, P, thin, cold, max_chunk, max_len, ws, st) : prompt_launch<float, 128>(d, P, thin, cold, max_chunk, max_len, ws, st);
    return d->head_dim == 64 ? prompt_launch<bf16_t, 64>(d, P, thin, cold, max_chunk, max_len, ws, st) : prompt_launch<bf16_t, 128>(d, P, thin, cold, max_chunk, max_len, ws, st);
}

}  // namespace fk
