// fk_paged_attn: its launches with chunks of many query rows, alone or with chunks of few beside them
#include "prompt.h"
#include "thin.h"

#include <algorithm>

namespace fk {

struct PromptParams {
    AttnPagedParams attn;
    int rest;                 // items that may be split, behind attn.whole others
    uint32_t rest_magic;
};

// workgroup -> item and split: the whole items, then every split of all others
template <typename T, int D> __device__ __forceinline__ void prompt_part(const PromptParams& P, int x) {
    const int y = x - P.attn.whole, split = y < 0 ? 0 : scalar(divide(y, P.rest, P.rest_magic));
    prompt_tile<T, D>(P.attn, y < 0 ? x : P.attn.whole + y - split * P.rest, split);
}
template <typename T, int D> __device__ __forceinline__ void prompt_merge(const PromptParams& P, int x) {
    merge_tile<T, D, kPromptRows, PromptCfg<T, D>::KT>(P.attn, P.attn.whole + x / (kPromptRows / 16), x % (kPromptRows / 16));
}

template <typename T, int D>
__global__ __launch_bounds__(256, 2) void prompt_kernel(const PromptParams P) { prompt_part<T, D>(P, blockIdx.x); }

template <typename T, int D>
__global__ __launch_bounds__(256) void prompt_merge_kernel(const PromptParams P) { prompt_merge<T, D>(P, blockIdx.x); }

// Both kinds of chunks in one launch, the long tiles first: one kind's products run beside the other's loads.  A small model's batch of four prompt chunks
// and twenty single tokens, with the append before it: 53 us in two launches and two merges, 38 in one and one.
struct MixedParams {
    PromptParams prompt;
    AttnPagedParams thin;
    int many, merge;          // workgroups of the prompt tiles, of the first launch and of the second
};
template <typename T, int D, bool NT_LOADS>
__global__ __launch_bounds__(256, 2) void mixed_kernel(const MixedParams P) {
    const int x = blockIdx.x;
    if (x < P.many) {
        prompt_part<T, D>(P.prompt, x);
    } else {
        const int items = P.thin.grid.places * P.thin.view.n_kv, split = scalar(divide(x - P.many, items));
        thin_tile<T, D, false, 4, NT_LOADS>(P.thin, x - P.many - split * items, split);
    }
}
template <typename T, int D>
__global__ __launch_bounds__(256) void mixed_merge_kernel(const MixedParams P) {
    const int x = blockIdx.x;
    if (x < P.merge) prompt_merge<T, D>(P.prompt, x);
    else merge_tile<T, D, 16, ThinCfg<T, D>::KT>(P.thin, x - P.merge, 0);
}

// ---- host side ---------------------------------------------------------------------------------------------------
// Which items (a tile of rows, a kv head) have their pairs split, and over how many workgroups.  256 CUs hold two workgroups each: 512 items are a turn, and
// those beyond a multiple of it, or all of fewer, another one that leaves CUs idle - five sixths of a turn where they are at most 256 (a workgroup alone
// on its CU is a little faster).  Splits make that turn shorter and cost a second launch and their records' way to memory and back.  In
// microseconds, with 2.1 for 64 pairs of bf16 and D = 128, 6 for the launch and 4 TB/s for the records; in fp32 one workgroup has the matrix units of its CU
// busy, 9.4 for 64 pairs, half of one more has a CU to share, and all items are split alike.  Whole / 2 / 3 / 4 / 8 splits measured for 8 heads of g 4, D 128: 512 tokens of 8192 pairs: 216 / 123 / 104 / 93 / 101; 1024 of
// 8192: 222 / 160 / 175 / 166 / 186; 4 chunks to 300 of 2048: 70 / 80 / 72 / 73 / 70.  A split has 512 pairs and more, or 256 where no
// sequence is longer than 2048: 2 chunks to 908 of 908, 2 heads 35 whole, 29 in two, fp32 896 of 896, one head of g 8, D 64 80 and 49; 4 to 100 of 1000 37 and 33; but a batch of 300 to 4096 pairs (mixed_kernel)
// 35 by splits of 512, 37 of 256.  The rest of the last turn alone split, against nothing and everything
// split: 2400 tokens of 16384 606, 822 and 662; two chunks to 1200 of 8192 298, 425 and 340.  How many chunks there are that are not single tokens the host
// does not know: as many as would have the longest one's length.
struct PromptPlan {
    int whole, splits, shift;
};
static PromptPlan prompt_plan(const fk_paged_desc* d, const TileGrid& G, int n_tokens, int max_chunk, long long pairs) {
    const bool bf16 = d->dtype == FK_BF16;
    const long long g = d->n_q_heads / d->n_kv_heads, chunk = max_chunk < n_tokens ? max_chunk : n_tokens, rest = n_tokens - d->batch;
    const long long chunks = chunk > 1 && rest > 0 ? (rest + chunk - 2) / (chunk - 1) : 1;
    const long long items = (n_tokens * g + chunks * (kPromptRows - 1)) / kPromptRows * d->n_kv_heads, places = (long long)G.places * d->n_kv_heads;
    long long whole = bf16 ? items / 512 * 512 : 0;
    whole -= whole % d->n_kv_heads;
    whole = std::min(whole, places);
    const long long left = items - whole;
    const int fewest = pairs <= 2048 ? 256 : 512;   // pairs of a split
    PromptPlan p = {(int)whole, 1, (fewest == 256 ? 2 : 3) + (bf16 ? 0 : 1)};
    const double one = (double)pairs / 64 * d->head_dim / 128 * (bf16 ? 2.1 : 9.4);
    double least = 0;
    for (int s = 1; s <= 16 && (s == 1 || (pairs / s >= fewest && (places - whole) * s <= 4096 /* a quarter of a GiB of records */)); ++s) {
        const long long all = left * s, over = all % 512;
        const double turns = bf16 ? (double)(all / 512) + (over == 0 ? 0. : over <= 256 ? 5. / 6 : 1.) : std::max(1., (double)(all + 128) / 256);
        const double time = turns * one / s + (s == 1 ? 0. : 6 + (double)all * kPromptRows * d->head_dim * 8 / 4e6);
        if (s == 1 || time < least) least = time, p.splits = s;
    }
    return p;
}
size_t prompt_workspace(const fk_paged_desc* d, const TileGrid& G, int n_tokens, int max_chunk, int max_len) {
    const PromptPlan p = prompt_plan(d, G, n_tokens, max_chunk, max_len);
    return record_bytes((long long)G.places * d->n_kv_heads - p.whole, p.splits, kPromptRows, d->head_dim);
}

template <typename T, int D, bool NT_LOADS> static fk_status mixed_launch(const MixedParams& P, hipStream_t st) {
    auto kern = mixed_kernel<T, D, NT_LOADS>;
    constexpr size_t lds = std::max(PromptCfg<T, D>::LDS_BYTES, ThinCfg<T, D>::lds(false, 4, 0));
    static bool lds_ok[kMaxDevices] = {};
    if (!allow_dynamic_lds((const void*)kern, lds, lds_ok)) return FK_ERR_LAUNCH;
    const int thin = P.thin.grid.places * P.thin.view.n_kv;
    hipLaunchKernelGGL(kern, dim3((unsigned)(P.many + thin * P.thin.splits)), dim3(256), lds, st, P);
    const int parts = P.merge + (P.thin.splits > 1 ? thin : 0);
    if (parts > 0) hipLaunchKernelGGL((mixed_merge_kernel<T, D>), dim3((unsigned)parts), dim3(256), 0, st, P);
    return launch_status();
}

template <typename T, int D>
static fk_status prompt_launch(const fk_paged_desc* d, AttnPagedParams& A, const AttnPagedParams* thin, bool cold, int max_chunk, int max_len, void* ws, hipStream_t st) {
    const PromptPlan p = prompt_plan(d, A.grid, A.view.n_tokens, max_chunk, max_len);   // (what the workspace is for)
    const long long seen = (long long)A.view.window + A.view.sink + kPromptRows;
    A.whole = p.whole;
    A.splits = seen < max_len ? std::min(p.splits, prompt_plan(d, A.grid, A.view.n_tokens, max_chunk, seen).splits) : p.splits;
    A.split_shift = p.shift;
    const int items = A.grid.places * d->n_kv_heads, rest = items - A.whole;
    A.rec_ml = reinterpret_cast<float2*>(ws);
    A.rec = reinterpret_cast<float*>(static_cast<char*>(ws) + up256((size_t)rest * A.splits * kPromptRows * sizeof(float2)));
    const PromptParams P = {A, rest, rest > 0 ? magic_of(rest) : 0};
    const int many = A.whole + rest * A.splits, merge = A.splits > 1 ? rest * (kPromptRows / 16) : 0;
    if (thin) {
        const MixedParams M = {P, *thin, many, merge};
        return cold ? mixed_launch<T, D, true>(M, st) : mixed_launch<T, D, false>(M, st);
    }
    auto kern = prompt_kernel<T, D>;
    constexpr size_t lds = PromptCfg<T, D>::LDS_BYTES;
    static bool lds_ok[kMaxDevices] = {};
    if (!allow_dynamic_lds((const void*)kern, lds, lds_ok)) return FK_ERR_LAUNCH;
    hipLaunchKernelGGL(kern, dim3((unsigned)many), dim3(256), lds, st, P);
    if (merge > 0) hipLaunchKernelGGL((prompt_merge_kernel<T, D>), dim3((unsigned)merge), dim3(256), 0, st, P);
    return launch_status();
}

fk_status prompt_paged(const fk_paged_desc* d, AttnPagedParams P, const AttnPagedParams* thin, bool cold, int max_chunk, int max_len, void* ws, hipStream_t st) {
    if (d->dtype == FK_F32)
        return d->head_dim == 64 ? prompt_launch<float, 64>(d, P, thin, cold, max_chunk, max_len, ws, st) : prompt_launch<float, 128>(d, P, thin, cold, max_chunk, max_len, ws, st);
    return d->head_dim == 64 ? prompt_launch<bf16_t, 64>(d, P, thin, cold, max_chunk, max_len, ws, st) : prompt_launch<bf16_t, 128>(d, P, thin, cold, max_chunk, max_len, ws, st);
}

}  // namespace fk
