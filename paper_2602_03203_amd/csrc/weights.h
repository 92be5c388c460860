// The weights that pairs receive from the queries of chunks (weights.hip), called by fk_paged_weights.
#pragma once
#include "paged.h"

namespace fk {

struct WeightsParams {
    PagedParams view;
    const float2* stats;   // [tokens][heads] (M, L)
    float* acc;            // [batch][n_kv][max_pages * page_size]
    float* part;           // [splits][batch * n_kv][part_len], with more than one split of the queries
    int splits, part_len;
    int keys, blocks;      // keys of a block, blocks of a sequence in the launch
    uint32_t blocks_magic;
};

size_t weights_workspace(const fk_paged_desc* d, int n_tokens, int max_chunk, int max_len);
fk_status weights_launch(const fk_paged_desc* d, WeightsParams P, int max_chunk, int max_len, void* workspace, hipStream_t st);

}  // namespace fk
