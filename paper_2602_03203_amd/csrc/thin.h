// Attention of few query rows over many pairs (thin.hip): single tokens and short chunks over a paged cache, and the decode step that
// accumulates its weights over the rows of a budgeted cache.
#pragma once
#include "paged.h"

namespace fk {

struct ThinParams {
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
__host__ __device__ inline int thin_splits(int total, int splits, int least) {
    const int s = total / least;
    return s < 1 ? 1 : s < splits ? s : splits;
}

size_t thin_paged_workspace(const fk_paged_desc* d, const TileGrid& G, int max_len);
fk_status thin_paged(const fk_paged_desc* d, ThinParams P, int max_len, void* workspace, hipStream_t st);
fk_status thin_rows(const fk_cache_desc* d, ThinParams P, int max_len, void* workspace, hipStream_t st);
size_t thin_rows_workspace(const fk_cache_desc* d);

}  // namespace fk
