// The paged cache of a prompt (fk_paged_*): its parameters, where a pair lies, what a query sees, and the checks of its calls.
#pragma once
#include "fk_common.h"

#include <cfloat>
#include <cmath>

namespace fk {

struct PagedParams {
    const void* q;
    const void *K, *V;
    const int32_t *table, *kv_len, *q_start;
    int batch, n_kv, g, page_shift, n_pages, max_pages, n_tokens;
    int window, sink;      // window: INT_MAX without one
    float scale_log2e;     // >= 0: queries are negated as they are read where softmax_scale is negative (exact)
    bool negate;
    uint32_t g_magic, kv_magic, batch_magic;   // for divisions by g, n_kv, batch (magic_of)
};

// x / n for 0 <= x < 2^31 by a multiplication: magic = floor(2^32 / n) (n = 1: 2^32 - 1) is short by less than one unit of the quotient
inline uint32_t magic_of(int n) { return n == 1 ? 0xffffffffu : (uint32_t)((1ull << 32) / n); }
__device__ __forceinline__ int divide(int x, int n, uint32_t magic) {
    int q = (int)__umulhi((uint32_t)x, magic);
    if (x - q * n >= n) ++q;
    return q;
}
// small quotients (x < 2^24) of numbers that only the device knows
__device__ __forceinline__ int divide(int x, int n) {
    int q = (int)((float)x * __builtin_amdgcn_rcpf((float)n));
    if (x - q * n >= n) ++q;
    if (x - q * n < 0) --q;
    return q;
}

// A value that is the same for every lane, in a scalar register.  (Opaque first: the builtin is dropped where the compiler knows as much; it then
// keeps what integer divisions gave, and all that follows from it, in vector registers: page numbers by vector loads, branches by exec masks, 60
// registers more.)
__device__ __forceinline__ int scalar(int x) {
    asm volatile("" : "+v"(x));
    return __builtin_amdgcn_readfirstlane(x);
}

template <typename T> __device__ __forceinline__ const T* scalar_ptr(const T* p) {
    const uint64_t x = reinterpret_cast<uint64_t>(p);
    const uint32_t lo = (uint32_t)scalar((int)(uint32_t)x), hi = (uint32_t)scalar((int)(uint32_t)(x >> 32));
    return reinterpret_cast<const T*>((uint64_t)hi << 32 | lo);
}

// An element of an array that nothing writes during the launch, at an index that is the same for a whole wavefront: a scalar load.  (Vector loads
// return in order: waiting for a page number would mean waiting for all pairs sent for before it.)
__device__ __forceinline__ int load_uniform(const int32_t* p, int i) {
    return ((const __attribute__((address_space(4))) int32_t*)p)[i];
}

// Tokens of sequence b in the packed buffers, and its pairs; whatever the arrays hold, inside the buffers.
__device__ __forceinline__ int chunk_begin(const PagedParams& P, int b) { return min(max(P.q_start[b], 0), P.n_tokens); }
__device__ __forceinline__ int chunk_end(const PagedParams& P, int b, int begin) { return min(max(P.q_start[b + 1], begin), P.n_tokens); }
__device__ __forceinline__ int pairs_of(const PagedParams& P, int b) { return min(max(P.kv_len[b], 0), P.max_pages << P.page_shift); }

__device__ __forceinline__ bool page_ok(const PagedParams& P, int page) { return (unsigned)page < (unsigned)P.n_pages; }

// The sequence that token t belongs to, -1 for none (q_start ascending: the first one that ends behind t), and its end.  `from`: the first token that
// any lane of the wavefront asks for; the ends are looked at 64 at a time, then a lane walks on from there.
__device__ __forceinline__ int sequence_of(const PagedParams& P, int t, int from) {
    const int lane = threadIdx.x & (kWave - 1);
    int b = P.batch;
    for (int base = 0; base < P.batch; base += kWave) {
        const unsigned long long m = __ballot(base + lane < P.batch && P.q_start[min(base + lane, P.batch - 1) + 1] > from);
        if (m) {
            b = base + __ffsll((long long)m) - 1;
            break;
        }
    }
    while (b < P.batch && P.q_start[b + 1] <= t) ++b;
    return b < P.batch && P.q_start[b] <= t ? b : -1;
}

// 16 bytes per lane from global memory to LDS, at `to` + lane * 16.  A barrier alone does not wait for them: arrived() before it.
__device__ __forceinline__ void load_to_lds(const void* from, unsigned char* to) {
    __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)from, (__attribute__((address_space(3))) void*)to, 16, 0, 0);
}
__device__ __forceinline__ void arrived() { asm volatile("s_waitcnt vmcnt(0)" ::: "memory"); }   // this wavefront's

// |logits| from which they are rounded before a maximum is subtracted from them, as the few-row kernel always does; below it they are left to the fma, where an
// exponent may be off by the rounding of the maximum, 2^-17 at most.  M and L are then the ones that the weights' exponents belong to, from whichever kernel
// they come.  Where a tile has such logits it costs more: 2048 tokens of 16384 pairs, 8 heads of g 4, D 128, attention 501 us -> 524, weights 276 -> 312.
static constexpr float kLargeLogit = 256.f;

// ---- tiles of query rows --------------------------------------------------------------------------------------------
// The queries of a (chunk, KV head) are rows: row r is head r % g of token r / g.  A tile is TM of them.  `slot` counts the places of a launch:
// either place i of sequence b is slot i * batch + b (spread == false; a sequence has `per_seq` places, whose workgroups take every
// per_seq-th of its tiles), or the slots are dealt to the tiles there are, sequence after sequence (`places` of them).  A sequence's last
// tiles come first: they see the most.
struct TileGrid {
    bool spread;
    int places;     // slots in all
    int per_seq;
    int least, most;   // rows of the chunks that the launch takes: least <= nq * g <= most
};

struct TileOf {
    int b, begin, nq, n, first;   // sequence, its first token, tokens, pairs, position of the first token
    int tile, step;               // tiles tile, tile - step, .. >= 0
    bool one;                     // no more tiles than places: each has its own
};

__device__ __forceinline__ bool chunk_of(const PagedParams& P, const TileGrid& G, int b, TileOf& t, int tm, int& tiles) {
    t.b = b;
    t.begin = chunk_begin(P, b);
    t.nq = chunk_end(P, b, t.begin) - t.begin;
    const int rows = t.nq * P.g;
    tiles = rows >= G.least && rows <= G.most ? (rows + tm - 1) / tm : 0;
    return tiles > 0;
}

// false: the slot has no tile
__device__ __forceinline__ bool tile_of(const PagedParams& P, const TileGrid& G, int slot, int tm, TileOf& t) {
    int tiles;
    if (!G.spread) {
        const int i = scalar(divide(slot, P.batch, P.batch_magic));
        t.b = slot - i * P.batch;
        t.begin = min(max(load_uniform(P.q_start, t.b), 0), P.n_tokens);
        t.nq = min(max(load_uniform(P.q_start, t.b + 1), t.begin), P.n_tokens) - t.begin;
        t.n = min(max(load_uniform(P.kv_len, t.b), 0), P.max_pages << P.page_shift);
        const int rows = t.nq * P.g;
        tiles = rows >= G.least && rows <= G.most ? (uint32_t)(rows + tm - 1) / (uint32_t)tm : 0;
        if (i >= tiles) return false;
        t.tile = tiles - 1 - i;
        t.step = G.per_seq;
        t.one = tiles <= G.per_seq;
    } else {
        const int lane = threadIdx.x & (kWave - 1);
        int left = slot, found = -1, at = 0;
        for (int base = 0; base < P.batch && found < 0; base += kWave) {
            int mine = 0;
            if (base + lane < P.batch) chunk_of(P, G, base + lane, t, tm, mine);
            int incl = mine;
#pragma unroll
            for (int off = 1; off < kWave; off <<= 1) {
                const int o = __shfl_up(incl, off);
                if (lane >= off) incl += o;
            }
            const unsigned long long m = __ballot(incl > left);
            if (m) {
                const int src = __ffsll((long long)m) - 1;
                found = base + src;
                at = left - __shfl(incl - mine, src);
            } else {
                left -= __shfl(incl, kWave - 1);
            }
        }
        found = scalar(found);
        if (found < 0) return false;
        chunk_of(P, G, found, t, tm, tiles);
        t.tile = tiles - 1 - scalar(at);
        t.n = pairs_of(P, found);
        t.step = 1 << 30;   // (as many slots as there can be tiles)
        t.one = true;
    }
    // (the same for every lane, which the compiler is told: branches on them are scalar)
    t.b = scalar(t.b);
    t.begin = scalar(t.begin);
    t.nq = scalar(t.nq);
    t.n = scalar(t.n);
    t.tile = scalar(t.tile);
    t.step = scalar(t.step);
    t.first = t.n - t.nq;
    return true;
}

// The key tiles of kt pairs that rows at positions lo .. hi see something of: na tiles from the first on, then those from b0 to b1.
struct KeyTiles {
    int na, b0, total;
    __device__ __forceinline__ int at(int i) const { return i < na ? i : i - na + b0; }
};
__device__ __forceinline__ KeyTiles key_tiles(const PagedParams& P, int lo, int hi, int kt) {
    KeyTiles k;
    const int end = hi + 1;                                         // pairs up to here
    const int from = P.window == 0x7fffffff ? 0 : max(0, lo - P.window + 1);
    k.na = (uint32_t)(min(P.sink, max(end, 0)) + kt - 1) / (uint32_t)kt;
    k.b0 = (uint32_t)from / (uint32_t)kt;
    if (k.b0 <= k.na) k.na = k.b0 = 0;
    const int b1 = (uint32_t)(max(end, 0) + kt - 1) / (uint32_t)kt;
    k.total = k.na + max(b1 - k.b0, 0);
    return k;
}

// ---- host side ---------------------------------------------------------------------------------------------------
// |softmax_scale| for exponents of 2; 0: as near to it as keeps what is not seen at -inf, all logits are equal; NaN stays NaN
inline float base2_scale(float softmax_scale) {
    const float s = std::fabs(softmax_scale) * 1.4426950408889634f;
    return s < FLT_MIN ? FLT_MIN : s;
}

inline fk_status check_paged(const fk_paged_desc* d) {
    if (!d) return FK_ERR_INVALID_ARG;
    if (d->batch <= 0 || d->n_q_heads <= 0 || d->n_kv_heads <= 0 || d->head_dim <= 0 || d->page_size <= 0 || d->n_pages <= 0 || d->max_pages <= 0)
        return FK_ERR_INVALID_ARG;
    if (d->n_q_heads % d->n_kv_heads != 0) return FK_ERR_INVALID_ARG;
    if (d->dtype != FK_F32 && d->dtype != FK_BF16) return FK_ERR_UNSUPPORTED;
    if (d->head_dim != 64 && d->head_dim != 128) return FK_ERR_UNSUPPORTED;
    if (d->n_q_heads / d->n_kv_heads > 8) return FK_ERR_UNSUPPORTED;
    if (d->page_size < 16 || d->page_size > 1024 || (d->page_size & (d->page_size - 1))) return FK_ERR_UNSUPPORTED;
    if ((int64_t)d->max_pages * d->page_size >= (1 << 24)) return FK_ERR_UNSUPPORTED;
    if ((int64_t)d->batch * d->n_kv_heads >= (1 << 24)) return FK_ERR_UNSUPPORTED;
    return FK_OK;
}

// sizes of a call on chunks; 32-bit counts of query rows
inline fk_status check_chunks(const fk_paged_desc* d, int32_t n_tokens, int32_t max_chunk, int32_t max_len) {
    if (n_tokens < 0 || max_chunk <= 0 || max_len <= 0 || (int64_t)max_len > (int64_t)d->max_pages * d->page_size) return FK_ERR_INVALID_ARG;
    if ((int64_t)n_tokens * d->n_q_heads >= (1 << 28)) return FK_ERR_UNSUPPORTED;
    return FK_OK;
}

// Places for the tiles of tm rows of a call, without knowing the chunks
inline TileGrid tile_grid(const fk_paged_desc* d, int32_t n_tokens, int32_t max_chunk, int tm) {
    const long long g = d->n_q_heads / d->n_kv_heads, most = (long long)n_tokens * g / tm + d->batch;
    const long long chunk = max_chunk < n_tokens ? max_chunk : n_tokens > 0 ? n_tokens : 1, per_seq = (chunk * g + tm - 1) / tm;
    if (per_seq * d->batch <= 2 * most) return {false, (int)(per_seq * d->batch), (int)per_seq, 1, 0x7fffffff};
    return {true, (int)most, 1, 1, 0x7fffffff};
}

inline PagedParams paged_params(const fk_paged_desc* d, const int32_t* table, const int32_t* kv_len, const int32_t* q_start, int32_t n_tokens) {
    PagedParams P = {};
    P.table = table;
    P.kv_len = kv_len;
    P.q_start = q_start;
    P.batch = d->batch;
    P.n_kv = d->n_kv_heads;
    P.g = d->n_q_heads / d->n_kv_heads;
    P.page_shift = __builtin_ctz(d->page_size);
    P.n_pages = d->n_pages;
    P.max_pages = d->max_pages;
    P.n_tokens = n_tokens;
    P.g_magic = magic_of(P.g);
    P.kv_magic = magic_of(P.n_kv);
    P.batch_magic = magic_of(P.batch);
    return P;
}

}  // namespace fk
