// fk_paged_append and fk_paged_compress: the ways into the pages of a prompt and out of them into the rows of a budgeted cache.
#include "paged.h"

namespace fk {

typedef unsigned int pu32x4_t __attribute__((ext_vector_type(4)));

// ---------------------------------------------------------------------------------------
// append: every new pair is read and written once.  A thread moves 16 bytes of K and of V; the threads of a wavefront, and of
// neighbouring wavefronts, take the chunks of a pair, the heads of a token, the tokens, in the order of k_new.  2 us for a few tokens, a chain of
// loads (sequence, length, page, pair); 7.8 us for 2048 tokens of 8 heads (34 MB moved).
// ---------------------------------------------------------------------------------------
__global__ __launch_bounds__(256) void paged_append_kernel(const PagedParams P, pu32x4_t* __restrict__ K, pu32x4_t* __restrict__ V,
                                                           const pu32x4_t* __restrict__ k_new, const pu32x4_t* __restrict__ v_new, int chunk_shift) {
    const size_t i = (size_t)blockIdx.x * 256 + threadIdx.x;
    const size_t pair = i >> chunk_shift;
    const int c = (int)(i & ((1u << chunk_shift) - 1));
    const int t = (int)(pair / P.n_kv), h = (int)(pair % P.n_kv);
    const int b = sequence_of(P, min(t, P.n_tokens - 1), min(__builtin_amdgcn_readfirstlane(t), P.n_tokens - 1));   // (all lanes take part)
    if (t >= P.n_tokens || b < 0) return;
    const int begin = chunk_begin(P, b), p = pairs_of(P, b) - (chunk_end(P, b, begin) - t);
    if (p < 0) return;
    const int page = P.table[(size_t)b * P.max_pages + (p >> P.page_shift)];
    if (!page_ok(P, page)) return;
    const size_t dst = (((((size_t)page * P.n_kv + h) << P.page_shift) + (p & ((1 << P.page_shift) - 1))) << chunk_shift) + c;
    K[dst] = k_new[i];
    V[dst] = v_new[i];
}

// ---------------------------------------------------------------------------------------
// compress: slot j of a row <- the pair at keep[j].  Bound by the memory system: a kept pair's K and V are read and written once.
// A workgroup owns 64 slots of a row: the indices and page numbers are looked up once, by one wavefront, positions and
// accumulated weights move beside them; then every thread moves 16 bytes of K and V a turn, all turns' loads ahead of the stores (the rows share no
// memory with the pool).  4 prompts, 8 heads, 2048 pairs kept (67 MB moved): 8.8 to 12 us.
// ---------------------------------------------------------------------------------------
static constexpr int kCompressSlots = 64;

struct CompressParams {
    const float* acc;
    const int32_t* keep;
    void *Kr, *Vr;
    int32_t *pos, *len;
    float* acc_rows;
    int budget, cap;
};

template <int CH /* 16-byte chunks of a pair's K */>
__device__ __forceinline__ void compress_slots(const PagedParams& P, const CompressParams& C, int row, long long (&s_src)[kCompressSlots]) {
    constexpr int U = kCompressSlots * CH / 256;
    const int b = row / P.n_kv, h = row % P.n_kv, tid = threadIdx.x;
    const int n = pairs_of(P, b), kept = min(n, C.budget), base = blockIdx.x * kCompressSlots;
    if (blockIdx.x == 0 && tid == 0) C.len[row] = kept;
    if (base >= kept) return;
    if (tid < kCompressSlots) {
        const int j = base + tid, p = j < kept ? C.keep[(size_t)row * C.budget + j] : -1;
        long long src = -1;
        if (p >= 0 && p < n) {
            const int page = P.table[(size_t)b * P.max_pages + (p >> P.page_shift)];
            if (page_ok(P, page)) src = ((((long long)page * P.n_kv + h) << P.page_shift) + (p & ((1 << P.page_shift) - 1)));
        }
        s_src[tid] = src;
        if (src >= 0) {
            C.pos[(size_t)row * C.cap + j] = p;
            if (C.acc) C.acc_rows[(size_t)row * C.cap + j] = C.acc[(size_t)row * ((size_t)P.max_pages << P.page_shift) + p];
        }
    }
    __syncthreads();
    const pu32x4_t *K = reinterpret_cast<const pu32x4_t*>(P.K), *V = reinterpret_cast<const pu32x4_t*>(P.V);
    pu32x4_t *Kr = reinterpret_cast<pu32x4_t*>(C.Kr) + ((size_t)row * C.cap + base) * CH, *Vr = reinterpret_cast<pu32x4_t*>(C.Vr) + ((size_t)row * C.cap + base) * CH;
    pu32x4_t k[U], v[U];
    long long src[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const int i = tid + u * 256;
        src[u] = s_src[i / CH];
        const size_t from = (size_t)(src[u] < 0 ? 0 : src[u]) * CH + i % CH;   // (none: the pool's first pair, not stored)
        k[u] = K[from];
        v[u] = V[from];
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const int i = tid + u * 256;
        if (src[u] < 0) continue;
        Kr[i] = k[u];
        Vr[i] = v[u];
    }
}

template <int CH>
__global__ __launch_bounds__(256) void paged_compress_kernel(const PagedParams P, const CompressParams C) {
    __shared__ long long s_src[kCompressSlots];   // pair of the pool, -1 for none
    for (int row = blockIdx.y;;) {   // (a grid's second dimension ends at 65535)
        compress_slots<CH>(P, C, row, s_src);
        row += gridDim.y;
        if (row >= P.batch * P.n_kv) break;
        __syncthreads();
    }
}

}  // namespace fk

using namespace fk;

extern "C" fk_status fk_paged_append(const fk_paged_desc* desc, void* K, void* V, const int32_t* page_table, const int32_t* kv_len,
                                     const int32_t* q_start, int32_t n_tokens, const void* k_new, const void* v_new, void* stream) {
    fk_status s = check_paged(desc);
    if (s == FK_OK) s = check_chunks(desc, n_tokens, 1, 1);
    if (s != FK_OK) return s;
    if (!K || !V || !page_table || !kv_len || !q_start || ((!k_new || !v_new) && n_tokens > 0)) return FK_ERR_INVALID_ARG;
    if (!aligned16(K) || !aligned16(V) || !aligned16(k_new) || !aligned16(v_new)) return FK_ERR_INVALID_ARG;
    if (n_tokens == 0) return FK_OK;
    const PagedParams P = paged_params(desc, page_table, kv_len, q_start, n_tokens);
    const int shift = __builtin_ctz(desc->head_dim * (desc->dtype == FK_F32 ? 4 : 2) / 16);
    const size_t threads = ((size_t)n_tokens * desc->n_kv_heads) << shift;
    hipLaunchKernelGGL(paged_append_kernel, dim3((unsigned)((threads + 255) / 256)), dim3(256), 0, (hipStream_t)stream, P, (pu32x4_t*)K, (pu32x4_t*)V,
                       (const pu32x4_t*)k_new, (const pu32x4_t*)v_new, shift);
    return launch_status();
}

extern "C" fk_status fk_paged_compress(const fk_paged_desc* desc, const void* K, const void* V, const int32_t* page_table,
                                       const int32_t* kv_len, const float* acc, const int32_t* keep_idx, int32_t budget,
                                       const fk_cache_desc* rows, void* K_rows, void* V_rows, int32_t* pos, int32_t* len,
                                       float* acc_rows, void* stream) {
    fk_status s = check_paged(desc);
    if (s == FK_OK) s = check_desc(rows);
    if (s != FK_OK) return s;
    if (rows->batch != desc->batch || rows->n_q_heads != desc->n_q_heads || rows->n_kv_heads != desc->n_kv_heads || rows->head_dim != desc->head_dim ||
        rows->dtype != desc->dtype)
        return FK_ERR_INVALID_ARG;
    if (!K || !V || !page_table || !kv_len || !keep_idx || !K_rows || !V_rows || !pos || !len || !acc != !acc_rows) return FK_ERR_INVALID_ARG;
    if (budget <= 0 || budget > rows->capacity) return FK_ERR_INVALID_ARG;
    if (!aligned16(K) || !aligned16(V) || !aligned16(K_rows) || !aligned16(V_rows)) return FK_ERR_INVALID_ARG;
    const int n_rows = desc->batch * desc->n_kv_heads;
    PagedParams P = paged_params(desc, page_table, kv_len, nullptr, 0);
    P.K = K;
    P.V = V;
    const CompressParams C = {acc, keep_idx, K_rows, V_rows, pos, len, acc_rows, budget, rows->capacity};
    const dim3 grid((budget + kCompressSlots - 1) / kCompressSlots, n_rows < 65536 ? n_rows : 65535);
    hipStream_t st = (hipStream_t)stream;
    switch (desc->head_dim * (desc->dtype == FK_F32 ? 4 : 2) / 16) {
        case 8: hipLaunchKernelGGL(paged_compress_kernel<8>, grid, dim3(256), 0, st, P, C); break;
        case 16: hipLaunchKernelGGL(paged_compress_kernel<16>, grid, dim3(256), 0, st, P, C); break;
        default: hipLaunchKernelGGL(paged_compress_kernel<32>, grid, dim3(256), 0, st, P, C); break;
    }
    return launch_status();
}
