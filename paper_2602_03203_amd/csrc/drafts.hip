// fk_verify_drafts: which drafted tokens the large model's probabilities accept, and the token behind them.
// fk_commit_drafts, fk_paged_commit_drafts: the pairs of the accepted path join the cache.
#include "paged.h"

#include <algorithm>
#include <type_traits>

namespace fk {

static constexpr int kNodes = FK_TREE_NODES;

// ---------------------------------------------------------------------------------------
// Verification.  At a node with distributions p (target) and q (draft) the first child x, drawn from q, is accepted with probability
// min(1, p(x) / q(x)); else what is left, r = max(p - q, 0) normalised, takes the place of p for the next child, and so on: the token that
// comes out is distributed as p whatever q is (speculative sampling, with several drafts).  Only two numbers carry from
// rejection to rejection: with r_k = max(p - c_k q, 0) / m_k, c_0 = 0, m_0 = 1,
//     r_k+1 ~ max(r_k - q, 0) = max(p - (c_k + m_k) q, 0) / m_k,   so   c_k+1 = c_k + m_k,   m_k+1 = sum max(p - c_k+1 q, 0).
// A child of a likeliest-token draft (no q) is accepted with probability p(x) / m; else p(x) becomes 0 and m goes down by it.
// Sums and comparisons in 64 bits: a 32-bit sum over a vocabulary is off by more than its smaller probabilities.
//
// One launch.  A sequence's vocabulary is cut into chunks, a workgroup each.  All of them walk the tree alike (a few hundred numbers, all sent for
// together) up to the first rejection whose sum is not known, or to the end; each sums its chunk of what is left, tells the others, and goes on with
// the sum of all chunks; the one whose chunk holds the last number draws the token.  Nobody has to wait: a sum that does not come in time (its
// workgroup may not have begun) is formed by whoever misses it, in the same order, so that it is the same bits.
// A sum on its way is two words of 32 bits of it and the call's number each: one that holds another number is not there yet.
// Bound by latencies, one after the other: sequence, nodes, their probabilities, the row, the others' sums, the chunk's numbers (16 chains of 4 drafted tokens, 32000
// numbers: 11.2 us), and another 3 us for every further sum (16 trees of 17 to 33 nodes, 131072 numbers: 25 us; one workgroup alone, which then
// summed whole rows, took 234; 4 nodes with 200 children each, all rejected: 0.6 ms, and 10.7 while the first 32 sums alone were told).
// ---------------------------------------------------------------------------------------
static constexpr int kVerifyThreads = 256, kVerifyWaves = kVerifyThreads / kWave, kMostChunks = 64;
static constexpr int kRounds = kNodes + 1; // sums of a sequence: one for every rejected node, the last token's, and the target's own where nothing is left
static constexpr int kPatience = 64;       // looks at a sum that is not there, 0.5 us and more each

struct VerifyParams {
    const float *target, *draft;
    const int32_t *tokens, *parent, *q_start;
    const float* uniform;
    int32_t *path, *accepted, *next;
    int n_tokens, batch, vocab, chunks, chunk;   // chunk: numbers of a chunk, a multiple of 4
    uint32_t *call, *done;                       // calls on this workspace so far, workgroups of this one that are done
    unsigned long long* told;                    // [batch][kRounds][chunks][2]
};

struct Tree {            // in LDS
    float p[kNodes], q[kNodes], u[kNodes];   // target's and draft's probability of a node's token behind its parent; its number
    int token[kNodes];
    short parent[kNodes], path[kNodes], gone[kNodes];
    int here[kNodes];                        // rejected tokens of a chunk
    double part[kMostChunks], wave[kVerifyWaves];
    double c, left;
    unsigned long long missing;
    int at, depth, n_gone, n_here, tried, state, chosen, first[kVerifyWaves];
};

// The walk as far as it needs no sums, by the first wavefront: children of `at` from `tried` on.  state 1: a sum with the new c is wanted before the next
// child; 2: no child is left.  m: the sum of what is left (before the first child 1).  All lanes have and store the same values: what a lane reads back it has
// written itself.
__device__ __forceinline__ void walk(Tree& T, int nodes, bool drawn, double m) {
    const int lane = threadIdx.x & (kWave - 1);
    int at = T.at, from = T.tried, depth = T.depth, n_gone = T.n_gone, state = 2;
    double c = T.c;
    for (;;) {
        int i = -1;
        for (int w = from / kWave; w * kWave < nodes; ++w) {
            const int j = w * kWave + lane;
            const unsigned long long child = __ballot(j < nodes && j >= from && T.parent[min(j, nodes - 1)] == at);
            if (child) {
                i = w * kWave + __ffsll((long long)child) - 1;
                break;
            }
        }
        if (i < 0) break;
        from = i + 1;
        const double p = T.p[i], u = T.u[i];
        bool yes, again = false;
        if (drawn) {
            yes = u * T.q[i] * m < p - c * T.q[i];
        } else {
            for (int k0 = 0; k0 < n_gone; k0 += kWave)
                again |= __ballot(k0 + lane < n_gone && T.token[T.gone[min(k0 + lane, n_gone - 1)]] == T.token[i]) != 0;
            yes = u * m < (again ? 0.0 : p);
        }
        if (yes) {
            T.path[depth] = (short)i;
            ++depth;
            at = i;
            c = 0.0;
            m = 1.0;
            n_gone = 0;
        } else if (drawn) {
            c += m;
            state = 1;
            break;
        } else if (!again) {
            T.gone[n_gone] = (short)i;
            ++n_gone;
            m = fmax(m - p, 0.0);
        }
    }
    T.at = at;
    T.tried = from;
    T.depth = depth;
    T.n_gone = n_gone;
    T.c = c;
    T.state = state;
}

// what is left of a number of the vocabulary at the current node; drawn: tokens of the draft have been rejected there
__device__ __forceinline__ double left_of(double c, float p, float q, bool drawn) {
    const double r = drawn ? (double)p - c * (double)q : (double)p;
    return r > 0.0 ? r : 0.0;
}

__device__ __forceinline__ double wave_sum(double x) {
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) x += __shfl_xor(x, off);
    return x;
}
__device__ __forceinline__ double wave_scan(double x) {   // inclusive
    const int lane = threadIdx.x & (kWave - 1);
#pragma unroll
    for (int off = 1; off < kWave; off <<= 1) {
        const double o = __shfl_up(x, off);
        if (lane >= off) x += o;
    }
    return x;
}

typedef float vf32x4_t __attribute__((ext_vector_type(4), aligned(4)));   // rows of an odd vocabulary start anywhere

// Four numbers of what is left, from v on; 0 from `end` on and where `gone` has a bit.
struct Four {
    double r[4];
};
__device__ __forceinline__ Four four_of(const float* p, const float* q, int v, int end, double c, uint32_t gone) {
    Four x;
    vf32x4_t a = {0.f, 0.f, 0.f, 0.f}, b = a;
    if (v + 4 <= end) {
        a = *reinterpret_cast<const vf32x4_t*>(p + v);
        if (q) b = *reinterpret_cast<const vf32x4_t*>(q + v);
    } else {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            if (v + j >= end) break;
            a[j] = p[v + j];
            if (q) b[j] = q[v + j];
        }
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) x.r[j] = gone >> j & 1 ? 0.0 : left_of(c, a[j], b[j], q != nullptr);
    return x;
}
// A bit for each rejected token among this thread's numbers v, v + 1, v + 2, v + 3, then those kStep on, sixteen times.
static constexpr int kStep = kVerifyThreads * 4;
__device__ __forceinline__ unsigned long long gone_of(const Tree& T, int v) {
    unsigned long long bits = 0;
    for (int k = 0; k < T.n_here; ++k) {
        const int x = T.here[k] - v;
        if (x >= 0 && x < 16 * kStep && x % kStep < 4) bits |= 1ull << (x / kStep * 4 + x % kStep);
    }
    return bits;
}

// The draft's row as far as it plays a part: with nothing rejected (c = 0) what is left is the target's row whatever the draft holds - nobody drew from the row
// of a node without children, which may not have been filled, and 0 times an infinity or a NaN is no 0.  The same for all threads of a sequence.
__device__ __forceinline__ const float* draft_of(const VerifyParams& P, const Tree& T, size_t row) { return P.draft && T.c != 0.0 ? P.draft + row : nullptr; }

// the rejected tokens that lie in a chunk; all threads
__device__ __forceinline__ void find_gone(const VerifyParams& P, Tree& T, int chunk) {
    if (threadIdx.x < kWave) {
        const int lane = threadIdx.x;
        int n = 0;
        for (int k0 = 0; k0 < T.n_gone; k0 += kWave) {
            const int x = k0 + lane < T.n_gone ? T.token[T.gone[k0 + lane]] : -1;
            const bool in = x >= chunk * P.chunk && x < (chunk + 1) * P.chunk;
            const unsigned long long all = __ballot(in);
            if (in) T.here[n + __popcll(all & ((1ull << lane) - 1))] = x;
            n += __popcll(all);
        }
        if (lane == 0) T.n_here = n;
    }
    __syncthreads();
}

// the sum of what is left in a chunk, into T.part; all threads
__device__ __forceinline__ void sum_chunk(const VerifyParams& P, Tree& T, int begin, int chunk) {
    const int tid = threadIdx.x, v0 = chunk * P.chunk, end = min(v0 + P.chunk, P.vocab);
    find_gone(P, T, chunk);
    const size_t row = (size_t)(begin + T.at) * P.vocab;
    const float *p = P.target + row, *q = draft_of(P, T, row);
    const double c = T.c;
    double sum = 0.0;
    auto add = [&](auto SOME) {   // SOME: tokens that do not count
        for (int first = v0 + tid * 4; first < end; first += 16 * kStep) {
            const unsigned long long gone = SOME ? gone_of(T, first) : 0;
            constexpr int U = 4;
            for (int g0 = 0; g0 < 16; g0 += U) {   // (all loads of a turn ahead of its sums)
                const int v = first + g0 * kStep;
                if (v >= end) break;
                const uint32_t bits = (uint32_t)(gone >> (g0 * 4));
                if (v + (U - 1) * kStep + 4 <= end) {
                    vf32x4_t a[U], b[U];
#pragma unroll
                    for (int u = 0; u < U; ++u) {
                        a[u] = *reinterpret_cast<const vf32x4_t*>(p + v + u * kStep);
                        b[u] = vf32x4_t{0.f, 0.f, 0.f, 0.f};
                        if (q) b[u] = *reinterpret_cast<const vf32x4_t*>(q + v + u * kStep);
                    }
#pragma unroll
                    for (int u = 0; u < U; ++u) {
                        double r[4];
#pragma unroll
                        for (int j = 0; j < 4; ++j) r[j] = SOME && bits >> (u * 4 + j) & 1 ? 0.0 : left_of(c, a[u][j], b[u][j], q != nullptr);
                        sum += (r[0] + r[1]) + (r[2] + r[3]);
                    }
                } else {
                    Four x[U];
#pragma unroll
                    for (int u = 0; u < U; ++u) x[u] = four_of(p, q, v + u * kStep, end, c, bits >> (u * 4));
#pragma unroll
                    for (int u = 0; u < U; ++u) sum += (x[u].r[0] + x[u].r[1]) + (x[u].r[2] + x[u].r[3]);
                }
            }
        }
    };
    if (T.n_here == 0) add(std::false_type());
    else add(std::true_type());
    sum = wave_sum(sum);
    if (tid % kWave == 0) T.wave[tid / kWave] = sum;
    __syncthreads();
    if (tid == 0) {
        double all = 0.0;
        for (int w = 0; w < kVerifyWaves; ++w) all += T.wave[w];
        T.part[chunk] = all;
    }
    __syncthreads();
}

__global__ __launch_bounds__(kVerifyThreads) void verify_kernel(const VerifyParams P) {
    __shared__ Tree T;
    const int tid = threadIdx.x, lane = tid & (kWave - 1), wave = tid / kWave, b = blockIdx.y, chunk = blockIdx.x;
    const bool drawn = P.draft != nullptr;
    const uint32_t call = P.chunks > 1 ? __hip_atomic_load(P.call, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) + 1 : 0;
    // the last one to be done with it: the next call, of whatever sizes, has another number
    auto be_done = [&]() {
        if (P.chunks == 1 || tid != 0) return;
        if (__hip_atomic_fetch_add(P.done, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == (uint32_t)(P.chunks * P.batch) - 1) {
            __hip_atomic_store(P.done, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
            __hip_atomic_store(P.call, call, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        }
    };
    const int begin = min(max(P.q_start[b], 0), P.n_tokens), nodes = min(max(P.q_start[b + 1], begin), P.n_tokens) - begin;
    if (nodes == 0 || nodes > kNodes) {
        if (chunk == 0 && tid == 0) {
            P.accepted[b] = 0;
            P.next[b] = -1;
        }
        be_done();
        return;
    }
    for (int i = tid; i < nodes; i += kVerifyThreads) {
        const int up = P.parent[begin + i], x = P.tokens[begin + i];
        const float u = P.uniform[begin + i];
        const bool there = i > 0 && up >= 0 && up < i && x >= 0 && x < P.vocab;
        const size_t at = (size_t)(begin + (there ? up : 0)) * P.vocab + (there ? x : 0);
        const float p = P.target[at], q = drawn ? P.draft[at] : 0.f;
        T.p[i] = there && p > 0.f ? p : 0.f;
        T.q[i] = there ? q : 0.f;
        T.u[i] = u;
        T.token[i] = x;
        T.parent[i] = (short)(i > 0 && up < i ? max(up, -1) : -1);
    }
    if (tid == 0) {
        T.at = 0;
        T.depth = 1;
        T.path[0] = 0;
        T.n_gone = 0;
        T.tried = 1;
        T.c = 0.0;
    }
    __syncthreads();
    if (wave == 0) walk(T, nodes, drawn, 1.0);
    __syncthreads();
    for (int round = 0;; ++round) {
        // the sums of what is left at T.at, chunk by chunk
        sum_chunk(P, T, begin, chunk);
        if (P.chunks > 1) {
            unsigned long long* told = P.told + ((size_t)b * kRounds + round) * P.chunks * 2;
            if (wave == 0) {
                if (lane < 2) {
                    const uint64_t bits = (uint64_t)__double_as_longlong(T.part[chunk]);
                    __hip_atomic_store(told + chunk * 2 + lane, (unsigned long long)call << 32 | (uint32_t)(bits >> (32 * lane)), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
                }
                bool here = lane >= P.chunks || lane == chunk;
                for (int look = 0; look < kPatience; ++look) {
                    if (!here) {
                        const unsigned long long lo = __hip_atomic_load(told + lane * 2, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
                        const unsigned long long hi = __hip_atomic_load(told + lane * 2 + 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
                        if ((uint32_t)(lo >> 32) == call && (uint32_t)(hi >> 32) == call) {
                            T.part[lane] = __longlong_as_double((long long)((uint64_t)(uint32_t)hi << 32 | (uint32_t)lo));
                            here = true;
                        }
                    }
                    if (__all(here)) break;
                    __builtin_amdgcn_s_sleep(2);
                }
                const unsigned long long missing = __ballot(!here);
                if (lane == 0) T.missing = missing;
            }
            __syncthreads();
            for (unsigned long long missing = T.missing; missing; missing &= missing - 1) sum_chunk(P, T, begin, __ffsll((long long)missing) - 1);
        }
        if (wave == 0) {
            const double all = wave_sum(lane < P.chunks ? T.part[lane] : 0.0);
            const int depth = T.depth, was = T.state;
            if (was == 1) walk(T, nodes, drawn, all);
            if (lane == 0) {
                if (was != 1 || (T.state == 2 && T.depth == depth)) T.state = 3;   // no child was left: the sums are those to draw from
                if (T.state == 3 && all == 0.0) {                                  // nothing is left, by rounding: the target's own distribution
                    const bool own = T.c == 0.0 && T.n_gone == 0;
                    T.c = 0.0;
                    T.n_gone = 0;
                    T.state = own ? 4 : 2;
                }
            }
        }
        __syncthreads();
        if (T.state >= 3) break;
    }
    be_done();
    if (chunk == 0) {
        for (int i = tid; i < nodes; i += kVerifyThreads) P.path[begin + i] = i < T.depth ? T.path[i] : -1;
        if (tid == 0) P.accepted[b] = T.depth;
        if (tid == 0 && T.state == 4) P.next[b] = -1;   // no mass at all
    }
    if (T.state == 4) return;
    if (wave == 0) {   // the chunk that holds the number, the last one with anything where rounding leaves it beyond all
        const double mine = lane < P.chunks ? T.part[lane] : 0.0, incl = wave_scan(mine), want = (double)T.u[0] * __shfl(incl, kWave - 1);
        const unsigned long long hit = __ballot(mine > 0.0 && incl > want), any = __ballot(mine > 0.0);
        const int chosen = hit ? __ffsll((long long)hit) - 1 : 63 - __clzll((long long)any);
        if (lane == chosen) {
            T.chosen = chosen;
            T.left = want - (incl - mine);
        }
    }
    __syncthreads();
    if (T.chosen != chunk) return;
    // in it: four numbers a thread at a time
    find_gone(P, T, chunk);
    const size_t row = (size_t)(begin + T.at) * P.vocab;
    const float *p = P.target + row, *q = draft_of(P, T, row);
    const int end = min((chunk + 1) * P.chunk, P.vocab);
    const double want = T.left, c = T.c;
    double below = 0.0;
    int found = -1;   // of this thread: the last number with anything
    unsigned long long gone = 0;
    for (int v0 = chunk * P.chunk, turn = 0;; v0 += kStep, ++turn) {
        const int v = v0 + tid * 4;
        if (turn % 16 == 0) gone = gone_of(T, v);
        const Four x = four_of(p, q, v, end, c, (uint32_t)(gone >> (turn % 16 * 4)));
        double to[4];
        to[0] = x.r[0];
#pragma unroll
        for (int j = 1; j < 4; ++j) to[j] = to[j - 1] + x.r[j];
#pragma unroll
        for (int j = 0; j < 4; ++j)
            if (x.r[j] > 0.0) found = v + j;
        const double incl = wave_scan(to[3]);
        __syncthreads();
        if (lane == kWave - 1) T.wave[wave] = incl;
        __syncthreads();
        double before = below + incl - to[3];
        for (int w = 0; w < wave; ++w) before += T.wave[w];
        int one = 0x7fffffff;
#pragma unroll
        for (int j = 3; j >= 0; --j)
            if (x.r[j] > 0.0 && before + to[j] > want) one = v + j;
        for (int w = 0; w < kVerifyWaves; ++w) below += T.wave[w];
        const unsigned long long hit = __ballot(one != 0x7fffffff);
        if (hit) one = __shfl(one, __ffsll((long long)hit) - 1);
        if (lane == 0) T.first[wave] = one;
        __syncthreads();
        int first = 0x7fffffff;
        for (int w = 0; w < kVerifyWaves; ++w) first = min(first, T.first[w]);
        if (first != 0x7fffffff) {
            if (tid == 0) P.next[b] = first;
            return;
        }
        if (v0 + kStep >= end) break;
    }
    // rounding has left it beyond all: the last number with anything
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) found = max(found, __shfl_xor(found, off));
    __syncthreads();
    if (lane == 0) T.first[wave] = found;
    __syncthreads();
    if (tid == 0) {
        for (int w = 1; w < kVerifyWaves; ++w) found = max(found, T.first[w]);
        P.next[b] = found;
    }
}

// ---------------------------------------------------------------------------------------
// Commit: bound by the latency of a chain of loads (length, path, pair); every accepted pair is read and written once.  A workgroup owns a row, or all
// heads of a sequence in pages: it alone reads and sets the length.  16 sequences, 8 heads, paths of up to 8 nodes: 3.2 us.
// ---------------------------------------------------------------------------------------
typedef unsigned int du32x4_t __attribute__((ext_vector_type(4)));

struct CommitParams {
    void *K, *V;
    int32_t *pos, *len;          // pages: len is kv_len
    float* acc;
    const void *k_tree, *v_tree;
    const int32_t *q_start, *path, *accepted, *pos_first;
    int n_tokens, batch, n_kv, cap;
    // pages
    const int32_t* table;
    int page_shift, n_pages, max_pages;
};

// nodes of the path, up to the first entry that is none; all lanes of the first wavefront
__device__ __forceinline__ int path_length(const CommitParams& P, int b, int begin, int nodes) {
    const int lane = threadIdx.x & (kWave - 1), n = min(max(P.accepted[b], 0), nodes);
    for (int i0 = 0; i0 < n; i0 += kWave) {
        const int node = i0 + lane < n ? P.path[begin + i0 + lane] : 0;
        const unsigned long long bad = __ballot(node < 0 || node >= nodes);
        if (bad) return i0 + __ffsll((long long)bad) - 1;
    }
    return n;
}

template <int CH>
__global__ __launch_bounds__(256) void commit_rows_kernel(const CommitParams P) {
    __shared__ int s_count;
    const int tid = threadIdx.x, row = blockIdx.x, b = row / P.n_kv, h = row - b * P.n_kv;
    const int begin = min(max(P.q_start[b], 0), P.n_tokens), nodes = min(max(P.q_start[b + 1], begin), P.n_tokens) - begin;
    const int start = P.len[row];
    if (tid < kWave) {
        const int n = path_length(P, b, begin, nodes);
        if (tid == 0) s_count = start < 0 ? 0 : min(n, max(P.cap - start, 0));
    }
    __syncthreads();
    const int n = s_count;
    const du32x4_t *k = reinterpret_cast<const du32x4_t*>(P.k_tree), *v = reinterpret_cast<const du32x4_t*>(P.v_tree);
    du32x4_t *K = reinterpret_cast<du32x4_t*>(P.K), *V = reinterpret_cast<du32x4_t*>(P.V);
    const int c = tid % CH;
    for (int i = tid / CH; i < n; i += 256 / CH) {
        const size_t from = ((size_t)(begin + P.path[begin + i]) * P.n_kv + h) * CH + c, to = ((size_t)row * P.cap + start + i) * CH + c;
        K[to] = k[from];
        V[to] = v[from];
    }
    const int first = P.pos_first[b];
    for (int i = tid; i < n; i += 256) {
        P.pos[(size_t)row * P.cap + start + i] = first + i;
        if (P.acc) P.acc[(size_t)row * P.cap + start + i] = 0.f;
    }
    if (tid == 0 && n > 0) P.len[row] = start + n;   // (this workgroup alone reads it)
}

template <int CH>
__global__ __launch_bounds__(1024) void commit_pages_kernel(const CommitParams P) {
    __shared__ int s_count;
    const int tid = threadIdx.x, b = blockIdx.x;
    const int begin = min(max(P.q_start[b], 0), P.n_tokens), nodes = min(max(P.q_start[b + 1], begin), P.n_tokens) - begin;
    const int start = P.len[b], most = P.max_pages << P.page_shift;
    if (tid < kWave) {
        const int n = path_length(P, b, begin, nodes);
        if (tid == 0) s_count = start < 0 ? 0 : min(n, max(most - start, 0));
    }
    __syncthreads();
    const int n = s_count, row = P.n_kv * CH;
    const du32x4_t *k = reinterpret_cast<const du32x4_t*>(P.k_tree), *v = reinterpret_cast<const du32x4_t*>(P.v_tree);
    du32x4_t *K = reinterpret_cast<du32x4_t*>(P.K), *V = reinterpret_cast<du32x4_t*>(P.V);
    // pair i of the path, 16 bytes hc of all its heads (together more than 32 bits count)
    for (int i = tid / row, hc = tid % row; i < n; i += 1024 / row, hc += 1024 % row) {
        if (hc >= row) {
            hc -= row;
            if (++i >= n) break;
        }
        const int h = hc / CH, p = start + i;
        const int page = P.table[(size_t)b * P.max_pages + (p >> P.page_shift)];
        if ((unsigned)page >= (unsigned)P.n_pages) continue;
        const size_t from = (size_t)(begin + P.path[begin + i]) * row + hc;
        const size_t to = ((((size_t)page * P.n_kv + h) << P.page_shift) + (p & ((1 << P.page_shift) - 1))) * CH + hc % CH;
        K[to] = k[from];
        V[to] = v[from];
    }
    if (tid == 0 && n > 0) P.len[b] = start + n;
}

// Chunks of 2048 numbers and more, up to 512 workgroups, two to a CU: all at work at once as a rule.
static int verify_chunks(int batch, int vocab) { return std::max(1, std::min(std::min(512 / batch, vocab / 2048), kMostChunks)); }

}  // namespace fk

using namespace fk;

extern "C" size_t fk_verify_drafts_workspace(int32_t batch, int32_t vocab) {
    if (batch <= 0 || vocab <= 0 || batch > 65535) return 0;
    // (a smaller batch has more chunks: the most workgroups of as many sequences or fewer)
    const int chunks = std::min(vocab / 2048, kMostChunks);
    return 256 + (chunks > 1 ? (size_t)std::min<int64_t>(512, (int64_t)batch * chunks) * kRounds * 2 * sizeof(unsigned long long) : 0);
}

extern "C" fk_status fk_verify_drafts(int32_t batch, int32_t vocab, const float* target, const float* draft, const int32_t* tokens,
                                      const int32_t* parent, const int32_t* q_start, int32_t n_tokens, const float* uniform, int32_t* path,
                                      int32_t* n_accepted, int32_t* next_token, void* workspace, size_t workspace_bytes, void* stream) {
    if (batch <= 0 || vocab <= 0 || n_tokens < 0) return FK_ERR_INVALID_ARG;
    if (vocab >= (1 << 30) || batch > 65535) return FK_ERR_UNSUPPORTED;
    if (!q_start || !n_accepted || !next_token) return FK_ERR_INVALID_ARG;
    if (n_tokens > 0 && (!target || !tokens || !parent || !uniform || !path)) return FK_ERR_INVALID_ARG;
    if (!workspace || workspace_bytes < fk_verify_drafts_workspace(batch, vocab) || !aligned16(workspace)) return FK_ERR_WORKSPACE;
    VerifyParams P = {target, draft, tokens, parent, q_start, uniform, path, n_accepted, next_token, n_tokens, batch, vocab, verify_chunks(batch, vocab), 0, nullptr, nullptr, nullptr};
    P.chunk = ((vocab + P.chunks - 1) / P.chunks + 3) / 4 * 4;
    P.call = static_cast<uint32_t*>(workspace);
    P.done = P.call + 1;
    P.told = reinterpret_cast<unsigned long long*>(static_cast<char*>(workspace) + 256);
    hipLaunchKernelGGL(verify_kernel, dim3(P.chunks, batch), dim3(kVerifyThreads), 0, (hipStream_t)stream, P);
    return launch_status();
}

extern "C" fk_status fk_commit_drafts(const fk_cache_desc* desc, void* K, void* V, int32_t* pos, int32_t* len, float* acc, const void* k_tree,
                                      const void* v_tree, const int32_t* q_start, int32_t n_tokens, const int32_t* path, const int32_t* n_accepted,
                                      const int32_t* pos_first, void* stream) {
    const fk_status s = check_desc(desc);
    if (s != FK_OK) return s;
    if ((int64_t)desc->batch * desc->n_kv_heads >= (1 << 24)) return FK_ERR_UNSUPPORTED;
    if (n_tokens < 0 || !K || !V || !pos || !len || !q_start || !n_accepted || !pos_first) return FK_ERR_INVALID_ARG;
    if (n_tokens > 0 && (!k_tree || !v_tree || !path)) return FK_ERR_INVALID_ARG;
    if (!aligned16(K) || !aligned16(V) || !aligned16(k_tree) || !aligned16(v_tree)) return FK_ERR_INVALID_ARG;
    if (n_tokens == 0) return FK_OK;
    CommitParams P = {};
    P.K = K;
    P.V = V;
    P.pos = pos;
    P.len = len;
    P.acc = acc;
    P.k_tree = k_tree;
    P.v_tree = v_tree;
    P.q_start = q_start;
    P.path = path;
    P.accepted = n_accepted;
    P.pos_first = pos_first;
    P.n_tokens = n_tokens;
    P.batch = desc->batch;
    P.n_kv = desc->n_kv_heads;
    P.cap = desc->capacity;
    const dim3 grid(desc->batch * desc->n_kv_heads);
    hipStream_t st = (hipStream_t)stream;
    switch (desc->head_dim * (desc->dtype == FK_F32 ? 4 : 2) / 16) {
        case 8: hipLaunchKernelGGL(commit_rows_kernel<8>, grid, dim3(256), 0, st, P); break;
        case 16: hipLaunchKernelGGL(commit_rows_kernel<16>, grid, dim3(256), 0, st, P); break;
        default: hipLaunchKernelGGL(commit_rows_kernel<32>, grid, dim3(256), 0, st, P); break;
    }
    return launch_status();
}

extern "C" fk_status fk_paged_commit_drafts(const fk_paged_desc* desc, void* K, void* V, const int32_t* page_table, int32_t* kv_len,
                                            const void* k_tree, const void* v_tree, const int32_t* q_start, int32_t n_tokens,
                                            const int32_t* path, const int32_t* n_accepted, void* stream) {
    const fk_status s = check_paged(desc);
    if (s != FK_OK) return s;
    if (desc->n_kv_heads >= (1 << 16)) return FK_ERR_UNSUPPORTED;
    if (n_tokens < 0 || !K || !V || !page_table || !kv_len || !q_start || !n_accepted) return FK_ERR_INVALID_ARG;
    if (n_tokens > 0 && (!k_tree || !v_tree || !path)) return FK_ERR_INVALID_ARG;
    if (!aligned16(K) || !aligned16(V) || !aligned16(k_tree) || !aligned16(v_tree)) return FK_ERR_INVALID_ARG;
    if (n_tokens == 0) return FK_OK;
    CommitParams P = {};
    P.K = K;
    P.V = V;
    P.len = kv_len;
    P.k_tree = k_tree;
    P.v_tree = v_tree;
    P.q_start = q_start;
    P.path = path;
    P.accepted = n_accepted;
    P.n_tokens = n_tokens;
    P.batch = desc->batch;
    P.n_kv = desc->n_kv_heads;
    P.table = page_table;
    P.page_shift = __builtin_ctz(desc->page_size);
    P.n_pages = desc->n_pages;
    P.max_pages = desc->max_pages;
    hipStream_t st = (hipStream_t)stream;
    switch (desc->head_dim * (desc->dtype == FK_F32 ? 4 : 2) / 16) {
        case 8: hipLaunchKernelGGL(commit_pages_kernel<8>, dim3(desc->batch), dim3(1024), 0, st, P); break;
        case 16: hipLaunchKernelGGL(commit_pages_kernel<16>, dim3(desc->batch), dim3(1024), 0, st, P); break;
        default: hipLaunchKernelGGL(commit_pages_kernel<32>, dim3(desc->batch), dim3(1024), 0, st, P); break;
    }
    return launch_status();
}
