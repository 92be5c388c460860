// fk_rope: rotary positions of queries and keys.
//
// A pair of channels (u, w) of a token at position p turns by the angle p * freq: (u cos - w sin, u sin + w cos), times a magnitude.  Angles of far
// positions lose their fraction in 32 bits (2^23 radians: 1 of 1), so they are formed in 64, in turns, and reduced to half a turn before
// they become 32 bits (off by 2^-25 of a turn at most).  A workgroup takes a few tokens: sine and cosine once for every pair
// of channels, in LDS, then all heads of these tokens pass by, 16 bytes a thread and load.
// Bound by the memory system: every element is read and written once.
#include "fk_common.h"

#include <cmath>

namespace fk {

typedef unsigned int ru32x4_t __attribute__((ext_vector_type(4)));

struct RopeParams {
    const void *q, *k;
    void *q_out, *k_out;
    const int32_t* pos;
    const double* freq;
    long long q_stride, k_stride, qo_stride, ko_stride;   // elements from token to token
    int n_tokens, hq, heads, dim, rot, tokens /* of a workgroup */, parts /* workgroups of the same tokens: each takes a share of the heads */;
    float magnitude;
    bool inverse, half, q_copy, k_copy;                   // copy: the channels behind the rotated ones go into another tensor
};

template <typename T> __device__ __forceinline__ void store16(T* p, const float* f) {
    if constexpr (sizeof(T) == 2) *reinterpret_cast<ru32x4_t*>(p) = ru32x4_t{pack_bf16(f[0], f[1]), pack_bf16(f[2], f[3]), pack_bf16(f[4], f[5]), pack_bf16(f[6], f[7])};
    else *reinterpret_cast<float4*>(p) = make_float4(f[0], f[1], f[2], f[3]);
}
__device__ __forceinline__ float load_in(const float* p) { return *p; }
__device__ __forceinline__ float load_in(const bf16_t* p) { return __uint_as_float((uint32_t)*p << 16); }

// VEC: whole 16-byte groups turn together; otherwise a thread turns one pair of channels or copies one channel
template <typename T, bool VEC>
__global__ __launch_bounds__(256) void rope_kernel(const RopeParams P) {
    extern __shared__ float2 s_turn[];   // [tokens][rot / 2] (cos, sin) times the magnitude
    const int tid = threadIdx.x, pairs = P.rot / 2, t0 = blockIdx.x / P.parts * P.tokens, part = blockIdx.x % P.parts, tokens = min(P.tokens, P.n_tokens - t0);
    for (int i = tid; i < tokens * pairs; i += 256) {
        const int t = i / pairs;
        double turns = (double)P.pos[t0 + t] * (P.freq[i - t * pairs] * 0.15915494309189535);
        turns -= rint(turns);
        float s, c;
        sincospif(2.f * (float)turns, &s, &c);
        s_turn[i] = make_float2(c * P.magnitude, (P.inverse ? -s : s) * P.magnitude);
    }
    __syncthreads();
    constexpr int N = VEC ? Vec16<T>::N : 1;
    // units of a head: those that turn, then those that are copied
    const int turning = VEC ? (P.half ? pairs / N : P.rot / N) : pairs, units = turning + (P.q_copy || P.k_copy ? (P.dim - P.rot) / N : 0);
    const int first = P.heads * part / P.parts, heads = P.heads * (part + 1) / P.parts - first;
    const int all = tokens * heads * units;
    for (int i = tid; i < all; i += 256) {
        const int u = i % units, th = i / units, h = first + th % heads, t = th / heads;
        const bool is_q = h < P.hq;
        const T* x = (is_q ? reinterpret_cast<const T*>(P.q) + (t0 + t) * P.q_stride : reinterpret_cast<const T*>(P.k) + (t0 + t) * P.k_stride) + (size_t)(is_q ? h : h - P.hq) * P.dim;
        T* y = (is_q ? reinterpret_cast<T*>(P.q_out) + (t0 + t) * P.qo_stride : reinterpret_cast<T*>(P.k_out) + (t0 + t) * P.ko_stride) + (size_t)(is_q ? h : h - P.hq) * P.dim;
        const float2* turn = s_turn + t * pairs;
        if (u >= turning) {
            if (!(is_q ? P.q_copy : P.k_copy)) continue;
            const int d = P.rot + (u - turning) * N;
            if constexpr (VEC) *reinterpret_cast<ru32x4_t*>(y + d) = *reinterpret_cast<const ru32x4_t*>(x + d);
            else y[d] = x[d];
            continue;
        }
        if constexpr (!VEC) {
            const int a = P.half ? u : 2 * u, b = P.half ? u + pairs : a + 1;
            const float v = load_in(x + a), w = load_in(x + b);
            const float2 cs = turn[u];
            store_out(y + a, v * cs.x - w * cs.y);
            store_out(y + b, v * cs.y + w * cs.x);
        } else if (P.half) {
            float v[N], w[N];
            Vec16<T>::unpack(*reinterpret_cast<const uint4*>(x + u * N), v);
            Vec16<T>::unpack(*reinterpret_cast<const uint4*>(x + pairs + u * N), w);
#pragma unroll
            for (int j = 0; j < N; ++j) {
                const float2 cs = turn[u * N + j];
                const float a = v[j] * cs.x - w[j] * cs.y;
                w[j] = v[j] * cs.y + w[j] * cs.x;
                v[j] = a;
            }
            store16(y + u * N, v);
            store16(y + pairs + u * N, w);
        } else {
            float v[N];
            Vec16<T>::unpack(*reinterpret_cast<const uint4*>(x + u * N), v);
#pragma unroll
            for (int j = 0; j < N; j += 2) {
                const float2 cs = turn[u * (N / 2) + j / 2];
                const float a = v[j] * cs.x - v[j + 1] * cs.y;
                v[j + 1] = v[j] * cs.y + v[j + 1] * cs.x;
                v[j] = a;
            }
            store16(y + u * N, v);
        }
    }
}

}  // namespace fk

using namespace fk;

extern "C" fk_status fk_rope_frequencies(int32_t rotary_dim, double base, int32_t scaling, double factor, double context, double low, double high,
                                         double* freq) {
    if (rotary_dim <= 0 || rotary_dim % 2 || !freq || !(base > 0) || !std::isfinite(base)) return FK_ERR_INVALID_ARG;
    if (scaling != FK_ROPE_PLAIN && (!(factor > 0) || !std::isfinite(factor))) return FK_ERR_INVALID_ARG;
    if (scaling == FK_ROPE_PARTS && (!(context > 0) || !(low >= 0) || !(high > low) || !std::isfinite(context) || !std::isfinite(high))) return FK_ERR_INVALID_ARG;
    if (scaling < FK_ROPE_PLAIN || scaling > FK_ROPE_PARTS) return FK_ERR_UNSUPPORTED;
    if (scaling == FK_ROPE_BASE && rotary_dim > 2) base *= std::pow(factor, rotary_dim / (rotary_dim - 2.0));
    for (int32_t i = 0; i < rotary_dim / 2; ++i) {
        double f = std::pow(base, -2.0 * i / rotary_dim);
        if (scaling == FK_ROPE_LINEAR) f /= factor;
        if (scaling == FK_ROPE_PARTS) {
            const double turns = context * f / 6.283185307179586;   // of this pair over the context it was trained on
            const double keep = turns <= low ? 0.0 : turns >= high ? 1.0 : (turns - low) / (high - low);
            f *= keep + (1.0 - keep) / factor;
        }
        freq[i] = f;
    }
    return FK_OK;
}

extern "C" fk_status fk_rope(const fk_rope_desc* d, const void* q, const void* k, const int32_t* pos, const double* freq, int32_t n_tokens,
                             void* q_out, void* k_out, void* stream) {
    if (!d || d->n_q_heads < 0 || d->n_kv_heads < 0 || d->n_q_heads + (int64_t)d->n_kv_heads <= 0 || d->head_dim <= 0 || n_tokens < 0) return FK_ERR_INVALID_ARG;
    if (d->rotary_dim <= 0 || d->rotary_dim % 2 || d->rotary_dim > d->head_dim || !std::isfinite(d->magnitude)) return FK_ERR_INVALID_ARG;
    if (d->dtype != FK_F32 && d->dtype != FK_BF16) return FK_ERR_UNSUPPORTED;
    if (d->layout != FK_ROPE_HALF && d->layout != FK_ROPE_INTERLEAVED) return FK_ERR_UNSUPPORTED;
    if (d->head_dim != 64 && d->head_dim != 128) return FK_ERR_UNSUPPORTED;
    if ((int64_t)d->n_q_heads + d->n_kv_heads >= (1 << 16)) return FK_ERR_UNSUPPORTED;
    const int es = d->dtype == FK_F32 ? 4 : 2;
    const long long q_row = (long long)d->n_q_heads * d->head_dim, k_row = (long long)d->n_kv_heads * d->head_dim;
    RopeParams P = {};
    P.q_stride = d->q_stride ? d->q_stride : q_row;
    P.k_stride = d->k_stride ? d->k_stride : k_row;
    P.qo_stride = d->q_out_stride ? d->q_out_stride : q_row;
    P.ko_stride = d->k_out_stride ? d->k_out_stride : k_row;
    if (P.q_stride < q_row || P.qo_stride < q_row || P.k_stride < k_row || P.ko_stride < k_row) return FK_ERR_INVALID_ARG;
    if ((P.q_stride | P.qo_stride | P.k_stride | P.ko_stride) * es % 16) return FK_ERR_INVALID_ARG;
    if (n_tokens > 0 && (!pos || !freq || (d->n_q_heads && (!q || !q_out)) || (d->n_kv_heads && (!k || !k_out)))) return FK_ERR_INVALID_ARG;
    if (!aligned16(q) || !aligned16(k) || !aligned16(q_out) || !aligned16(k_out) || (reinterpret_cast<uintptr_t>(freq) & 7)) return FK_ERR_INVALID_ARG;
    if ((q == q_out && P.q_stride != P.qo_stride) || (k == k_out && P.k_stride != P.ko_stride)) {
        if ((q && q == q_out && d->n_q_heads) || (k && k == k_out && d->n_kv_heads)) return FK_ERR_INVALID_ARG;
    }
    if (n_tokens == 0) return FK_OK;
    P.q = q;
    P.k = k;
    P.q_out = q_out;
    P.k_out = k_out;
    P.pos = pos;
    P.freq = freq;
    P.n_tokens = n_tokens;
    P.hq = d->n_q_heads;
    P.heads = d->n_q_heads + d->n_kv_heads;
    P.dim = d->head_dim;
    P.rot = d->rotary_dim;
    P.magnitude = d->magnitude;
    P.inverse = d->inverse != 0;
    P.half = d->layout == FK_ROPE_HALF;
    P.q_copy = q != q_out;
    P.k_copy = k != k_out;
    P.tokens = n_tokens >= 2048 ? 4 : 1;
    P.parts = 1;
    const bool vec = (P.half ? P.rot / 2 : P.rot) * es % 16 == 0;
    const dim3 grid((unsigned)((n_tokens + P.tokens - 1) / P.tokens) * P.parts);
    const size_t lds = (size_t)P.tokens * P.rot / 2 * sizeof(float2);
    hipStream_t st = (hipStream_t)stream;
    if (d->dtype == FK_F32) {
        if (vec) hipLaunchKernelGGL((rope_kernel<float, true>), grid, dim3(256), lds, st, P);
        else hipLaunchKernelGGL((rope_kernel<float, false>), grid, dim3(256), lds, st, P);
    } else {
        if (vec) hipLaunchKernelGGL((rope_kernel<bf16_t, true>), grid, dim3(256), lds, st, P);
        else hipLaunchKernelGGL((rope_kernel<bf16_t, false>), grid, dim3(256), lds, st, P);
    }
    return launch_status();
}
