// fk_rope: rotary positions of queries and keys.
//
// A pair of channels (u, w) of a token at position p turns by the angle p * freq: (u cos - w sin, u sin + w cos), times a magnitude.  Angles of far
// positions have no fraction left in 32 bits (from 2^23 radians on), so they are formed in 64, in turns, and reduced to half a turn before
// they become 32 bits (off by 2^-25 of a turn at most).  A workgroup takes a few tokens: sine and cosine once for every pair
// of channels, in LDS, then all heads of these tokens pass by, 16 bytes a thread and load.
// Bound by the memory system: every element is read and written once.  65000 tokens of 40 heads of 128 channels (1.33 GB) 253 us, 5.3 TB/s (a copy of 2 GiB 4.9);
// 4096 tokens 15 us; 16 tokens 3.8, a launch and two loads one after the other.  Where rotated channels are no whole 16-byte groups (50 of 128) a thread takes a pair of channels or
// copies one, 2 or 4 bytes a load, bound by the number of its loads: 16384 tokens 177 us (interleaved 173), 66 where all 128 turn.
#include "paged.h"

#include <cmath>

namespace fk {

struct RopeParams {
    const void *q, *k;
    void *q_out, *k_out;
    const int32_t* pos;
    const double* freq;
    long long q_stride, k_stride, qo_stride, ko_stride;   // elements from token to token
    int n_tokens, hq, heads, dim, rot, tokens;            // tokens: of a workgroup
    uint32_t token_magic, unit_magic, pair_magic;         // for divisions by a token's units, a head's, the pairs of channels
    float magnitude;
    bool inverse, q_copy, k_copy;                         // copy: the channels behind the rotated ones go into another tensor
};

template <typename T> __device__ __forceinline__ void store16(T* p, const float* f) {
    if constexpr (sizeof(T) == 2) *reinterpret_cast<uint4*>(p) = make_uint4(pack_bf16(f[0], f[1]), pack_bf16(f[2], f[3]), pack_bf16(f[4], f[5]), pack_bf16(f[6], f[7]));
    else *reinterpret_cast<float4*>(p) = make_float4(f[0], f[1], f[2], f[3]);
}
__device__ __forceinline__ float load_in(const float* p) { return *p; }
__device__ __forceinline__ float load_in(const bf16_t* p) { return __uint_as_float((uint32_t)*p << 16); }

template <typename T> __device__ __forceinline__ T copy_of(uint32_t x) {   // what load_in's bits came from, a NaN's own ones among them
    if constexpr (sizeof(T) == 2) return (T)(x >> 16);
    else return __uint_as_float(x);
}

// VEC: whole 16-byte groups turn together; otherwise a thread turns one pair of channels or copies one channel.  A thread's units are two turns' loads ahead
// of their stores.
template <typename T, bool VEC, bool HALF>
__global__ __launch_bounds__(256) void rope_kernel(const RopeParams P) {
    extern __shared__ float2 s_turn[];   // [tokens][rot / 2] (cos, sin) times the magnitude
    constexpr int N = VEC ? Vec16<T>::N : 1, U = !VEC ? 2 : HALF ? 4 : 8;   // units of a thread under way: eight loads
    const int tid = threadIdx.x, pairs = P.rot / 2, t0 = blockIdx.x * P.tokens, tokens = min(P.tokens, P.n_tokens - t0);
    // units of a head: those that turn, then those that are copied
    const int turning = VEC ? (HALF ? pairs / N : P.rot / N) : pairs, units = turning + (P.q_copy || P.k_copy ? (P.dim - P.rot) / N : 0);
    const int per_token = P.heads * units, all = tokens * per_token;
    struct Unit {
        T* y;
        int t, u;              // u < 0: nothing to do
        uint4 a, b;
    };
    auto fetch = [&](int i) {
        Unit x;
        x.u = -1;
        if (i >= all) return x;
        const int t = divide(i, per_token, P.token_magic), r = i - t * per_token, h = divide(r, units, P.unit_magic), u = r - h * units;
        const bool is_q = h < P.hq;
        if (u >= turning && !(is_q ? P.q_copy : P.k_copy)) return x;
        const size_t token = (size_t)(t0 + t);
        const T* from = is_q ? reinterpret_cast<const T*>(P.q) + token * P.q_stride + (size_t)h * P.dim : reinterpret_cast<const T*>(P.k) + token * P.k_stride + (size_t)(h - P.hq) * P.dim;
        x.y = is_q ? reinterpret_cast<T*>(P.q_out) + token * P.qo_stride + (size_t)h * P.dim : reinterpret_cast<T*>(P.k_out) + token * P.ko_stride + (size_t)(h - P.hq) * P.dim;
        x.t = t;
        x.u = u;
        if constexpr (VEC) {
            const int d = u < turning ? u * N : P.rot + (u - turning) * N;
            x.a = *reinterpret_cast<const uint4*>(from + d);
            if (HALF && u < turning) x.b = *reinterpret_cast<const uint4*>(from + d + pairs);
        } else {
            const int a = u >= turning ? P.rot + u - turning : HALF ? u : 2 * u;
            x.a.x = __float_as_uint(load_in(from + a));
            if (u < turning) x.b.x = __float_as_uint(load_in(from + (HALF ? a + pairs : a + 1)));
        }
        return x;
    };
    auto finish = [&](const Unit& x) {
        if (x.u < 0) return;
        const float2* turn = s_turn + x.t * pairs;
        if constexpr (VEC) {
            if (x.u >= turning) {
                *reinterpret_cast<uint4*>(x.y + P.rot + (x.u - turning) * N) = x.a;
                return;
            }
            float v[N], w[N];
            Vec16<T>::unpack(x.a, v);
            if constexpr (HALF) {
                Vec16<T>::unpack(x.b, w);
#pragma unroll
                for (int j = 0; j < N; ++j) {
                    const float2 cs = turn[x.u * N + j];
                    const float a = v[j] * cs.x - w[j] * cs.y;
                    w[j] = v[j] * cs.y + w[j] * cs.x;
                    v[j] = a;
                }
                store16(x.y + x.u * N, v);
                store16(x.y + pairs + x.u * N, w);
            } else {
#pragma unroll
                for (int j = 0; j < N; j += 2) {
                    const float2 cs = turn[x.u * (N / 2) + j / 2];
                    const float a = v[j] * cs.x - v[j + 1] * cs.y;
                    v[j + 1] = v[j] * cs.y + v[j + 1] * cs.x;
                    v[j] = a;
                }
                store16(x.y + x.u * N, v);
            }
        } else {
            const float v = __uint_as_float(x.a.x);
            if (x.u >= turning) {
                x.y[P.rot + x.u - turning] = copy_of<T>(x.a.x);
                return;
            }
            const float w = __uint_as_float(x.b.x);
            const int a = HALF ? x.u : 2 * x.u, b = HALF ? a + pairs : a + 1;
            const float2 cs = turn[x.u];
            store_out(x.y + a, v * cs.x - w * cs.y);
            store_out(x.y + b, v * cs.y + w * cs.x);
        }
    };
    Unit x[U];
#pragma unroll
    for (int k = 0; k < U; ++k) x[k] = fetch(tid + k * 256);   // (on their way while the angles are formed)
    for (int i = tid; i < tokens * pairs; i += 256) {
        const int t = divide(i, pairs, P.pair_magic);
        double turns = (double)P.pos[t0 + t] * (P.freq[i - t * pairs] * 0.15915494309189535);
        turns -= rint(turns);
        float s, c;
        sincospif(2.f * (float)turns, &s, &c);
        s_turn[i] = make_float2(c * P.magnitude, (P.inverse ? -s : s) * P.magnitude);
    }
    __syncthreads();
    for (int i = tid;;) {
#pragma unroll
        for (int k = 0; k < U; ++k) finish(x[k]);
        i += U * 256;
        if (i >= all) break;
#pragma unroll
        for (int k = 0; k < U; ++k) x[k] = fetch(i + k * 256);
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
    if (d->n_q_heads && q && q == q_out && P.q_stride != P.qo_stride) return FK_ERR_INVALID_ARG;
    if (d->n_kv_heads && k && k == k_out && P.k_stride != P.ko_stride) return FK_ERR_INVALID_ARG;
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
    const bool half = d->layout == FK_ROPE_HALF;
    P.q_copy = q != q_out;
    P.k_copy = k != k_out;
    P.tokens = n_tokens >= 2048 ? 4 : 1;
    const bool vec = (half ? P.rot / 2 : P.rot) * es % 16 == 0;
    const int n = vec ? 16 / es : 1, turning = vec && !half ? P.rot / n : P.rot / 2 / n, units = turning + (P.q_copy || P.k_copy ? (P.dim - P.rot) / n : 0);
    P.token_magic = magic_of(P.heads * units);
    P.unit_magic = magic_of(units);
    P.pair_magic = magic_of(P.rot / 2);
    const dim3 grid((unsigned)((n_tokens + P.tokens - 1) / P.tokens));
    const size_t lds = (size_t)P.tokens * P.rot / 2 * sizeof(float2);
    hipStream_t st = (hipStream_t)stream;
    auto kern = d->dtype == FK_F32 ? (vec ? (half ? rope_kernel<float, true, true> : rope_kernel<float, true, false>) : half ? rope_kernel<float, false, true> : rope_kernel<float, false, false>)
                                   : (vec ? (half ? rope_kernel<bf16_t, true, true> : rope_kernel<bf16_t, true, false>) : half ? rope_kernel<bf16_t, false, true> : rope_kernel<bf16_t, false, false>);
    hipLaunchKernelGGL(kern, grid, dim3(256), lds, st, P);
    return launch_status();
}
