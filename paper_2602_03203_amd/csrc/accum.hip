// fk_decode_step_acc: the decode step that adds its attention weights to those that the retained pairs have accumulated.
// The plain form: the step, then a workgroup per row that forms the logits once more.
#include "fk_common.h"

namespace fk {

template <typename T> __device__ __forceinline__ float load_one(const T* p);
template <> __device__ __forceinline__ float load_one<float>(const float* p) { return *p; }
template <> __device__ __forceinline__ float load_one<bf16_t>(const bf16_t* p) { return bf16_lo(*p); }

template <typename T>
__global__ __launch_bounds__(256) void acc_plain_kernel(const T* q, const T* K, const int32_t* len, float* acc, float* logit, float scale, int g, int D, int cap,
                                                        const int32_t* old_len) {
    const int row = blockIdx.x, tid = threadIdx.x, n = min(max(len[row], 0), cap), fresh = old_len[row] < n ? n - 1 : n;
    __shared__ float s_red[256];
    float* lg = logit + (size_t)row * cap;
    for (int h = 0; h < g; ++h) {
        const T* qr = q + ((size_t)row * g + h) * D;
        float mx = -INFINITY, sum = 0.f;
        for (int j = tid; j < n; j += 256) {
            float s = 0.f;
            for (int e = 0; e < D; ++e) s = fmaf(load_one(qr + e), load_one(K + ((size_t)row * cap + j) * D + e), s);
            lg[j] = s * scale;
            mx = fmaxf(mx, s * scale);
        }
        s_red[tid] = mx;
        __syncthreads();
        for (int w = 128; w; w /= 2) {
            if (tid < w) s_red[tid] = fmaxf(s_red[tid], s_red[tid + w]);
            __syncthreads();
        }
        mx = s_red[0];
        __syncthreads();
        for (int j = tid; j < n; j += 256) sum += exp2f(lg[j] - mx);
        s_red[tid] = sum;
        __syncthreads();
        for (int w = 128; w; w /= 2) {
            if (tid < w) s_red[tid] += s_red[tid + w];
            __syncthreads();
        }
        sum = s_red[0];
        __syncthreads();
        float* a = acc + (size_t)row * cap;
        for (int j = tid; j < n; j += 256) a[j] = (h == 0 && j == fresh ? 0.f : a[j]) + exp2f(lg[j] - mx) / sum;
    }
}

__global__ void acc_lengths_kernel(const int32_t* len, int32_t* to, int rows) {
    const int r = blockIdx.x * 256 + threadIdx.x;
    if (r < rows) to[r] = len[r];
}
__global__ void acc_clear_kernel(uint32_t* p, size_t n) {
    for (size_t i = (size_t)blockIdx.x * 256 + threadIdx.x; i < n; i += (size_t)gridDim.x * 256) p[i] = 0;
}

}  // namespace fk

using namespace fk;

// decode workspace | row lengths before the step | logits
static size_t align256(size_t n) { return (n + 255) / 256 * 256; }

extern "C" size_t fk_decode_step_acc_workspace(const fk_cache_desc* desc) {
    if (check_desc(desc) != FK_OK) return 0;
    const size_t rows = (size_t)desc->batch * desc->n_kv_heads;
    return align256(fk_decode_attn_workspace(desc, desc->capacity)) + align256(rows * 4) + rows * desc->capacity * 4;
}

extern "C" fk_status fk_decode_step_acc(const fk_cache_desc* desc, const void* q, void* K, void* V, int32_t* pos, int32_t* len,
                                        const void* k_new, const void* v_new, const int32_t* pos_new, int32_t max_len,
                                        float softmax_scale, float* acc, void* out, void* workspace, size_t workspace_bytes, void* stream) {
    fk_status s = check_desc(desc);
    if (s != FK_OK) return s;
    if (!q || !K || !V || !pos || !len || !k_new || !v_new || !pos_new || !acc || !out) return FK_ERR_INVALID_ARG;
    if (!aligned16(q) || !aligned16(K) || !aligned16(V) || !aligned16(out) || !aligned16(k_new) || !aligned16(v_new) || !aligned16(acc)) return FK_ERR_INVALID_ARG;
    if (max_len <= 0 || max_len > desc->capacity) return FK_ERR_INVALID_ARG;
    if (!workspace || workspace_bytes < fk_decode_step_acc_workspace(desc) || !aligned16(workspace)) return FK_ERR_WORKSPACE;
    const size_t step_ws = align256(fk_decode_attn_workspace(desc, desc->capacity));
    const int rows = desc->batch * desc->n_kv_heads;
    hipStream_t st = (hipStream_t)stream;
    int32_t* old_len = reinterpret_cast<int32_t*>((char*)workspace + step_ws);
    float* logit = reinterpret_cast<float*>((char*)workspace + step_ws + align256((size_t)rows * 4));
    hipLaunchKernelGGL(acc_clear_kernel, dim3(64), dim3(256), 0, st, (uint32_t*)workspace, step_ws / 4);
    hipLaunchKernelGGL(acc_lengths_kernel, dim3((rows + 255) / 256), dim3(256), 0, st, len, old_len, rows);
    s = fk_decode_step(desc, q, K, V, pos, len, k_new, v_new, pos_new, max_len, softmax_scale, out, workspace, step_ws, stream);
    if (s != FK_OK) return s;
    const int g = desc->n_q_heads / desc->n_kv_heads;
    const float scale = softmax_scale * 1.4426950408889634f;
    if (desc->dtype == FK_F32)
        hipLaunchKernelGGL(acc_plain_kernel<float>, dim3(rows), dim3(256), 0, st, (const float*)q, (const float*)K, len, acc, logit, scale, g, desc->head_dim, desc->capacity, old_len);
    else
        hipLaunchKernelGGL(acc_plain_kernel<bf16_t>, dim3(rows), dim3(256), 0, st, (const bf16_t*)q, (const bf16_t*)K, len, acc, logit, scale, g, desc->head_dim, desc->capacity, old_len);
    return launch_status();
}
