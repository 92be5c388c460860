// fk_decode_step_acc: the decode step that adds its attention weights to those that the retained pairs have accumulated (thin.h).
#include "attn_paged.h"
#include <climits>
#include <cmath>

using namespace fk;

extern "C" size_t fk_decode_step_acc_workspace(const fk_cache_desc* desc) {
    if (check_desc(desc) != FK_OK) return 0;
    return thin_rows_workspace(desc);
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
    AttnPagedParams P = {};
    P.view.q = q;
    P.view.K = K;
    P.view.V = V;
    P.view.batch = desc->batch * desc->n_kv_heads;
    P.view.n_kv = 1;
    P.view.g = desc->n_q_heads / desc->n_kv_heads;
    P.view.window = INT_MAX;
    P.view.negate = std::signbit(softmax_scale);
    P.view.scale_log2e = base2_scale(softmax_scale);
    P.out = out;
    P.cap = desc->capacity;
    P.pos = pos;
    P.len = len;
    P.pos_new = pos_new;
    P.k_new = k_new;
    P.v_new = v_new;
    P.batch_of_pos = desc->n_kv_heads;
    P.acc = acc;
    return thin_rows(desc, P, max_len, workspace, (hipStream_t)stream);
}
