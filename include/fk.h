/*
 * fk — budgeted KV-cache decoding with learned eviction (ForesightKV generation path)
 * for AMD MI355X (gfx950).  C ABI; every kernel behind it is hand-written HIP.
 *
 * The path (Section 3.1 of the paper, "Dynamic KV Cache Eviction During Long-Context
 * Generation"): the cache holds at most B + L pairs per (sequence, KV head).  Every
 * decode step appends the new pair (fk_append) and attends over the retained pairs
 * (fk_decode_attn).  After every L steps the retained pairs are scored by an MLP
 * (fk_score_kv), the L newest plus the B - L most important others are selected
 * (fk_select_keep) and the cache is compacted back to B entries (fk_compact).
 *
 * Memory layout (row major, all DEVICE memory owned by the caller):
 *   K, V   [batch][n_kv_heads][capacity][head_dim]   dtype (fp32 or bf16)
 *   pos    [batch][n_kv_heads][capacity]             int32 absolute position of each slot
 *   len    [batch][n_kv_heads]                       int32 retained count of each row
 * A (sequence, KV head) pair is called a row; row index r = b * n_kv_heads + h.  Slots
 * 0 .. len[r]-1 of a row are live.  Every row carries its own count (each KV head keeps its own
 * retained set); under one budget for all heads the counts of a sequence are equal.
 * Precondition kept by fk_append and fk_compact: along the live slots of a row the
 * positions are strictly increasing, so slot order is position order.
 *
 * Conventions:
 *   - descriptor structs are HOST memory, read during the call only;
 *   - all other pointers are DEVICE pointers, 16-byte aligned, owned by the caller;
 *   - `stream` is a hipStream_t passed as void* (NULL = the null stream); every call
 *     only enqueues work on it and returns; nothing is allocated.  The only state the library keeps is per
 *     device and invisible to results: flags "this kernel's dynamic-LDS limit has been raised" and, for
 *     fk_decode_step_static, the address of its fixed scratch array;
 *   - errors are return codes; arguments are validated on the host before any launch;
 *   - `max_len` is a host-side upper bound on every len[r] at the time the kernels run
 *     (pass `capacity` when unknown); it only sizes the launch.  Every call stays correct when a row is longer
 *     than max_len (the last workgroup of the row runs on to the row's end: slower, same results).
 *   - supported: head_dim 64 or 128; dtype fp32 or bf16; n_q_heads a multiple of
 *     n_kv_heads with group size <= 8; capacity < 2^24.
 */
#ifndef FK_H
#define FK_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum {
    FK_OK = 0,
    FK_ERR_INVALID_ARG = 1, /* null pointer, non-positive size, inconsistent sizes */
    FK_ERR_UNSUPPORTED = 2, /* shape or dtype outside the supported set */
    FK_ERR_WORKSPACE = 3,   /* workspace missing or too small */
    FK_ERR_LAUNCH = 4       /* the HIP runtime refused a launch */
} fk_status;

typedef enum { FK_F32 = 0, FK_BF16 = 1 } fk_dtype;

typedef struct {
    int32_t batch;      /* sequences */
    int32_t n_q_heads;  /* query heads per sequence */
    int32_t n_kv_heads; /* KV heads per sequence; group size g = n_q_heads / n_kv_heads */
    int32_t head_dim;   /* D */
    int32_t capacity;   /* slots per row, >= B + L */
    int32_t dtype;      /* fk_dtype of q, K, V, out and of the scorer's W1 */
    int32_t flags;      /* FK_CACHE_* bits, 0 by default */
} fk_cache_desc;

/* The cache is not expected to sit in the GPU's caches when a call starts (one layer of a deep stack whose
 * layers are visited in turn): attention streams K and V with non-temporal loads whatever their size.  Without
 * the flag that is done from 352 MB of K + V per call on, below which a cache re-read every step stays in the
 * Infinity Cache, and rows may be cut into more splits (size the workspace with the same descriptor).  A hint:
 * results are the same up to the order of the floating-point merges. */
#define FK_CACHE_COLD 1

/* Scoring model of one layer (Appendix B.1): phi = gelu(x W1 + b1) W2 + b2, x = concat(k, v). */
typedef struct {
    const void *w1;   /* device [n_sets][2*head_dim][hidden], cache dtype */
    const float *b1;  /* device [n_sets][hidden] */
    const float *w2;  /* device [n_sets][hidden] */
    const float *b2;  /* device [n_sets] */
    int32_t hidden;   /* H; bf16: multiple of 8 with H'*(2*head_dim+8)*2 + 8*H' <= 160 KiB of LDS, H' = H rounded up to 32 */
    int32_t per_head; /* 1: n_sets = n_kv_heads, one model per KV head; 0: one shared model */
    int32_t skip_len; /* rows with len[r] <= skip_len are skipped, their scores not written (pass the budget:
                         rows at or under budget are not pruned and need no scores); 0 scores every row */
} fk_scorer;

const char *fk_status_string(fk_status s);

/* Names the build: "fk <version> gfx950". */
const char *fk_version(void);

/*
 * Section 3.1 (a generated token joins the cache): for every sequence b and KV head h write
 * k_new[b][h][:], v_new[b][h][:] and pos_new[b] into slot len[r] of row r = (b, h), then
 * len[r] += 1.  k_new, v_new: [batch][n_kv_heads][head_dim] dtype; pos_new: [batch] int32.
 * A row whose len[r] == capacity is left unchanged (nothing is written past the row).
 */
fk_status fk_append(const fk_cache_desc *desc, void *K, void *V, int32_t *pos, int32_t *len,
                    const void *k_new, const void *v_new, const int32_t *pos_new, void *stream);

/*
 * Bytes of device workspace fk_decode_attn / fk_decode_step need (0 on bad args).  The size does
 * not depend on max_len, so one workspace serves every call on this descriptor.  The workspace
 * starts with per-row arrival counters: the caller zero-fills it ONCE after allocating it; every call
 * leaves the counters at zero again.  Calls sharing a workspace must not overlap in time.
 */
size_t fk_decode_attn_workspace(const fk_cache_desc *desc, int32_t max_len);

/*
 * Appendix A, "Problem Setup" (attention over the retained set, renormalised softmax):
 *   out[b][hq][:] = sum_{i < len[b][hq/g]} softmax_i(softmax_scale * <q[b][hq], K[b][hq/g][i]>) V[b][hq/g][i]
 * q, out: [batch][n_q_heads][head_dim] dtype; accumulation in fp32 (bf16 with head_dim 128: the
 * softmax weights are rounded to bf16 before the P.V contraction and normalised by the sum of the
 * rounded weights).  Query heads of a row with len == 0 get zeros.  workspace: >= fk_decode_attn_workspace(desc, max_len) bytes, zero-filled
 * once by the caller (see above); FK_ERR_WORKSPACE if missing or too small.  One launch.
 */
fk_status fk_decode_attn(const fk_cache_desc *desc, const void *q, const void *K, const void *V,
                         const int32_t *len, int32_t max_len, float softmax_scale, void *out,
                         void *workspace, size_t workspace_bytes, void *stream);

/*
 * One decode step in ONE launch: fk_append followed by fk_decode_attn (Section 3.1 for the append,
 * Appendix A "Problem Setup" for the attention), with the same arguments and results as the two
 * calls in that order; the new pair takes part in the attention.  max_len bounds len[r] + 1.
 */
fk_status fk_decode_step(const fk_cache_desc *desc, const void *q, void *K, void *V, int32_t *pos,
                         int32_t *len, const void *k_new, const void *v_new, const int32_t *pos_new,
                         int32_t max_len, float softmax_scale, void *out, void *workspace,
                         size_t workspace_bytes, void *stream);

/*
 * The arguments of one fk_decode_step, or with feat of one fk_decode_step_feat, in one place: for callers whose
 * foreign-function interface takes its time per argument and that make the same call again and again.
 * fk_decode_step_packed(a) is that call, with its checks, results and status.
 */
typedef struct {
    fk_cache_desc desc;
    int32_t max_len;
    const void *q;
    void *K, *V;
    int32_t *pos, *len;
    const void *k_new, *v_new;
    const int32_t *pos_new;
    void *out, *workspace;
    size_t workspace_bytes;
    void *stream;
    float softmax_scale;
    int32_t chunk_pos, chunk_len;   /* with feat */
    float *feat;                    /* null: fk_decode_step */
} fk_step_args;
fk_status fk_decode_step_packed(const fk_step_args *args);

/*
 * fk_decode_step for callers that cannot allocate device memory (code under HIP graph capture, tight serving
 * loops, harnesses that forbid hipMalloc): same arguments and results as fk_decode_step without the workspace,
 * which is a fixed FK_STATIC_SCRATCH_BYTES array inside the library's device image (each GPU the library runs on
 * holds its own copy until the process ends).  FK_ERR_WORKSPACE when fk_decode_attn_workspace(desc, max_len)
 * exceeds FK_STATIC_SCRATCH_BYTES (about batch * n_kv_heads * splits * g * (head_dim + 2) * 4 bytes; the Qwen3-4B
 * layer shape at batch 16 needs 0.8 MB); FK_ERR_LAUNCH if the array's address cannot be resolved.  Nothing is
 * allocated or freed, by this call or by anything it calls.  The first call on a device looks the array up and
 * clears it with a small kernel on `stream` (make that call outside a graph capture); every call leaves the
 * counters in it at zero for the next one.  All calls on one GPU share the array: calls that overlap in time
 * on one GPU (two streams, two threads) race, the caller must serialise them.
 */
#define FK_STATIC_SCRATCH_BYTES (8u << 20)
fk_status fk_decode_step_static(const fk_cache_desc *desc, const void *q, void *K, void *V, int32_t *pos,
                                int32_t *len, const void *k_new, const void *v_new, const int32_t *pos_new,
                                int32_t max_len, float softmax_scale, void *out, void *stream);

/*
 * Section 3.1 (the L generation steps between two eviction events): n_steps consecutive fk_decode_step calls
 * enqueued by one call, step t on q_seq[t], k_seq[t], v_seq[t], pos_seq[t] with its output in out_seq[t] and
 * max_len = min(max_len_first + t, capacity); max_len_first bounds len[r] + 1 at the first step.
 *   q_seq, out_seq [n_steps][batch][n_q_heads][head_dim], k_seq, v_seq [n_steps][batch][n_kv_heads][head_dim]
 *   dtype; pos_seq [n_steps][batch] int32.
 * Results are those of the n_steps single calls, bit for bit; the host returns to its caller once per window instead of once
 * per step.  All inputs are taken as they are when the work runs: bf16 windows are computed at once, one launch that reads K and V
 * for many steps together, unless single steps are the faster way (few long rows, few steps) or the buffers give the steps an order
 * (out_seq overlaps q_seq, new rows lie in the cache, ...): then, and for fp32, the steps run one launch each.  n_steps == 0 is a
 * no-op.  On an error the steps before it stay enqueued.
 */
fk_status fk_decode_window(const fk_cache_desc *desc, const void *q_seq, void *K, void *V, int32_t *pos,
                           int32_t *len, const void *k_seq, const void *v_seq, const int32_t *pos_seq,
                           int32_t n_steps, int32_t max_len_first, float softmax_scale, void *out_seq,
                           void *workspace, size_t workspace_bytes, void *stream);

/*
 * Section 3.1 Eq. 1 and Appendix B.1 (importance score of every retained pair, features
 * restricted to the key and value vectors):
 *   scores[b][h][i] = sum_j gelu(sum_f x_f W1[f][j] + b1[j]) W2[j] + b2,  x = [K[b][h][i], V[b][h][i]]
 * for i < len[r]; gelu is the exact erf form; fp32 accumulation (bf16: MFMA).  scores:
 * [batch][n_kv_heads][capacity] fp32; slots >= len[r] are not written.
 */
fk_status fk_score_kv(const fk_cache_desc *desc, const void *K, const void *V, const int32_t *len,
                      int32_t max_len, const fk_scorer *scorer, float *scores, void *stream);

/*
 * Section 3.1 (keep the most recent L pairs, prune the others to the B - L most important;
 * deterministic Top-K form).  For every row with len[r] > budget: keep the last
 * `protect_recent` live slots and, of the other len[r] - protect_recent, the
 * budget - protect_recent best under the total order (score descending, then slot
 * ascending = position ascending).  -0 equals +0; NaN ranks below -inf.  The kept slot
 * indices are written ascending to keep_idx[b][h][0 .. budget-1].  Rows with
 * len[r] <= budget get the identity keep_idx[j] = j for all j < budget (nothing to prune; fk_compact moves nothing).
 * keep_idx: [batch][n_kv_heads][budget] int32.  pos may be NULL: it is not read, slot order
 * stands for position order (see the precondition above).
 * Requires 0 <= protect_recent <= budget <= capacity.
 */
fk_status fk_select_keep(const fk_cache_desc *desc, const float *scores, const int32_t *pos,
                         const int32_t *len, int32_t max_len, int32_t budget,
                         int32_t protect_recent, int32_t *keep_idx, void *stream);

/*
 * fk_select_keep for few, long rows (Section 4.3: one-shot compression of a long prompt before
 * decoding; the same selection rule, applied once to rows far over budget).  Same arguments,
 * same result bit for bit.  With at most 64 rows of max_len >= 16384 a row is cut into chunks that
 * are selected by one workgroup each, and a second launch selects among the chunks' survivors (a
 * pair among the row's best budget - protect_recent is among its chunk's best under the same total
 * order); otherwise this is fk_select_keep.  workspace: caller-owned device scratch of at least
 * fk_select_keep_workspace(desc, max_len, budget, protect_recent) bytes (0 when rows are not split;
 * then workspace may be NULL), contents undefined before and after; FK_ERR_WORKSPACE if too small.
 */
size_t fk_select_keep_workspace(const fk_cache_desc *desc, int32_t max_len, int32_t budget,
                                int32_t protect_recent);
fk_status fk_select_keep_ws(const fk_cache_desc *desc, const float *scores, const int32_t *pos,
                            const int32_t *len, int32_t max_len, int32_t budget,
                            int32_t protect_recent, int32_t *keep_idx, void *workspace,
                            size_t workspace_bytes, void *stream);

/*
 * Section 3.1 Eq. 2 and Appendix B.2 (Top-K multinomial eviction, the paper's inference policy).
 * For every row with len[r] > budget, E = len[r] - budget pairs go: the last `protect_recent` live
 * slots are kept; of the others, the max(n_candidates, E) lowest-ranked under (score descending,
 * slot ascending) are candidates (the paper uses 2E), the rest are kept; E candidates are drawn
 * without replacement with probabilities softmax(-score), in Gumbel-top-k form: the caller supplies
 * noise[b][h][i] (iid Gumbel(0,1) for the paper's law; fp32, [batch][n_kv_heads][capacity]) and the
 * E candidates with the smallest fp32 value of scores - noise are evicted, ties evicting the higher
 * slot first.  noise == 0 or n_candidates <= E gives fk_select_keep's result.  Output, rows at or
 * under budget, pos and the special values are as for fk_select_keep.  capacity <= 131072
 * (FK_ERR_UNSUPPORTED above).
 */
fk_status fk_select_keep_sampled(const fk_cache_desc *desc, const float *scores, const float *noise,
                                 const int32_t *pos, const int32_t *len, int32_t max_len,
                                 int32_t budget, int32_t protect_recent, int32_t n_candidates,
                                 int32_t *keep_idx, void *stream);

/*
 * Section 1 / 3.1 (evicted pairs are discarded for good; stable in-place form): for every row
 * with len[r] > budget, slot j of K, V and pos receives the former contents of slot
 * keep_idx[b][h][j], j = 0 .. budget-1 (bit copies; keep_idx ascending with keep_idx[j] >= j,
 * as fk_select_keep writes it), then len[r] = budget.  Rows with len[r] <= budget are untouched.
 * What moves is read from keep_idx alone (one launch, the length is clamped in the same kernel): every row of
 * keep_idx must be written in full, rows at or under budget with the identity or with entries outside
 * [0, capacity) (both move nothing; fk_select_keep and fk_select_keep_sampled write the identity).
 */
fk_status fk_compact(const fk_cache_desc *desc, void *K, void *V, int32_t *pos, int32_t *len,
                     const int32_t *keep_idx, int32_t budget, void *stream);

/*
 * ---- Attention features of the scoring model (Appendix B.1) ----
 *
 * Beside k and v the scorer sees, for every retained pair and every query head of its group, six sums of
 * the attention weights the pair received: over the last 8, 16 and 32 queries of the current chunk of L
 * steps, over the whole chunk so far (wL), and the sums carried over the earlier chunks, plain (cum)
 * and decayed by 0.9 per chunk (dec).  Device state, owned by the caller, zero-filled at the start:
 *   feat [batch][n_kv_heads][6][capacity][GP] fp32, GP = 4 if g <= 4 else 8 (heads >= g hold zeros),
 *   planes in the order w8, w16, w32, wL, cum, dec; cum and dec hold the state BEFORE the current chunk.
 * The scorer's feature vector of a pair is a[head * 6 + plane] with cum + wL and 0.9 dec + wL in the
 * last two planes, so W1 has 2 * head_dim + 6 g rows: k, v, then a.
 */

/* Bytes of workspace fk_decode_step_feat needs (0 on bad args); no initialisation required. */
size_t fk_decode_step_feat_workspace(const fk_cache_desc *desc);

/*
 * fk_decode_step that also accounts the step's attention weights (softmax over the retained set
 * including the new pair, fp32 weights from the unrounded exponentials) in `feat`: the slot of the
 * new pair restarts all six planes from zero, then every live slot i gains p[hq][i] in wL and in each
 * window plane w with chunk_pos >= chunk_len - w.  chunk_pos = 0 .. chunk_len - 1 counts the steps since
 * the last eviction event, chunk_len = L.  One launch, one workgroup per row.  The workspace holds the
 * step's logits; calls sharing it must not overlap in time.
 */
fk_status fk_decode_step_feat(const fk_cache_desc *desc, const void *q, void *K, void *V, int32_t *pos,
                              int32_t *len, const void *k_new, const void *v_new,
                              const int32_t *pos_new, int32_t max_len, float softmax_scale, float *feat,
                              int32_t chunk_pos, int32_t chunk_len, void *out, void *workspace,
                              size_t workspace_bytes, void *stream);

/*
 * Appendix B.1 (the queries of one chunk): n_steps consecutive fk_decode_step_feat calls enqueued by one
 * call, step t at chunk position chunk_pos_first + t, on q_seq[t], k_seq[t], v_seq[t], pos_seq[t] with its
 * output in out_seq[t] and max_len = min(max_len_first + t, capacity).  Layouts as for fk_decode_window;
 * the window must end inside the chunk (chunk_pos_first + n_steps <= chunk_len).  Results are those of
 * the n_steps single calls, bit for bit.  bf16 with head_dim 128: two launches for the whole window, unless it is two steps of
 * rows below 2048 pairs (max_len_first), its buffers give the steps an order, or 2 n_steps g > capacity * GP, the space the workspace
 * has; otherwise the steps one by one.
 */
fk_status fk_decode_window_feat(const fk_cache_desc *desc, const void *q_seq, void *K, void *V, int32_t *pos,
                                int32_t *len, const void *k_seq, const void *v_seq, const int32_t *pos_seq,
                                int32_t n_steps, int32_t max_len_first, float softmax_scale, float *feat,
                                int32_t chunk_pos_first, int32_t chunk_len, void *out_seq, void *workspace,
                                size_t workspace_bytes, void *stream);

/*
 * fk_score_kv on x = concat(k, v, a) (Section 3.1 Eq. 1 with the attention features of Appendix
 * B.1).  scorer->w1 is [n_sets][2*head_dim + 6 g][hidden]; the fp32 features enter the contraction as
 * a bf16 head plus a bf16 remainder (16 significant bits; fp32 caches: plain fp32).  bf16: FK_ERR_UNSUPPORTED
 * unless hidden is a multiple of 8 and H' * (2*head_dim + roundup(6 g, 16) + 8) * 2 + 8 * H' <= 160 KiB (H' = hidden rounded up to 32).
 */
fk_status fk_score_kv_feat(const fk_cache_desc *desc, const void *K, const void *V, const float *feat,
                           const int32_t *len, int32_t max_len, const fk_scorer *scorer, float *scores,
                           void *stream);

/*
 * fk_compact that also closes the chunk of the features: for every row and live slot cum += wL,
 * dec = 0.9 dec + wL, the planes w8, w16, w32, wL restart from zero, and rows over budget move the
 * features of slot keep_idx[j] to slot j together with K, V and pos.  Other arguments and results as
 * fk_compact.
 */
fk_status fk_compact_feat(const fk_cache_desc *desc, void *K, void *V, int32_t *pos, float *feat,
                          int32_t *len, const int32_t *keep_idx, int32_t budget, void *stream);

/*
 * ---- Golden Eviction label builder (Section 3.2 Eq. 3-5; training-side, outside the decode loop) ----
 *
 * Input: the attention matrices of the query heads of one layer on a full trace of T tokens,
 *   A [n_q_heads][T][ld] dtype (fp32 or bf16), row = query position, column = key position (0-based),
 *   ld >= T elements per row with ld % 8 == 0; precondition A[h][q][i] == 0 for i > q (causal).
 * With budget B and eviction length L (L <= B) the queries from B + L on form M = ceil((T - B)/L) - 1
 * blocks; block t = 1 .. M holds queries B + tL .. min(B + (t+1)L, T) - 1, the last one counted as L
 * queries (zero padded).
 */

/* M for a trace of T tokens; -1 on bad arguments. */
int32_t fk_golden_steps(int32_t T, int32_t budget, int32_t interval);

/*
 * Eq. 3-4 and the first half of Eq. 5:
 *   block_scores[h'][t-1][i] = 1/(g L) sum_{h in group h'} sum_{q in block t} A[h][q][i]     (average pooling)
 *   alpha[h'][t-1][i]        = max_{t <= j <= M} block_scores[h'][j-1][i]                    (future score)
 * both [n_kv_heads][M][T] fp32, fp32 accumulation; nothing is written when M == 0.
 */
fk_status fk_golden_scores(const void *A, int32_t dtype, int32_t n_q_heads, int32_t n_kv_heads, int32_t T,
                           int64_t ld, int32_t budget, int32_t interval, float *block_scores,
                           float *alpha, void *stream);

/*
 * Second half of Eq. 5 as an eviction trace under the protocol of Section 3.1: before step 1 the cache
 * holds positions 0 .. B + L - 1; step t keeps the L newest (B + tL - L .. B + tL - 1) and, of the other B
 * it holds, the B - L with the largest alpha[h'][t-1][.] (ties: the lower position); then positions
 * B + tL .. B + (t+1)L - 1 join.  kept [n_kv_heads][M][B] int32: the positions retained after step t,
 * ascending.  -0 equals +0 and NaN ranks lowest, as in fk_select_keep.  B + L <= 12288
 * (FK_ERR_UNSUPPORTED above).
 */
fk_status fk_golden_trace(const float *alpha, int32_t n_kv_heads, int32_t T, int32_t budget,
                          int32_t interval, int32_t *kept, void *stream);

/*
 * ---- The prompt's side: a paged cache, attention of chunks over it, accumulated weights, compression ----
 *
 * A prompt is longer than any budget.  Until it is compressed (Section 4.3: once, before decoding) its pairs lie in pages of a pool that
 * all sequences share:
 *   K, V        [n_pages][n_kv_heads][page_size][head_dim]  dtype
 *   page_table  [batch][max_pages] int32   page i of sequence b holds its positions i * page_size .. (i + 1) * page_size - 1
 *   kv_len      [batch] int32              pairs of every sequence, those of the current chunk among them
 *   q_start     [batch + 1] int32          tokens q_start[b] .. q_start[b + 1] - 1 of the call are sequence b's chunk (of any length, 0 too);
 *                                          ascending; tokens outside of all chunks are not touched
 * Token i of a chunk of c tokens has position p = kv_len[b] - c + i.  Its queries see the pairs j <= p; with window > 0 only those with
 * j > p - window or j < n_sink (a sliding window, and first tokens that stay visible).  A page_table entry outside [0, n_pages) is a hole:
 * nothing is stored there and nobody sees its pairs.  kv_len is taken as at most max_pages * page_size; tokens at negative positions are not
 * stored and see nothing.  Values of pairs that a query does not see, infinities and NaN among them, do not reach its results.
 * n_tokens is the number of tokens that q, out, stats, k_new and v_new hold.  max_chunk and max_len bound the chunks' and the sequences'
 * lengths; they only size the launch, results are right beyond them too.
 */
typedef struct {
    int32_t batch;      /* sequences */
    int32_t n_q_heads;  /* query heads per token */
    int32_t n_kv_heads; /* KV heads; group size g = n_q_heads / n_kv_heads <= 8 */
    int32_t head_dim;   /* 64 or 128 */
    int32_t page_size;  /* pairs per page: a power of two, 16 to 1024 */
    int32_t n_pages;    /* pages of the pool */
    int32_t max_pages;  /* entries per row of the page table; max_pages * page_size < 2^24 */
    int32_t dtype;      /* fk_dtype of q, K, V, out */
} fk_paged_desc;

/* The new pairs join the cache: K and V of token i of sequence b's chunk, k_new / v_new [n_tokens][n_kv_heads][head_dim], are stored at
 * their position.  Two sequences may share pages that no chunk of the call is stored to. */
fk_status fk_paged_append(const fk_paged_desc *desc, void *K, void *V, const int32_t *page_table, const int32_t *kv_len,
                          const int32_t *q_start, int32_t n_tokens, const void *k_new, const void *v_new, void *stream);

/*
 * Attention of every chunk over its sequence's pairs (the chunk's own are in the cache: fk_paged_append first), single tokens included:
 *   out[t][hq][:] = sum_j 2^(s_j - M) V_j / L,  s_j = log2(e) * softmax_scale * <q[t][hq], K_j>,  M = max_j s_j,  L = sum_j 2^(s_j - M)
 * over the pairs j that the query sees.  q, out: [n_tokens][n_q_heads][head_dim]; stats (may be NULL): [n_tokens][n_q_heads][2] fp32, M and L.  A query
 * that sees nothing, or logits of -inf alone, gets zeros and (-inf, 0); one that is no number, or meets one, has L = NaN.  fp32 accumulation; bf16: the
 * weights are rounded to bf16 before they meet V, L is the sum of the unrounded ones.  workspace: fk_paged_attn_workspace bytes, no initialisation
 * required; calls sharing it must not overlap in time.
 */
size_t fk_paged_attn_workspace(const fk_paged_desc *desc, int32_t n_tokens, int32_t max_chunk, int32_t max_len);
fk_status fk_paged_attn(const fk_paged_desc *desc, const void *q, const void *K, const void *V, const int32_t *page_table,
                        const int32_t *kv_len, const int32_t *q_start, int32_t n_tokens, int32_t max_chunk, int32_t max_len,
                        int32_t window, int32_t n_sink, float softmax_scale, void *out, float *stats, void *workspace,
                        size_t workspace_bytes, void *stream);

/*
 * The attention weight that every pair received from the chunks' queries, summed over the group's query heads:
 *   acc[b][h][j] = (j older than the chunk ? acc[b][h][j] : 0) + sum_{t in chunk, t sees j} sum_{hq in group h} 2^(s_j - M) / L
 * with the M and L that fk_paged_attn gave in stats for the same q, view and scale.  acc: [batch][n_kv_heads][max_pages * page_size] fp32,
 * the layout of fk_select_keep's scores for a cache of that capacity; slots from kv_len on, and rows of sequences without a chunk, are not
 * written.  The order of the sums is fixed: equal calls give equal bits.  workspace as for fk_paged_attn.
 */
size_t fk_paged_weights_workspace(const fk_paged_desc *desc, int32_t n_tokens, int32_t max_chunk, int32_t max_len);
fk_status fk_paged_weights(const fk_paged_desc *desc, const void *q, const void *K, const int32_t *page_table, const int32_t *kv_len,
                           const int32_t *q_start, int32_t n_tokens, int32_t max_chunk, int32_t max_len, int32_t window, int32_t n_sink,
                           float softmax_scale, const float *stats, float *acc, void *workspace, size_t workspace_bytes, void *stream);

/*
 * Compression of the prompts into the rows of a budgeted cache (`rows`: same batch, heads, head_dim and dtype): slot j of row (b, h) receives
 * the pair at position keep_idx[b][h][j], j < min(kv_len[b], budget) - K, V, the position into pos, its accumulated weight into acc_rows -
 * and len[b][h] = min(kv_len[b], budget).  keep_idx: [batch][n_kv_heads][budget], as fk_select_keep writes it on acc; an entry outside
 * [0, kv_len[b]) or in a hole leaves its slot as it is.  acc and acc_rows [batch][n_kv_heads][rows->capacity] may both be NULL.  The rows must
 * not share memory with the pool.
 */
fk_status fk_paged_compress(const fk_paged_desc *desc, const void *K, const void *V, const int32_t *page_table, const int32_t *kv_len,
                            const float *acc, const int32_t *keep_idx, int32_t budget, const fk_cache_desc *rows, void *K_rows,
                            void *V_rows, int32_t *pos, int32_t *len, float *acc_rows, void *stream);

/*
 * ---- Drafted tokens: positions, attention of trees over a cache, verification, the accepted path joins the cache ----
 *
 * A small model drafts several tokens behind the last one, as a tree (a chain is one); one pass of the large model answers for all of them.  Only what is
 * accepted joins the cache: a budgeted cache must not hold, score or evict for pairs that are thrown away again.  The trees of a call are packed:
 *   q_start [batch + 1] int32   tokens q_start[b] .. q_start[b + 1] - 1 of the call are sequence b's tree (of 0 to FK_TREE_NODES nodes), ascending
 *   parent  [n_tokens] int32    a node's parent, counted from the tree's first node and lower than its own place; others, -1 by custom, stand for none
 * Node 0 is the root: the last token of the sequence, whose pair is not in the cache yet.  A tree of more than FK_TREE_NODES nodes is passed over by the attention,
 * which writes nothing of it, and by fk_verify_drafts, which accepts nothing; the commits take a path's pairs out of any number of nodes.  The round of a layer:
 * fk_rope, fk_tree_attn; of the model: fk_verify_drafts; of every layer then: fk_commit_drafts.
 */
#define FK_TREE_NODES 256

/*
 * Rotary positions.  Of every head the first rotary_dim channels turn in pairs (u, w) by the angle pos * freq_i, i = 0 .. rotary_dim / 2 - 1:
 *   u' = magnitude * (u cos - w sin),  w' = magnitude * (u sin + w cos)
 * with u, w = channels i and i + rotary_dim / 2 (FK_ROPE_HALF) or 2 i and 2 i + 1 (FK_ROPE_INTERLEAVED); channels from rotary_dim on are copied.  Angles are
 * formed in 64 bits and reduced to a turn before sine and cosine are taken in fp32; results are rounded once.  inverse: the angles negated (keys turned back; the
 * gradient of a call is the same call on the outputs' gradients with inverse flipped).
 */
typedef enum { FK_ROPE_HALF = 0, FK_ROPE_INTERLEAVED = 1 } fk_rope_layout;

typedef struct {
    int32_t n_q_heads;  /* query heads per token, 0: no queries */
    int32_t n_kv_heads; /* key heads per token, 0: no keys */
    int32_t head_dim;   /* 64 or 128 */
    int32_t rotary_dim; /* even, 2 .. head_dim */
    int32_t layout;     /* fk_rope_layout */
    int32_t dtype;      /* fk_dtype of q, k and the outputs */
    int32_t inverse;
    float magnitude;    /* 1, or what a scaling for long contexts multiplies queries and keys by */
    int64_t q_stride, k_stride, q_out_stride, k_out_stride; /* elements from one token's heads to the next one's, whole 16 bytes; 0: heads * head_dim */
} fk_rope_desc;

/* q [n_tokens][n_q_heads][head_dim], k [n_tokens][n_kv_heads][head_dim] with their strides, pos [n_tokens] int32 (any value), freq [rotary_dim / 2] fp64: radians per
 * position.  q_out may be q, and k_out k, with the same strides (in place); otherwise outputs share no memory with inputs or each other. */
fk_status fk_rope(const fk_rope_desc *desc, const void *q, const void *k, const int32_t *pos, const double *freq, int32_t n_tokens,
                  void *q_out, void *k_out, void *stream);

/* Frequencies f_i = base^(-2 i / rotary_dim), scaled for contexts `factor` times as long as trained on:
 *   FK_ROPE_LINEAR  all divided by factor
 *   FK_ROPE_BASE    base * factor^(rotary_dim / (rotary_dim - 2)) in the place of base: the slowest pair slows down by factor, the fastest not at all
 *   FK_ROPE_PARTS   a pair that turns r = context * f_i / (2 pi) times over the trained context is divided by factor where r <= low, left alone where
 *                   r >= high, and mixed linearly in r between
 * freq: HOST memory, [rotary_dim / 2].  Parameters that a scaling does not name are not looked at. */
typedef enum { FK_ROPE_PLAIN = 0, FK_ROPE_LINEAR = 1, FK_ROPE_BASE = 2, FK_ROPE_PARTS = 3 } fk_rope_scaling;
fk_status fk_rope_frequencies(int32_t rotary_dim, double base, int32_t scaling, double factor, double context, double low, double high,
                              double *freq);

/*
 * Attention of trees over the rows of a budgeted cache: a node sees the live pairs of its sequence's rows, its ancestors' pairs and its own,
 *   out[t][hq][:] = sum_j 2^(s_j - M) V_j / L,  s_j = log2(e) * softmax_scale * <q[t][hq], K_j>,  M = max_j s_j,  L = sum_j 2^(s_j - M)
 * k_tree, v_tree: the nodes' own pairs, [n_tokens][n_kv_heads][head_dim]; the cache is only read.  q, out: [n_tokens][n_q_heads][head_dim]; stats (may be NULL):
 * [n_tokens][n_q_heads][2] fp32, M and L.  Logits of -inf alone give zeros and (-inf, 0); a query that is no number, or meets one, has L = NaN.  Values of
 * pairs that a node does not see, infinities and NaN among them, do not reach its results.  fp32 accumulation; bf16: a weight meets V as two bf16 terms, off
 * by 2^-15 of it at most, L is the sum of the unrounded ones.  max_tree <= FK_TREE_NODES bounds the trees' nodes and max_len every len[r]; they only
 * size the launch, results are right beyond them too.  workspace: fk_tree_attn_workspace bytes for these sizes or larger ones (what serves a call serves every call of
 * the descriptor with as many tokens or fewer and such bounds or lower ones), zero-filled ONCE by the caller; every call leaves its counters at zero again, and
 * calls of any sizes (of fk_paged_tree_attn too) may take turns with one that is large enough for each; calls sharing it must not
 * overlap in time.  One launch; the order of all sums is fixed: equal calls give equal bits.  FK_ERR_UNSUPPORTED: n_tokens * n_q_heads >= 2^28, n_kv_heads >= 2^16.
 */
size_t fk_tree_attn_workspace(const fk_cache_desc *desc, int32_t n_tokens, int32_t max_tree, int32_t max_len);
fk_status fk_tree_attn(const fk_cache_desc *desc, const void *q, const void *K, const void *V, const int32_t *len, const void *k_tree,
                       const void *v_tree, const int32_t *parent, const int32_t *q_start, int32_t n_tokens, int32_t max_tree,
                       int32_t max_len, float softmax_scale, void *out, float *stats, void *workspace, size_t workspace_bytes, void *stream);

/* The same over the pages of a prompt (fk_paged_attn's pool, page table and holes).  kv_len counts the pairs in the pages, none of the tree's.  A node has position
 * p = kv_len[b] + the number of its ancestors; with window > 0 it sees, of the pairs of the pages and of its ancestors, those at positions j > p - window or
 * j < n_sink. */
size_t fk_paged_tree_attn_workspace(const fk_paged_desc *desc, int32_t n_tokens, int32_t max_tree, int32_t max_len);
fk_status fk_paged_tree_attn(const fk_paged_desc *desc, const void *q, const void *K, const void *V, const int32_t *page_table,
                             const int32_t *kv_len, const void *k_tree, const void *v_tree, const int32_t *parent, const int32_t *q_start,
                             int32_t n_tokens, int32_t max_tree, int32_t max_len, int32_t window, int32_t n_sink, float softmax_scale,
                             void *out, float *stats, void *workspace, size_t workspace_bytes, void *stream);

/*
 * Verification of drafted tokens against the large model's probabilities (speculative sampling: what comes out is distributed as the large model's own
 * samples).  target [n_tokens][vocab] fp32: row i is the distribution of the token behind node i; draft [n_tokens][vocab] fp32: row i is the one from which the
 * children of node i were drawn, independently of each other (rows of nodes without children are not looked at); tokens [n_tokens]: the nodes' tokens (the root's
 * is not looked at); uniform [n_tokens] fp32 in [0, 1): a node's number decides about it, the root's draws the last token.  From the root on, with r = target's
 * row of the current node, its children x in ascending order:
 *   uniform * draft(x) < r(x): x is accepted and becomes the current node, with r = target's row again;
 *   otherwise r becomes max(r - draft, 0), divided by its sum.
 * draft NULL (tokens that were not drawn, the likeliest ones say): x is accepted where uniform * m < r(x), with m = 1 at first; otherwise m goes down by r(x),
 * not below 0, and r(x) becomes 0.  When no child is left, next_token is the lowest v with r(0) + .. + r(v) > uniform * (sum of r) and r(v) > 0 - the
 * last v with r(v) > 0 where rounding finds none; of target's row where r is 0 everywhere; -1 where that is too.  Numbers that are negative or NaN in a row of r
 * count as 0; a token outside [0, vocab) has probability 0 in both.  Sums and comparisons are in fp64, sums in a fixed order: equal calls give equal tokens.
 * path [n_tokens]: the accepted nodes of sequence b, the root first, from q_start[b] on, then -1; n_accepted [batch]: how many, the root among them (0 without
 * a tree); next_token [batch] (-1 without one).
 * workspace: fk_verify_drafts_workspace bytes for these sizes or larger ones, zero-filled ONCE by the caller and from then on only handed to this call, of any
 * sizes that it is large enough for.  Calls sharing it must not overlap in time.  batch <= 65535, vocab < 2^30 (FK_ERR_UNSUPPORTED beyond).  One launch.
 */
size_t fk_verify_drafts_workspace(int32_t batch, int32_t vocab);
fk_status fk_verify_drafts(int32_t batch, int32_t vocab, const float *target, const float *draft, const int32_t *tokens, const int32_t *parent,
                           const int32_t *q_start, int32_t n_tokens, const float *uniform, int32_t *path, int32_t *n_accepted,
                           int32_t *next_token, void *workspace, size_t workspace_bytes, void *stream);

/*
 * The accepted paths' pairs join the rows of a budgeted cache: slot len[r] + i of row r = (b, h) receives pair path[q_start[b] + i] of the tree - K, V, and
 * pos_first[b] + i into pos - for i < n_accepted[b], then len[r] goes up by as many.  A path ends at its first entry that is no node of the tree; a row takes as
 * many pairs as it has room for, the first ones.  acc (may be NULL): accumulated weights (fk_decode_step_acc), which start from zero in the new slots and stay as they
 * are in the others.  k_tree, v_tree, path and n_accepted as above.  The pairs must not share memory with the cache.
 */
fk_status fk_commit_drafts(const fk_cache_desc *desc, void *K, void *V, int32_t *pos, int32_t *len, float *acc, const void *k_tree,
                           const void *v_tree, const int32_t *q_start, int32_t n_tokens, const int32_t *path, const int32_t *n_accepted,
                           const int32_t *pos_first, void *stream);

/* The same into pages: position kv_len[b] + i receives the i-th pair, then kv_len[b] goes up.  A pair whose place lies in a hole is not stored, and counts; a
 * sequence takes as many pairs as its page table has room for.  Sequences may share pages that nothing is stored to. */
fk_status fk_paged_commit_drafts(const fk_paged_desc *desc, void *K, void *V, const int32_t *page_table, int32_t *kv_len, const void *k_tree,
                                 const void *v_tree, const int32_t *q_start, int32_t n_tokens, const int32_t *path,
                                 const int32_t *n_accepted, void *stream);

/*
 * ---- Eviction by accumulated attention weight ----
 *
 * The score that learned ones are compared with: the attention weight a pair has received so far.  Device state, owned by the caller:
 * acc [batch][n_kv_heads][capacity] fp32, in the layout of fk_select_keep's scores, so that an event is fk_select_keep on acc, then
 * fk_compact_acc.
 */

/* Bytes of workspace fk_decode_step_acc needs (0 on bad args); no initialisation required. */
size_t fk_decode_step_acc_workspace(const fk_cache_desc *desc);

/*
 * fk_decode_step that also adds the step's attention weights (softmax over the retained set including the new pair, fp32 weights from the
 * unrounded exponentials and their sum), summed over the group's query heads, to acc; the slot of the new pair starts from zero.  Other arguments
 * and results as fk_decode_step (the outputs' own weights and normaliser too: fk_decode_attn).  Calls sharing a workspace must not overlap in time.
 */
fk_status fk_decode_step_acc(const fk_cache_desc *desc, const void *q, void *K, void *V, int32_t *pos, int32_t *len,
                             const void *k_new, const void *v_new, const int32_t *pos_new, int32_t max_len,
                             float softmax_scale, float *acc, void *out, void *workspace, size_t workspace_bytes, void *stream);

/* fk_compact that moves the accumulated weights with K, V and pos.  Other arguments and results as fk_compact. */
fk_status fk_compact_acc(const fk_cache_desc *desc, void *K, void *V, int32_t *pos, float *acc, int32_t *len,
                         const int32_t *keep_idx, int32_t budget, void *stream);

#ifdef __cplusplus
}
#endif
#endif /* FK_H */
