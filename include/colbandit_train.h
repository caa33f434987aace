/*
 * colbandit_train.h - C-ABI of the training operators of the Col-Bandit library.
 *
 * The scoring calls (colbandit.h) read token embeddings that an encoder made.  These calls
 * are one fine-tuning step of such an encoder, on the score that the scoring calls compute
 * and over the layout that they read:
 *
 *   colbandit_attention            attention over ragged packed sequences, with an optional
 *                                  key mask, causal limit, shared key heads and learned
 *                                  relative position bias by buckets of distance
 *   colbandit_attention_backward   its gradients; the probabilities are recomputed
 *   colbandit_maxsim_scores        MaxSim score of every (query, document) pair and the
 *                                  document token that each query token chose
 *   colbandit_contrastive_loss     cross-entropy over each query's scores, and its gradient
 *   colbandit_maxsim_backward      gradients of the embeddings from those of the scores
 *   colbandit_clip_gradients       global norm of many tensors, and the tensors clipped to it
 *
 * Conventions are those of colbandit.h: DEVICE pointers are the caller's memory on the
 * current HIP device, HOST pointers are plain memory that is read before the call returns;
 * all kernels go to `stream`, nothing is allocated, nothing is synchronised and nothing is
 * read from the workspace that the same call has not written, so every call may be captured
 * in a HIP graph.  Results do not depend on the order in which workgroups run: the same
 * inputs give the same bits.  On an argument error nothing is enqueued.
 */
#ifndef COLBANDIT_TRAIN_H
#define COLBANDIT_TRAIN_H

#include "colbandit.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Limits (requests beyond them return COLBANDIT_ERR_UNSUPPORTED).
 * Head width and embedding width: 32, 64, 96 or 128.  Rows: below 2^31 - 2^16.  Heads: 4,096.
 * A launch has less than 2^32 threads, which bounds attention at some 2^31 query rows (key rows)
 * times heads, and at 2^24 sequences times heads (one head a workgroup of 256 threads), and the
 * gradients of MaxSim at 2^24 documents, 64-token tiles and query tokens together. */
#define COLBANDIT_MAX_DISTANCE 256   /* last distance with a bucket of its own range     */
#define COLBANDIT_MAX_BUCKETS 128    /* rows of the bias table                           */

/*
 * One attention problem.  Sequence s has query rows q_offsets[s] .. q_offsets[s+1]-1 and key
 * rows k_offsets[s] .. k_offsets[s+1]-1, Lq and Lk of them, either of which may be zero; query
 * row i (from 0) stands at key position p_i = i + Lk - Lq, so that both ends coincide.
 *   S_ij   = scale * <q_i, k_j> + bias[bucket(j - p_i)][head]
 *   seen   : keep == NULL or keep[key row j] != 0, and not causal or j <= p_i
 *   out_i  = sum_j exp(S_ij - lse_i) v_j,   lse_i = log sum_j exp(S_ij)   over the seen j
 * A row that sees nothing has out = 0 and lse = -inf, and takes no part in any gradient (its q
 * and dout may hold anything where the mask, the causal limit or lengths hide its keys, and are
 * finite where biases of -inf do).
 * Query head h reads key head h / (heads / kv_heads).  Keys that the mask hides may hold
 * anything, infinities and NaN included.
 * Scores are held in 32 bits: of a bias of 1e9 in size a row's products leave nothing.  Rows whose
 * scores are all that far from zero (a table may hide distances by any finite value, down to the
 * type's lowest) have outputs and gradients like any other; lse has a 32-bit value's rounding.
 * Products are summed in 32 bits.  fp32 values are multiplied as three bf16 pieces each, whose
 * sum is the value; the three smallest of the nine products of pieces, 2^-22 of a product
 * together, are left out.  fp32 values that are seen must be finite.
 * Rows of q, k and v lie q_row elements apart and heads q_head apart (likewise k, v); the d
 * values of a row and head are consecutive.  Pointers and strides are whole multiples of 16
 * bytes; rows lie at most 32 MiB apart.  out and all gradients are dense, [rows][heads][d].
 * Rows behind the last sequence (a batch padded to a round size) belong to none: out 0, lse -inf,
 * all gradients 0, whatever they hold.
 * Preconditions the host cannot check without a copy: offsets are non-decreasing, from 0 to at
 * most total_q (total_k).  Kernels clamp them, so a violation gives meaningless results and rows
 * that are not written, never an out-of-bounds access.
 */
typedef struct {
    int dt;                        /* colbandit_dtype of q, k, v, bias, out, gradients   */
    int n_seqs, heads, kv_heads, d;
    int causal;
    int n_buckets, max_distance;   /* of the bias table; ignored without one             */
    float scale;
    int64_t total_q, total_k;
    const int64_t *q_offsets, *k_offsets;      /* DEVICE [n_seqs + 1]                    */
    const void *q, *k, *v;                     /* DEVICE                                 */
    int64_t q_row, q_head, k_row, k_head, v_row, v_head;
    const uint8_t *keep;           /* DEVICE [total_k] or NULL                           */
    const void *bias;              /* DEVICE [n_buckets][heads] or NULL                  */
} colbandit_attn;

/* sizeof(colbandit_attn) as this library was compiled. */
size_t colbandit_sizeof_attn(void);

/*
 * Buckets of the relative position bias.  Without `causal` each direction has n_buckets/2 of
 * them (keys behind the query from n_buckets/2 on), with it the keys before it have all.  Of a
 * direction's n buckets the first n/2 are the distances 0 .. n/2-1; bucket n/2+i begins at
 * distance (n/2) * (max_distance / (n/2))^(i/(n - n/2)), rounded up, and the last one has no
 * end.  (causal: keys behind the query, which no row sees, count as distance 0.)
 *   starts   HOST [n]: first distance of each bucket of one direction
 * Returns n, or COLBANDIT_ERR_SHAPE / COLBANDIT_ERR_UNSUPPORTED.  Pure host code.
 */
int colbandit_bias_buckets(int n_buckets, int max_distance, int causal, int32_t *starts);

/*
 * out   DEVICE, [total_q][heads][d] of the storage type
 * lse   DEVICE float [heads][total_q] (natural logarithm)
 * workspace  256-byte aligned, >= colbandit_attention_workspace_bytes(a, 0); may be NULL
 *            where that is 0
 */
size_t colbandit_attention_workspace_bytes(const colbandit_attn *a, int backward);
int colbandit_attention(const colbandit_attn *a, void *out, float *lse, void *workspace,
                        size_t workspace_bytes, void *stream);

/*
 * Gradients from that of `out`; out and lse as colbandit_attention gave them.
 *   dout   DEVICE [total_q][heads][d]
 *   dq     DEVICE [total_q][heads][d];  dk, dv  DEVICE [total_k][kv_heads][d]
 *   dbias  DEVICE [n_buckets][heads], required with a bias
 * Key rows that no query row sees get zeros.
 * workspace  >= colbandit_attention_workspace_bytes(a, 1)
 */
int colbandit_attention_backward(const colbandit_attn *a, const void *out, const float *lse,
                                 const void *dout, void *dq, void *dk, void *dv, void *dbias,
                                 void *workspace, size_t workspace_bytes, void *stream);

/*
 * MaxSim of all pairs, for training: scores[q][i] = sum_t max_j <Q[q][t], docs[offsets[i]+j]>.
 *   Q        DEVICE [n_queries][T][d], docs DEVICE [total_tokens][d], 16-byte aligned
 *   offsets  DEVICE int64 [N+1]; a document may be empty: its score is -inf
 *   T        1 .. COLBANDIT_MAX_T
 *   scores   DEVICE float [n_queries][N]
 *   argmax   DEVICE int32 [n_queries][N][T]: the j that token t chose, the lowest of equal
 *            ones; -1 in an empty document
 * Products are summed in 32 bits; precision is that of the attention calls' products.
 * Embeddings are finite.
 */
int colbandit_maxsim_scores(const void *Q, int n_queries, int T, int d, colbandit_dtype dt,
                            const void *docs, const int64_t *offsets, int64_t N,
                            int64_t total_tokens, float *scores, int32_t *argmax, void *stream);

/*
 * loss[q] = log sum_i exp(scores[q][i] / temperature) - scores[q][targets[q]] / temperature
 * dscores[q][i] = d(mean of loss) / d(scores[q][i])
 * A target outside 0 .. N-1 takes its query out of the mean: loss 0, dscores 0.  Scores of
 * -inf have no weight; a target's makes a loss of +inf, and if all are -inf the loss and its
 * gradient are NaN, as the formula has it.
 *   temperature  > 0, finite, and so is its inverse in 32 bits
 *   targets  DEVICE int64 [n_queries];  loss DEVICE float [n_queries]
 *   dscores  DEVICE float [n_queries][N]
 */
int colbandit_contrastive_loss(const float *scores, int n_queries, int64_t N,
                               const int64_t *targets, float temperature, float *loss,
                               float *dscores, void *stream);

/*
 * dQ[q][t]       = sum_i dscores[q][i] * docs[offsets[i] + argmax[q][i][t]]
 * ddocs[row]     = sum of dscores[q][i] * Q[q][t] over the (q, t) that chose the row
 * Sums in 32 bits, in a fixed order.  dQ [n_queries][T][d] and ddocs [total_tokens][d] have the
 * storage type and are 16-byte aligned; tokens that nobody chose get zeros, and so do those
 * behind the last document.
 */
int colbandit_maxsim_backward(const float *dscores, const int32_t *argmax, const void *Q,
                              int n_queries, int T, int d, colbandit_dtype dt, const void *docs,
                              const int64_t *offsets, int64_t N, int64_t total_tokens, void *dQ,
                              void *ddocs, void *stream);

/*
 * norm = sqrt of the sum of the squares of all values of all tensors; every output is its
 * input times min(1, max_norm / (norm + 1e-6)): the factor is rounded to 32 bits, the product
 * as well, and to 16 bits after that where the tensor has them.
 *   n_tensors  >= 1
 *   grads, out HOST arrays of DEVICE pointers (out[i] may be grads[i]: clipped in place, and
 *              not written where nothing has to change); each aligned to its type; no other two
 *              of all these tensors overlap
 *   sizes      HOST [n_tensors]: values of each tensor, >= 0
 *   dts        HOST [n_tensors]: colbandit_dtype of each tensor and its output
 *   max_norm   > 0, may be +inf
 *   norm       DEVICE float [1]
 * Squares are summed in 64 bits, so no finite gradient overflows (a norm beyond 32 bits is
 * written as +inf, the tensors are clipped right).  A norm that is infinite or
 * NaN follows the formula (as torch's clip_grad_norm_ does): read `norm` to skip such a step.
 * out == NULL: only the norm.
 */
size_t colbandit_clip_workspace_bytes(int64_t n_tensors, const int64_t *sizes);
int colbandit_clip_gradients(int64_t n_tensors, const void *const *grads, void *const *out,
                             const int64_t *sizes, const int32_t *dts, float max_norm,
                             float *norm, void *workspace, size_t workspace_bytes, void *stream);

#ifdef __cplusplus
}
#endif
#endif /* COLBANDIT_TRAIN_H */
