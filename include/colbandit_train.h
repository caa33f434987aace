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
 *   colbandit_embedding            rows of a token table, scaled; its gradient by sorted tokens
 *   colbandit_norm_rotate          queries and keys, each head normalised, weighted and rotated by
 *                                  its row's position; its gradients
 *   colbandit_attention_window     attention through a window around each row, and to the first
 *                                  keys of its sequence; its gradients
 *   colbandit_orthogonalise        matrices (updates of weights) made nearly orthogonal
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
 * The same attention, of rows that see less of their sequence:
 *   seen   : as above, and (p_i - before <= j <= p_i + after or j < sinks)
 * Under a causal limit `after` says nothing.  Keys and values that the mask leaves are finite
 * (also those that no row's window reaches).  Rows: at most 2^28.  The gradients' workgroups for
 * the first keys count towards a launch's, one for 128 to 512 rows of a sequence, each key head and
 * 64 to 128 first keys.
 */
#define COLBANDIT_MAX_SINKS 1024
typedef struct {
    int64_t before, after;         /* >= 0; of any size                                   */
    int64_t sinks;                 /* 0 .. COLBANDIT_MAX_SINKS                            */
} colbandit_window;
size_t colbandit_sizeof_window(void);

size_t colbandit_attention_window_workspace_bytes(const colbandit_attn *a, const colbandit_window *w,
                                                  int backward);
int colbandit_attention_window(const colbandit_attn *a, const colbandit_window *w, void *out,
                               float *lse, void *workspace, size_t workspace_bytes, void *stream);
int colbandit_attention_window_backward(const colbandit_attn *a, const colbandit_window *w,
                                        const void *out, const float *lse, const void *dout,
                                        void *dq, void *dk, void *dv, void *dbias, void *workspace,
                                        size_t workspace_bytes, void *stream);

/*
 * out[i] = scale * table[tokens[i]], zeros where the token is none of 0 .. vocab-1 (padding)
 *   table    DEVICE [vocab][width], rows table_row elements apart
 *   tokens   DEVICE int64 [n];  out DEVICE [n][width]
 * Products in 32 bits, rounded once; table and out may differ in type.
 * n below 2^31 - 2^16, vocab at most 2^24, width at most 2^16.  Values looked up below 2^34 (2^36
 * where rows begin at whole multiples of 16 bytes and width is one of 8), of the gradient, n / 64
 * rows more than the table's, below 2^32 (2^34).
 */
int colbandit_embedding(const void *table, colbandit_dtype table_dt, int64_t table_row,
                        const int64_t *tokens, int64_t n, int64_t vocab, int64_t width, float scale,
                        void *out, colbandit_dtype out_dt, void *stream);
/*
 * dtable[v] = scale * sum of dout[i] over the i whose token is v; zeros for tokens that do not occur
 *   dout     DEVICE [n][width], rows dout_row elements apart;  dtable DEVICE [vocab][width]
 * Sums in 32 bits, in the order of i (of more than 64 in groups of 64 of the sorted tokens).  What
 * stands in rows of padding tokens is not read.
 */
size_t colbandit_embedding_workspace_bytes(int64_t n, int64_t vocab, int64_t width);
int colbandit_embedding_backward(const void *dout, colbandit_dtype dout_dt, int64_t dout_row,
                                 const int64_t *tokens, int64_t n, int64_t vocab, int64_t width,
                                 float scale, void *dtable, colbandit_dtype table_dt,
                                 void *workspace, size_t workspace_bytes, void *stream);

/*
 * Norms and rotation of queries and keys.  Of a head's d values x
 *   y = x / sqrt(mean of x^2 + eps) * weight
 * and of each pair (y_a, y_b), whose cosine c and sine s are the table's at the row's position,
 *   out_a = y_a c - y_b s,  out_b = y_b c + y_a s
 * Pair i is values 2i and 2i + 1 (interleaved) or i and i + d/2.  Arithmetic in 32 bits, rounded
 * once; squares must not overflow there (|x| below 2^60).
 * Rows whose position is none of the table's (padding) get zeros, and take no part in any gradient.
 * Rows of q and k lie q_row elements apart and heads q_head apart (likewise k); the d values are
 * consecutive.  Pointers to q, k, the table, outputs and gradients, and strides, are whole multiples
 * of 16 bytes.  Outputs and their gradients are dense, [rows][heads][d].  Heads: at most 4,096.
 */
typedef struct {
    int dt;                        /* colbandit_dtype of q, k, outputs, their gradients   */
    int heads, kv_heads, d;        /* d: 32, 64, 96 or 128                                */
    int interleaved;
    float eps;                     /* >= 0                                                */
    int64_t rows, n_positions;
    const void *q, *k;             /* DEVICE                                              */
    int64_t q_row, q_head, k_row, k_head;
    const float *q_weight, *k_weight;          /* DEVICE [d], or NULL: ones               */
    const float *table;            /* DEVICE [n_positions][d/2][2], or NULL: no rotation  */
    const int64_t *positions;      /* DEVICE [rows]; not read without a table             */
} colbandit_rotation;
size_t colbandit_sizeof_rotation(void);

/*
 * The usual table, in HOST memory [n_positions][d/2][2]: cosine and sine of position * base^(-2i/d),
 * computed in 64 bits.  Pure host code.
 */
int colbandit_rotary_table(int64_t n_positions, int d, double base, float *table);

/* q_out, k_out: may be q and k, where these are dense; otherwise they overlap nothing. */
int colbandit_norm_rotate(const colbandit_rotation *r, void *q_out, void *k_out, void *stream);
/*
 * dq, dk from the gradients of the outputs; dq_weight, dk_weight DEVICE float [d], either may be
 * NULL.  Sums in 32 bits, in a fixed order.
 */
size_t colbandit_norm_rotate_workspace_bytes(const colbandit_rotation *r);
int colbandit_norm_rotate_backward(const colbandit_rotation *r, const void *dq_out, const void *dk_out,
                                   void *dq, void *dk, float *dq_weight, float *dk_weight,
                                   void *workspace, size_t workspace_bytes, void *stream);

/*
 * Each matrix G, in the singular value decomposition U S V^T of it divided by its Frobenius norm,
 * becomes U p(..p(S)) V^T with p(s) = a s + b s^3 + c s^5, `steps` times: with the usual
 * coefficients singular values come near to one.  Computed by matrix products,
 *   X <- a X + (b A + c A^2) X,  A = X X^T
 * whose sums are 32 bits.  X, A and the bracket are held as two 16-bit pieces each: 22 bits of a
 * value, but some 2^-40 of the matrix' norm is lost of what is small beside it, and each step raises
 * that with the value.  They are held in 32 bits instead, with products to 2^-26 and in up to 2.3
 * times the time, where that loss could come to 2^-19 of the result, and where |a| < 1: where the
 * product of all steps' largest factors of a singular value (3.4 for the usual coefficients) and of the
 * root of rows times columns is beyond 2^22, or up to four times less where steps make singular
 * values of more than 1.5.  (Usual steps: more than five for 7,500 x 7,500 values, six for 2,200,
 * seven for 640.  Matrices that follow one another in a list, up to 40, are held alike.)  So a
 * matrix is about as far off as by plain 32-bit products, whatever its rows' and columns' sizes.  Rows
 * that are small beside the others at the end are right on their own in 32 bits, in pieces only up to
 * the loss.  What is below 2^-100 of the norm may be lost.
 * A matrix of zeros stays zeros, one that holds an infinity or NaN is NaN everywhere.
 *   n_matrices    >= 1
 *   in, out       HOST arrays of DEVICE pointers [rows][cols], dense, each aligned to its type
 *                 (out[i] may be in[i]; no other two overlap)
 *   rows, cols    HOST, >= 0; the smaller of the two at most 2^14, the other 2^26
 *                 (matrices that follow one another, up to 40: below 2^33 values in all, each side
 *                 rounded up to 64)
 *   dts           HOST: colbandit_dtype of each matrix and its output
 *   steps         1 .. 64
 *   coefficients  HOST float [3]: a, b, c.  Refused (COLBANDIT_ERR_KNOB) where singular values from
 *                 0 to 1 would pass 4 in size in some step, or b s^2 + c s^4 would pass 32.
 */
size_t colbandit_orthogonalise_workspace_bytes(int64_t n_matrices, const int64_t *rows,
                                               const int64_t *cols);
int colbandit_orthogonalise(int64_t n_matrices, const void *const *in, void *const *out,
                            const int64_t *rows, const int64_t *cols, const int32_t *dts, int steps,
                            const float *coefficients, void *workspace, size_t workspace_bytes,
                            void *stream);

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
