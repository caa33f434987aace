// Host-side launch interface of the training operators, and what their kernels share.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace cb {

enum { TR_F32 = 0, TR_BF16 = 1 };

// An attention problem as the kernels take it (by value).
struct AttnArgs {
    const void *q, *k, *v;
    int64_t q_row, q_head, k_row, k_head, v_row, v_head;   // strides in elements
    const int64_t *qoff, *koff;
    const uint8_t* keep;
    const void* bias;            // [n_buckets][heads]
    int n_seqs, heads, kv_heads, group;
    int pack;                    // heads of a group whose rows share a tile: all of them, or one
    int total_q, total_k;
    int causal;
    float scale;
    int n_buckets, n_dir;        // buckets in all, and of one direction
    int reach;                   // first distance of a direction's last bucket
    int16_t starts[128];         // first distance of each bucket of one direction
    int windowed;                // rows see `before` keys before them, `after` behind them, and the first `sinks`
    int before, after, sinks;
    int sink_rows;               // rows of a sequence that one workgroup adds up for the gradients of its first keys
};

// Wavefronts of a workgroup, 32 columns each.  (Of one, for sequences of up to 32 columns: one query of 32 tokens, forward pass and both
// kernels of the backward pass, 9.2, 15.1 and 8.8 us where four take 7.2, 12.3 and 6.2; 128 fp32 sequences of 32 tokens alike.)
constexpr int kWavefronts = 4;
// Wide heads take all registers: their workgroups do not go on to the next one.
constexpr bool goes_on_to_next_head(int d) { return d <= 64; }
// In 16 bits the gradients of wide heads' keys and values take a wavefront each.
constexpr bool two_for_keys(int d, int bytes) { return bytes == 2 && d >= 96; }
constexpr int kMostRun = 2;      // heads that a workgroup takes one after the other (four: the histograms leave half the workgroups no LDS)

enum { AS_THEY_COME, BY_XCD, LONGEST_FIRST };         // order of workgroups

struct AttnPlan {
    int d, dt;
    int64_t q_slots, k_slots;    // places for tiles of all sequences
    int q_order, k_order;
    int units;                   // head units: heads / pack
    int run, kv_run;             // head units (key heads) that a workgroup takes one after the other
    int splits;                  // parts that the keys of a forward call's tiles are cut into
    int64_t sink_groups;         // workgroups for the first keys' gradients
    size_t o_part, ml_part, delta, bias_part, sink_part, bytes;
};
AttnPlan plan_attention(const AttnArgs& A, int d, int dt, bool backward);

hipError_t launch_attention_bf16(const AttnArgs& A, const AttnPlan& P, void* out, float* lse, char* ws, hipStream_t st);
hipError_t launch_attention_f32(const AttnArgs& A, const AttnPlan& P, void* out, float* lse, char* ws, hipStream_t st);
struct AttnGrads {
    const void *out, *dout;
    const float* lse;
    void *dq, *dk, *dv, *dbias;
};
hipError_t launch_attention_backward_bf16(const AttnArgs& A, const AttnPlan& P, const AttnGrads& G, char* ws, hipStream_t st);
hipError_t launch_attention_backward_f32(const AttnArgs& A, const AttnPlan& P, const AttnGrads& G, char* ws, hipStream_t st);

hipError_t launch_attention_window_bf16(const AttnArgs& A, const AttnPlan& P, void* out, float* lse, char* ws, hipStream_t st);
hipError_t launch_attention_window_f32(const AttnArgs& A, const AttnPlan& P, void* out, float* lse, char* ws, hipStream_t st);
hipError_t launch_attention_window_backward_bf16(const AttnArgs& A, const AttnPlan& P, const AttnGrads& G, char* ws, hipStream_t st);
hipError_t launch_attention_window_backward_f32(const AttnArgs& A, const AttnPlan& P, const AttnGrads& G, char* ws, hipStream_t st);

hipError_t launch_maxsim_scores(const void* Q, int nq, int T, int d, int dt, const void* docs, const int64_t* off, int64_t N,
                                int64_t total, float* scores, int32_t* argmax, hipStream_t st);
hipError_t launch_contrastive_loss(const float* scores, int nq, int64_t N, const int64_t* targets, float temperature,
                                   float* loss, float* dscores, hipStream_t st);
int64_t maxsim_backward_groups(int nq, int T, int64_t N, int64_t total);     // of 256 threads
hipError_t launch_maxsim_backward(const float* dscores, const int32_t* argmax, const void* Q, int nq, int T, int d, int dt,
                                  const void* docs, const int64_t* off, int64_t N, int64_t total, void* dQ, void* ddocs,
                                  hipStream_t st);

size_t clip_workspace_bytes(int64_t n, const int64_t* sizes);
hipError_t launch_clip(int64_t n, const void* const* grads, void* const* out, const int64_t* sizes, const int32_t* dts,
                       float max_norm, float* norm, void* ws, hipStream_t st);

int embedding_piece(const void* rows, int rows_dt, int64_t row, const void* dense, int dense_dt, int64_t width);      // values of a piece
bool embedding_launchable(int64_t n, int64_t vocab, int64_t width, int piece, bool backward);
hipError_t launch_embedding(const void* table, int table_dt, int64_t table_row, const int64_t* tokens, int64_t n, int64_t vocab, int64_t width,
                            float scale, void* out, int out_dt, hipStream_t st);
size_t embedding_workspace_bytes(int64_t n, int64_t vocab, int64_t width);
hipError_t launch_embedding_backward(const void* dout, int dout_dt, int64_t dout_row, const int64_t* tokens, int64_t n, int64_t vocab,
                                     int64_t width, float scale, void* dtable, int table_dt, char* ws, hipStream_t st);

// Norms of queries and keys with rotation, as the kernels take them (by value).
struct RotateArgs {
    const void *q, *k;
    int64_t q_row, q_head, k_row, k_head;
    const float *q_weight, *k_weight, *table;        // table [n_positions][d / 2][2]: cosine, sine
    const int64_t* positions;
    int64_t rows, n_positions;
    int heads, kv_heads, near;
    float eps;
    const void *dq_out, *dk_out;                     // (backward pass) gradients of the outputs
    void *q_to, *k_to;                               // outputs, or gradients of the inputs
    float* part;                                     // the workgroups' sums for the weights' gradients
};
size_t rotate_workspace_bytes(const RotateArgs& A, int d);
hipError_t launch_rotate(const RotateArgs& A, int d, int dt, hipStream_t st);
hipError_t launch_rotate_backward(const RotateArgs& A, int d, int dt, float* dq_weight, float* dk_weight, hipStream_t st);

// A's scale is X's squared times this, so that what the product of its pieces is multiplied by is a constant: X's is at most 2^15, and
// 49,152 by the largest singular value, which leaves A below 36,864.  (As an argument it cost an encoder's matrices 1,608 us for 1,585.)
constexpr float kGramScale = 0x1p-16f;
// A polynomial a s + b s^3 + c s^5 and what is known of its steps from singular values of up to one on.
struct OrthoPolynomial {
    float a, b, c;
    float scale_x, scale_a, scale_b; // powers of two that X, A and B are held times in 16-bit pieces (1 in 32 bits)
    double raised;                   // factor by which the steps raise small values at most; infinite where they lower them
};
size_t ortho_workspace_bytes(int64_t n, const int64_t* rows, const int64_t* cols);
bool ortho_launchable(int64_t n, const int64_t* rows, const int64_t* cols);
hipError_t launch_ortho(int64_t n, const void* const* in, void* const* out, const int64_t* rows, const int64_t* cols, const int32_t* dts,
                        int steps, const OrthoPolynomial& polynomial, char* ws, hipStream_t st);

}  // namespace cb
