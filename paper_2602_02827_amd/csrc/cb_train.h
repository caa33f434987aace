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
};

// Wavefronts of a workgroup, 32 columns each.  (Of one, for sequences of up to 32 columns: one query of 32 tokens, forward pass and both
// kernels of the backward pass, 9.2, 15.1 and 8.8 us where four take 7.2, 12.3 and 6.2; 128 fp32 sequences of 32 tokens alike.)
constexpr int kWavefronts = 4;
// Wide heads take all registers: their workgroups do not go on to the next one.
constexpr bool goes_on_to_next_head(int d) { return d <= 64; }
constexpr int kMostRun = 2;      // heads that a workgroup takes one after the other (four: the histograms leave half the workgroups no LDS)

enum { AS_THEY_COME, BY_XCD, LONGEST_FIRST };         // order of workgroups

struct AttnPlan {
    int d, dt;
    int64_t q_slots, k_slots;    // places for tiles of all sequences
    int q_order, k_order;
    int units;                   // head units: heads / pack
    int run, kv_run;             // head units (key heads) that a workgroup takes one after the other
    int splits;                  // parts that the keys of a forward call's tiles are cut into
    size_t o_part, ml_part, delta, bias_part, bytes;
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

}  // namespace cb
