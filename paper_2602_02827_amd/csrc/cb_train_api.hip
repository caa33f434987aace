// C-ABI of the training operators: argument validation, plans and workspace layout.  No device arithmetic lives here.
#include <math.h>
#include <string.h>

#include "../../include/colbandit_train.h"
#include "cb_train.h"

namespace cb {

namespace {
constexpr int64_t kShortRows = 384;                   // up to six tiles of the other side's rows
int64_t round_up(int64_t x) { return (x + 255) / 256 * 256; }
}

AttnPlan plan_attention(const AttnArgs& A, int d, int dt, bool backward) {
    AttnPlan P = {};
    P.d = d;
    P.dt = dt;
    P.units = A.heads / A.pack;
    const int64_t k_rows = A.total_k / A.n_seqs;
    P.q_slots = A.total_q / (32 * kWavefronts / A.pack) + A.n_seqs;
    P.k_slots = A.total_k / (32 * kWavefronts) + A.n_seqs;
    auto order_of = [&](int64_t slots, int64_t rows) {
        return rows <= kShortRows ? BY_XCD : A.causal && slots >= 4 * (int64_t)A.n_seqs ? LONGEST_FIRST : AS_THEY_COME;
    };
    P.q_order = order_of(P.q_slots, k_rows);
    P.k_order = order_of(P.k_slots, (int64_t)A.total_q * A.group / A.n_seqs);
    P.splits = 1;
    // Short sequences: a workgroup goes on to the next heads, as long as enough workgroups are left (six a CU).
    // 512 passages, forward and backward: 691 us, one head each 706.
    auto run_of = [](int64_t slots, int units, int64_t rows) {
        int r = 1;
        while (rows <= kShortRows && 2 * r <= kMostRun && 2 * r <= units && slots * (units / (2 * r)) >= 1536) r *= 2;
        return r;
    };
    P.run = goes_on_to_next_head(d) ? run_of(P.q_slots, P.units, k_rows) : 1;
    P.kv_run = goes_on_to_next_head(d) ? run_of(P.k_slots, A.kv_heads, (int64_t)A.total_q * A.group / A.n_seqs) : 1;
    if (A.bias && A.reach > 128) P.run = 1;          // (histograms of all its heads are in LDS)
    const int64_t groups = P.q_slots * P.units;
    ++P.q_slots;                                     // the rows behind the last sequence may end in a tile of their own
    ++P.k_slots;
    size_t o = 0;
    auto take = [&](int64_t bytes) {
        const size_t at = o;
        o += (size_t)round_up(bytes);
        return at;
    };
    if (!backward) {
        // Few tiles over long keys: their keys are cut into parts of 128 rows or more (on average; the longest sequence's are
        // longer) until there are 2,048 workgroups.  16 tokens over 1 to 16,385 keys, us: 40 so, 46 with 256 rows and 1,024, 42 with
        // 128 and 4,096, 66 with 512 and 1,024.
        if (groups < 512 && k_rows >= 512) {
            int64_t s = (2048 - 1 + groups) / groups;
            s = s < k_rows / 128 ? s : k_rows / 128;
            P.splits = (int)(s < 1 ? 1 : s > 256 ? 256 : s);
        }
        if (P.splits > 1) {
            const int64_t rows = (int64_t)A.heads * A.total_q * P.splits;
            P.o_part = take(rows * d * 4);
            P.ml_part = take(rows * 8);
        }
    } else {
        P.delta = take((int64_t)A.heads * A.total_q * 8);        // and a value of rows that are far (is_far)
        if (A.bias) P.bias_part = take(P.q_slots * A.heads * A.n_buckets * 4);
    }
    P.bytes = o;
    return P;
}

}  // namespace cb

using namespace cb;

namespace {

constexpr int64_t kMostRows = 0x7fffffff - (1 << 16), kMostRowBytes = 1 << 25;

bool misaligned(const void* p, size_t to = 16) { return ((uintptr_t)p & (to - 1)) != 0; }

int workspace_ok(const void* ws, size_t bytes, size_t need) {
    if (need == 0) return COLBANDIT_OK;
    if (!ws) return COLBANDIT_ERR_NULL;
    if (misaligned(ws, 256)) return COLBANDIT_ERR_ALIGNMENT;
    return bytes < need ? COLBANDIT_ERR_WORKSPACE : COLBANDIT_OK;
}

// First distance of each bucket of a direction with n of them.
void bucket_starts(int n, int max_distance, int32_t* starts) {
    const int single = n / 2;
    for (int i = 0; i < n; ++i) {
        if (i < single) {
            starts[i] = i;
        } else {
            const double x = single * pow((double)max_distance / single, (double)(i - single) / (n - single));
            starts[i] = (int32_t)ceil(x - 1e-9);
        }
    }
}
int check_buckets(int n_buckets, int max_distance, int causal, int* n_dir) {
    if (n_buckets < 1 || max_distance < 1) return COLBANDIT_ERR_SHAPE;
    if (!causal && n_buckets % 2) return COLBANDIT_ERR_SHAPE;
    const int n = causal ? n_buckets : n_buckets / 2;
    if (n < 2 || max_distance <= n / 2) return COLBANDIT_ERR_SHAPE;
    if (n_buckets > COLBANDIT_MAX_BUCKETS || max_distance > COLBANDIT_MAX_DISTANCE) return COLBANDIT_ERR_UNSUPPORTED;
    *n_dir = n;
    return COLBANDIT_OK;
}

int attn_args(const colbandit_attn* a, AttnArgs& A) {
    if (!a) return COLBANDIT_ERR_NULL;
    if (a->dt != COLBANDIT_F32 && a->dt != COLBANDIT_BF16) return COLBANDIT_ERR_SHAPE;
    if (a->n_seqs < 1 || a->heads < 1 || a->kv_heads < 1 || a->d < 1 || a->total_q < 0 || a->total_k < 0 || a->heads % a->kv_heads)
        return COLBANDIT_ERR_SHAPE;
    if (!(a->scale > -INFINITY && a->scale < INFINITY)) return COLBANDIT_ERR_KNOB;
    if (a->d != 32 && a->d != 64 && a->d != 96 && a->d != 128) return COLBANDIT_ERR_UNSUPPORTED;
    if (a->total_q > kMostRows || a->total_k > kMostRows || a->n_seqs > kMostRows) return COLBANDIT_ERR_UNSUPPORTED;
    if (!a->q_offsets || !a->k_offsets || (a->total_q && !a->q) || (a->total_k && (!a->k || !a->v))) return COLBANDIT_ERR_NULL;
    const int64_t eb = a->dt == COLBANDIT_BF16 ? 2 : 4;
    const int64_t strides[] = {a->q_row, a->q_head, a->k_row, a->k_head, a->v_row, a->v_head};
    for (int64_t s : strides) {
        if (s < 0) return COLBANDIT_ERR_SHAPE;
        if (s * eb % 16) return COLBANDIT_ERR_ALIGNMENT;
    }
    // a tile's rows are addressed in 32 bits from its first one
    if (a->k_row * eb > kMostRowBytes || a->v_row * eb > kMostRowBytes || a->q_row * eb > kMostRowBytes ||
        (int64_t)a->heads * a->d * eb > kMostRowBytes)
        return COLBANDIT_ERR_UNSUPPORTED;
    if (misaligned(a->q) || misaligned(a->k) || misaligned(a->v) || misaligned(a->q_offsets, 8) || misaligned(a->k_offsets, 8))
        return COLBANDIT_ERR_ALIGNMENT;
    A = AttnArgs{};
    if (a->bias) {
        int32_t starts[COLBANDIT_MAX_BUCKETS];
        const int rc = check_buckets(a->n_buckets, a->max_distance, a->causal, &A.n_dir);
        if (rc) return rc;
        if (misaligned(a->bias, (size_t)eb)) return COLBANDIT_ERR_ALIGNMENT;
        bucket_starts(A.n_dir, a->max_distance, starts);
        for (int i = 0; i < A.n_dir; ++i) A.starts[i] = (int16_t)starts[i];
        A.reach = starts[A.n_dir - 1];
        A.n_buckets = a->n_buckets;
        A.bias = a->bias;
    }
    A.q = a->q;
    A.k = a->k;
    A.v = a->v;
    A.q_row = a->q_row;
    A.q_head = a->q_head;
    A.k_row = a->k_row;
    A.k_head = a->k_head;
    A.v_row = a->v_row;
    A.v_head = a->v_head;
    A.qoff = a->q_offsets;
    A.koff = a->k_offsets;
    A.keep = a->keep;
    A.n_seqs = a->n_seqs;
    A.heads = a->heads;
    A.kv_heads = a->kv_heads;
    A.group = a->heads / a->kv_heads;
    // (16 single tokens, four heads to a key head: 40 us, a tile for each head 85; 24 causal pages, with gradients: 507 and 541)
    A.pack = !a->bias && A.group <= 16 && a->q_head * eb <= kMostRowBytes && a->total_q <= kMostRows / A.group &&
                     a->total_k <= kMostRows / A.group ? A.group : 1;      // columns are counted in 31 bits
    A.total_q = (int)a->total_q;
    A.total_k = (int)a->total_k;
    A.causal = a->causal != 0;
    A.scale = a->scale;
    return COLBANDIT_OK;
}

// Threads of one launch, below 2^32.
bool fits_a_grid(int64_t groups, int64_t threads) { return groups <= 0xffffffffll / threads; }

// Every launch of the plan can be made.
bool launchable(const AttnArgs& A, const AttnPlan& P) {
    if (A.heads > 1 << 12 || P.bytes >= (1ull << 46)) return false;
    const int64_t rows = (int64_t)A.heads * A.total_q, entries = A.bias ? (int64_t)A.n_buckets * A.heads : 0;
    return fits_a_grid(P.q_slots * ((P.units + P.run - 1) / P.run) * P.splits, 64 * kWavefronts) &&
           fits_a_grid(P.k_slots * ((A.kv_heads + P.kv_run - 1) / P.kv_run) + entries, 128 * kWavefronts) &&      // (some have twice as many)
           (P.splits == 1 || fits_a_grid((rows + 3) / 4, 256));
}

int check_maxsim(const void* Q, int nq, int T, int d, int dt, const void* docs, const int64_t* off, int64_t N, int64_t total) {
    if (!Q || !off || (total > 0 && !docs)) return COLBANDIT_ERR_NULL;
    if (nq < 1 || T < 1 || d < 1 || N < 1 || total < 0) return COLBANDIT_ERR_SHAPE;
    if (dt != COLBANDIT_F32 && dt != COLBANDIT_BF16) return COLBANDIT_ERR_SHAPE;
    if (d != 32 && d != 64 && d != 96 && d != 128) return COLBANDIT_ERR_UNSUPPORTED;
    // places of documents' tiles and entries are counted in 31 bits
    if (T > COLBANDIT_MAX_T || nq > 65535 || total > kMostRows || N > (1 << 28)) return COLBANDIT_ERR_UNSUPPORTED;
    if (misaligned(Q) || misaligned(docs) || misaligned(off, 8)) return COLBANDIT_ERR_ALIGNMENT;
    return COLBANDIT_OK;
}

int hip(hipError_t e) { return e == hipSuccess ? COLBANDIT_OK : COLBANDIT_ERR_HIP; }

}  // namespace

extern "C" {

size_t colbandit_sizeof_attn(void) { return sizeof(colbandit_attn); }

int colbandit_bias_buckets(int n_buckets, int max_distance, int causal, int32_t* starts) {
    if (!starts) return COLBANDIT_ERR_NULL;
    int n = 0;
    const int rc = check_buckets(n_buckets, max_distance, causal, &n);
    if (rc) return rc;
    bucket_starts(n, max_distance, starts);
    return n;
}

size_t colbandit_attention_workspace_bytes(const colbandit_attn* a, int backward) {
    AttnArgs A;
    if (attn_args(a, A)) return 0;
    return plan_attention(A, a->d, a->dt, backward != 0).bytes;
}

int colbandit_attention(const colbandit_attn* a, void* out, float* lse, void* workspace, size_t workspace_bytes, void* stream) {
    AttnArgs A;
    int rc = attn_args(a, A);
    if (rc) return rc;
    if (A.total_q && (!out || !lse)) return COLBANDIT_ERR_NULL;
    if (misaligned(out) || misaligned(lse, 4)) return COLBANDIT_ERR_ALIGNMENT;
    const AttnPlan P = plan_attention(A, a->d, a->dt, false);
    if (!launchable(A, P)) return COLBANDIT_ERR_UNSUPPORTED;
    rc = workspace_ok(workspace, workspace_bytes, P.bytes);
    if (rc) return rc;
    const hipStream_t st = (hipStream_t)stream;
    return hip(a->dt == COLBANDIT_BF16 ? launch_attention_bf16(A, P, out, lse, (char*)workspace, st)
                                       : launch_attention_f32(A, P, out, lse, (char*)workspace, st));
}

int colbandit_attention_backward(const colbandit_attn* a, const void* out, const float* lse, const void* dout, void* dq, void* dk,
                                 void* dv, void* dbias, void* workspace, size_t workspace_bytes, void* stream) {
    AttnArgs A;
    int rc = attn_args(a, A);
    if (rc) return rc;
    if (A.total_q && (!out || !lse || !dout || !dq)) return COLBANDIT_ERR_NULL;
    if (A.total_k && (!dk || !dv)) return COLBANDIT_ERR_NULL;
    if (A.bias && !dbias) return COLBANDIT_ERR_NULL;
    if (misaligned(out) || misaligned(dout) || misaligned(dq) || misaligned(dk) || misaligned(dv) || misaligned(lse, 4) ||
        misaligned(dbias, a->dt == COLBANDIT_BF16 ? 2 : 4))
        return COLBANDIT_ERR_ALIGNMENT;
    const AttnPlan P = plan_attention(A, a->d, a->dt, true);
    if (!launchable(A, P)) return COLBANDIT_ERR_UNSUPPORTED;
    rc = workspace_ok(workspace, workspace_bytes, P.bytes);
    if (rc) return rc;
    const AttnGrads G = {out, dout, lse, dq, dk, dv, dbias};
    const hipStream_t st = (hipStream_t)stream;
    return hip(a->dt == COLBANDIT_BF16 ? launch_attention_backward_bf16(A, P, G, (char*)workspace, st)
                                       : launch_attention_backward_f32(A, P, G, (char*)workspace, st));
}

int colbandit_maxsim_scores(const void* Q, int n_queries, int T, int d, colbandit_dtype dt, const void* docs, const int64_t* offsets,
                            int64_t N, int64_t total_tokens, float* scores, int32_t* argmax, void* stream) {
    const int rc = check_maxsim(Q, n_queries, T, d, dt, docs, offsets, N, total_tokens);
    if (rc) return rc;
    if (!scores || !argmax) return COLBANDIT_ERR_NULL;
    if (misaligned(scores, 4) || misaligned(argmax, 4)) return COLBANDIT_ERR_ALIGNMENT;
    return hip(launch_maxsim_scores(Q, n_queries, T, d, dt, docs, offsets, N, total_tokens, scores, argmax, (hipStream_t)stream));
}

int colbandit_contrastive_loss(const float* scores, int n_queries, int64_t N, const int64_t* targets, float temperature, float* loss,
                               float* dscores, void* stream) {
    if (!scores || !targets || !loss || !dscores) return COLBANDIT_ERR_NULL;
    if (n_queries < 1 || N < 1) return COLBANDIT_ERR_SHAPE;
    if (!(temperature > 0.f && temperature < INFINITY && 1.f / temperature < INFINITY)) return COLBANDIT_ERR_KNOB;
    if (n_queries > 65535) return COLBANDIT_ERR_UNSUPPORTED;
    if (misaligned(scores, 4) || misaligned(targets, 8) || misaligned(loss, 4) || misaligned(dscores, 4)) return COLBANDIT_ERR_ALIGNMENT;
    return hip(launch_contrastive_loss(scores, n_queries, N, targets, temperature, loss, dscores, (hipStream_t)stream));
}

int colbandit_maxsim_backward(const float* dscores, const int32_t* argmax, const void* Q, int n_queries, int T, int d,
                              colbandit_dtype dt, const void* docs, const int64_t* offsets, int64_t N, int64_t total_tokens, void* dQ,
                              void* ddocs, void* stream) {
    const int rc = check_maxsim(Q, n_queries, T, d, dt, docs, offsets, N, total_tokens);
    if (rc) return rc;
    if (!fits_a_grid(maxsim_backward_groups(n_queries, T, N, total_tokens), 256)) return COLBANDIT_ERR_UNSUPPORTED;
    if (!dscores || !argmax || !dQ || (total_tokens && !ddocs)) return COLBANDIT_ERR_NULL;
    if (misaligned(dscores, 4) || misaligned(argmax, 4) || misaligned(dQ) || misaligned(ddocs)) return COLBANDIT_ERR_ALIGNMENT;
    return hip(launch_maxsim_backward(dscores, argmax, Q, n_queries, T, d, dt, docs, offsets, N, total_tokens, dQ, ddocs,
                                      (hipStream_t)stream));
}

size_t colbandit_clip_workspace_bytes(int64_t n_tensors, const int64_t* sizes) {
    return n_tensors < 1 || !sizes ? 0 : clip_workspace_bytes(n_tensors, sizes);
}

int colbandit_clip_gradients(int64_t n_tensors, const void* const* grads, void* const* out, const int64_t* sizes, const int32_t* dts,
                             float max_norm, float* norm, void* workspace, size_t workspace_bytes, void* stream) {
    if (!grads || !sizes || !dts || !norm) return COLBANDIT_ERR_NULL;
    if (n_tensors < 1) return COLBANDIT_ERR_SHAPE;
    if (!(max_norm > 0.f)) return COLBANDIT_ERR_KNOB;
    int64_t all = 0;
    for (int64_t i = 0; i < n_tensors; ++i) {
        if (sizes[i] < 0 || (dts[i] != COLBANDIT_F32 && dts[i] != COLBANDIT_BF16)) return COLBANDIT_ERR_SHAPE;
        if (sizes[i] && (!grads[i] || (out && !out[i]))) return COLBANDIT_ERR_NULL;
        const size_t eb = dts[i] == COLBANDIT_BF16 ? 2 : 4;
        if (misaligned(grads[i], eb) || (out && misaligned(out[i], eb))) return COLBANDIT_ERR_ALIGNMENT;
        // chunks of one launch's tensors are counted in 32 bits
        if (sizes[i] > ((int64_t)1 << 42) || (all += sizes[i]) > ((int64_t)1 << 44)) return COLBANDIT_ERR_UNSUPPORTED;
    }
    if (misaligned(norm, 4)) return COLBANDIT_ERR_ALIGNMENT;
    const int rc = workspace_ok(workspace, workspace_bytes, clip_workspace_bytes(n_tensors, sizes));
    if (rc) return rc;
    return hip(launch_clip(n_tensors, grads, out, sizes, dts, max_norm, norm, workspace, (hipStream_t)stream));
}

}  // extern "C"
