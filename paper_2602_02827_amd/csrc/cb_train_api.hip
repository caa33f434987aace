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
    int64_t k_rows = A.total_k / A.n_seqs, q_rows = (int64_t)A.total_q * A.group / A.n_seqs;
    if (A.windowed) {                                // what a tile sees of them
        const int64_t tile = 32 * kWavefronts, span = (int64_t)A.before + A.after + tile;
        k_rows = span + A.sinks < k_rows ? span + A.sinks : k_rows;
        q_rows = span * A.group < q_rows ? span * A.group : q_rows;
    }
    P.q_slots = A.total_q / (32 * kWavefronts / A.pack) + A.n_seqs;
    const int64_t key_tile = A.windowed && two_for_keys(d, dt == TR_BF16 ? 2 : 4) ? 16 * kWavefronts : 32 * kWavefronts;
    P.k_slots = A.total_k / key_tile + A.n_seqs;
    auto order_of = [&](int64_t slots, int64_t rows) {
        return rows <= kShortRows ? BY_XCD : A.causal && slots >= 4 * (int64_t)A.n_seqs ? LONGEST_FIRST : AS_THEY_COME;
    };
    P.q_order = order_of(P.q_slots, k_rows);
    P.k_order = order_of(P.k_slots, q_rows);
    P.splits = 1;
    // Short sequences: a workgroup goes on to the next heads, as long as enough workgroups are left (six a CU).
    // 512 passages, forward and backward, before later steps: 691 us, one head each 706.
    auto run_of = [](int64_t slots, int units, int64_t rows) {
        int r = 1;
        while (rows <= kShortRows && 2 * r <= kMostRun && 2 * r <= units && slots * (units / (2 * r)) >= 1536) r *= 2;
        return r;
    };
    P.run = goes_on_to_next_head(d) ? run_of(P.q_slots, P.units, k_rows) : 1;
    P.kv_run = goes_on_to_next_head(d) ? run_of(P.k_slots, A.kv_heads, q_rows) : 1;
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
        // 128 and 4,096, 66 with 512 and 1,024.  Through a window rows see fewer keys than there are: parts of 64 (16 that see 1,028
        // keys: 17 us, of 128 rows 18.4).
        const int64_t part = A.windowed ? 64 : 128;
        if (groups < 512 && k_rows >= 4 * part) {
            int64_t s = (2048 - 1 + groups) / groups;
            s = s < k_rows / part ? s : k_rows / part;
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
        if (A.windowed && A.sinks) {
            const int64_t slots = A.total_q / A.sink_rows + A.n_seqs;
            P.sink_groups = slots * A.kv_heads * ((A.sinks + key_tile - 1) / key_tile);
            P.sink_part = take(2 * (A.total_q / A.sink_rows + 1) * (int64_t)A.kv_heads * A.sinks * 2 * d * 4);
        }
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
    // (16 single tokens, four heads to a key head: 40 us, a tile for each head 85; 24 causal pages, with gradients, before later steps: 507 and 541)
    A.pack = !a->bias && A.group <= 16 && a->q_head * eb <= kMostRowBytes && a->total_q <= kMostRows / A.group &&
                     a->total_k <= kMostRows / A.group ? A.group : 1;      // columns are counted in 31 bits
    A.total_q = (int)a->total_q;
    A.total_k = (int)a->total_k;
    A.causal = a->causal != 0;
    A.scale = a->scale;
    return COLBANDIT_OK;
}

// Distances and their sums with rows are counted in 31 bits.
constexpr int64_t kMostWindowRows = 1 << 28;
constexpr int kWholeWindow = 1 << 29;

int64_t size_of(int dt) { return dt == COLBANDIT_BF16 ? 2 : 4; }
int window_args(const colbandit_attn* a, const colbandit_window* w, AttnArgs& A) {
    if (!w) return COLBANDIT_ERR_NULL;
    if (w->before < 0 || w->after < 0 || w->sinks < 0) return COLBANDIT_ERR_SHAPE;
    if (w->sinks > COLBANDIT_MAX_SINKS || A.total_q > kMostWindowRows || A.total_k > kMostWindowRows) return COLBANDIT_ERR_UNSUPPORTED;
    A.windowed = 1;
    A.before = w->before < kWholeWindow ? (int)w->before : kWholeWindow;
    A.after = A.causal ? 0 : w->after < kWholeWindow ? (int)w->after : kWholeWindow;
    A.sinks = (int)w->sinks;
    // Short enough for an even load, since workgroups of the first keys have little to do at a time, as long as that costs little
    // workspace.  (8 documents of 2,048 tokens, two key heads of 128 under eight, a window of 256 rows and four first keys, with
    // gradients: 216 us, with 256 rows 232, with 512 242; of up to 4,095 tokens, heads of 64: 175, 164 and 167.
    // More first keys are more workgroups, and more shares to add up: backward pass of the first documents with 200 of them, in chunks of
    // 256 and of 512 rows, 231 and 237 us, with 300 266 and 254; 26 pages of 1,030 tokens, six heads of 64, 100 first keys, 142 and 137,
    // with 300 223 and 198.)
    A.sink_rows = A.sinks > 256 ? 512 : A.sinks > 64 || !two_for_keys(a->d, (int)size_of(a->dt)) ? 256 : 128;
    return COLBANDIT_OK;
}

// Threads of one launch, below 2^32.
bool fits_a_grid(int64_t groups, int64_t threads) { return groups <= 0xffffffffll / threads; }

// Every launch of the plan can be made.
bool launchable(const AttnArgs& A, const AttnPlan& P) {
    if (A.heads > 1 << 12 || P.bytes >= (1ull << 46)) return false;
    const int64_t rows = (int64_t)A.heads * A.total_q, entries = A.bias ? (int64_t)A.n_buckets * A.heads : 0;
    return fits_a_grid(P.q_slots * ((P.units + P.run - 1) / P.run) * P.splits, 64 * kWavefronts) &&
           fits_a_grid(P.k_slots * ((A.kv_heads + P.kv_run - 1) / P.kv_run) + P.sink_groups + entries, 128 * kWavefronts) &&      // (some have twice as many)
           fits_a_grid(((int64_t)A.n_seqs * A.kv_heads * A.sinks + 3) / 4, 256) &&
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

int attention(const colbandit_attn* a, AttnArgs& A, void* out, float* lse, void* workspace, size_t workspace_bytes, void* stream) {
    if (A.total_q && (!out || !lse)) return COLBANDIT_ERR_NULL;
    if (misaligned(out) || misaligned(lse, 4)) return COLBANDIT_ERR_ALIGNMENT;
    const AttnPlan P = plan_attention(A, a->d, a->dt, false);
    if (!launchable(A, P)) return COLBANDIT_ERR_UNSUPPORTED;
    const int rc = workspace_ok(workspace, workspace_bytes, P.bytes);
    if (rc) return rc;
    const auto launch = A.windowed ? (a->dt == COLBANDIT_BF16 ? launch_attention_window_bf16 : launch_attention_window_f32)
                                   : (a->dt == COLBANDIT_BF16 ? launch_attention_bf16 : launch_attention_f32);
    return hip(launch(A, P, out, lse, (char*)workspace, (hipStream_t)stream));
}

int attention_backward(const colbandit_attn* a, AttnArgs& A, const AttnGrads& G, void* workspace, size_t workspace_bytes, void* stream) {
    if (A.total_q && (!G.out || !G.lse || !G.dout || !G.dq)) return COLBANDIT_ERR_NULL;
    if (A.total_k && (!G.dk || !G.dv)) return COLBANDIT_ERR_NULL;
    if (A.bias && !G.dbias) return COLBANDIT_ERR_NULL;
    if (misaligned(G.out) || misaligned(G.dout) || misaligned(G.dq) || misaligned(G.dk) || misaligned(G.dv) || misaligned(G.lse, 4) ||
        misaligned(G.dbias, a->dt == COLBANDIT_BF16 ? 2 : 4))
        return COLBANDIT_ERR_ALIGNMENT;
    const AttnPlan P = plan_attention(A, a->d, a->dt, true);
    if (!launchable(A, P)) return COLBANDIT_ERR_UNSUPPORTED;
    const int rc = workspace_ok(workspace, workspace_bytes, P.bytes);
    if (rc) return rc;
    const auto launch = A.windowed ? (a->dt == COLBANDIT_BF16 ? launch_attention_window_backward_bf16 : launch_attention_window_backward_f32)
                                   : (a->dt == COLBANDIT_BF16 ? launch_attention_backward_bf16 : launch_attention_backward_f32);
    return hip(launch(A, P, G, (char*)workspace, (hipStream_t)stream));
}

bool is_type(int dt) { return dt == COLBANDIT_F32 || dt == COLBANDIT_BF16; }

constexpr int64_t kMostVocab = 1 << 24, kMostWidth = 1 << 16;
int check_embedding(int64_t n, int64_t vocab, int64_t width, int64_t row, int dt, int other) {
    if (n < 0 || vocab < 1 || width < 1 || !is_type(dt) || !is_type(other)) return COLBANDIT_ERR_SHAPE;
    if (row < width) return COLBANDIT_ERR_SHAPE;
    if (n > kMostRows || vocab > kMostVocab || width > kMostWidth || row > ((int64_t)1 << 32)) return COLBANDIT_ERR_UNSUPPORTED;
    return COLBANDIT_OK;
}

int rotate_args(const colbandit_rotation* r, RotateArgs& A) {
    if (!r) return COLBANDIT_ERR_NULL;
    if (!is_type(r->dt) || r->rows < 0 || r->heads < 1 || r->kv_heads < 1 || r->d < 1) return COLBANDIT_ERR_SHAPE;
    if (!(r->eps >= 0.f && r->eps < INFINITY)) return COLBANDIT_ERR_KNOB;
    if (r->d != 32 && r->d != 64 && r->d != 96 && r->d != 128) return COLBANDIT_ERR_UNSUPPORTED;
    if (r->rows > kMostRows || r->heads > 1 << 12) return COLBANDIT_ERR_UNSUPPORTED;
    if (r->kv_heads > 1 << 12 || r->n_positions > ((int64_t)1 << 40)) return COLBANDIT_ERR_UNSUPPORTED;
    if (r->table && r->n_positions < 1) return COLBANDIT_ERR_SHAPE;
    if (r->rows && (!r->q || !r->k || (r->table && !r->positions))) return COLBANDIT_ERR_NULL;
    const int64_t strides[] = {r->q_row, r->q_head, r->k_row, r->k_head};
    for (int64_t s : strides) {
        if (s < 0) return COLBANDIT_ERR_SHAPE;
        if (s * size_of(r->dt) % 16) return COLBANDIT_ERR_ALIGNMENT;
    }
    if (misaligned(r->q) || misaligned(r->k) || misaligned(r->table) || misaligned(r->positions, 8) || misaligned(r->q_weight, 4) ||
        misaligned(r->k_weight, 4))
        return COLBANDIT_ERR_ALIGNMENT;
    A = RotateArgs{};
    A.q = r->q;
    A.k = r->k;
    A.q_row = r->q_row;
    A.q_head = r->q_head;
    A.k_row = r->k_row;
    A.k_head = r->k_head;
    A.q_weight = r->q_weight;
    A.k_weight = r->k_weight;
    A.table = r->table;
    A.positions = r->positions;
    A.rows = r->rows;
    A.n_positions = r->n_positions;
    A.heads = r->heads;
    A.kv_heads = r->kv_heads;
    A.near = r->interleaved != 0;
    A.eps = r->eps;
    return COLBANDIT_OK;
}

// The largest power of two that takes what is at most `limit` in size to no more than three quarters of what 16 bits hold.
float scale_for(double limit) { return (float)exp2(floor(log2(49152.0 / fmax(limit, 1.0)))); }

// Whether singular values from 0 to 1 stay within what the pieces of X, A and B can hold (4, 16 and 32 in size) over all steps of
// s <- a s + b s^3 + c s^5, and what the kernels have to know of them.  A polynomial's extremes are where its derivative is zero, and
// at the ends.
bool polynomial_holds(const float* k, int steps, OrthoPolynomial& P) {
    const double a = k[0], b = k[1], c = k[2];
    if (!isfinite(a) || !isfinite(b) || !isfinite(c)) return false;
    double most = 1.0, most_x = 1.0, most_b = 0.0, raised = 1.0;
    for (int s = 0; s < steps; ++s) {
        most *= 1.0001;                              // (roundings)
        if (most > 4.0) return false;
        const double u1 = most * most;
        auto square = [&](double u) { return fabs(b * u + c * u * u); };
        double side = square(u1);
        if (c != 0.0 && -b / (2 * c) > 0.0 && -b / (2 * c) < u1) side = fmax(side, square(-b / (2 * c)));
        if (side > 32.0) return false;
        most_x = fmax(most_x, most);
        most_b = fmax(most_b, side);
        auto factor = [&](double u) { return fabs(a + b * u + c * u * u); };      // of a singular value sqrt(u)
        double most_factor = fmax(factor(0.0), factor(u1));
        if (c != 0.0 && -b / (2 * c) > 0.0 && -b / (2 * c) < u1) most_factor = fmax(most_factor, factor(-b / (2 * c)));
        raised *= most_factor;
        auto value = [&](double u) { return fabs(sqrt(u) * (a + b * u + c * u * u)); };
        double next = value(u1);
        const double q[3] = {5 * c, 3 * b, a};       // of u = s^2
        const double under = q[1] * q[1] - 4 * q[0] * q[2];
        double roots[2];
        int n = 0;
        if (under >= 0.0) {                          // without a difference, which a small q[0] would leave nothing of
            const double sum = -0.5 * (q[1] + copysign(sqrt(under), q[1]));
            if (q[0] != 0.0) roots[n++] = sum / q[0];
            if (sum != 0.0) roots[n++] = q[2] / sum;
        }
        for (int i = 0; i < n; ++i)
            if (roots[i] > 0.0 && roots[i] < u1) next = fmax(next, value(roots[i]));
        most = next;
    }
    const float x = scale_for(most_x);
    P = {k[0], k[1], k[2], x, x * x * kGramScale, scale_for(most_b), fabs(a) < 1.0 ? (double)INFINITY : raised};
    return most <= 4.0;
}

constexpr int64_t kMostSide = 1 << 14, kMostLength = 1 << 26;
int check_matrices(int64_t n, const int64_t* rows, const int64_t* cols) {
    if (!rows || !cols) return COLBANDIT_ERR_NULL;
    if (n < 1) return COLBANDIT_ERR_SHAPE;
    for (int64_t i = 0; i < n; ++i)
        if (rows[i] < 0 || cols[i] < 0) return COLBANDIT_ERR_SHAPE;
    for (int64_t i = 0; i < n; ++i) {
        const int64_t m = rows[i] < cols[i] ? rows[i] : cols[i], longer = rows[i] < cols[i] ? cols[i] : rows[i];
        if (m > kMostSide || longer > kMostLength) return COLBANDIT_ERR_UNSUPPORTED;
    }
    return ortho_launchable(n, rows, cols) ? COLBANDIT_OK : COLBANDIT_ERR_UNSUPPORTED;
}

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
    const int rc = attn_args(a, A);
    return rc ? rc : attention(a, A, out, lse, workspace, workspace_bytes, stream);
}

int colbandit_attention_backward(const colbandit_attn* a, const void* out, const float* lse, const void* dout, void* dq, void* dk,
                                 void* dv, void* dbias, void* workspace, size_t workspace_bytes, void* stream) {
    AttnArgs A;
    const int rc = attn_args(a, A);
    return rc ? rc : attention_backward(a, A, {out, dout, lse, dq, dk, dv, dbias}, workspace, workspace_bytes, stream);
}

size_t colbandit_sizeof_window(void) { return sizeof(colbandit_window); }

size_t colbandit_attention_window_workspace_bytes(const colbandit_attn* a, const colbandit_window* w, int backward) {
    AttnArgs A;
    if (attn_args(a, A) || window_args(a, w, A)) return 0;
    return plan_attention(A, a->d, a->dt, backward != 0).bytes;
}

int colbandit_attention_window(const colbandit_attn* a, const colbandit_window* w, void* out, float* lse, void* workspace,
                               size_t workspace_bytes, void* stream) {
    AttnArgs A;
    int rc = attn_args(a, A);
    if (!rc) rc = window_args(a, w, A);
    return rc ? rc : attention(a, A, out, lse, workspace, workspace_bytes, stream);
}

int colbandit_attention_window_backward(const colbandit_attn* a, const colbandit_window* w, const void* out, const float* lse, const void* dout,
                                        void* dq, void* dk, void* dv, void* dbias, void* workspace, size_t workspace_bytes, void* stream) {
    AttnArgs A;
    int rc = attn_args(a, A);
    if (!rc) rc = window_args(a, w, A);
    return rc ? rc : attention_backward(a, A, {out, dout, lse, dq, dk, dv, dbias}, workspace, workspace_bytes, stream);
}

int colbandit_embedding(const void* table, colbandit_dtype table_dt, int64_t table_row, const int64_t* tokens, int64_t n, int64_t vocab,
                        int64_t width, float scale, void* out, colbandit_dtype out_dt, void* stream) {
    const int rc = check_embedding(n, vocab, width, table_row, table_dt, out_dt);
    if (rc) return rc;
    if (!table || (n && (!tokens || !out))) return COLBANDIT_ERR_NULL;
    if (!embedding_launchable(n, vocab, width, embedding_piece(table, table_dt, table_row, out, out_dt, width), false)) return COLBANDIT_ERR_UNSUPPORTED;
    if (misaligned(table, size_of(table_dt)) || misaligned(out, size_of(out_dt)) || misaligned(tokens, 8)) return COLBANDIT_ERR_ALIGNMENT;
    return hip(launch_embedding(table, table_dt, table_row, tokens, n, vocab, width, scale, out, out_dt, (hipStream_t)stream));
}

size_t colbandit_embedding_workspace_bytes(int64_t n, int64_t vocab, int64_t width) {
    return check_embedding(n, vocab, width, width, COLBANDIT_F32, COLBANDIT_F32) ? 0 : embedding_workspace_bytes(n, vocab, width);
}

int colbandit_embedding_backward(const void* dout, colbandit_dtype dout_dt, int64_t dout_row, const int64_t* tokens, int64_t n, int64_t vocab,
                                 int64_t width, float scale, void* dtable, colbandit_dtype table_dt, void* workspace, size_t workspace_bytes,
                                 void* stream) {
    int rc = check_embedding(n, vocab, width, dout_row, table_dt, dout_dt);
    if (rc) return rc;
    if (!dtable || (n && (!tokens || !dout))) return COLBANDIT_ERR_NULL;
    if (!embedding_launchable(n, vocab, width, embedding_piece(dout, dout_dt, dout_row, dtable, table_dt, width), true))
        return COLBANDIT_ERR_UNSUPPORTED;
    if (misaligned(dtable, size_of(table_dt)) || misaligned(dout, size_of(dout_dt)) || misaligned(tokens, 8)) return COLBANDIT_ERR_ALIGNMENT;
    rc = workspace_ok(workspace, workspace_bytes, embedding_workspace_bytes(n, vocab, width));
    if (rc) return rc;
    return hip(launch_embedding_backward(dout, dout_dt, dout_row, tokens, n, vocab, width, scale, dtable, table_dt, (char*)workspace,
                                         (hipStream_t)stream));
}

int colbandit_rotary_table(int64_t n_positions, int d, double base, float* table) {
    if (!table) return COLBANDIT_ERR_NULL;
    if (n_positions < 1 || d < 2 || d % 2) return COLBANDIT_ERR_SHAPE;
    if (!(base > 0.0 && base < INFINITY)) return COLBANDIT_ERR_KNOB;
    for (int i = 0; i < d / 2; ++i) {
        const double frequency = pow(base, -2.0 * i / d);
        for (int64_t p = 0; p < n_positions; ++p) {
            float* to = table + (p * (d / 2) + i) * 2;
            to[0] = (float)cos((double)p * frequency);
            to[1] = (float)sin((double)p * frequency);
        }
    }
    return COLBANDIT_OK;
}

size_t colbandit_sizeof_rotation(void) { return sizeof(colbandit_rotation); }

int colbandit_norm_rotate(const colbandit_rotation* r, void* q_out, void* k_out, void* stream) {
    RotateArgs A;
    const int rc = rotate_args(r, A);
    if (rc) return rc;
    if (A.rows && (!q_out || !k_out)) return COLBANDIT_ERR_NULL;
    if (misaligned(q_out) || misaligned(k_out)) return COLBANDIT_ERR_ALIGNMENT;
    A.q_to = q_out;
    A.k_to = k_out;
    return hip(launch_rotate(A, r->d, r->dt, (hipStream_t)stream));
}

size_t colbandit_norm_rotate_workspace_bytes(const colbandit_rotation* r) {
    RotateArgs A;
    return rotate_args(r, A) ? 0 : rotate_workspace_bytes(A, r->d);
}

int colbandit_norm_rotate_backward(const colbandit_rotation* r, const void* dq_out, const void* dk_out, void* dq, void* dk, float* dq_weight,
                                   float* dk_weight, void* workspace, size_t workspace_bytes, void* stream) {
    RotateArgs A;
    int rc = rotate_args(r, A);
    if (rc) return rc;
    if (A.rows && (!dq_out || !dk_out || !dq || !dk)) return COLBANDIT_ERR_NULL;
    if (misaligned(dq_out) || misaligned(dk_out) || misaligned(dq) || misaligned(dk) || misaligned(dq_weight, 4) || misaligned(dk_weight, 4))
        return COLBANDIT_ERR_ALIGNMENT;
    rc = workspace_ok(workspace, workspace_bytes, rotate_workspace_bytes(A, r->d));
    if (rc) return rc;
    A.dq_out = dq_out;
    A.dk_out = dk_out;
    A.q_to = dq;
    A.k_to = dk;
    A.part = (float*)workspace;
    return hip(launch_rotate_backward(A, r->d, r->dt, dq_weight, dk_weight, (hipStream_t)stream));
}

size_t colbandit_orthogonalise_workspace_bytes(int64_t n_matrices, const int64_t* rows, const int64_t* cols) {
    return check_matrices(n_matrices, rows, cols) ? 0 : ortho_workspace_bytes(n_matrices, rows, cols);
}

int colbandit_orthogonalise(int64_t n_matrices, const void* const* in, void* const* out, const int64_t* rows, const int64_t* cols,
                            const int32_t* dts, int steps, const float* coefficients, void* workspace, size_t workspace_bytes, void* stream) {
    if (!in || !out || !dts || !coefficients) return COLBANDIT_ERR_NULL;
    int rc = check_matrices(n_matrices, rows, cols);
    if (rc) return rc;
    if (steps < 1) return COLBANDIT_ERR_SHAPE;
    OrthoPolynomial polynomial;
    if (steps > 64 || !polynomial_holds(coefficients, steps, polynomial)) return COLBANDIT_ERR_KNOB;
    for (int64_t i = 0; i < n_matrices; ++i) {
        if (!is_type(dts[i])) return COLBANDIT_ERR_SHAPE;
        if (rows[i] && cols[i] && (!in[i] || !out[i])) return COLBANDIT_ERR_NULL;
        if (misaligned(in[i], size_of(dts[i])) || misaligned(out[i], size_of(dts[i]))) return COLBANDIT_ERR_ALIGNMENT;
    }
    rc = workspace_ok(workspace, workspace_bytes, ortho_workspace_bytes(n_matrices, rows, cols));
    if (rc) return rc;
    return hip(launch_ortho(n_matrices, in, out, rows, cols, dts, steps, polynomial, (char*)workspace, (hipStream_t)stream));
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
