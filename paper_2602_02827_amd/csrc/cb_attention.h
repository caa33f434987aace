// Attention over ragged packed sequences and its backward pass: kernels (templates of the storage type) and launches.
//
// Columns of a tile are query rows (forward, gradients of queries) or key rows (gradients of keys and values), 32 to a
// wavefront; the other side's rows pass through LDS.  Scores are made with the columns' rows as the B operand, so a
// column's statistics, limit and log-sum-exp are one value of its two lanes, and scores that were turned into
// probabilities or their gradients are the next product's B operand without leaving their registers (cb_tile.h).
// Where several query heads share a key head and there is no bias, their rows share tiles: column c is row c / pack of
// head c % pack, so keys and values are staged once for all of them, and a single token still fills its columns.
#pragma once
#include "cb_tile.h"
#include "cb_train.h"

namespace cb {

// First columns' row, rows and key limits of a tile of query columns.
struct QueryTile {
    int seq, row0, Lq, Lk, q0, k0;      // sequence, first local row, lengths, first global rows
    bool none;
};
__device__ __forceinline__ QueryTile query_tile(const AttnArgs& A, int slot, int per, int lane) {
    QueryTile t;
    t.seq = find_sequence(A.qoff, A.n_seqs, per, A.total_q, slot, lane);
    const Range q = sequence_rows(A.qoff, t.seq, A.total_q), k = sequence_rows(A.koff, t.seq, A.total_k);
    t.row0 = (slot - place_of(A.qoff, t.seq, per, A.total_q)) * per;
    t.Lq = q.n;
    t.Lk = k.n;
    t.q0 = q.lo;
    t.k0 = k.lo;
    t.none = t.row0 < 0 || t.row0 >= q.n;
    return t;
}

// Bias of a head by distance key - query, -reach .. reach, in powers of two.  Finite values stay finite.
template <class E>
__device__ __forceinline__ int bucket_of(const AttnArgs& A, int dist) {
    const int far = A.causal ? (dist < 0 ? -dist : 0) : (dist < 0 ? -dist : dist);
    int lo = 0, hi = A.n_dir;
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (A.starts[mid] <= far) lo = mid; else hi = mid;
    }
    return lo + (!A.causal && dist > 0 ? A.n_dir : 0);
}
template <class E>
__device__ __forceinline__ void fill_bias(const AttnArgs& A, int head, float* table, int tid, int threads) {
    for (int i = tid; i <= 2 * A.reach; i += threads) {
        const float x = (float)((const E*)A.bias)[(int64_t)bucket_of<E>(A, i - A.reach) * A.heads + head];
        const float y = x * LOG2E;
        table[i] = fabsf(x) < INFINITY ? fminf(fmaxf(y, -3.4028235e38f), 3.4028235e38f) : y;
    }
}
__device__ __forceinline__ float bias_at(const float* table, int reach, int dist) {
    const int i = dist < -reach ? -reach : dist > reach ? reach : dist;
    return table[i + reach];
}

// A tile of two matrices' rows on its way from memory to LDS: loads are issued a tile ahead and wait in registers.
template <class E, int D, int THREADS> struct Staged {
    using T = Tile<E, D>;
    static constexpr int N = T::ROWS * T::PIECES / THREADS;
    u32x4 x[N], y[N];
    uint8_t keep[N];
    static __device__ __forceinline__ int row(int i, int tid) { return (i * THREADS + tid) / T::PIECES; }
    static __device__ __forceinline__ int piece(int i, int tid) { return (i * THREADS + tid) % T::PIECES; }
    __device__ __forceinline__ void put(char* a, char* b, int tid) const {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int at = T::at(row(i, tid), piece(i, tid));
            const u32x4 zero = {0u, 0u, 0u, 0u};
            *(u32x4*)(a + at) = keep[i] ? x[i] : zero;       // what the mask hides may be anything
            *(u32x4*)(b + at) = keep[i] ? y[i] : zero;
        }
    }
    // rows first .. of the keys and values of a head, zeros from `end` on and where the mask hides them
    __device__ __forceinline__ void keys(const AttnArgs& A, int kv_head, int k0, int first, int end, int tid) {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int r = first + row(i, tid);
            x[i] = y[i] = u32x4{0u, 0u, 0u, 0u};
            keep[i] = 1;
            if (r < end) {
                const int64_t at = k0 + r;
                const int p = piece(i, tid) * 16;
                x[i] = *(const u32x4*)((const char*)A.k + (at * A.k_row + kv_head * A.k_head) * (int64_t)sizeof(E) + p);
                y[i] = *(const u32x4*)((const char*)A.v + (at * A.v_row + kv_head * A.v_head) * (int64_t)sizeof(E) + p);
                if (A.keep) keep[i] = A.keep[at];
            }
        }
    }
};

// The eight-value pieces of one column's row (B operand of all steps); zeros for a column that is none.
template <class E, int D> struct Column {
    typename Oper<E>::Frag v[D / 16];
    __device__ __forceinline__ void load(const E* row, bool real, int h) {
#pragma unroll
        for (int c = 0; c < D / 16; ++c) {
            v[c] = {};
            if (real) v[c] = Oper<E>::load(row + 16 * c + 8 * h);
        }
    }
};

// Which of a tile's key rows are seen at all, one bit each.
__device__ __forceinline__ uint64_t seen_keys(const AttnArgs& A, int k0, int first, int end, int rows, int lane) {
    bool ok = lane < rows && first + lane < end;
    if (A.keep && ok) ok = A.keep[(int64_t)k0 + first + lane] != 0;
    return __ballot(ok);
}

// ---- forward -------------------------------------------------------------------------------------------------
// One pass over the keys with the running maximum and sum of the softmax, in 32 bits; probabilities are rounded to the
// storage type for the second product (their sum is not).
template <class E, int D, int NW, bool BIAS>
__global__ __launch_bounds__(64 * NW) void k_attention(const AttnArgs A, int slots, int units, int splits, E* out, float* lse,
                                                       float* o_part, float2* ml_part) {
    using O = Oper<E>;
    using T = Tile<E, D>;
    constexpr int NB = T::ROWS / 32, DB = D / 32, THREADS = 64 * NW;
    __shared__ __align__(16) char lk[T::BYTES], lv[T::BYTES];
    extern __shared__ float table[];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, h = lane >> 5;
    const int slot = blockIdx.x % slots, unit = blockIdx.x / slots % units, split = blockIdx.x / slots / units;
    const int G = A.pack, per = 32 * NW / G;
    const QueryTile t = query_tile(A, slot, per, lane);
    if (t.none) return;
    const int head0 = unit * G, kv = head0 / A.group;
    if constexpr (BIAS) fill_bias<E>(A, head0, table, tid, THREADS);

    const int col = wave * 32 + (lane & 31);
    const int local = col / G, row = t.row0 + local, head = head0 + col % G;
    const bool real = local < per && row < t.Lq;
    const int shift = t.Lk - t.Lq, lim = row + shift;
    const int last = (t.row0 + per < t.Lq ? t.row0 + per : t.Lq) - 1;
    int end = A.causal ? last + shift + 1 : t.Lk;                 // keys that any column sees
    end = end < 0 ? 0 : end > t.Lk ? t.Lk : end;
    const int tiles = (end + T::ROWS - 1) / T::ROWS, each = (tiles + splits - 1) / splits;
    const int first_tile = split * each, end_tile = first_tile + each < tiles ? first_tile + each : tiles;
    // this wavefront's columns: their first and last row
    const int wrow = t.row0 + wave * 32 / G;
    const bool busy = wave * 32 / G < per && wrow < t.Lq;
    const int wlast = t.row0 + (wave * 32 + 31) / G;
    const int wend = A.causal ? (wlast < last ? wlast : last) + shift + 1 : t.Lk, wlim = wrow + shift;

    Column<E, D> q;
    q.load((const E*)A.q + (int64_t)(t.q0 + row) * A.q_row + head * A.q_head, real, h);
    f32x16 acc[DB] = {};
    float m = -INFINITY, l = 0.f;
    const float scale2 = A.scale * LOG2E;
    Staged<E, D, THREADS> next;
    if (first_tile < end_tile) next.keys(A, kv, t.k0, first_tile * T::ROWS, end, tid);
    for (int i = first_tile; i < end_tile; ++i) {
        const int base = i * T::ROWS;
        const uint64_t seen = seen_keys(A, t.k0, base, end, T::ROWS, lane);
        __syncthreads();
        next.put(lk, lv, tid);
        __syncthreads();
        if (i + 1 < end_tile) next.keys(A, kv, t.k0, base + T::ROWS, end, tid);
        if (!busy || base >= wend) continue;
        f32x16 s[NB];
#pragma unroll
        for (int b = 0; b < NB; ++b) {
            s[b] = {};
#pragma unroll
            for (int c = 0; c < D / 16; ++c) O::mma(s[b], T::rows(lk, lane, b, c), q.v[c]);
        }
        const uint64_t all = T::ROWS == 64 ? ~0ull : (1ull << (T::ROWS & 63)) - 1ull;
        const bool part = seen != all || (A.causal && base + T::ROWS - 1 > wlim);
        const int room = A.causal ? lim - base - 4 * h : 1 << 20;
        const uint64_t mine = seen >> (4 * h);
        float top = -INFINITY;
#pragma unroll
        for (int b = 0; b < NB; ++b)
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                const int k = 32 * b + 8 * (r >> 2) + (r & 3);
                float x = s[b][r] * scale2;
                if constexpr (BIAS) x += bias_at(table, A.reach, base + k + 4 * h - lim);
                if (part && !(k <= room && ((uint32_t)(mine >> (32 * b)) >> (k & 31) & 1u))) x = -INFINITY;
                s[b][r] = x;
                top = fmaxf(top, x);
            }
        top = fmaxf(top, other_half(top));
        const float m_new = fmaxf(m, top), m_use = m_new == -INFINITY ? 0.f : m_new;
        if (__ballot(m_new > m)) {
            const float down = exp2_fast(m - m_use);
            l *= down;
#pragma unroll
            for (int db = 0; db < DB; ++db) acc[db] *= down;
            m = m_new;
        }
#pragma unroll
        for (int b = 0; b < NB; ++b) {
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                s[b][r] = exp2_fast(s[b][r] - m_use);
                l += s[b][r];
            }
#pragma unroll
            for (int c = 0; c < 2; ++c) {
                const auto x = c ? __builtin_shufflevector(s[b], s[b], 8, 9, 10, 11, 12, 13, 14, 15)
                                 : __builtin_shufflevector(s[b], s[b], 0, 1, 2, 3, 4, 5, 6, 7);
                const typename O::Frag p = O::round(x);
#pragma unroll
                for (int db = 0; db < DB; ++db) O::mma(acc[db], T::turned(lv, lane, b, c, db), p);
            }
        }
    }
    l += other_half(l);
    if (!real) return;
    const int64_t at = (int64_t)(t.q0 + row);
    if (splits > 1) {
        const int64_t place = ((int64_t)split * A.heads + head) * A.total_q + at;
        if (h == 0) ml_part[place] = make_float2(m, l);
#pragma unroll
        for (int db = 0; db < DB; ++db)
#pragma unroll
            for (int j = 0; j < 4; ++j)
                *(f32x4*)(o_part + place * D + 32 * db + 8 * j + 4 * h) =
                    f32x4{acc[db][4 * j], acc[db][4 * j + 1], acc[db][4 * j + 2], acc[db][4 * j + 3]};
        return;
    }
    const float inv = l == 0.f ? 0.f : 1.f / l;
    if (h == 0) lse[(int64_t)head * A.total_q + at] = l == 0.f ? -INFINITY : m * LN2 + logf(l);
    E* o = out + (at * A.heads + head) * D;
#pragma unroll
    for (int db = 0; db < DB; ++db)
#pragma unroll
        for (int j = 0; j < 4; ++j)
            O::store4(o + 32 * db + 8 * j + 4 * h, f32x4{acc[db][4 * j] * inv, acc[db][4 * j + 1] * inv,
                                                          acc[db][4 * j + 2] * inv, acc[db][4 * j + 3] * inv});
}

// Joins the parts of rows whose keys were split: a quarter of a row's values a thread and row.
template <class E, int D>
__global__ __launch_bounds__(256) void k_attention_join(const AttnArgs A, int splits, const float* o_part, const float2* ml_part,
                                                        E* out, float* lse) {
    constexpr int PER = D / 4;
    const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
    const int64_t rows = (int64_t)A.heads * A.total_q, place = i / PER;
    const int dim = (int)(i % PER) * 4;
    if (place >= rows) return;
    // rows that no sequence holds have no parts: they are not written by any call, nor is their output
    const int64_t row = place % A.total_q;
    int64_t lo = A.qoff[0], hi = A.qoff[A.n_seqs];
    if (row < lo || row >= hi) return;
    float m = -INFINITY;
    for (int s = 0; s < splits; ++s) m = fmaxf(m, ml_part[s * rows + place].x);
    const float m_use = m == -INFINITY ? 0.f : m;
    float l = 0.f;
    f32x4 o = {0.f, 0.f, 0.f, 0.f};
    for (int s = 0; s < splits; ++s) {
        const float2 ml = ml_part[s * rows + place];
        if (ml.y == 0.f) continue;
        const float w = exp2_fast(ml.x - m_use);
        l += ml.y * w;
        o += *(const f32x4*)(o_part + (s * rows + place) * D + dim) * w;
    }
    const float inv = l == 0.f ? 0.f : 1.f / l;
    if (dim == 0) lse[place] = l == 0.f ? -INFINITY : m * LN2 + logf(l);
    Oper<E>::store4(out + (row * A.heads + place / A.total_q) * D + dim, o * inv);
}

// ---- backward ------------------------------------------------------------------------------------------------
// dS_ij = P_ij (<dO_i, V_j> - delta_i), delta_i = <dO_i, O_i>, P_ij = exp(S_ij - lse_i), all in 32 bits; P and dS are rounded
// to the storage type as operands of the last products.  Queries' and keys' gradients are made by a kernel each, which
// recomputes the scores twice (seven products where one kernel would need five) but adds in a fixed order, where one
// kernel would have to add either side's gradients by atomics.

// Gradients of queries, delta, and the bias table's share of each tile.
// The table's gradient: dS of a 32 x 32 block is added to a histogram by distance in LDS, one of each half wavefront: the 32
// lanes of a half have as many distances, so no two lanes add to one place at once and the order of the sums is the
// program's.  Blocks whose distances all lie in a direction's last bucket are summed in a register instead.
template <class E, int D, int NW, bool BIAS>
__global__ __launch_bounds__(64 * NW) void k_attention_dq(const AttnArgs A, int slots, int units, const E* out, const E* dout,
                                                          const float* lse, E* dq, float* delta, float* bias_part) {
    using O = Oper<E>;
    using T = Tile<E, D>;
    constexpr int NB = T::ROWS / 32, DB = D / 32, THREADS = 64 * NW;
    __shared__ __align__(16) char lk[T::BYTES], lv[T::BYTES];
    __shared__ float far_sum[NW][2];
    extern __shared__ float table[];                  // [2 reach + 1], then the histograms
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, h = lane >> 5;
    const int slot = blockIdx.x % slots, unit = blockIdx.x / slots;
    const int G = A.pack, per = 32 * NW / G;
    const QueryTile t = query_tile(A, slot, per, lane);
    const int head0 = unit * G, kv = head0 / A.group;
    if (t.none) {
        if constexpr (BIAS)
            for (int b = tid; b < A.n_buckets; b += THREADS) bias_part[((int64_t)slot * A.heads + head0) * A.n_buckets + b] = 0.f;
        return;
    }
    const int width = 2 * A.reach + 125, mid = A.reach + 62;      // distances of blocks that are not far: below reach + 63
    float* hist = table + 2 * A.reach + 1;
    if constexpr (BIAS) {
        fill_bias<E>(A, head0, table, tid, THREADS);
        for (int i = tid; i < 2 * NW * width; i += THREADS) hist[i] = 0.f;
    }
    float* mine_hist = hist + (2 * wave + h) * width + mid;
    float far_lo = 0.f, far_hi = 0.f;

    const int col = wave * 32 + (lane & 31);
    const int local = col / G, row = t.row0 + local, head = head0 + col % G;
    const bool real = local < per && row < t.Lq;
    const int shift = t.Lk - t.Lq, lim = row + shift;
    const int last = (t.row0 + per < t.Lq ? t.row0 + per : t.Lq) - 1;
    int end = A.causal ? last + shift + 1 : t.Lk;
    end = end < 0 ? 0 : end > t.Lk ? t.Lk : end;
    const int tiles = (end + T::ROWS - 1) / T::ROWS;
    const int wrow = t.row0 + wave * 32 / G;
    const bool busy = wave * 32 / G < per && wrow < t.Lq;
    const int wlast = t.row0 + (wave * 32 + 31) / G;
    const int wend = A.causal ? (wlast < last ? wlast : last) + shift + 1 : t.Lk, wlim = wrow + shift;

    const int64_t at = (int64_t)(t.q0 + row), place = (int64_t)head * A.total_q + at, dense = (at * A.heads + head) * D;
    const float row_lse = real ? lse[place] : -INFINITY;
    const bool seeing = row_lse != -INFINITY;         // rows that see nothing take no part, whatever their gradient is
    const float lse2 = row_lse * LOG2E;
    Column<E, D> q, g;
    q.load((const E*)A.q + at * A.q_row + head * A.q_head, seeing, h);
    g.load(dout + dense, seeing, h);
    float dot = 0.f;
    {
        Column<E, D> o;
        o.load(out + dense, seeing, h);
#pragma unroll
        for (int c = 0; c < D / 16; ++c) {
            const f32x8 x = O::wide(g.v[c]), y = O::wide(o.v[c]);
#pragma unroll
            for (int e = 0; e < 8; ++e) dot += x[e] * y[e];
        }
        dot += other_half(dot);
        if (real && h == 0) delta[place] = dot;
    }
    f32x16 acc[DB] = {};
    const float scale2 = A.scale * LOG2E;
    Staged<E, D, THREADS> next;
    if (tiles > 0) next.keys(A, kv, t.k0, 0, end, tid);
    for (int i = 0; i < tiles; ++i) {
        const int base = i * T::ROWS;
        const uint64_t seen = seen_keys(A, t.k0, base, end, T::ROWS, lane);
        __syncthreads();
        next.put(lk, lv, tid);
        __syncthreads();
        if (i + 1 < tiles) next.keys(A, kv, t.k0, base + T::ROWS, end, tid);
        if (!busy || base >= wend) continue;
        const uint64_t all = T::ROWS == 64 ? ~0ull : (1ull << (T::ROWS & 63)) - 1ull;
        const bool part = seen != all || !__all(seeing) || (A.causal && base + T::ROWS - 1 > wlim);
        const int room = !seeing ? -1 : A.causal ? lim - base - 4 * h : 1 << 20;
        const uint64_t mine = seen >> (4 * h);
#pragma unroll
        for (int b = 0; b < NB; ++b) {
            f32x16 s = {}, dp = {};
#pragma unroll
            for (int c = 0; c < D / 16; ++c) O::mma(s, T::rows(lk, lane, b, c), q.v[c]);
#pragma unroll
            for (int c = 0; c < D / 16; ++c) O::mma(dp, T::rows(lv, lane, b, c), g.v[c]);
            f32x16 ds;
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                const int k = 32 * b + 8 * (r >> 2) + (r & 3);
                float x = s[r] * scale2;
                if constexpr (BIAS) x += bias_at(table, A.reach, base + k + 4 * h - lim);
                float y = exp2_fast(x - lse2) * (dp[r] - dot);
                if (part && !(k <= room && ((uint32_t)(mine >> (32 * b)) >> (k & 31) & 1u))) y = 0.f;
                ds[r] = y;
            }
            if constexpr (BIAS) {
                const int d0 = base + 32 * b - wlim;              // distance of the block's first key and row
                if (d0 - 31 >= A.reach || d0 + 31 <= -A.reach) {
                    float sum = 0.f;
#pragma unroll
                    for (int r = 0; r < 16; ++r) sum += ds[r];
                    (d0 > 0 ? far_hi : far_lo) += sum;
                } else {
                    const int d = base + 32 * b + 4 * h - lim;
#pragma unroll
                    for (int r = 0; r < 16; ++r) atomicAdd(mine_hist + d + 8 * (r >> 2) + (r & 3), ds[r]);
                }
            }
#pragma unroll
            for (int c = 0; c < 2; ++c) {
                const auto x = c ? __builtin_shufflevector(ds, ds, 8, 9, 10, 11, 12, 13, 14, 15)
                                 : __builtin_shufflevector(ds, ds, 0, 1, 2, 3, 4, 5, 6, 7);
                const typename O::Frag p = O::round(x);
#pragma unroll
                for (int db = 0; db < DB; ++db) O::mma(acc[db], T::turned(lk, lane, b, c, db), p);
            }
        }
    }
    if (real) {
        E* o = dq + dense;
#pragma unroll
        for (int db = 0; db < DB; ++db)
#pragma unroll
            for (int j = 0; j < 4; ++j)
                O::store4(o + 32 * db + 8 * j + 4 * h,
                          f32x4{acc[db][4 * j] * A.scale, acc[db][4 * j + 1] * A.scale, acc[db][4 * j + 2] * A.scale,
                                acc[db][4 * j + 3] * A.scale});
    }
    if constexpr (BIAS) {
#pragma unroll
        for (int m = 1; m < 64; m <<= 1) {
            far_lo += __shfl_xor(far_lo, m);
            far_hi += __shfl_xor(far_hi, m);
        }
        if (lane == 0) {
            far_sum[wave][0] = far_lo;
            far_sum[wave][1] = far_hi;
        }
        __syncthreads();
        for (int b = tid; b < A.n_buckets; b += THREADS) {
            const bool behind = b >= A.n_dir;                     // keys behind the query
            const int i = behind ? b - A.n_dir : b;
            const bool open = i == A.n_dir - 1;                   // the last one of its direction
            const int lo = A.starts[i], hi = open ? mid : A.starts[i + 1] - 1;
            float sum = 0.f;
            for (int w = 0; w < 2 * NW; ++w) {
                const float* x = hist + w * width + mid;
                // distance 0 belongs to the keys before; with a causal limit so do all keys behind, of which none is seen
                for (int j = lo; j <= hi; ++j) sum += behind ? (j > 0 ? x[j] : 0.f) : x[-j];
            }
            if (open)
                for (int w = 0; w < NW; ++w) sum += far_sum[w][behind ? 1 : 0];
            bias_part[((int64_t)slot * A.heads + head0) * A.n_buckets + b] = sum;
        }
    }
}

// Gradients of keys and values; workgroups from `main` on add up the bias table's shares of all tiles.
template <class E, int D, int NW, bool BIAS>
__global__ __launch_bounds__(64 * NW) void k_attention_dkv(const AttnArgs A, int slots, int main, int q_slots, const E* dout,
                                                           const float* lse, const float* delta, const float* bias_part, E* dk, E* dv,
                                                           E* dbias) {
    using O = Oper<E>;
    using T = Tile<E, D>;
    constexpr int NB = T::ROWS / 32, DB = D / 32, THREADS = 64 * NW, COLS = 32 * NW;
    __shared__ __align__(16) char lq[T::BYTES], lg[T::BYTES];
    __shared__ __align__(16) float row_lse[T::ROWS], row_delta[T::ROWS];
    __shared__ __align__(16) int row_lim[T::ROWS];
    extern __shared__ float table[];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, h = lane >> 5;
    if constexpr (BIAS) {
        if ((int)blockIdx.x >= main) {                // one entry of the table each wavefront
            const int e = ((int)blockIdx.x - main) * NW + wave;
            if (e >= A.n_buckets * A.heads) return;
            const int head = e / A.n_buckets, b = e % A.n_buckets;
            float sum = 0.f;
            for (int s = lane; s < q_slots; s += 64) sum += bias_part[((int64_t)s * A.heads + head) * A.n_buckets + b];
#pragma unroll
            for (int m = 1; m < 64; m <<= 1) sum += __shfl_xor(sum, m);
            if (lane == 0) dbias[(int64_t)b * A.heads + head] = (E)sum;
            return;
        }
    }
    const int slot = blockIdx.x % slots, kv = blockIdx.x / slots;
    const int seq = find_sequence(A.koff, A.n_seqs, COLS, A.total_k, slot, lane);
    const Range ks = sequence_rows(A.koff, seq, A.total_k), qs = sequence_rows(A.qoff, seq, A.total_q);
    const int key0 = (slot - place_of(A.koff, seq, COLS, A.total_k)) * COLS;
    if (key0 < 0 || key0 >= ks.n) return;
    const int key = key0 + wave * 32 + (lane & 31), shift = ks.n - qs.n;
    const bool real = key < ks.n;
    const int64_t at = ks.lo + key;
    const bool seen = real && (!A.keep || A.keep[at]);
    Column<E, D> k, v;
    k.load((const E*)A.k + at * A.k_row + kv * A.k_head, seen, h);
    v.load((const E*)A.v + at * A.v_row + kv * A.v_head, seen, h);
    f32x16 ak[DB] = {}, av[DB] = {};
    const float scale2 = A.scale * LOG2E;
    const int G = A.pack;
    const int first = A.causal && key0 > shift ? key0 - shift : 0;       // first row that sees a key of the tile
    const int wfirst = A.causal && key0 + wave * 32 > shift ? key0 + wave * 32 - shift : 0;
    const bool busy = key0 + wave * 32 < ks.n;
    const int cols = qs.n * G, col0 = (int)((int64_t)first * G / T::ROWS * T::ROWS);
    for (int head0 = kv * A.group; head0 < (kv + 1) * A.group; head0 += G) {
        if constexpr (BIAS) {
            __syncthreads();
            fill_bias<E>(A, head0, table, tid, THREADS);
        }
        Staged<E, D, THREADS> next;
        float n_lse = 0.f, n_delta = 0.f;
        auto fetch = [&](int c0) {
#pragma unroll
            for (int i = 0; i < next.N; ++i) {
                const int c = c0 + next.row(i, tid);
                next.x[i] = next.y[i] = u32x4{0u, 0u, 0u, 0u};
                next.keep[i] = 1;
                if (c < cols) {
                    const int64_t r = qs.lo + c / G;
                    const int head = head0 + c % G, p = next.piece(i, tid) * 16;
                    next.x[i] = *(const u32x4*)((const char*)A.q + (r * A.q_row + head * A.q_head) * (int64_t)sizeof(E) + p);
                    next.y[i] = *(const u32x4*)((const char*)dout + (r * A.heads + head) * (int64_t)(D * sizeof(E)) + p);
                    next.keep[i] = lse[(int64_t)head * A.total_q + r] != -INFINITY;
                }
            }
            if (tid < T::ROWS) {
                const int c = c0 + tid;
                n_lse = -INFINITY;
                n_delta = 0.f;
                if (c < cols) {
                    const int64_t place = (int64_t)(head0 + c % G) * A.total_q + qs.lo + c / G;
                    n_lse = lse[place];
                    n_delta = delta[place];
                }
            }
        };
        if (col0 < cols) fetch(col0);
        for (int c0 = col0; c0 < cols; c0 += T::ROWS) {
            __syncthreads();
            next.put(lq, lg, tid);
            if (tid < T::ROWS) {
                row_lse[tid] = n_lse == -INFINITY ? INFINITY : n_lse * LOG2E;     // exp2(x - inf) = 0
                row_delta[tid] = n_delta;
                row_lim[tid] = (c0 + tid) / G + shift;
            }
            __syncthreads();
            if (c0 + T::ROWS < cols) fetch(c0 + T::ROWS);
            if (!busy || (c0 + T::ROWS - 1) / G < wfirst) continue;
            const bool part = A.causal && key0 + wave * 32 + 31 > c0 / G + shift;
#pragma unroll
            for (int b = 0; b < NB; ++b) {
                f32x16 s = {}, dp = {};
#pragma unroll
                for (int c = 0; c < D / 16; ++c) O::mma(s, T::rows(lq, lane, b, c), k.v[c]);
#pragma unroll
                for (int c = 0; c < D / 16; ++c) O::mma(dp, T::rows(lg, lane, b, c), v.v[c]);
                f32x16 ds;
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const int r0 = 32 * b + 8 * j + 4 * h;
                    const f32x4 e = *(const f32x4*)(row_lse + r0), dl = *(const f32x4*)(row_delta + r0);
                    const int4 lm = *(const int4*)(row_lim + r0);
                    const int lims[4] = {lm.x, lm.y, lm.z, lm.w};
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const int r = 4 * j + i;
                        float x = s[r] * scale2;
                        if constexpr (BIAS) x += bias_at(table, A.reach, key - lims[i]);
                        float p = exp2_fast(x - e[i]);
                        if (part && key > lims[i]) p = 0.f;
                        s[r] = p;
                        ds[r] = p * (dp[r] - dl[i]);
                    }
                }
#pragma unroll
                for (int c = 0; c < 2; ++c) {
                    const auto x = c ? __builtin_shufflevector(s, s, 8, 9, 10, 11, 12, 13, 14, 15)
                                     : __builtin_shufflevector(s, s, 0, 1, 2, 3, 4, 5, 6, 7);
                    const auto y = c ? __builtin_shufflevector(ds, ds, 8, 9, 10, 11, 12, 13, 14, 15)
                                     : __builtin_shufflevector(ds, ds, 0, 1, 2, 3, 4, 5, 6, 7);
                    const typename O::Frag p = O::round(x), q = O::round(y);
#pragma unroll
                    for (int db = 0; db < DB; ++db) O::mma(av[db], T::turned(lg, lane, b, c, db), p);
#pragma unroll
                    for (int db = 0; db < DB; ++db) O::mma(ak[db], T::turned(lq, lane, b, c, db), q);
                }
            }
        }
    }
    if (!real) return;
    const int64_t dense = (at * A.kv_heads + kv) * D;
#pragma unroll
    for (int db = 0; db < DB; ++db)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            f32x4 x = {ak[db][4 * j], ak[db][4 * j + 1], ak[db][4 * j + 2], ak[db][4 * j + 3]};
            f32x4 y = {av[db][4 * j], av[db][4 * j + 1], av[db][4 * j + 2], av[db][4 * j + 3]};
            const f32x4 zero = {0.f, 0.f, 0.f, 0.f};
            O::store4(dk + dense + 32 * db + 8 * j + 4 * h, seen ? x * A.scale : zero);
            O::store4(dv + dense + 32 * db + 8 * j + 4 * h, seen ? y : zero);
        }
}

// ---- launches ------------------------------------------------------------------------------------------------
template <class F> hipError_t by_width(int d, F&& f) {
    switch (d) {
        case 32: return f(std::integral_constant<int, 32>{});
        case 64: return f(std::integral_constant<int, 64>{});
        case 96: return f(std::integral_constant<int, 96>{});
        default: return f(std::integral_constant<int, 128>{});
    }
}
template <class F> hipError_t by_waves(int waves, bool bias, F&& f) {
    using One = std::integral_constant<int, 1>;
    using Four = std::integral_constant<int, 4>;
    if (bias) return waves == 1 ? f(One{}, std::true_type{}) : f(Four{}, std::true_type{});
    return waves == 1 ? f(One{}, std::false_type{}) : f(Four{}, std::false_type{});
}

template <class E>
hipError_t launch_attention(const AttnArgs& A, const AttnPlan& P, E* out, float* lse, char* ws, hipStream_t st) {
    if (P.q_slots == 0 || A.total_q == 0) return hipSuccess;
    return by_width(P.d, [&](auto dc) {
        constexpr int D = decltype(dc)::value;
        float* o_part = (float*)(ws + P.o_part);
        float2* ml_part = (float2*)(ws + P.ml_part);
        const hipError_t e = by_waves(P.q_waves, A.bias != nullptr, [&](auto nw, auto bias) {
            constexpr int NW = decltype(nw)::value;
            constexpr bool BIAS = decltype(bias)::value;
            const size_t lds = BIAS ? 4 * (size_t)(2 * A.reach + 1) : 0;
            k_attention<E, D, NW, BIAS><<<dim3((unsigned)(P.q_slots * P.units * P.splits)), 64 * NW, lds, st>>>(
                A, (int)P.q_slots, P.units, P.splits, out, lse, o_part, ml_part);
            return hipGetLastError();
        });
        if (e != hipSuccess || P.splits == 1) return e;
        const int64_t threads = (int64_t)A.heads * A.total_q * (D / 4);
        k_attention_join<E, D><<<dim3((unsigned)((threads + 255) / 256)), 256, 0, st>>>(A, P.splits, o_part, ml_part, out, lse);
        return hipGetLastError();
    });
}

template <class E>
hipError_t launch_attention_backward(const AttnArgs& A, const AttnPlan& P, const AttnGrads& G, char* ws, hipStream_t st) {
    float* delta = (float*)(ws + P.delta);
    float* bias_part = (float*)(ws + P.bias_part);
    return by_width(P.d, [&](auto dc) {
        constexpr int D = decltype(dc)::value;
        hipError_t e = hipSuccess;
        if (A.total_q > 0) {
            e = by_waves(P.q_waves, A.bias != nullptr, [&](auto nw, auto bias) {
                constexpr int NW = decltype(nw)::value;
                constexpr bool BIAS = decltype(bias)::value;
                const size_t lds = BIAS ? 4 * (size_t)(2 * A.reach + 1 + 2 * NW * (2 * A.reach + 125)) : 0;
                k_attention_dq<E, D, NW, BIAS><<<dim3((unsigned)(P.q_slots * P.units)), 64 * NW, lds, st>>>(
                    A, (int)P.q_slots, P.units, (const E*)G.out, (const E*)G.dout, G.lse, (E*)G.dq, delta, bias_part);
                return hipGetLastError();
            });
            if (e != hipSuccess) return e;
        }
        const int q_slots = A.total_q > 0 ? (int)P.q_slots : 0;
        return by_waves(P.k_waves, A.bias != nullptr, [&](auto nw, auto bias) {
            constexpr int NW = decltype(nw)::value;
            constexpr bool BIAS = decltype(bias)::value;
            const size_t lds = BIAS ? 4 * (size_t)(2 * A.reach + 1) : 0;
            const int main = A.total_k > 0 ? (int)(P.k_slots * A.kv_heads) : 0;
            const int more = BIAS ? (A.n_buckets * A.heads + NW - 1) / NW : 0;
            if (main + more == 0) return hipSuccess;
            k_attention_dkv<E, D, NW, BIAS><<<dim3((unsigned)(main + more)), 64 * NW, lds, st>>>(
                A, (int)P.k_slots, main, q_slots, (const E*)G.dout, G.lse, delta, bias_part, (E*)G.dk, (E*)G.dv, (E*)G.dbias);
            return hipGetLastError();
        });
    });
}

}  // namespace cb
