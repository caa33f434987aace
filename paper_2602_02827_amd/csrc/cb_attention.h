// Attention over ragged packed sequences and its backward pass: kernels (templates of the storage type) and launches.
//
// Columns of a tile are query rows (forward, gradients of queries) or key rows (gradients of keys and values), 32 to a
// wavefront; the other side's rows pass through LDS.  Scores are made with the columns' rows as the B operand, so a
// column's statistics, limit and log-sum-exp are one value of its two lanes, and scores that were turned into
// probabilities or their gradients are the next product's B operand without leaving their registers (cb_tile.h).
// Where several query heads share a key head and there is no bias, their rows share tiles: column c is row c / pack of
// head c % pack, so keys and values are staged once for all of them, and a single token still fills its columns.
#pragma once
#include <type_traits>

#include "cb_tile.h"
#include "cb_train.h"

namespace cb {

// Bias of a head by distance key - query, as it is in the table.  A block of 32 x 32 distances that
// is not all in one direction's last bucket reaches less than kBlock beyond `reach`: the table is that much longer, so that no
// distance is clamped when it is looked up, and a lane's sixteen places differ by constants.
constexpr int kBlock = 62;
__device__ __host__ __forceinline__ int bias_middle(int reach) { return reach + kBlock; }
__device__ __host__ __forceinline__ int bias_width(int reach) { return 2 * bias_middle(reach) + 1; }
// Eight threads write a bucket's distances; its first one is in `starts`, in LDS.  They are put there by way of scalar registers:
// vector loads of a kernel's arguments take microseconds.
__device__ __forceinline__ void load_starts(const AttnArgs& A, int16_t* starts, int tid, int threads) {
    for (int first = 0; first <= A.n_dir; first += threads) {
        const int own = first + tid;
        int x = bias_middle(A.reach) + 1;             // behind the last one
        const int end = A.n_dir < first + threads ? A.n_dir : first + threads;
#pragma unroll 8
        for (int j = first; j < end; ++j) x = j == own ? A.starts[j] : x;
        if (own <= A.n_dir) starts[own] = (int16_t)x;
    }
}
template <class E>
__device__ __forceinline__ void fill_bias(const AttnArgs& A, int head, const int16_t* starts, float* table, int tid, int threads) {
    const int middle = bias_middle(A.reach);
    for (int b = tid >> 3; b < A.n_buckets; b += threads >> 3) {
        const bool behind = b >= A.n_dir;             // keys behind the query
        const int i = behind ? b - A.n_dir : b;
        const float z = (float)((const E*)A.bias)[(int64_t)b * A.heads + head];
        const int end = starts[i + 1];
        for (int j = starts[i] + (tid & 7); j < end; j += 8)
            if (!behind) table[middle - j] = z; else if (j > 0) table[middle + j] = z;
        if (A.causal && b == 0)                       // no row sees a key behind it: as distance 0
            for (int j = 1 + (tid & 7); j <= middle; j += 8) table[middle + j] = z;
    }
}
// LDS of the starts and of `tables` tables.
constexpr int kStartsBytes = 272;                     // of up to 129
__host__ __forceinline__ size_t bias_bytes(int reach, int tables) { return kStartsBytes + 4 * (size_t)(tables * bias_width(reach)); }

// Places of tiles, in the order in which workgroups (and what each has several of: `inner`) take them.
// BY_XCD: workgroups are dealt to the eight XCDs in turn; numbered so that each XCD has runs of consecutive ones (64, or as many as
// leave each eight runs), the heads of a short sequence, whose values lie side by side, are read through one L2 (512 passages,
// forward and backward: 691 us, as they come 709; 48 pages, where a head's tiles are kept together as they come: 576 and 563).
// LONGEST_FIRST: under a causal limit the later rows see more keys (earlier keys are seen by more rows): places go round the
// sequences, each one's longest tiles first (`down`: its last ones), so that short ones are left for the end.  Sequences are taken
// to be of one length; others are only in another order; the last place, which only rows behind the last sequence can have, stays (24 causal pages, forward and backward: 508 us, as they come 585).
__device__ __forceinline__ int in_order(int block, int blocks) {
    const int lg = blocks < 128 ? 0 : blocks >= 4096 ? 6 : 25 - __builtin_clz(blocks);
    const int whole = blocks >> (lg + 3) << (lg + 3), xcd = block & 7, i = block >> 3;
    return block < whole ? (((i >> lg) * 8 + xcd) << lg) + (i & ((1 << lg) - 1)) : block;
}
__device__ __forceinline__ int longest_first(int x, int slots, int n, bool down) {
    const int f = slots / n, rest = slots - f * n, j = x / n;      // sequence i has the places from i f + floor(i rest / n)
    int i = x - j * n;
    if (j >= f) i = (int)(((int64_t)(x - f * n + 1) * n + rest - 1) / rest) - 1;      // of those with one more
    return i * f + (int)((int64_t)i * rest / n) + (down && j < f ? f - 1 - j : j);
}
struct Work { int slot, inner; };
__device__ __forceinline__ Work work_of(int block, int slots, int inner, int n, int order, bool down) {
    const int x = order == BY_XCD ? in_order(block, slots * inner) : block, slot = x / inner;
    return {order == LONGEST_FIRST && slot < slots - 1 ? longest_first(slot, slots - 1, n, down) : slot, x - slot * inner};
}
// Which way a block of 32 rows and columns lies whose first key and row are d0 apart: -1 or 1: all beyond reach, 0: not.
__device__ __forceinline__ int block_side(int d0, int reach) { return d0 + 31 <= -reach ? -1 : d0 - 31 >= reach ? 1 : 0; }

// The columns' rows take the scale's sign (exact), and are zeros where it is zero, so that the maximum of the raw products is that
// of the scores.  Without a bias scores stay raw products; with one they are scaled by |scale| and natural, as the table is.
// The exponential takes powers of two, and is given fma(score, k, -(maximum * k)), one instruction.  Where the maximum is far from
// zero (a table that hides distances by values down to the type's lowest, in rows that see no other distance; scores of millions) the
// rounding of that product, or its overflow, is larger than the differences that matter: there it is (score - maximum) * k, which is
// 0 for the maximum itself.  kFar is where that begins, in powers of two: up to it the product's rounding is 2^-18.
constexpr float kFar = 128.f;
__device__ __forceinline__ float unit_of_scores(float scale) { return scale == 0.f ? 1.f : fabsf(scale); }
// A product that is rounded before anything is added to it.
__device__ __forceinline__ float rounded_product(float a, float b) {
#pragma clang fp contract(off)
    return a * b;
}
// Exponent of a probability's share whose own maximum is m, from where the maximum is `to` (both finite).
__device__ __forceinline__ float exponent_between(float m, float to, float k) {
    const float a = m * k, b = to * k;
    return fabsf(a) > kFar || fabsf(b) > kFar ? (m - to) * k : a - b;
}
// From here on a sum's logarithm is taken to be the maximum: the sum of up to 2^31 exponentials adds less than three of its last
// places, and the backward pass finds the maximum in it, to the bit.
constexpr float kLostLog = 134217728.f;
// Natural logarithm of a sum l of exponentials from the maximum m on, a score's unit being `unit`.
__device__ __forceinline__ float log_of_sum(float m, float l, float k, float unit) {
    if (l == 0.f) return -INFINITY;
    if (l != l) return l;                            // the row saw a NaN
    const float a = m * k, b = rounded_product(m, unit);
    return fabsf(a) <= kFar ? fmaf(a, LN2, logf(l)) : fabsf(b) < kLostLog ? b + logf(l) : b;
}

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
    __device__ __forceinline__ void take_sign(float scale) {
        if (scale > 0.f) return;
#pragma unroll
        for (int c = 0; c < D / 16; ++c) v[c] = scale < 0.f ? -v[c] : typename Oper<E>::Frag{};
    }
};

// Two matrices' rows on their way to tiles in LDS.  What a mask hides may be anything: zeros are written in its place.
template <class E, int D, int THREADS, bool MASKED, int ROWS> struct Staged {
    using T = Tile<E, D, ROWS>;
    using R = Rows<E, D, THREADS, ROWS>;
    R x, y;
    uint8_t keep[MASKED ? R::N : 1];
    // a_at(row), b_at(row): byte offsets of the matrices' rows; kept(row): whether the mask leaves it.  rows: how many are left.
    template <class AtA, class AtB, class Kept>
    __device__ __forceinline__ void issue(const char* a, const char* b, char* lds, int rows, int tid0, AtA&& a_at, AtB&& b_at, Kept&& kept) {
        const int tid = here(tid0), wave = __builtin_amdgcn_readfirstlane(tid0 >> 6);
        x.issue(a, lds, rows, tid, wave, a_at);
        y.issue(b, lds + T::BYTES, rows, tid, wave, b_at);
        if constexpr (MASKED) {
#pragma unroll
            for (int i = 0; i < R::N; ++i) {
                const int r = R::row(i, tid);
                keep[i] = kept(r < rows ? r : rows - 1);
            }
        }
    }
    __device__ __forceinline__ void finish(char* lds, int tid) const {
        auto whole = [&](int i) { return !MASKED || keep[MASKED ? i : 0]; };
        x.finish(lds, tid, whole);
        y.finish(lds + T::BYTES, tid, whole);
    }
};

// A workgroup's tile of query columns, and which keys its rows see.
struct QueryTile {
    int row0, Lq, Lk, q0, k0, shift, end;     // first row, lengths, first global rows, Lk - Lq, keys that any row sees
    bool none;
    __device__ __forceinline__ QueryTile(const AttnArgs& A, int slot, int per, int lane) {
        const int seq = find_sequence(A.qoff, A.n_seqs, per, A.total_q, slot, lane);
        bool rest;
        const Range q = rows_of_place(A.qoff, seq, A.n_seqs, A.total_q, per, slot, rest);
        const Range k = rest ? Range{0, 0, 0} : sequence_rows(A.koff, seq, A.total_k);
        row0 = (slot - q.place) * per;
        Lq = q.n;
        Lk = k.n;
        q0 = q.lo;
        k0 = k.lo;
        shift = Lk - Lq;
        none = row0 < 0 || row0 >= Lq;
        const int last = (row0 + per < Lq ? row0 + per : Lq) - 1;
        end = A.causal ? last + shift + 1 : Lk;
        end = end < 0 ? 0 : end > Lk ? Lk : end;
    }
};

// A wavefront's 32 columns of it.
struct QueryColumns {
    int row, head, lim, first_lim, end;       // own row, head in its unit, key limit; that of the first column; keys that any sees
    bool real, busy;
    __device__ __forceinline__ QueryColumns(const AttnArgs& A, const QueryTile& t, int G, int per, int wave, int lane) {
        const int local = (wave * 32 + (lane & 31)) / G;
        row = t.row0 + local;
        head = (wave * 32 + (lane & 31)) % G;
        real = local < per && row < t.Lq;
        lim = row + t.shift;
        const int first = t.row0 + wave * 32 / G, last = t.row0 + (wave * 32 + 31) / G;
        first_lim = first + t.shift;
        busy = wave * 32 / G < per && first < t.Lq;
        const int e = last + t.shift + 1;
        end = A.causal && e < t.end ? e : t.end;
    }
};

template <int LO> __device__ __forceinline__ f32x8 eight(const f32x16& x) {
    return __builtin_shufflevector(x, x, LO, LO + 1, LO + 2, LO + 3, LO + 4, LO + 5, LO + 6, LO + 7);
}

// Values of a block's rows, as its accumulators have them (LDS).  Tiles whose rows are not all seen by every column get minus
// infinity added to the scores of rows that none sees (past the end, or hidden by the mask), and causal ones a limit on the row as
// well.  These, and all that not every tile needs, are branches around a few instructions: a copy of the whole tile's code for each
// case costs some sixty registers, since the accumulators are in other places in each.
__device__ __forceinline__ f32x16 of_rows(const float* v, int b, int h) {
    f32x16 x;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const f32x4 y = *(const f32x4*)(v + 32 * b + 8 * j + 4 * h);
#pragma unroll
        for (int i = 0; i < 4; ++i) x[4 * j + i] = y[i];
    }
    return x;
}

// Rows of a block that a lane's column sees under a limit, as bits: a lane's rows lie at 8 (r / 4) + r % 4 from its first one.  One
// register instead of sixteen comparisons' masks, which take scalar registers that other values are then moved out of.
__device__ __forceinline__ uint32_t bits_up_to(int room) { return room < 0 ? 0u : room >= 31 ? ~0u : (2u << room) - 1u; }
__device__ __forceinline__ uint32_t all_if(uint32_t bits, int r) { return (uint32_t)((int)(bits << (31 - 8 * (r >> 2) - (r & 3))) >> 31); }
__device__ __forceinline__ float hidden_unless(float x, uint32_t all) {
    return __uint_as_float((__float_as_uint(x) & all) | (0xff800000u & ~all));
}

// Wavefronts per SIMD that the registers are shared out for: forward pass, gradients of queries, of keys and values (one more each
// makes the compiler spill, and is slower; 512 passages: forward pass with three and four 150 and 227 us, forward and backward with
// two and three for the queries 765 and 691, with two and three for the keys 691 and 850).
template <class E, int D> constexpr int kWaves = sizeof(E) == 2 || D <= 32 ? 3 : D <= 96 ? 2 : 1;
template <class E, int D> constexpr int kGradientWaves = sizeof(E) == 2 || D <= 32 ? 2 : 1;
template <class E, int D> constexpr int kQueryWaves = sizeof(E) == 2 && D <= 64 ? 3 : kGradientWaves<E, D>;
// Key rows of the forward pass's tiles: of wide heads 32, so that LDS and registers hold three workgroups (48 pages of 1,030 rows,
// d = 128: 563 us; with 64 rows the compiler spills, 1,215; the gradients' kernels, which have registers for two, lose by 32).
template <class E, int D> constexpr int kForwardRows = D >= 96 ? 32 : Oper<E>::ROWS;
template <int D> constexpr bool kRuns = goes_on_to_next_head(D);

// ---- forward -------------------------------------------------------------------------------------------------
// One pass over the keys with the running maximum and sum of the softmax, in 32 bits; probabilities are rounded to the
// storage type for the second product (their sum is not; outputs in 16 bits are off by 2.3e-3 of their norm, their own rounding
// is 1.7e-3; probabilities in two values would make three products of two).  The maximum that is subtracted may lag by up to kLag: sums and
// outputs are rescaled only when it is passed, which few tiles after the first do; probabilities up to 2^kLag are no less exact
// (48 pages of 1,030 rows, 16 heads of 128 over 8: 563 us, without a lag 613).
constexpr float kLag = 8.f;
// A workgroup takes its tile for `run` head units one after the other, the first keys of the next on their way while it
// computes: short sequences have one to three tiles of keys, whose latency would otherwise be most of the time.
// Long sequences are bound by the matrix and vector units' turns (an exponential, a maximum, a sum and half a conversion for every
// score: as many clocks as the products): the pages above 552 to 565 us, 750 TFLOP/s where this library's scoring of all documents
// reaches 1,504.  Short ones by latency and what a workgroup does before its first product: 512 passages, 12 heads of 64 with bias and
// mask, 151 us.  Single tokens by memory: 16 over 1 to 16,385 keys, two key heads of 128, 134 MB in 30 us and 7.3 us to join their
// parts.
template <class E, int D, bool BIAS, bool MASKED>
__global__ __launch_bounds__(64 * kWavefronts, (kWaves<E, D>)) void k_attention(const AttnArgs A, int slots, int order, int units, int run,
                                                                           int splits, E* out, float* lse, float* o_part,
                                                                           float2* ml_part) {
    using O = Oper<E>;
    using T = Tile<E, D, kForwardRows<E, D>>;
    constexpr int NB = T::ROWS / 32, DB = D / 32, THREADS = 64 * kWavefronts;
    __shared__ __align__(256) char lds[2][2 * T::BYTES];
    __shared__ __align__(16) float hidden[2][T::ROWS];           // 0, or minus infinity for rows that no column sees
    extern __shared__ __align__(16) char dyn[];
    const int tid = threadIdx.x, lane0 = tid & 63, lane = lane0, wave = __builtin_amdgcn_readfirstlane(tid >> 6), h = lane >> 5;
    const Work work = work_of(blockIdx.x, slots, (units + run - 1) / run * splits, A.n_seqs, order, true);
    const int split = work.inner % splits, slot = work.slot;
    int unit = work.inner / splits * run;
    const int end_unit = unit + run < units ? unit + run : units;
    const int G = A.pack, per = 32 * kWavefronts / G;
    const QueryTile t(A, slot, per, lane);
    if (t.none) return;
    const QueryColumns w(A, t, G, per, wave, lane);
    const int tiles = (t.end + T::ROWS - 1) / T::ROWS, each = (tiles + splits - 1) / splits;
    const int first_tile = split * each, end_tile = first_tile + each < tiles ? first_tile + each : tiles;

    const int64_t krow = A.k_row * (int64_t)sizeof(E), vrow = A.v_row * (int64_t)sizeof(E);
    Staged<E, D, THREADS, MASKED, T::ROWS> next;
    uint8_t next_keep = 0;
    auto issue = [&](int u, int base, char* to) {
        const int kv = u * G / A.group;
        next.issue((const char*)A.k + (t.k0 + base) * krow + kv * A.k_head * (int64_t)sizeof(E),
                   (const char*)A.v + (t.k0 + base) * vrow + kv * A.v_head * (int64_t)sizeof(E), to, t.end - base, tid,
                   [&](int r) { return (uint32_t)r * (uint32_t)krow; }, [&](int r) { return (uint32_t)r * (uint32_t)vrow; },
                   [&](int r) { return A.keep[(int64_t)t.k0 + base + r]; });
        next_keep = base + lane < t.end;
        if constexpr (MASKED) next_keep = lane < T::ROWS && base + lane < t.end ? A.keep[(int64_t)t.k0 + base + lane] : 0;
    };
    constexpr uint64_t kAllRows = T::ROWS == 64 ? ~0ull : (1ull << (T::ROWS & 63)) - 1ull;
    uint64_t seen = 0;                                           // rows of the tile that some column sees
    auto finish = [&](int buf) {
        next.finish(lds[buf], tid);
        if (tid < T::ROWS) hidden[buf][tid] = next_keep ? 0.f : -INFINITY;
        seen = __ballot(next_keep != 0) & kAllRows;
    };
    Column<E, D> q;
    auto load_q = [&](int u) {
        const int h = here(lane0) >> 5;
        q.load((const E*)A.q + (int64_t)(t.q0 + w.row) * A.q_row + (u * G + w.head) * A.q_head, w.real, h);
        q.take_sign(A.scale);
    };
    const bool any = first_tile < end_tile;
    if (any) issue(unit, first_tile * T::ROWS, lds[0]);
    load_q(unit);
    int16_t* starts = (int16_t*)dyn;
    float* table = (float*)(dyn + kStartsBytes);
    const int middle = bias_middle(A.reach);
    if constexpr (BIAS) {
        load_starts(A, starts, tid, THREADS);
        __syncthreads();
        fill_bias<E>(A, unit, starts, table, tid, THREADS);
    }
    f32x16 acc[DB] = {};
    float m = -INFINITY, l = 0.f, off = 0.f;                     // off: -m k, of a row with a maximum
    bool far = false;                                            // of some row of the wavefront
    bool sees = !MASKED;                                         // the mask leaves the row some key
    const float unit_scale = unit_of_scores(A.scale), k = BIAS ? LOG2E : unit_scale * LOG2E, lag = fminf(kLag / k, 1e38f);
    if (any) finish(0);
    __syncthreads();
    const typename T::At at_tiles(lds[0], lane);
    int i = first_tile, buf = 0;
    while (true) {
        const int base = i * T::ROWS;
        const typename T::At lk = at_tiles + buf * 2 * T::BYTES, lv = lk + T::BYTES;
        const bool last = i + 1 >= end_tile;                     // of the unit
        const int n_unit = last ? unit + 1 : unit, n_i = last ? first_tile : i + 1;
        const bool more = kRuns<D> ? n_unit < end_unit : !last;
        if (more && any) issue(n_unit, n_i * T::ROWS, lds[buf ^ 1]);
        if (any && w.busy && base < w.end) {
            const bool one = NB > 1 && base + 32 >= w.end;       // its second block has no keys
            const bool diagonal = A.causal && base + T::ROWS - 1 > w.first_lim, part = seen != kAllRows;
            if constexpr (MASKED) {
                const int room = A.causal ? w.lim - base : 63;
                sees |= (seen & (room < 0 ? 0ull : room >= 63 ? ~0ull : (2ull << room) - 1ull)) != 0;
            }
            f32x16 s[NB];
            float top = -INFINITY;
#pragma unroll
            for (int b = 0; b < NB; ++b) {
                if (b && one) break;
                s[b] = {};
#pragma unroll
                for (int c = 0; c < D / 16; ++c) O::mma(s[b], T::rows(lk, b, c), q.v[c]);
                if constexpr (BIAS) {
                    const int d0 = base + 32 * b - w.first_lim, side = block_side(d0, A.reach);
                    if (side) {
                        const float x = table[side < 0 ? 0 : 2 * middle];
#pragma unroll
                        for (int r = 0; r < 16; ++r) s[b][r] = fmaf(s[b][r], unit_scale, x);
                    } else {
                        const float* x = table + middle + base + 32 * b + 4 * h - w.lim;
#pragma unroll
                        for (int r = 0; r < 16; ++r) s[b][r] = fmaf(s[b][r], unit_scale, x[8 * (r >> 2) + (r & 3)]);
                    }
                }
                if (part) s[b] += of_rows(hidden[buf], b, h);
                if (diagonal) {
                    const uint32_t own = bits_up_to(w.lim - base - 32 * b - 4 * h);
#pragma unroll
                    for (int r = 0; r < 16; ++r) s[b][r] = hidden_unless(s[b][r], all_if(own, r));
                }
#pragma unroll
                for (int r = 0; r < 16; ++r) top = __builtin_elementwise_maximum(top, s[b][r]);
            }
            top = max_of_halves(top);
            const bool passed = top > m + lag;
            if (__ballot(passed)) {
                const float to = passed ? top : m;
                const float down = m == -INFINITY ? 0.f : exp2_fast(exponent_between(m, to, k));
                off = to == -INFINITY ? 0.f : -(to * k);
                far = __ballot(fabsf(off) > kFar) != 0;
                l *= down;
#pragma unroll
                for (int db = 0; db < DB; ++db) acc[db] *= down;
                m = to;
            }
#pragma unroll
            for (int b = 0; b < NB; ++b) {
                if (b && one) break;
                if (far) {
                    const float from = m == -INFINITY ? 0.f : m;
#pragma unroll
                    for (int r = 0; r < 16; ++r) s[b][r] = (s[b][r] - from) * k;
                } else {
#pragma unroll
                    for (int r = 0; r < 16; ++r) s[b][r] = fmaf(s[b][r], k, off);
                }
#pragma unroll
                for (int r = 0; r < 16; ++r) {
                    s[b][r] = exp2_fast(s[b][r]);
                    l += s[b][r];
                }
                const typename O::Frag p0 = O::round(eight<0>(s[b])), p1 = O::round(eight<8>(s[b]));
#pragma unroll
                for (int db = 0; db < DB; ++db) O::mma(acc[db], T::turned(lv, b, 0, db), p0);
#pragma unroll
                for (int db = 0; db < DB; ++db) O::mma(acc[db], T::turned(lv, b, 1, db), p1);
            }
        }
        if (last) {
            if (kRuns<D> && more) load_q(n_unit);
            l = sum_of_halves(l);
            if (MASKED && !sees) {                               // whatever its row held
                m = -INFINITY;
                l = 0.f;
#pragma unroll
                for (int db = 0; db < DB; ++db) acc[db] = {};
            }
            const int head = unit * G + w.head;
            const int64_t at = (int64_t)(t.q0 + w.row);
            if (w.real && splits > 1) {
                const int64_t place = ((int64_t)split * A.heads + head) * A.total_q + at;
                if (h == 0) ml_part[place] = make_float2(m, l);
#pragma unroll
                for (int db = 0; db < DB; ++db)
#pragma unroll
                    for (int j = 0; j < 4; ++j)
                        *(f32x4*)(o_part + place * D + 32 * db + 8 * j + 4 * h) =
                            f32x4{acc[db][4 * j], acc[db][4 * j + 1], acc[db][4 * j + 2], acc[db][4 * j + 3]};
            } else if (w.real) {
                const float inv = l == 0.f ? 0.f : 1.f / l;
                if (h == 0) lse[(int64_t)head * A.total_q + at] = log_of_sum(m, l, k, BIAS ? 1.f : unit_scale);
                E* o = out + (at * A.heads + head) * D;
#pragma unroll
                for (int db = 0; db < DB; ++db)
#pragma unroll
                    for (int j = 0; j < 4; ++j)
                        O::store4(o + 32 * db + 8 * j + 4 * h, f32x4{acc[db][4 * j] * inv, acc[db][4 * j + 1] * inv,
                                                                      acc[db][4 * j + 2] * inv, acc[db][4 * j + 3] * inv});
            }
            if (!more) return;
            m = -INFINITY;
            l = off = 0.f;
            far = false;
            sees = !MASKED;
#pragma unroll
            for (int db = 0; db < DB; ++db) acc[db] = {};
        }
        if (any) finish(buf ^ 1);
        __syncthreads();
        if (BIAS && last) {                                      // nobody reads the table of the unit before any more
            fill_bias<E>(A, n_unit, starts, table, tid, THREADS);
            __syncthreads();
        }
        unit = n_unit;
        i = n_i;
        buf ^= 1;
    }
}

// Joins the parts of rows whose keys were split: a wavefront for each row and head, its lanes over the parts for their maximum, then
// over the row's values, four each, and several parts at a time.
template <class E, int D>
__global__ __launch_bounds__(256) void k_attention_join(const AttnArgs A, int splits, const float* o_part, const float2* ml_part,
                                                        E* out, float* lse) {
    const float unit = A.bias ? 1.f : unit_of_scores(A.scale), k = unit * LOG2E;
    constexpr int LANES = D / 4 <= 8 ? 8 : D / 4 <= 16 ? 16 : 32, PARTS = 64 / LANES, AHEAD = 4;
    const int lane = threadIdx.x & 63;
    const int64_t rows = (int64_t)A.heads * A.total_q, place = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
    if (place >= rows) return;
    const int64_t row = place % A.total_q;
    if (row < A.qoff[0]) return;                     // no sequence's, and no parts either
    float m = -INFINITY;
    for (int s = lane; s < splits; s += 64) m = fmaxf(m, ml_part[s * rows + place].x);
#pragma unroll
    for (int x = 1; x < 64; x <<= 1) m = fmaxf(m, __shfl_xor(m, x));
    const int dim = lane % LANES * 4;
    float l = 0.f;
    f32x4 o = {0.f, 0.f, 0.f, 0.f};
    for (int s0 = lane / LANES; s0 < splits; s0 += PARTS * AHEAD) {
        float2 ml[AHEAD];
        f32x4 x[AHEAD];
#pragma unroll
        for (int j = 0; j < AHEAD; ++j) {
            const int s = s0 + j * PARTS;
            ml[j] = make_float2(-INFINITY, 0.f);
            x[j] = f32x4{0.f, 0.f, 0.f, 0.f};
            if (s < splits && dim < D) {
                ml[j] = ml_part[s * rows + place];
                x[j] = *(const f32x4*)(o_part + (s * rows + place) * D + dim);
            }
        }
#pragma unroll
        for (int j = 0; j < AHEAD; ++j) {
            if (ml[j].y == 0.f) continue;
            const float w = exp2_fast(exponent_between(ml[j].x, m, k));
            l += ml[j].y * w;
            o += x[j] * w;
        }
    }
#pragma unroll
    for (int x = LANES; x < 64; x <<= 1) {
        l += __shfl_xor(l, x);
#pragma unroll
        for (int e = 0; e < 4; ++e) o[e] += __shfl_xor(o[e], x);
    }
    if (lane >= LANES || dim >= D) return;
    const float inv = l == 0.f ? 0.f : 1.f / l;
    if (lane == 0) lse[place] = log_of_sum(m, l, k, unit);
    Oper<E>::store4(out + (row * A.heads + place / A.total_q) * D + dim, o * inv);
}

// ---- backward ------------------------------------------------------------------------------------------------
// dS_ij = P_ij (<dO_i, V_j> - delta_i), delta_i = <dO_i, O_i>, P_ij = exp(S_ij - lse_i), all in 32 bits; P and dS are rounded
// to the storage type as operands of the last products.  Queries' and keys' gradients are made by a kernel each, which
// recomputes the scores twice (seven products where one kernel would need five) but adds in a fixed order, where one
// kernel would have to add either side's gradients by atomics.
// The rounding of O reaches dS through delta, the same for all of a row.  Rows of dS sum to zero, so what a row's sum is
// instead is the error of its delta: the first kernel adds it to the delta that the second one takes.  In the first, 16-bit dS goes
// into its product as two values of eight bits each, which leaves O's rounding as the only error beside the result's own (gradients
// of queries, against 64 bits, 512 passages: 2.6e-3 with one value, 2.0e-3 with two; the result's own rounding is 1.7e-3).  Those of
// keys and values are made from dS and P in one value each: 2.35e-3, as a second one would be two more products of four.  Rows that
// see few keys have small gradients and a large O, so that its rounding counts most there: tiles that see up to kTwice keys go over
// them twice, first for delta in 32 bits (60 causal sequences of 1 to 17 tokens: 2.8e-3, so 1.7e-3; of 1 to 301: 2.2e-3 and 1.7e-3.
// It costs the 512 passages 22 us of 691, with 64 keys 2 us, which leaves 2.1e-3 for sequences of up to 131 tokens).
constexpr int kTwice = 128;
// P's error is the rounding of a log-sum-exp in 32 bits, 2^-24 of its size.  Rows where that would show (is_far: from 2^-16 on) are
// normalised again: exponents are score - lse, which is exact or nearly so, and the first kernel goes over the keys of their tiles
// twice, first for the sum of what they give, by whose logarithm it and the second kernel correct them, and for delta.
constexpr float kFarRow = 256.f;
// (A log-sum-exp is also divided by the scale, where accumulators start from it: that must not overflow.)
__device__ __forceinline__ bool is_far(float lse, float scale2) {
    const float a = fabsf(lse);
    return a < INFINITY && (a > kFarRow || a * LOG2E > 1e30f * scale2);
}
// Bound by the matrix and vector units' turns where sequences are long (24 causal pages, 8 heads of 128 over 2: 178 and 227 us, 451
// TFLOP/s of the three and four products that each cannot do without), by latency and by what surrounds the products where they are
// short (the 512 passages: 289 and 265 us).

// Sums of a 32 x 32 block along its diagonals, added to a histogram by distance.  The block is in accumulators: a lane has sixteen
// keys of a column.  Lane p of a half takes key k's value from column (p + k) mod 32: it lies on diagonal -p, or 32 - p where that
// wraps.  Both sums of a lane are complete with those of the other half's keys; the lower half has the first, the upper the second.
// No atomics, which take 2.5 clocks a lane there, and a fixed order.
__device__ __forceinline__ void add_diagonals(const f32x16& x, float* hist, int lane) {
    const int own = here(lane), p = own & 31, h = own >> 5, from = p + 4 * h;
    float a = 0.f, w = 0.f;
#pragma unroll
    for (int r = 0; r < 16; ++r) {
        const int n = from + 8 * (r >> 2) + (r & 3);
        const float y = __int_as_float(__builtin_amdgcn_ds_bpermute((n & 31) << 2 | h << 7, __float_as_int(x[r])));
        a += n < 32 ? y : 0.f;
        w += n < 32 ? 0.f : y;
    }
    const auto s = __builtin_amdgcn_permlane32_swap(__float_as_uint(a), __float_as_uint(w), false, false);
    const uint32_t lo = s[0], hi = s[1];
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    hist[32 * h - p] += __uint_as_float(lo) + __uint_as_float(hi);
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
}

// Gradients of queries, delta, and the bias table's share of each tile; head units one after the other, as the forward pass.
template <class E, int D, bool BIAS, bool MASKED>
__global__ __launch_bounds__(64 * kWavefronts, (kQueryWaves<E, D>)) void
k_attention_dq(const AttnArgs A, int slots, int order, int units, int run, const E* out, const E* dout, const float* lse, E* dq,
               float* delta, float* bias_part) {
    using O = Oper<E>;
    using T = Tile<E, D>;
    constexpr int NB = T::ROWS / 32, DB = D / 32, THREADS = 64 * kWavefronts;
    __shared__ __align__(256) char lds[2][2 * T::BYTES];
    __shared__ __align__(16) float hidden[2][T::ROWS];
    __shared__ float far_sum[kMostRun][kWavefronts][2];
    __shared__ float far_lse[THREADS];                // own log-sum-exp, for far tiles
    __shared__ int any_row_far[2][kWavefronts];                // of a wavefront's rows, for this head unit and the next
    extern __shared__ __align__(16) char dyn[];       // the bias by distance, then histograms of each head and wavefront
    const int tid = threadIdx.x, lane0 = tid & 63, lane = lane0, wave = __builtin_amdgcn_readfirstlane(tid >> 6), h = lane >> 5;
    const Work work = work_of(blockIdx.x, slots, (units + run - 1) / run, A.n_seqs, order, true);
    const int slot = work.slot, first_unit = work.inner * run;
    int unit = first_unit;
    const int end_unit = unit + run < units ? unit + run : units;
    const int G = A.pack, per = 32 * kWavefronts / G;
    const QueryTile t(A, slot, per, lane);
    if (t.none) {
        if constexpr (BIAS)
            for (int b = tid; b < (end_unit - unit) * A.n_buckets; b += THREADS)
                bias_part[((int64_t)slot * A.heads + unit) * A.n_buckets + b] = 0.f;
        return;
    }
    const QueryColumns w(A, t, G, per, wave, lane);
    const int tiles = (t.end + T::ROWS - 1) / T::ROWS;
    const bool few = sizeof(E) == 2 && t.end <= kTwice;
    bool far = false, twice = few;                               // some row of the tile is far; twice: first for delta and sums
    const int64_t krow = A.k_row * (int64_t)sizeof(E), vrow = A.v_row * (int64_t)sizeof(E);
    Staged<E, D, THREADS, MASKED, T::ROWS> next;
    uint8_t next_keep = 0;
    auto issue = [&](int u, int base, char* to) {
        const int kv = u * G / A.group;
        next.issue((const char*)A.k + (t.k0 + base) * krow + kv * A.k_head * (int64_t)sizeof(E),
                   (const char*)A.v + (t.k0 + base) * vrow + kv * A.v_head * (int64_t)sizeof(E), to, t.end - base, tid,
                   [&](int r) { return (uint32_t)r * (uint32_t)krow; }, [&](int r) { return (uint32_t)r * (uint32_t)vrow; },
                   [&](int r) { return A.keep[(int64_t)t.k0 + base + r]; });
        next_keep = base + lane < t.end;
        if constexpr (MASKED) next_keep = lane < T::ROWS && base + lane < t.end ? A.keep[(int64_t)t.k0 + base + lane] : 0;
    };
    constexpr uint64_t kAllRows = T::ROWS == 64 ? ~0ull : (1ull << (T::ROWS & 63)) - 1ull;
    uint64_t seen = 0;                                           // rows of the tile that some column sees
    auto finish = [&](int buf) {
        next.finish(lds[buf], tid);
        if (tid < T::ROWS) hidden[buf][tid] = next_keep ? 0.f : -INFINITY;
        seen = __ballot(next_keep != 0) & kAllRows;
    };
    const bool any = tiles > 0;
    if (any) issue(unit, 0, lds[0]);
    Column<E, D> q, g;
    float dot = 0.f, own_lse = 0.f;                              // own_lse: what is added to the exponent
    const float unit_scale = unit_of_scores(A.scale), scale2 = unit_scale * LOG2E;
    auto load_rows = [&](int u) {
        const int64_t at = t.q0 + here(w.row);
        const int h = here(lane0) >> 5, head = u * G + w.head;
        const int64_t dense = (at * A.heads + head) * D;
        const float row_lse = w.real ? lse[(int64_t)head * A.total_q + at] : -INFINITY;
        Column<E, D> o;
        q.load((const E*)A.q + at * A.q_row + head * A.q_head, w.real, h);
        g.load(dout + dense, w.real, h);
        o.load(out + dense, w.real, h);
        // rows that see nothing take no part, whatever their gradient is: exp2(x - inf) = 0
        const bool seeing = row_lse != -INFINITY;
        own_lse = seeing ? -row_lse * LOG2E : -INFINITY;
        far_lse[tid] = seeing ? row_lse : INFINITY;
        const bool is = __ballot(is_far(row_lse, scale2)) != 0;
        if (lane0 == 0) any_row_far[u & 1][wave] = is;
        dot = 0.f;
#pragma unroll
        for (int c = 0; c < D / 16; ++c) {
            if (!seeing) {
                q.v[c] = {};
                g.v[c] = {};
            }
            const f32x8 x = O::wide(g.v[c]), y = O::wide(o.v[c]);
#pragma unroll
            for (int e = 0; e < 8; ++e) dot += x[e] * y[e];
        }
        dot = few ? 0.f : sum_of_halves(dot);
        q.take_sign(A.scale);
    };
    load_rows(unit);
    const int middle = bias_middle(A.reach), width = bias_width(A.reach);
    int16_t* starts = (int16_t*)dyn;
    float* table = (float*)(dyn + kStartsBytes);
    float* hist = table + width;
    float* own_hist = hist + wave * width + middle;
    if constexpr (BIAS) {
        for (int i = tid; i < (end_unit - unit) * kWavefronts * width; i += THREADS) hist[i] = 0.f;
        load_starts(A, starts, tid, THREADS);
        __syncthreads();
        fill_bias<E>(A, unit, starts, table, tid, THREADS);
    }
    float far_lo = 0.f, far_hi = 0.f, weight_lo = 0.f, weight_hi = 0.f;
    f32x16 acc[DB] = {};
    float row_sum = 0.f;
    if (any) finish(0);
    __syncthreads();
    const typename T::At at_tiles(lds[0], lane);
    float weight = 0.f;                                          // sum of a row's probabilities, in a far tile's first pass
    int i = 0, buf = 0;
    while (true) {
        if (i == 0) {                                            // a head unit begins
            int is = 0;
#pragma unroll
            for (int v = 0; v < kWavefronts; ++v) is |= any_row_far[unit & 1][v];
            far = __builtin_amdgcn_readfirstlane(is) != 0;
            twice = few || far;
            if (far) {
                own_lse = dot = weight = 0.f;
            }
        }
        const bool before = twice && i < tiles;
        const float k = BIAS || far ? LOG2E : scale2;
        const int base = (i < tiles ? i : i - tiles) * T::ROWS;
        const typename T::At lk = at_tiles + buf * 2 * T::BYTES, lv = lk + T::BYTES;
        const bool last = i + 1 >= (twice ? 2 * tiles : tiles);
        const int n_unit = last ? unit + 1 : unit, n_i = last ? 0 : i + 1;
        const bool more = kRuns<D> ? n_unit < end_unit : !last;
        if (more && any) issue(n_unit, (n_i < tiles ? n_i : n_i - tiles) * T::ROWS, lds[buf ^ 1]);
        if (any && w.busy && base < w.end) {
            const bool diagonal = A.causal && base + T::ROWS - 1 > w.first_lim, part = seen != kAllRows;
#pragma unroll 1
            for (int b = 0; b < NB && base + 32 * b < w.end; ++b) {
                f32x16 s = {}, dp;
#pragma unroll
                for (int c = 0; c < D / 16; ++c) O::mma(s, T::rows(lk, b, c), q.v[c]);
                phase();
#pragma unroll
                for (int r = 0; r < 16; ++r) dp[r] = -dot;
#pragma unroll
                for (int c = 0; c < D / 16; ++c) O::mma(dp, T::rows(lv, b, c), g.v[c]);
                phase();
                const int d0 = base + 32 * b - w.first_lim, side = BIAS ? block_side(d0, A.reach) : 0;
                if (BIAS && !side) {
                    const float* x = table + middle + base + 32 * b + 4 * h - w.lim;
#pragma unroll
                    for (int r = 0; r < 16; ++r) s[r] = fmaf(s[r], unit_scale, x[8 * (r >> 2) + (r & 3)]);
                } else if constexpr (BIAS) {
                    const float x = table[side < 0 ? 0 : 2 * middle];
#pragma unroll
                    for (int r = 0; r < 16; ++r) s[r] = fmaf(s[r], unit_scale, x);
                }
                if (part) s += of_rows(hidden[buf], b, h);
                if (diagonal) {                       // (dp as well: what the row does not see may be anything)
                    const uint32_t own = bits_up_to(w.lim - base - 32 * b - 4 * h);
#pragma unroll
                    for (int r = 0; r < 16; ++r) {
                        s[r] = hidden_unless(s[r], all_if(own, r));
                        dp[r] = __uint_as_float(__float_as_uint(dp[r]) & all_if(own, r));
                    }
                }
                if (far) {
                    const float from = far_lse[tid];
#pragma unroll
                    for (int r = 0; r < 16; ++r) s[r] = (BIAS ? s[r] : rounded_product(s[r], unit_scale)) - from;
                    if (before)
#pragma unroll
                        for (int r = 0; r < 16; ++r) weight += exp2_fast(s[r] * LOG2E);
                }
#pragma unroll
                for (int r = 0; r < 16; ++r) s[r] = exp2_fast(fmaf(s[r], k, own_lse));
                if (BIAS && side && !before) {
                    float weight = 0.f;
#pragma unroll
                    for (int r = 0; r < 16; ++r) weight += s[r];
                    (side < 0 ? weight_lo : weight_hi) += weight;
                }
                float sum = 0.f;
#pragma unroll
                for (int r = 0; r < 16; ++r) {
                    s[r] *= dp[r];
                    sum += s[r];
                }
                row_sum += sum;
                if (before) continue;
                if constexpr (BIAS) {
                    if (side) (side < 0 ? far_lo : far_hi) += sum;
                    else add_diagonals(s, own_hist + d0, lane);
                }
                phase();
                if constexpr (sizeof(E) == 2) {
#pragma unroll
                    for (int c = 0; c < 2; ++c) {
                        const f32x8 x = c ? eight<8>(s) : eight<0>(s);
                        f32x8 most;
#pragma unroll
                        for (int e = 0; e < 8; ++e) most[e] = __uint_as_float(__float_as_uint(x[e]) & 0xffff0000u);
                        const typename O::Frag p = O::round(most), rest = O::round(x - most);
#pragma unroll
                        for (int db = 0; db < DB; ++db) {
                            const typename O::Frag x = T::turned(lk, b, c, db);
                            O::mma(acc[db], x, rest);
                            O::mma(acc[db], x, p);
                        }
                    }
                } else {
#pragma unroll
                    for (int db = 0; db < DB; ++db) O::mma(acc[db], T::turned(lk, b, 0, db), O::round(eight<0>(s)));
#pragma unroll
                    for (int db = 0; db < DB; ++db) O::mma(acc[db], T::turned(lk, b, 1, db), O::round(eight<8>(s)));
                }
            }
        }
        if (before && i + 1 == tiles) {
            dot = sum_of_halves(row_sum);
            row_sum = 0.f;
            if (far) {
                weight = sum_of_halves(weight);
                dot = weight == 0.f ? 0.f : dot / weight;
                own_lse = weight == 0.f ? 0.f : -log2f(weight);
            }
        }
        if (last) {
            row_sum = sum_of_halves(row_sum);
            const int64_t at = t.q0 + here(w.row);
            const int head = unit * G + w.head;
            if (w.real) {
                if (h == 0) delta[(int64_t)head * A.total_q + at] = dot + row_sum;
                if (far && h == 0) delta[((int64_t)A.heads + head) * A.total_q + at] = own_lse;
                E* o = dq + (at * A.heads + head) * D;
#pragma unroll
                for (int db = 0; db < DB; ++db)
#pragma unroll
                    for (int j = 0; j < 4; ++j)
                        O::store4(o + 32 * db + 8 * j + 4 * h,
                                  f32x4{acc[db][4 * j] * A.scale, acc[db][4 * j + 1] * A.scale, acc[db][4 * j + 2] * A.scale,
                                        acc[db][4 * j + 3] * A.scale});
            }
            if (kRuns<D> && more) load_rows(n_unit);
        }
        if (more && any) finish(buf ^ 1);
        if constexpr (BIAS) {
            if (last) {
                // what delta was off by, over the many keys of the open buckets
                far_lo -= row_sum * weight_lo;
                far_hi -= row_sum * weight_hi;
#pragma unroll
                for (int m = 1; m < 64; m <<= 1) {
                    far_lo += __shfl_xor(far_lo, m);
                    far_hi += __shfl_xor(far_hi, m);
                }
                if (lane == 0) {
                    far_sum[unit - first_unit][wave][0] = far_lo;
                    far_sum[unit - first_unit][wave][1] = far_hi;
                }
                far_lo = far_hi = weight_lo = weight_hi = 0.f;
                own_hist += kWavefronts * width;
                __syncthreads();
                if (more) fill_bias<E>(A, n_unit, starts, table, tid, THREADS);
            }
        }
        if (last) {
            if (!more) break;
            row_sum = 0.f;
#pragma unroll
            for (int db = 0; db < DB; ++db) acc[db] = {};
        }
        __syncthreads();
        unit = n_unit;
        i = n_i;
        buf ^= 1;
    }
    if constexpr (BIAS) {                             // the histograms of all heads: by wavefront, by bucket
        const int heads = end_unit - first_unit;
        for (int i = tid; i < heads * width; i += THREADS) {
            float* x = hist + i / width * kWavefronts * width + i % width;
#pragma unroll
            for (int v = 1; v < kWavefronts; ++v) x[0] += x[v * width];
        }
        __syncthreads();
        for (int i = tid >> 3; i < heads * A.n_buckets; i += THREADS / 8) {
            const int u = i / A.n_buckets, b = i % A.n_buckets;
            const float* x = hist + u * kWavefronts * width + middle;
            const bool behind = b >= A.n_dir;                             // buckets of keys behind the query
            const int j0 = behind ? b - A.n_dir : b, end = starts[j0 + 1];
            float sum = 0.f;
            for (int j = starts[j0] + (tid & 7); j < end; j += 8) sum += behind ? (j > 0 ? x[j] : 0.f) : x[-j];
#pragma unroll
            for (int m = 1; m < 8; m <<= 1) sum += __shfl_xor(sum, m);
            if ((tid & 7) == 0) {
                if (j0 == A.n_dir - 1)                                    // the open one of its direction
#pragma unroll
                    for (int v = 0; v < kWavefronts; ++v) sum += far_sum[u][v][behind ? 1 : 0];
                bias_part[((int64_t)slot * A.heads + first_unit + u) * A.n_buckets + b] = sum;
            }
        }
    }
}

// Gradients of keys and values, `run` key heads one after the other; workgroups from `main` on add up the bias table's shares
// of all tiles.
// A wavefront with both gradients of 32 wide rows takes more than half of the registers, so nothing runs beside its waits.
// In 16 bits wide heads have two wavefronts for the same rows, one for either gradient: the scores are made twice (five products
// where there were four), but two wavefronts share a SIMD (24 causal pages, forward and backward: 508 us, with one 828).
template <class E, int D> constexpr bool kApart = sizeof(E) == 2 && D >= 96;
template <class E, int D, bool BIAS, bool MASKED>
__global__ __launch_bounds__((kApart<E, D> ? 128 : 64) * kWavefronts, (kGradientWaves<E, D>)) void
k_attention_dkv(const AttnArgs A, int slots, int order, int run, int main, int q_slots, const E* dout, const float* lse,
                const float* delta, const float* bias_part, E* dk, E* dv, E* dbias) {
    using O = Oper<E>;
    using T = Tile<E, D>;
    constexpr int NB = T::ROWS / 32, DB = D / 32, COLS = 32 * kWavefronts;
    constexpr bool APART = kApart<E, D>;
    constexpr int WAVES = APART ? 2 * kWavefronts : kWavefronts, THREADS = 64 * WAVES;
    const bool keys = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6) >= kWavefronts;        // (APART) this wavefront has the keys' gradient
    __shared__ __align__(256) char lds[2][2 * T::BYTES];
    __shared__ __align__(16) float row_lse[2][T::ROWS], row_delta[2][T::ROWS], row_far[2][2][T::ROWS];
    __shared__ int tile_far[2];                       // some row is far: row_far has log-sum-exps, and what is added to far rows' exponents
    extern __shared__ __align__(16) char dyn[];
    const int tid = threadIdx.x, lane0 = tid & 63, lane = lane0, wave = __builtin_amdgcn_readfirstlane(tid >> 6), h = lane >> 5;
    if constexpr (BIAS) {
        if ((int)blockIdx.x >= main) {                // one entry of the table each wavefront
            const int e = ((int)blockIdx.x - main) * WAVES + wave;
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
    const Work work = work_of(blockIdx.x, slots, (A.kv_heads + run - 1) / run, A.n_seqs, order, false);
    const int slot = work.slot, kv0 = work.inner * run;
    const int kv_end = kv0 + run < A.kv_heads ? kv0 + run : A.kv_heads;
    const int seq = find_sequence(A.koff, A.n_seqs, COLS, A.total_k, slot, lane);
    bool rest;
    const Range ks = rows_of_place(A.koff, seq, A.n_seqs, A.total_k, COLS, slot, rest);
    const Range qs = rest ? Range{0, 0, 0} : sequence_rows(A.qoff, seq, A.total_q);
    const int key0 = (slot - ks.place) * COLS;
    if (key0 < 0 || key0 >= ks.n) return;
    const int wkey = key0 + wave % kWavefronts * 32, key = wkey + (lane & 31), shift = ks.n - qs.n;
    const bool real = key < ks.n;
    const int64_t at = ks.lo + key;
    const bool seen = real && (!MASKED || A.keep[at]);
    const int G = A.pack, cols = qs.n * G;
    // columns from the first row that sees a key of the tile: rows before it may see nothing at all
    const int col0 = A.causal && key0 > shift ? (key0 - shift) * G : 0;

    const int64_t qrow = A.q_row * (int64_t)sizeof(E), qhead = A.q_head * (int64_t)sizeof(E);
    const int64_t grow = (int64_t)A.heads * D * (int64_t)sizeof(E), ghead = D * (int64_t)sizeof(E);
    const char* qp = (const char*)A.q + qs.lo * qrow;
    const char* gp = (const char*)dout + qs.lo * grow;
    Staged<E, D, THREADS, MASKED, T::ROWS> next;
    float n_lse = 0.f, n_delta = 0.f;
    const float unit_scale = unit_of_scores(A.scale), scale2 = unit_scale * LOG2E, per_unit = BIAS ? LOG2E : scale2;
    // 16 bits: a row's log-sum-exp and delta are what its accumulators start from (in 32 bits that would cost the scores an
    // error of some roundings of the log-sum-exp, which 16-bit results do not show: it is at most kFarRow there)
    constexpr bool START = sizeof(E) == 2;
    auto place_of_row = [&](int head0, int c0, int r) {           // of a tile's row among all heads'
        const int row0 = c0 / G, c1 = c0 - row0 * G, row = G == 1 ? r : (int)((uint32_t)(c1 + r) / (uint32_t)G);
        return (int64_t)head0 * A.total_q + qs.lo + row0 + row + (int64_t)(c1 + r - row * G) * A.total_q;
    };
    auto issue = [&](int head0, int c0, char* to) {
        const int row0 = c0 / G, c1 = c0 - row0 * G;              // the tile's first row, and its first column's place in it
        auto row_of = [&](int r) { return G == 1 ? r : (int)((uint32_t)(c1 + r) / (uint32_t)G); };
        auto offset = [&](int r, uint32_t per_row, uint32_t per_head) {
            const int row = row_of(r);
            return G == 1 ? (uint32_t)row * per_row : (uint32_t)row * per_row + (uint32_t)(c1 + r - row * G) * per_head;
        };
        auto place = [&](int r) { return place_of_row(head0, c0, r); };
        next.issue(qp + row0 * qrow + head0 * qhead, gp + row0 * grow + head0 * ghead, to, cols - c0, tid,
                   [&](int r) { return offset(r, (uint32_t)qrow, (uint32_t)qhead); },
                   [&](int r) { return offset(r, (uint32_t)grow, (uint32_t)ghead); },
                   [&](int r) { return (uint8_t)(lse[place(r)] != -INFINITY); });
        if (tid < T::ROWS) {
            n_lse = -INFINITY;
            n_delta = 0.f;
            if (c0 + tid < cols) {
                n_lse = lse[place(tid)];
                n_delta = delta[place(tid)];
            }
        }
    };
    auto finish = [&](int buf, int head0, int c0) {
        next.finish(lds[buf], tid);
        if (tid < T::ROWS) {
            const bool own = is_far(n_lse, scale2), far = __ballot(own) != 0;
            // exp2(x - inf) = 0
            const float add = n_lse == -INFINITY ? -INFINITY : -n_lse * (START ? LOG2E / scale2 : LOG2E);
            if (far) {
                row_far[buf][0][tid] = n_lse == -INFINITY ? INFINITY : n_lse;
                row_far[buf][1][tid] = own ? delta[(int64_t)A.heads * A.total_q + place_of_row(head0, c0, tid)] : 0.f;
            }
            row_lse[buf][tid] = far ? 0.f : add;
            row_delta[buf][tid] = -n_delta;
            if (tid == 0) tile_far[buf] = far;
        }
    };
    int head0 = kv0 * A.group, c0 = col0;
    const int head_end = kv_end * A.group;
    const bool any = col0 < cols;
    if (any) issue(head0, c0, lds[0]);
    Column<E, D> k, v;
    auto load_keys = [&](int kv) {
        k.load((const E*)A.k + at * A.k_row + kv * A.k_head, seen, h);
        k.take_sign(A.scale);
        if (!APART || keys) v.load((const E*)A.v + at * A.v_row + kv * A.v_head, seen, h);
    };
    load_keys(kv0);
    f32x16 acc[DB] = {}, acc2[APART ? 1 : DB] = {};              // of keys and of values, or of the wavefront's own
    const int middle = bias_middle(A.reach);
    const bool busy = wkey < ks.n;
    const int wfirst = A.causal && wkey > shift ? (wkey - shift) * G : 0;             // first column that sees a key of the wavefront
    int16_t* starts = (int16_t*)dyn;
    float* table = (float*)(dyn + kStartsBytes);
    if constexpr (BIAS) {
        load_starts(A, starts, tid, THREADS);
        __syncthreads();
        fill_bias<E>(A, head0, starts, table, tid, THREADS);
    }
    if (any) finish(0, head0, c0);
    __syncthreads();
    const typename T::At at_tiles(lds[0], lane);
    int buf = 0;
    while (true) {
        const int far_now = tile_far[buf];
        const bool last_tile = c0 + T::ROWS >= cols;
        const int n_head = last_tile ? head0 + G : head0, n_c = last_tile ? col0 : c0 + T::ROWS;
        const bool last = last_tile && n_head % A.group == 0;                           // of a key head
        const bool more = kRuns<D> ? n_head < head_end : !last;
        if (more && any) issue(n_head, n_c, lds[buf ^ 1]);
        const typename T::At lq = at_tiles + buf * 2 * T::BYTES, lg = lq + T::BYTES;
        if (any && busy && c0 + T::ROWS > wfirst) {
            const bool diagonal = A.causal && (wkey + 31 - shift) * G > c0;
            const typename T::At own = APART && !keys ? lg : lq;           // (own gradient's other operand)
#pragma unroll 1
            for (int b = 0; b < NB && c0 + 32 * b < cols; ++b) {
                f32x16 s = {}, dp = {};
                const bool far = __builtin_amdgcn_readfirstlane(far_now) != 0;
                if constexpr (START) s = of_rows(row_lse[buf], b, h);
#pragma unroll
                for (int c = 0; c < D / 16; ++c) O::template mma<true>(s, T::rows(lq, b, c), k.v[c]);
                phase();
                if (!APART || keys) {
                    if constexpr (START) dp = of_rows(row_delta[buf], b, h);
#pragma unroll
                    for (int c = 0; c < D / 16; ++c) O::mma(dp, T::rows(lg, b, c), v.v[c]);
                    phase();
                }
                if constexpr (!START) dp += of_rows(row_delta[buf], b, h);
                if constexpr (BIAS) {
                    const int d0 = wkey - (c0 + 32 * b + shift), side = block_side(d0, A.reach);
                    if (!side) {
                        const float* x = table + middle + key - (c0 + 32 * b + shift) - 4 * h - 27;    // of the lane's last row
#pragma unroll
                        for (int r = 0; r < 16; ++r) s[r] = fmaf(s[r], unit_scale, x[27 - 8 * (r >> 2) - (r & 3)]);
                    } else {
                        const float x = table[side < 0 ? 0 : 2 * middle];
#pragma unroll
                        for (int r = 0; r < 16; ++r) s[r] = fmaf(s[r], unit_scale, x);
                    }
                }
                if (far) {
                    const f32x16 from = of_rows(row_far[buf][0], b, h), x = of_rows(row_far[buf][1], b, h);
#pragma unroll
                    for (int r = 0; r < 16; ++r) s[r] = fmaf((BIAS ? s[r] : rounded_product(s[r], unit_scale)) - from[r], LOG2E, x[r]);
                } else if constexpr (START) {
                    s *= per_unit;
                } else {
                    const f32x16 x = of_rows(row_lse[buf], b, h);
#pragma unroll
                    for (int r = 0; r < 16; ++r) s[r] = fmaf(s[r], per_unit, x[r]);
                }
                if (diagonal) {                       // a lane's key is seen by columns from (key - shift) G on
                    const uint32_t own = ~bits_up_to((key - shift) * G - c0 - 32 * b - 4 * h - 1);
#pragma unroll
                    for (int r = 0; r < 16; ++r) s[r] = hidden_unless(s[r], all_if(own, r));
                }
#pragma unroll
                for (int r = 0; r < 16; ++r) s[r] = exp2_fast(s[r]);
                if constexpr (!APART) {
                    const typename O::Frag p0 = O::round(eight<0>(s)), p1 = O::round(eight<8>(s));
                    phase();
#pragma unroll
                    for (int db = 0; db < DB; ++db) O::mma(acc2[db], T::turned(lg, b, 0, db), p0);
#pragma unroll
                    for (int db = 0; db < DB; ++db) O::mma(acc2[db], T::turned(lg, b, 1, db), p1);
                    phase();
                }
                if (!APART || keys) s *= dp;
                const typename O::Frag p0 = O::round(eight<0>(s)), p1 = O::round(eight<8>(s));
                phase();
#pragma unroll
                for (int db = 0; db < DB; ++db) O::mma(acc[db], T::turned(own, b, 0, db), p0);
#pragma unroll
                for (int db = 0; db < DB; ++db) O::mma(acc[db], T::turned(own, b, 1, db), p1);
            }
        }
        if (last) {
            const int kv = head0 / A.group;
            if (kRuns<D> && more) load_keys(kv + 1);
            if (real) {
                const int64_t dense = (at * A.kv_heads + kv) * D;
                auto store = [&](E* to, const f32x16(&a)[DB], float by) {
#pragma unroll
                    for (int db = 0; db < DB; ++db)
#pragma unroll
                        for (int j = 0; j < 4; ++j) {
                            const f32x4 x = {a[db][4 * j] * by, a[db][4 * j + 1] * by, a[db][4 * j + 2] * by, a[db][4 * j + 3] * by};
                            O::store4(to + dense + 32 * db + 8 * j + 4 * h, seen ? x : f32x4{0.f, 0.f, 0.f, 0.f});
                        }
                };
                if constexpr (!APART) {
                    store(dk, acc, A.scale);
                    store(dv, acc2, 1.f);
                } else {
                    store(keys ? dk : dv, acc, keys ? A.scale : 1.f);
                }
            }
            if (!more) return;
#pragma unroll
            for (int db = 0; db < DB; ++db) {
                acc[db] = {};
                if constexpr (!APART) acc2[db] = {};
            }
        }
        if (more && any) finish(buf ^ 1, n_head, n_c);
        __syncthreads();
        if (BIAS && n_head != head0) {
            fill_bias<E>(A, n_head, starts, table, tid, THREADS);
            __syncthreads();
        }
        head0 = n_head;
        c0 = n_c;
        buf ^= 1;
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
template <class F> hipError_t by_form(bool bias, bool masked, F&& f) {
    if (bias) return masked ? f(std::true_type{}, std::true_type{}) : f(std::true_type{}, std::false_type{});
    return masked ? f(std::false_type{}, std::true_type{}) : f(std::false_type{}, std::false_type{});
}

template <class E>
hipError_t launch_attention(const AttnArgs& A, const AttnPlan& P, E* out, float* lse, char* ws, hipStream_t st) {
    if (A.total_q == 0) return hipSuccess;
    return by_width(P.d, [&](auto dc) {
        constexpr int D = decltype(dc)::value;
        float* o_part = (float*)(ws + P.o_part);
        float2* ml_part = (float2*)(ws + P.ml_part);
        const hipError_t e = by_form(A.bias != nullptr, A.keep != nullptr, [&](auto bias, auto masked) {
            constexpr bool BIAS = decltype(bias)::value, MASKED = decltype(masked)::value;
            const size_t lds = BIAS ? bias_bytes(A.reach, 1) : 0;
            const int64_t runs = (P.units + P.run - 1) / P.run;
            k_attention<E, D, BIAS, MASKED><<<dim3((unsigned)(P.q_slots * runs * P.splits)), 64 * kWavefronts, lds, st>>>(
                A, (int)P.q_slots, P.q_order, P.units, P.run, P.splits, out, lse, o_part, ml_part);
            return hipGetLastError();
        });
        if (e != hipSuccess || P.splits == 1) return e;
        const int64_t rows = (int64_t)A.heads * A.total_q;
        k_attention_join<E, D><<<dim3((unsigned)((rows + 3) / 4)), 256, 0, st>>>(A, P.splits, o_part, ml_part, out, lse);
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
            e = by_form(A.bias != nullptr, A.keep != nullptr, [&](auto bias, auto masked) {
                constexpr bool BIAS = decltype(bias)::value, MASKED = decltype(masked)::value;
                const size_t lds = BIAS ? bias_bytes(A.reach, 1 + P.run * kWavefronts) : 0;
                const int64_t runs = (P.units + P.run - 1) / P.run;
                k_attention_dq<E, D, BIAS, MASKED><<<dim3((unsigned)(P.q_slots * runs)), 64 * kWavefronts, lds, st>>>(
                    A, (int)P.q_slots, P.q_order, P.units, P.run, (const E*)G.out, (const E*)G.dout, G.lse, (E*)G.dq, delta, bias_part);
                return hipGetLastError();
            });
            if (e != hipSuccess) return e;
        }
        const int q_slots = A.total_q > 0 ? (int)P.q_slots : 0;
        return by_form(A.bias != nullptr, A.keep != nullptr, [&](auto bias, auto masked) {
            constexpr bool BIAS = decltype(bias)::value, MASKED = decltype(masked)::value;
            const size_t lds = BIAS ? bias_bytes(A.reach, 1) : 0;
            const int main = A.total_k > 0 ? (int)(P.k_slots * ((A.kv_heads + P.kv_run - 1) / P.kv_run)) : 0;
            constexpr int WAVES = kApart<E, D> ? 2 * kWavefronts : kWavefronts;
            const int more = BIAS ? (A.n_buckets * A.heads + WAVES - 1) / WAVES : 0;
            if (main + more == 0) return hipSuccess;
            k_attention_dkv<E, D, BIAS, MASKED><<<dim3((unsigned)(main + more)), 64 * WAVES, lds, st>>>(
                A, (int)P.k_slots, P.k_order, P.kv_run, main, q_slots, (const E*)G.dout, G.lse, delta, bias_part, (E*)G.dk, (E*)G.dv, (E*)G.dbias);
            return hipGetLastError();
        });
    });
}

}  // namespace cb
