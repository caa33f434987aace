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
        int j = starts[i] + (tid & 7);
        if (behind && j == 0) j = 8;                  // (distance 0 is not behind)
        const int step = behind ? 8 : -8;
        for (float* to = table + middle + (behind ? j : -j); j < end; j += 8, to += step) *to = z;
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
// forward and backward, before later steps: 691 us, as they come 709; 48 pages, where a head's tiles are kept together as they come: 576 and
// 563).
// LONGEST_FIRST: under a causal limit the later rows see more keys (earlier keys are seen by more rows): places go round the
// sequences, each one's longest tiles first (`down`: its last ones), so that short ones are left for the end.  Sequences are taken
// to be of one length; others are only in another order; the last place, which only rows behind the last sequence can have, stays (24
// causal pages, forward and backward, before later steps: 508 us, as they come 585).
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

// Tiles of the keys that a workgroup's rows see: all of them from the first one on or, with a window, those of the first keys
// that all rows see (`first` of them) and then the ones from the first row's first key to the last row's last.  Where they meet they are
// one run.
template <bool WIN, int ROWS> struct KeyTiles {
    int count;
    __device__ __forceinline__ KeyTiles(const AttnArgs&, QueryTile& t, int) : count((t.end + ROWS - 1) / ROWS) {}
    __device__ __forceinline__ int base(int i) const { return i * ROWS; }
};
template <int ROWS> struct KeyTiles<true, ROWS> {
    int count, first, lo;
    __device__ __forceinline__ KeyTiles(const AttnArgs& A, QueryTile& t, int per) {
        const int last = (t.row0 + per < t.Lq ? t.row0 + per : t.Lq) - 1 + t.shift;
        int sinks = A.sinks < t.Lk ? A.sinks : t.Lk;
        if (A.causal && last + 1 < sinks) sinks = last + 1 < 0 ? 0 : last + 1;
        int hi = last + A.after + 1;
        hi = hi < 0 ? 0 : hi > t.Lk ? t.Lk : hi;
        lo = t.row0 + t.shift - A.before;
        lo = lo < 0 ? 0 : lo > hi ? hi : lo;
        first = (sinks + ROWS - 1) / ROWS;
        if (lo < first * ROWS) {
            first = lo = 0;
            hi = hi > sinks ? hi : sinks;
        }
        t.end = hi;
        count = first + (hi - lo + ROWS - 1) / ROWS;
    }
    __device__ __forceinline__ int base(int i) const { return i < first ? i * ROWS : lo + (i - first) * ROWS; }
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

// What a wavefront's columns, and a lane's, see of the keys through a window.  The first keys of a sequence are seen by all rows (under
// a causal limit, by those that are not before them).
__device__ __forceinline__ uint32_t bits_up_to(int room);
struct ColumnWindow {
    int lo, hi, sink;                         // of the lane's column: first and last key, last of the first keys
    int any_lo, any_hi, any_sink;             // of all columns: from the first key of any to the last of any
    int all_lo, all_hi, all_sink;             // from the last one's first key to the first one's last
    __device__ __forceinline__ ColumnWindow(const AttnArgs& A, const QueryTile& t, const QueryColumns& w, int G, int wave) {
        const int first = w.first_lim, last = t.row0 + (wave * 32 + 31) / G + t.shift;
        lo = w.lim - A.before;
        hi = w.lim + A.after;
        any_lo = first - A.before;
        all_lo = last - A.before;
        all_hi = first + A.after;
        any_hi = last + A.after < t.end ? last + A.after : t.end - 1;
        auto limit = [&](int p) { return A.causal && p < A.sinks - 1 ? p : A.sinks - 1; };
        sink = limit(w.lim);
        any_sink = limit(last);
        all_sink = limit(first);
    }
    // whether some column sees some of the n keys from `base` on; whether every one sees all of them
    __device__ __forceinline__ bool some(int base, int n) const { return (base <= any_hi && base + n > any_lo) || base <= any_sink; }
    __device__ __forceinline__ bool every(int base, int n) const { return (base >= all_lo && base + n - 1 <= all_hi) || base + n - 1 <= all_sink; }
    // keys that the column sees, of those that a lane has (from `base` on), as bits
    __device__ __forceinline__ uint32_t bits(int base) const {
        return (bits_up_to(hi - base) & ~bits_up_to(lo - 1 - base)) | bits_up_to(sink - base);
    }
    static __device__ __forceinline__ uint64_t up_to(int room) { return room < 0 ? 0ull : room >= 63 ? ~0ull : (2ull << room) - 1ull; }
    __device__ __forceinline__ uint64_t wide_bits(int base) const {
        return (up_to(hi - base) & ~up_to(lo - 1 - base)) | up_to(sink - base);
    }
};
struct NoWindow {
    __device__ __forceinline__ NoWindow(const AttnArgs&, const QueryTile&, const QueryColumns&, int, int) {}
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

// Products of a block's rows with the wavefront's columns.  The compiler, which would save registers, asks for an operand before its
// product, which then waits for it: a third wavefront on the SIMD goes on meanwhile, a second one often waits as well.  EARLY: operands
// are asked for three products ahead.
template <class T, bool EARLY, bool TURNED = false, int N>
__device__ __forceinline__ void add_rows(f32x16& x, const typename T::At& t, int b, const typename T::Frag (&own)[N]) {
    if constexpr (EARLY) {
        constexpr int AHEAD = 3;
        typename T::Frag f[N];
#pragma unroll
        for (int c = 0; c < AHEAD && c < N; ++c) f[c] = T::rows(t, b, c);
        in_turn();
#pragma unroll
        for (int c = 0; c < N; ++c) {
            T::O::template mma<TURNED>(x, f[c], own[c]);
            if (c + AHEAD < N) f[c + AHEAD] = T::rows(t, b, c + AHEAD);
            in_turn();
        }
    } else {
#pragma unroll
        for (int c = 0; c < N; ++c) T::O::template mma<TURNED>(x, T::rows(t, b, c), own[c]);
    }
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
// d = 128, before copies were a tile ahead: 563 us; with 64 rows the compiler spills, 1,215; the gradients' kernels, which have registers
// for two, lose by 32).
template <class E, int D> constexpr int kForwardRows = D >= 96 ? 32 : Oper<E>::ROWS;
template <int D> constexpr bool kRuns = goes_on_to_next_head(D);

// ---- forward -------------------------------------------------------------------------------------------------
// One pass over the keys with the running maximum and sum of the softmax, in 32 bits; probabilities are rounded to the
// storage type for the second product (their sum is not; outputs in 16 bits are off by 2.3e-3 of their norm, their own rounding
// is 1.7e-3; probabilities in two values would make three products of two).  The maximum that is subtracted may lag by up to kLag: sums and
// outputs are rescaled only when it is passed, which few tiles after the first do; probabilities up to 2^kLag are no less exact
// (48 pages of 1,030 rows, 16 heads of 128 over 8, before copies were a tile ahead: 563 us, without a lag 613).
constexpr float kLag = 8.f;
// A workgroup takes its tile for `run` head units one after the other, the first keys of the next on their way while it
// computes: short sequences have one to three tiles of keys, whose latency would otherwise be most of the time.
// Long sequences are bound by the matrix and vector units' turns (an exponential, a maximum, a sum and half a conversion for every
// score: as many clocks as the products): the pages above 518 to 530 us, 800 TFLOP/s where this library's scoring of all documents
// reaches 1,504.  Short ones by latency and what a workgroup does before its first product: 512 passages, 12 heads of 64 with bias and
// mask, 141 us.  Single tokens by memory: 16 over 1 to 16,385 keys, two key heads of 128, 134 MB in 29 us and 7.5 us to join their
// parts.
// Through a window (WIN) only tiles that some row sees are gone over, and tiles of the first keys; what a row sees of a tile is a bit a key.
// 6 documents of 500 to 8,191 tokens, 12 heads of 64, 64 keys to either side, one first key: 58 us, 10.3 GFLOP of 161 MB (38
// with a window of one key).  A workgroup's 128 rows see 256 keys together and 129 each.  A wavefront's 32 rows see 160, and it passes over
// tiles, and halves of them, that are not among them: it multiplies six and a half blocks of 32 keys, of which 37 % of the scores are hidden,
// and waits at the nine or ten that the others need.  Vector instructions (1,500 of a wavefront) and what comes before the first product
// bound it.  16 single tokens that see 1,028 of up to 16,385 keys: 9 us and 4 us to join.
template <class E, int D, bool BIAS, bool MASKED, bool WIN>
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
    QueryTile t(A, slot, per, lane);
    if (t.none) return;
    const KeyTiles<WIN, T::ROWS> at_key(A, t, per);
    const QueryColumns w(A, t, G, per, wave, lane);
    const std::conditional_t<WIN, ColumnWindow, NoWindow> win(A, t, w, G, wave);
    const int tiles = at_key.count, each = (tiles + splits - 1) / splits;
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
    if (any) issue(unit, at_key.base(first_tile), lds[0]);
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
        settle<E>();
        const int base = at_key.base(i);
        const typename T::At lk = at_tiles + buf * 2 * T::BYTES, lv = lk + T::BYTES;
        const bool last = i + 1 >= end_tile;                     // of the unit
        const int n_unit = last ? unit + 1 : unit, n_i = last ? first_tile : i + 1;
        const bool more = kRuns<D> ? n_unit < end_unit : !last;
        if (more && any) issue(n_unit, at_key.base(n_i), lds[buf ^ 1]);
        bool visit = any && w.busy, one, diagonal;               // one: its second block has no keys
        const bool part = seen != kAllRows;
        if constexpr (WIN) {
            visit = visit && win.some(base, T::ROWS);
            one = NB > 1 && !win.some(base + 32, 32);
            diagonal = false;
        } else {
            visit = visit && base < w.end;
            one = NB > 1 && base + 32 >= w.end;
            diagonal = A.causal && base + T::ROWS - 1 > w.first_lim;
        }
        if (visit) {
            if constexpr (MASKED && WIN) {
                sees |= (seen & win.wide_bits(base)) != 0;
            } else if constexpr (MASKED) {
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
                if constexpr (WIN) diagonal = !win.every(base + 32 * b, 32);
                if (diagonal) {
                    uint32_t own;
                    if constexpr (WIN) own = win.bits(base + 32 * b + 4 * h);
                    else own = bits_up_to(w.lim - base - 32 * b - 4 * h);
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
// It costs the 512 passages 22 us of 659, with 64 keys 2 us, which leaves 2.1e-3 for sequences of up to 131 tokens).
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
// Bound by the matrix and vector units' turns where sequences are long (24 causal pages, 8 heads of 128 over 2: 169 and 190 us, 510
// TFLOP/s of the three and four products that each cannot do without), by latency and by what surrounds the products where they are
// short (the 512 passages: 286 and 262 us).  8 documents of up to 4,095 tokens through a window of 256 rows and four first keys, 8 heads
// of 128 over 2: forward 51 us, queries 82, keys and values 127, 6.5 to join the first keys'.

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
template <class E, int D, bool BIAS, bool MASKED, bool WIN>
__global__ __launch_bounds__(64 * kWavefronts, (kQueryWaves<E, D>)) void
k_attention_dq(const AttnArgs A, int slots, int order, int units, int run, const E* out, const E* dout, const float* lse, E* dq,
               float* delta, float* bias_part) {
    using O = Oper<E>;
    using T = Tile<E, D>;
    constexpr bool EARLY = sizeof(E) == 2 && kQueryWaves<E, D> < 3;
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
    QueryTile t(A, slot, per, lane);
    if (t.none) {
        if constexpr (BIAS)
            for (int b = tid; b < (end_unit - unit) * A.n_buckets; b += THREADS)
                bias_part[((int64_t)slot * A.heads + unit) * A.n_buckets + b] = 0.f;
        return;
    }
    const KeyTiles<WIN, T::ROWS> at_key(A, t, per);
    const QueryColumns w(A, t, G, per, wave, lane);
    const std::conditional_t<WIN, ColumnWindow, NoWindow> win(A, t, w, G, wave);
    const int tiles = at_key.count;
    const bool few = sizeof(E) == 2 && (WIN ? tiles * T::ROWS <= kTwice || A.before + A.after + A.sinks < kTwice : t.end <= kTwice);
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
    if (any) issue(unit, at_key.base(0), lds[0]);
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
        settle<E>();
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
        const int base = at_key.base(i < tiles ? i : i - tiles);
        const typename T::At lk = at_tiles + buf * 2 * T::BYTES, lv = lk + T::BYTES;
        const bool last = i + 1 >= (twice ? 2 * tiles : tiles);
        const int n_unit = last ? unit + 1 : unit, n_i = last ? 0 : i + 1;
        const bool more = kRuns<D> ? n_unit < end_unit : !last;
        if (more && any) issue(n_unit, at_key.base(n_i < tiles ? n_i : n_i - tiles), lds[buf ^ 1]);
        bool visit = any && w.busy, diagonal;
        const bool part = seen != kAllRows;
        if constexpr (WIN) {
            visit = visit && win.some(base, T::ROWS);
            diagonal = false;
        } else {
            visit = visit && base < w.end;
            diagonal = A.causal && base + T::ROWS - 1 > w.first_lim;
        }
        if (visit) {
#pragma unroll 1
            for (int b = 0; b < NB && (WIN || base + 32 * b < w.end); ++b) {
                if constexpr (WIN)
                    if (!win.some(base + 32 * b, 32)) continue;
                if constexpr (WIN) diagonal = !win.every(base + 32 * b, 32);
                f32x16 s = {}, dp;
                add_rows<T, EARLY>(s, lk, b, q.v);
                phase();
#pragma unroll
                for (int r = 0; r < 16; ++r) dp[r] = -dot;
                add_rows<T, EARLY>(dp, lv, b, g.v);
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
                    uint32_t own;
                    if constexpr (WIN) own = win.bits(base + 32 * b + 4 * h);
                    else own = bits_up_to(w.lim - base - 32 * b - 4 * h);
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
                        if constexpr (EARLY) {
                            typename O::Frag f[DB];
#pragma unroll
                            for (int db = 0; db < DB; ++db) f[db] = T::turned(lk, b, c, db);
                            in_turn();
#pragma unroll
                            for (int db = 0; db < DB; ++db) O::mma(acc[db], f[db], rest);
#pragma unroll
                            for (int db = 0; db < DB; ++db) O::mma(acc[db], f[db], p);
                        } else {
#pragma unroll
                            for (int db = 0; db < DB; ++db) {
                                const typename O::Frag x = T::turned(lk, b, c, db);
                                O::mma(acc[db], x, rest);
                                O::mma(acc[db], x, p);
                            }
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

// Where a sequence's chunk of A.sink_rows rows leaves its shares.  Sequences of more than one chunk begin further apart than a chunk is
// long, so that their first chunks have places of their own, and so have the others, which begin after them.
__device__ __forceinline__ int64_t sink_place(const Range& rows, int chunk, int per) { return 2 * (int64_t)(rows.lo / per + chunk) + (chunk == 0); }

// Gradients of keys and values, `run` key heads one after the other; workgroups from `main` on add up the bias table's shares
// of all tiles.
// A wavefront with both gradients of 32 wide rows takes more than half of the registers, so nothing runs beside its waits.
// In 16 bits wide heads have two wavefronts for the same rows, one for either gradient, so that two share a SIMD (24 causal pages,
// forward and backward: 508 us, with one 828).  The values' one makes the probabilities and hands them over in LDS, in 32 bits; the
// keys' one is a block of 32 rows behind, which costs a barrier a block and a third tile in LDS (500 us where both make the scores and
// take their exponentials; so 476, and 456 with operands asked for ahead).
// Through a window such a workgroup has 64 key rows instead of 128, and tiles of 32 rows: two share a CU, and fewer rows that see only
// some of its keys are gone over (26 pages of 1,030 tokens, 6 heads of 128, 64 to either side, with gradients: 258 and 241 us; without
// a window, where each goes over all rows, 24 causal pages 456 and 468, of heads of 96 with a bias 705 and 753).
template <class E, int D> constexpr bool kApart = two_for_keys(D, sizeof(E));
template <class E, int D, bool WIN> constexpr int kKeyWaves = kApart<E, D> && !WIN ? 2 * kWavefronts : kWavefronts;
// Rows (of all heads that share a key head) that a 32-bit sum through a window takes before it is added to the result.  (11 documents of
// 1,030 tokens, seven fp32 heads of 64 to a key head, a window of 719 rows: keys' and values' gradients are 7.3e-7 of their norm off, 1.3e-6
// in one sum, plain 32-bit products 7.3e-7; 1,037 us, in one sum 1,055.  Heads of 128, four to a key head: 967 and 900.)
constexpr int kMostSum = 1024;
// With a window the first keys are left to workgroups of their own (the first `sink_groups` ones), since all of a sequence's rows see
// them: a key tile's others see some rows only.  Such a workgroup takes A.sink_rows rows of a sequence, and, where the sequence has
// more, leaves its shares of the first keys' gradients to k_attention_join_sinks.  They come first: the others, which are all of about
// one length, then do not begin at the same time, nor end so.
template <class E, int D, bool BIAS, bool MASKED, bool WIN>
__global__ __launch_bounds__(64 * (kKeyWaves<E, D, WIN>), (kGradientWaves<E, D>)) void
k_attention_dkv(const AttnArgs A, int slots, int order, int run, int main, int sink_groups, int q_slots, const E* dout, const float* lse,
                const float* delta, const float* bias_part, E* dk, E* dv, E* dbias, float* sink_part) {
    using O = Oper<E>;
    constexpr bool APART = kApart<E, D>;
    using T = Tile<E, D, APART && WIN ? 32 : Oper<E>::ROWS>;
    constexpr int WAVES = kKeyWaves<E, D, WIN>, GROUPS = APART ? WAVES / 2 : WAVES;      // of 32 key rows
    constexpr int NB = T::ROWS / 32, DB = D / 32, COLS = 32 * GROUPS, THREADS = 64 * WAVES;
    constexpr int BUFS = APART ? 3 : 2;               // tiles in LDS
    // (APART) This wavefront has the keys' gradient.  Of two workgroups on a CU (with a window; the second ones are about 256 on) one has its
    // values' wavefronts, with the exponentials, on the SIMDs where the other has its keys' (8 documents of up to 4,095 tokens, a window
    // of 256 rows and four first keys, with gradients: 269 us, so 261).
    const bool keys = (__builtin_amdgcn_readfirstlane(threadIdx.x >> 6) >= GROUPS) != (WIN && (blockIdx.x >> 8 & 1));
    __shared__ __align__(256) char lds[BUFS][2 * T::BYTES];
    __shared__ __align__(16) float row_lse[BUFS][T::ROWS], row_delta[BUFS][T::ROWS], row_far[BUFS][2][T::ROWS];
    __shared__ int tile_far[BUFS];                    // some row is far: row_far has log-sum-exps, and what is added to far rows' exponents
    __shared__ f32x4 handed[APART ? 2 : 1][APART ? GROUPS : 1][4][64];      // (APART) a block's probabilities
    extern __shared__ __align__(16) char dyn[];
    const int tid = threadIdx.x, lane0 = tid & 63, lane = lane0, wave = __builtin_amdgcn_readfirstlane(tid >> 6), h = lane >> 5;
    if constexpr (BIAS) {
        if ((int)blockIdx.x >= main + (WIN ? sink_groups : 0)) {      // one entry of the table each wavefront
            const int e = ((int)blockIdx.x - main - (WIN ? sink_groups : 0)) * WAVES + wave;
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
    const bool sinks = WIN && (int)blockIdx.x < sink_groups;
    int slot, kv0, kv_end, seq, key0;
    bool rest = false;
    Range ks, qs;
    if (!sinks) {
        const Work work = work_of((int)blockIdx.x - (WIN ? sink_groups : 0), slots, (A.kv_heads + run - 1) / run, A.n_seqs, order, false);
        slot = work.slot;
        kv0 = work.inner * run;
        kv_end = kv0 + run < A.kv_heads ? kv0 + run : A.kv_heads;
        seq = find_sequence(A.koff, A.n_seqs, COLS, A.total_k, slot, lane);
        ks = rows_of_place(A.koff, seq, A.n_seqs, A.total_k, COLS, slot, rest);
        qs = rest ? Range{0, 0, 0} : sequence_rows(A.qoff, seq, A.total_q);
        key0 = (slot - ks.place) * COLS;
        if (key0 < 0 || key0 >= ks.n) return;
    } else {
        const int x = (int)blockIdx.x, inner = A.kv_heads * ((A.sinks + COLS - 1) / COLS);
        slot = x / inner;
        kv0 = x % inner % A.kv_heads;
        kv_end = kv0 + 1;
        key0 = x % inner / A.kv_heads * COLS;
        seq = find_sequence(A.qoff, A.n_seqs, A.sink_rows, A.total_q, slot, lane);
        qs = rows_of_place(A.qoff, seq, A.n_seqs, A.total_q, A.sink_rows, slot, rest);
        if (rest) return;
        ks = sequence_rows(A.koff, seq, A.total_k);
    }
    const int wkey = key0 + wave % GROUPS * 32, key = wkey + (lane & 31), shift = ks.n - qs.n;
    const int G = A.pack;
    int key_from = 0, key_to = ks.n;                              // keys that are this workgroup's
    int cols = qs.n * G;
    // columns from the first row that sees a key of the tile: rows before it may see nothing at all
    int col0 = A.causal && key0 > shift ? (key0 - shift) * G : 0;
    int wfirst = A.causal && wkey > shift ? (wkey - shift) * G : 0;             // first column that sees a key of the wavefront
    int wend = cols, see_from = 0, see_to = 0, all_from = 0, all_to = 0;        // (WIN) columns that see the lane's key; all of the wavefront's
    if constexpr (WIN) {
        auto row = [&](int r) { return r < 0 ? 0 : r > qs.n ? qs.n : r; };      // ends of ranges of rows
        if (sinks) {
            const int begin = (slot - qs.place) * A.sink_rows, end = row(begin + A.sink_rows);
            key_to = A.sinks < ks.n ? A.sinks : ks.n;
            if (begin < 0 || begin >= qs.n || key0 >= key_to) return;
            const int from = A.causal ? row(key0 - shift) : 0;
            col0 = (from > begin ? from : begin) * G;
            cols = wend = end * G;
            see_from = A.causal ? row(key - shift) * G : 0;
            see_to = cols;
            all_from = A.causal ? row(wkey + 31 - shift) * G : 0;
            all_to = cols;
        } else {
            key_from = rest ? 0 : A.sinks;
            if (key0 + COLS <= key_from) return;
            const int last = key0 + COLS < ks.n ? key0 + COLS : ks.n, wlast = wkey + 32 < ks.n ? wkey + 32 : ks.n;
            col0 = row((key0 > key_from ? key0 : key_from) - A.after - shift) * G;
            cols = row(last + A.before - shift) * G;
            wfirst = row((wkey > key_from ? wkey : key_from) - A.after - shift) * G;
            wend = row(wlast + A.before - shift) * G;
            see_from = row(key - A.after - shift) * G;
            see_to = row(key + 1 + A.before - shift) * G;
            all_from = row(wkey + 31 - A.after - shift) * G;
            all_to = row(wkey + 1 + A.before - shift) * G;
        }
    }
    const bool real = key < key_to && key >= key_from;
    const int64_t at = ks.lo + key;
    const bool seen = real && (!MASKED || A.keep[at]);

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
    // A tile's first row, and its first column's place in it; what a tile adds to them.  Divisions by the number of heads that share a
    // tile, at most 16, are products (of fewer than 2^8 columns, exact): they were a quarter of the vector instructions.
    struct Place { int row, c; };
    const Place step = {T::ROWS / G, T::ROWS % G}, first_place = {col0 / G, 0};
    const uint32_t inverse = (65536u + (uint32_t)G - 1u) / (uint32_t)G;
    auto row_of = [&](int x) { return G == 1 ? x : (int)((uint32_t)x * inverse >> 16); };
    auto place_of_row = [&](int head0, const Place& p, int r) {   // of a tile's row among all heads'
        const int row = row_of(p.c + r);
        return (int64_t)head0 * A.total_q + qs.lo + p.row + row + (int64_t)(p.c + r - row * G) * A.total_q;
    };
    auto issue = [&](int head0, int c0, const Place& p, char* to) {
        auto offset = [&](int r, uint32_t per_row, uint32_t per_head) {
            const int row = row_of(p.c + r);
            return G == 1 ? (uint32_t)row * per_row : (uint32_t)row * per_row + (uint32_t)(p.c + r - row * G) * per_head;
        };
        auto place = [&](int r) { return place_of_row(head0, p, r); };
        next.issue(qp + p.row * qrow + head0 * qhead, gp + p.row * grow + head0 * ghead, to, cols - c0, tid,
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
    auto finish = [&](int buf, int head0, const Place& p) {
        next.finish(lds[buf], tid);
        if (tid < T::ROWS) {
            const bool own = is_far(n_lse, scale2), far = __ballot(own) != 0;
            // exp2(x - inf) = 0
            const float add = n_lse == -INFINITY ? -INFINITY : -n_lse * (START ? LOG2E / scale2 : LOG2E);
            if (far) {
                row_far[buf][0][tid] = n_lse == -INFINITY ? INFINITY : n_lse;
                row_far[buf][1][tid] = own ? delta[(int64_t)A.heads * A.total_q + place_of_row(head0, p, tid)] : 0.f;
            }
            row_lse[buf][tid] = far ? 0.f : add;
            row_delta[buf][tid] = -n_delta;
            if (tid == 0) tile_far[buf] = far;
        }
    };
    int head0 = kv0 * A.group, c0 = col0;
    Place at_c0 = first_place;
    const int head_end = kv_end * A.group;
    const bool any = col0 < cols;
    if (any) issue(head0, c0, at_c0, lds[0]);
    Column<E, D> k, v;                                // (APART) k: the wavefront's own, of keys or of values
    auto load_keys = [&](int kv) {
        if (APART && keys) {
            k.load((const E*)A.v + at * A.v_row + kv * A.v_head, seen, h);
        } else {
            k.load((const E*)A.k + at * A.k_row + kv * A.k_head, seen, h);
            k.take_sign(A.scale);
        }
        if constexpr (!APART) v.load((const E*)A.v + at * A.v_row + kv * A.v_head, seen, h);
    };
    load_keys(kv0);
    f32x16 acc[DB] = {}, acc2[APART ? 1 : DB] = {};              // of keys and of values, or of the wavefront's own
    int summed = 0;                                   // tiles since they were last added to the result, which holds some: again
    bool again = false;
    const int middle = bias_middle(A.reach);
    const bool busy = wkey < key_to && wkey + 32 > key_from;
    int16_t* starts = (int16_t*)dyn;
    float* table = (float*)(dyn + kStartsBytes);
    if constexpr (BIAS) {
        load_starts(A, starts, tid, THREADS);
        __syncthreads();
        fill_bias<E>(A, head0, starts, table, tid, THREADS);
    }
    if (any) finish(0, head0, at_c0);
    __syncthreads();
    const typename T::At at_tiles(lds[0], lane);
    // Of block b of the tile in `buf`, whose rows are the columns from c0 on: scores' probabilities,
    auto exponentials = [&](f32x16& s, int buf, int b, bool far, bool diagonal) {
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
        if (diagonal) {                               // a lane's key is seen by columns from (key - shift) G on
            uint32_t own;
            if constexpr (WIN) {
                const int from = c0 + 32 * b + 4 * h;
                own = bits_up_to(see_to - 1 - from) & ~bits_up_to(see_from - 1 - from);
            } else {
                own = ~bits_up_to((key - shift) * G - c0 - 32 * b - 4 * h - 1);
            }
#pragma unroll
            for (int r = 0; r < 16; ++r) s[r] = hidden_unless(s[r], all_if(own, r));
        }
#pragma unroll
        for (int r = 0; r < 16; ++r) s[r] = exp2_fast(s[r]);
    };
    // and what the block adds to a gradient.
    auto add_up = [&](f32x16(&to)[DB], const typename T::At& t, int b, const f32x16& x) {
        const typename O::Frag p0 = O::round(eight<0>(x)), p1 = O::round(eight<8>(x));
        phase();
#pragma unroll
        for (int db = 0; db < DB; ++db) O::mma(to[db], T::turned(t, b, 0, db), p0);
#pragma unroll
        for (int db = 0; db < DB; ++db) O::mma(to[db], T::turned(t, b, 1, db), p1);
    };
    // (APART) The keys' wavefronts are a block behind, whose probabilities have been handed over; held: its tile's buffer and its number,
    // or none that the wavefront's keys are seen by.
    int held = -1, turn = 0;
    int buf = 0;
    while (true) {
        settle<E>();
        const bool last_tile = c0 + T::ROWS >= cols;
        const int n_head = last_tile ? head0 + G : head0, n_c = last_tile ? col0 : c0 + T::ROWS, n_buf = buf + 1 < BUFS ? buf + 1 : 0;
        Place n_place = {at_c0.row + step.row, at_c0.c + step.c};
        if (n_place.c >= G) n_place = {n_place.row + 1, n_place.c - G};
        if (last_tile) n_place = first_place;
        const bool last = last_tile && n_head % A.group == 0;                           // of a key head
        const bool more = kRuns<D> ? n_head < head_end : !last;
        if (more && any) issue(n_head, n_c, n_place, lds[n_buf]);
        const typename T::At lq = at_tiles + buf * 2 * T::BYTES, lg = lq + T::BYTES;
        const bool seen_by = busy && c0 + T::ROWS > wfirst && (!WIN || c0 < wend);      // some of the wavefront's keys, by some of the rows
        if (any && (APART || seen_by)) {
            bool diagonal;
            if constexpr (!WIN) diagonal = A.causal && (wkey + 31 - shift) * G > c0;
            const int blocks = WIN && !APART ? (wend - c0 + 31) / 32 : (cols - c0 + 31) / 32, all = blocks < NB ? blocks : NB;
#pragma unroll 1
            for (int b = 0; b < all + (APART && last); ++b) {
                const bool on = !WIN || (c0 + 32 * b + 32 > wfirst && c0 + 32 * b < wend);
                if constexpr (WIN) diagonal = c0 + 32 * b < all_from || c0 + 32 * b + 32 > all_to;
                if constexpr (!APART) {
                    if (!on) continue;
                    f32x16 s = {}, dp = {};
                    const bool far = __builtin_amdgcn_readfirstlane(tile_far[buf]) != 0;
                    if constexpr (START) s = of_rows(row_lse[buf], b, h);
                    add_rows<T, false, true>(s, lq, b, k.v);
                    phase();
                    if constexpr (START) dp = of_rows(row_delta[buf], b, h);
                    add_rows<T, false>(dp, lg, b, v.v);
                    phase();
                    if constexpr (!START) dp += of_rows(row_delta[buf], b, h);
                    exponentials(s, buf, b, far, diagonal);
                    add_up(acc2, lg, b, s);
                    phase();
                    s *= dp;
                    add_up(acc, lq, b, s);
                } else {
                    if (b) __syncthreads();
                    const int now = b < all && seen_by && on ? buf * NB + b : -1, own = keys ? held : now;
                    if (own >= 0) {
                        const int of = own / NB, block = own % NB;
                        const typename T::At scored = at_tiles + (2 * of + keys) * T::BYTES, added = at_tiles + (2 * of + !keys) * T::BYTES;
                        const bool far = __builtin_amdgcn_readfirstlane(tile_far[buf]) != 0;
                        f32x16 x = of_rows(keys ? row_delta[of] : row_lse[of], block, h);
                        add_rows<T, true>(x, scored, block, k.v);
                        phase();
                        typename O::Frag f[2][DB];
#pragma unroll
                        for (int db = 0; db < DB; ++db) f[0][db] = T::turned(added, block, 0, db);
                        phase();
                        if (keys) {
#pragma unroll
                            for (int j = 0; j < 4; ++j) {
                                const f32x4 p = handed[turn ^ 1][wave % GROUPS][j][lane0];
#pragma unroll
                                for (int i = 0; i < 4; ++i) x[4 * j + i] *= p[i];
                            }
                        } else {
                            exponentials(x, buf, b, far, diagonal);
#pragma unroll
                            for (int j = 0; j < 4; ++j) handed[turn][wave % GROUPS][j][lane0] = f32x4{x[4 * j], x[4 * j + 1], x[4 * j + 2], x[4 * j + 3]};
                        }
                        const typename O::Frag p0 = O::round(eight<0>(x)), p1 = O::round(eight<8>(x));
#pragma unroll
                        for (int db = 0; db < DB; ++db) f[1][db] = T::turned(added, block, 1, db);
                        phase();
#pragma unroll
                        for (int db = 0; db < DB; ++db) O::mma(acc[db], f[0][db], p0);
#pragma unroll
                        for (int db = 0; db < DB; ++db) O::mma(acc[db], f[1][db], p1);
                    }
                    held = now;
                    turn ^= 1;
                }
            }
        }
        // fp32 through a window: all heads' rows of a wide window are one sum, whose rounding with each of six products of pieces shows, so
        // every kMostSum rows it is added to what the result holds
        constexpr bool PARTS = WIN && sizeof(E) == 4;
        const bool part = PARTS && !last && any && ++summed == kMostSum / T::ROWS;
        if (last || part) {
            const int kv = head0 / A.group;
            if (kRuns<D> && more && last) load_keys(kv + 1);
            if (real) {
                const int64_t dense = (at * A.kv_heads + kv) * D;
                auto store = [&](E* to, const f32x16(&a)[DB], float by) {
#pragma unroll
                    for (int db = 0; db < DB; ++db)
#pragma unroll
                        for (int j = 0; j < 4; ++j) {
                            f32x4 x = {a[db][4 * j] * by, a[db][4 * j + 1] * by, a[db][4 * j + 2] * by, a[db][4 * j + 3] * by};
                            E* at = to + dense + 32 * db + 8 * j + 4 * h;
                            if constexpr (PARTS)
                                if (again) x += *(const f32x4*)at;
                            O::store4(at, seen ? x : f32x4{0.f, 0.f, 0.f, 0.f});
                        }
                };
                if (WIN && sinks && qs.n > A.sink_rows) {
                    float* to = sink_part + ((sink_place(qs, slot - qs.place, A.sink_rows) * A.kv_heads + kv) * A.sinks + key) * 2 * D;
                    auto leave = [&](int which, const f32x16(&a)[DB], float by) {
#pragma unroll
                        for (int db = 0; db < DB; ++db)
#pragma unroll
                            for (int j = 0; j < 4; ++j) {
                                f32x4 x = {a[db][4 * j] * by, a[db][4 * j + 1] * by, a[db][4 * j + 2] * by, a[db][4 * j + 3] * by};
                                float* at = to + which * D + 32 * db + 8 * j + 4 * h;
                                if constexpr (PARTS)
                                    if (again) x += *(const f32x4*)at;
                                *(f32x4*)at = seen ? x : f32x4{0.f, 0.f, 0.f, 0.f};
                            }
                    };
                    if constexpr (!APART) {
                        leave(0, acc, A.scale);
                        leave(1, acc2, 1.f);
                    } else {
                        leave(keys ? 0 : 1, acc, keys ? A.scale : 1.f);
                    }
                } else if constexpr (!APART) {
                    store(dk, acc, A.scale);
                    store(dv, acc2, 1.f);
                } else {
                    store(keys ? dk : dv, acc, keys ? A.scale : 1.f);
                }
            }
            if (last && !more) return;
            again = part;
            summed = 0;
#pragma unroll
            for (int db = 0; db < DB; ++db) {
                acc[db] = {};
                if constexpr (!APART) acc2[db] = {};
            }
        }
        if (more && any) finish(n_buf, n_head, n_place);
        __syncthreads();
        if (BIAS && n_head != head0) {
            fill_bias<E>(A, n_head, starts, table, tid, THREADS);
            __syncthreads();
        }
        head0 = n_head;
        c0 = n_c;
        at_c0 = n_place;
        buf = n_buf;
    }
}

// Adds up the shares of the first keys' gradients, in the order of the rows: a wavefront for each of them and key head.  Of sequences
// without rows they are zeros.
template <class E, int D>
__global__ __launch_bounds__(256) void k_attention_join_sinks(const AttnArgs A, const float* part, E* dk, E* dv) {
    const int lane = threadIdx.x & 63;
    const int64_t place = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
    const int64_t of = place / A.sinks;
    const int key = (int)(place - of * A.sinks), seq = (int)(of / A.kv_heads), kv = (int)(of % A.kv_heads);
    if (seq >= A.n_seqs || lane >= D / 2) return;
    const Range ks = sequence_rows(A.koff, seq, A.total_k), qs = sequence_rows(A.qoff, seq, A.total_q, A.sink_rows);
    if (key >= ks.n) return;
    const int parts = (qs.n + A.sink_rows - 1) / A.sink_rows;
    if (parts == 1) return;                          // written as they are
    f32x4 sum = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 8
    for (int p = 0; p < parts; ++p)
        sum += *(const f32x4*)(part + ((sink_place(qs, p, A.sink_rows) * A.kv_heads + kv) * A.sinks + key) * 2 * D + 4 * lane);
    E* to = lane < D / 4 ? dk : dv;
    Oper<E>::store4(to + ((int64_t)(ks.lo + key) * A.kv_heads + kv) * D + 4 * (lane % (D / 4)), sum);
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

template <class E, bool WIN>
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
            k_attention<E, D, BIAS, MASKED, WIN><<<dim3((unsigned)(P.q_slots * runs * P.splits)), 64 * kWavefronts, lds, st>>>(
                A, (int)P.q_slots, P.q_order, P.units, P.run, P.splits, out, lse, o_part, ml_part);
            return hipGetLastError();
        });
        if (e != hipSuccess || P.splits == 1) return e;
        const int64_t rows = (int64_t)A.heads * A.total_q;
        k_attention_join<E, D><<<dim3((unsigned)((rows + 3) / 4)), 256, 0, st>>>(A, P.splits, o_part, ml_part, out, lse);
        return hipGetLastError();
    });
}

template <class E, bool WIN>
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
                k_attention_dq<E, D, BIAS, MASKED, WIN><<<dim3((unsigned)(P.q_slots * runs)), 64 * kWavefronts, lds, st>>>(
                    A, (int)P.q_slots, P.q_order, P.units, P.run, (const E*)G.out, (const E*)G.dout, G.lse, (E*)G.dq, delta, bias_part);
                return hipGetLastError();
            });
            if (e != hipSuccess) return e;
        }
        const int q_slots = A.total_q > 0 ? (int)P.q_slots : 0;
        e = by_form(A.bias != nullptr, A.keep != nullptr, [&](auto bias, auto masked) {
            constexpr bool BIAS = decltype(bias)::value, MASKED = decltype(masked)::value;
            const size_t lds = BIAS ? bias_bytes(A.reach, 1) : 0;
            const int main = A.total_k > 0 ? (int)(P.k_slots * ((A.kv_heads + P.kv_run - 1) / P.kv_run)) : 0;
            constexpr int WAVES = kKeyWaves<E, D, WIN>;
            const int more = BIAS ? (A.n_buckets * A.heads + WAVES - 1) / WAVES : 0;
            const int sinks = WIN && main ? (int)P.sink_groups : 0;
            if (main + more == 0) return hipSuccess;
            k_attention_dkv<E, D, BIAS, MASKED, WIN><<<dim3((unsigned)(main + sinks + more)), 64 * WAVES, lds, st>>>(
                A, (int)P.k_slots, P.k_order, P.kv_run, main, sinks, q_slots, (const E*)G.dout, G.lse, delta, bias_part, (E*)G.dk, (E*)G.dv,
                (E*)G.dbias, (float*)(ws + P.sink_part));
            return hipGetLastError();
        });
        if constexpr (WIN) {
            if (e != hipSuccess || !A.sinks || !A.total_k) return e;
            const int64_t places = (int64_t)A.n_seqs * A.kv_heads * A.sinks;
            k_attention_join_sinks<E, D><<<dim3((unsigned)((places + 3) / 4)), 256, 0, st>>>(A, (const float*)(ws + P.sink_part), (E*)G.dk, (E*)G.dv);
            e = hipGetLastError();
        }
        return e;
    });
}

}  // namespace cb
