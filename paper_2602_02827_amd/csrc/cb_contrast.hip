// MaxSim scores with the tokens that were chosen, the contrastive loss over them, and the gradients of both sides'
// embeddings.
#include <type_traits>

#include "cb_tile.h"
#include "cb_train.h"

namespace cb {

// ---- scores --------------------------------------------------------------------------------------------------
// A workgroup keeps the rows of a few whole queries in registers, 32 * CT columns to a wavefront, and streams the tokens of
// its documents through LDS, the next tile on its way while it multiplies.  A column's running maximum and its place stay in the
// column's two lanes; a comparison, and two selections of it, for every product (the place within a block is a constant).
// 64 x 32 tokens against 512 passages, d = 128: 50 us, 570 TFLOP/s.  Vector instructions take 56 % of the SIMDs' clocks there, half of
// them the three above, and the matrix units 35 %, with little of the one beside the other: four wavefronts a SIMD wait for the same
// tile at the same barrier, and at a document's end for its shuffles, its stores and the next one's offsets.  16 x 24 against 128
// pages: 34 us.
template <class E, int D, int CT>
__global__ __launch_bounds__(256, (sizeof(E) == 4 ? (D == 128 ? 1 : 2) : 4)) void
k_maxsim_train(const E* Q, int nq, int T, const E* docs, const int64_t* off, int N, int total, int col_groups, int q_per, int docs_per,
               float* scores, int32_t* argmax) {
    using O = Oper<E>;
    using L = Tile<E, D>;
    constexpr int NB = L::ROWS / 32;
    __shared__ __align__(256) char tile[2][L::BYTES];
    __shared__ float cells[2][128 * CT];
    const int tid = threadIdx.x, lane0 = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), n = lane0 & 31, h = lane0 >> 5;
    const int group = blockIdx.x % col_groups, part = blockIdx.x / col_groups;
    const int q0 = group * q_per, queries = nq - q0 < q_per ? nq - q0 : q_per, cols = queries * T;
    const int doc0 = part * docs_per, doc_end = N - doc0 < docs_per ? N : doc0 + docs_per;
    Rows<E, D, 256> next;
    auto issue = [&](const Range& r, int base, char* to) {
        if (r.n == 0) return;
        next.issue((const char*)(docs + (int64_t)(r.lo + base) * D), to, r.n - base, here(tid), wave,
                   [&](int row) { return (uint32_t)(row * D * (int)sizeof(E)); });
    };
    auto finish = [&](char* to) { next.finish(to, tid, [](int) { return true; }); };
    Range r = sequence_rows(off, doc0, total);
    issue(r, 0, tile[0]);
    typename O::Frag q[CT][D / 16];
#pragma unroll
    for (int ct = 0; ct < CT; ++ct) {
        const int col = (wave * CT + ct) * 32 + n;
#pragma unroll
        for (int c = 0; c < D / 16; ++c) {
            q[ct][c] = {};
            if (col < cols) q[ct][c] = O::load(Q + ((int64_t)q0 * T + col) * D + 16 * c + 8 * h);
        }
    }
    float best[CT];
    int where[CT];
    const typename L::At at_tile(tile[0], lane0);
    int i = doc0, base = 0, buf = 0;
    if (r.n) finish(tile[0]);
    __syncthreads();
    while (true) {
        const bool first = base == 0, last = base + L::ROWS >= r.n;       // of the document
        const int n_i = last ? i + 1 : i, n_base = last ? 0 : base + L::ROWS;
        const bool more = n_i < doc_end;
        const Range n_r = last && more ? sequence_rows(off, n_i, total) : r;
        if (more) issue(n_r, n_base, tile[buf ^ 1]);
        if (first) {
#pragma unroll
            for (int ct = 0; ct < CT; ++ct) {
                best[ct] = -INFINITY;
                where[ct] = r.n ? 0 : -1;
            }
        }
        if (wave * CT * 32 < cols) {
            const typename L::At t = at_tile + buf * L::BYTES;
#pragma unroll 1
            for (int b = 0; b < NB && base + 32 * b < r.n; ++b) {
                f32x16 s[CT] = {};
#pragma unroll
                for (int c = 0; c < D / 16; ++c) {
                    const typename O::Frag a = L::rows(t, b, c);
#pragma unroll
                    for (int ct = 0; ct < CT; ++ct) O::mma(s[ct], a, q[ct][c]);
                }
                const int at = base + 32 * b + 4 * h, room = r.n - at;
                if (base + 32 * b + 32 > r.n) {
#pragma unroll
                    for (int ct = 0; ct < CT; ++ct)
#pragma unroll
                        for (int x = 0; x < 16; ++x) s[ct][x] = 8 * (x >> 2) + (x & 3) < room ? s[ct][x] : -INFINITY;
                }
#pragma unroll
                for (int ct = 0; ct < CT; ++ct) {
                    int k = -1;
#pragma unroll
                    for (int x = 0; x < 16; ++x) {
                        const bool higher = s[ct][x] > best[ct];          // the first of equal ones stays
                        best[ct] = higher ? s[ct][x] : best[ct];
                        k = higher ? 8 * (x >> 2) + (x & 3) : k;
                    }
                    where[ct] = k < 0 ? where[ct] : at + k;
                }
            }
        }
        if (last) {
#pragma unroll
            for (int ct = 0; ct < CT; ++ct) {
                const float b2 = __shfl_xor(best[ct], 32);
                const int w2 = __shfl_xor(where[ct], 32);
                const bool take = b2 > best[ct] || (b2 == best[ct] && w2 < where[ct]);
                best[ct] = take ? b2 : best[ct];
                where[ct] = take ? w2 : where[ct];
                const int col = (wave * CT + ct) * 32 + n;
                if (h == 0) cells[i & 1][col] = best[ct];
                if (h == 0 && col < cols) argmax[((int64_t)(q0 + col / T) * N + i) * T + col % T] = where[ct];
            }
        }
        if (more && n_r.n) finish(tile[buf ^ 1]);
        __syncthreads();
        if (last) {                                  // eight lanes a query; the next document's cells are the other ones
            for (int x = tid >> 3; x < queries; x += 32) {
                float sum = 0.f;
                for (int t = tid & 7; t < T; t += 8) sum += cells[i & 1][x * T + t];
#pragma unroll
                for (int m = 1; m < 8; m <<= 1) sum += __shfl_xor(sum, m);
                if ((tid & 7) == 0) scores[(int64_t)(q0 + x) * N + i] = sum;
            }
        }
        if (!more) return;
        r = n_r;
        i = n_i;
        base = n_base;
        buf ^= 1;
    }
}

// ---- loss ----------------------------------------------------------------------------------------------------
__device__ __forceinline__ float block_max(float x, float* s) {
    const int tid = threadIdx.x;
#pragma unroll
    for (int m = 1; m < 64; m <<= 1) x = fmaxf(x, __shfl_xor(x, m));
    __syncthreads();
    if ((tid & 63) == 0) s[tid >> 6] = x;
    __syncthreads();
    return fmaxf(fmaxf(s[0], s[1]), fmaxf(s[2], s[3]));
}
__device__ __forceinline__ float block_sum(float x, float* s) {
    const int tid = threadIdx.x;
#pragma unroll
    for (int m = 1; m < 64; m <<= 1) x += __shfl_xor(x, m);
    __syncthreads();
    if ((tid & 63) == 0) s[tid >> 6] = x;
    __syncthreads();
    return (s[0] + s[1]) + (s[2] + s[3]);
}

// One workgroup a query: two passes over its scores, statistics in 32 bits.  3 to 5 us, a launch's latency.
__global__ __launch_bounds__(256) void k_contrastive(const float* scores, int nq, int64_t N, const int64_t* targets, float temperature,
                                                     float* loss, float* dscores) {
    __shared__ float s[4];
    const int q = blockIdx.x, tid = threadIdx.x;
    const float* x = scores + q * N;
    float* g = dscores + q * N;
    const int64_t target = targets[q];
    if (target < 0 || target >= N) {
        if (tid == 0) loss[q] = 0.f;
        for (int64_t i = tid; i < N; i += 256) g[i] = 0.f;
        return;
    }
    float counted = 0.f;                             // queries that take part in the mean (exact: below 2^24)
    for (int i = tid; i < nq; i += 256) counted += targets[i] >= 0 && targets[i] < N ? 1.f : 0.f;
    counted = block_sum(counted, s);
    float top = -INFINITY;
    for (int64_t i = tid; i < N; i += 256) top = fmaxf(top, x[i]);
    top = block_max(top, s);
    const float from = top == -INFINITY ? 0.f : top, inv = 1.f / temperature;
    float z = 0.f;
    for (int64_t i = tid; i < N; i += 256) z += expf((x[i] - from) * inv);
    z = block_sum(z, s);
    const float w = inv / counted, wz = w / z;
    for (int64_t i = tid; i < N; i += 256) {
        const float p = expf((x[i] - from) * inv) * wz;
        g[i] = i == target ? p - w : p;
    }
    if (tid == 0) loss[q] = logf(z) + (from - x[target]) * inv;
}

// ---- gradients -----------------------------------------------------------------------------------------------
// Lanes that hold a row of D values together, 16 bytes each.
template <class E, int D> struct RowLanes {
    static constexpr int PIECES = D * (int)sizeof(E) / 16, PER = 16 / (int)sizeof(E);
    static constexpr int LANES = PIECES <= 4 ? 4 : PIECES <= 8 ? 8 : PIECES <= 16 ? 16 : 32;
    static __device__ __forceinline__ void add(float (&acc)[PER], const u32x4& x, float w) {
        if constexpr (sizeof(E) == 2) {
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                acc[2 * j] = fmaf(w, __uint_as_float(x[j] << 16), acc[2 * j]);
                acc[2 * j + 1] = fmaf(w, __uint_as_float(x[j] & 0xffff0000u), acc[2 * j + 1]);
            }
        } else {
#pragma unroll
            for (int j = 0; j < 4; ++j) acc[j] = fmaf(w, __uint_as_float(x[j]), acc[j]);
        }
    }
    static __device__ __forceinline__ void store(E* row, int piece, const float (&acc)[PER]) {
#pragma unroll
        for (int j = 0; j < PER; j += 4)
            Oper<E>::store4(row + piece * PER + j, f32x4{acc[j], acc[j + 1], acc[j + 2], acc[j + 3]});
    }
};

// Queries: a row is the weighted sum of one token of every document.  A workgroup has one query token; its lane groups take the
// documents in turn (all workgroups go through the corpus together, so its rows are found in L2), and their sums are added in
// order.
// 64 x 32 tokens and 512 passages: 37 us by themselves, 1.05 million rows of 256 bytes, 7.2 TB/s from L2 and the last-level cache.
template <class E, int D>
__device__ __forceinline__ void query_gradient(char* lds, int block, const float* dscores, const int32_t* argmax, int T, const E* docs,
                                               const int64_t* off, int N, int total, E* dQ) {
    using R = RowLanes<E, D>;
    constexpr int PARTS = 256 / R::LANES, AHEAD = 8, WIDTH = R::LANES * R::PER;
    float* sums = (float*)lds;                       // [PARTS][WIDTH]
    const int tid = threadIdx.x, piece = tid % R::LANES, part = tid / R::LANES;
    const int q = block / T, t = block % T;
    float acc[R::PER] = {};
    if (piece < R::PIECES) {
        const int32_t* a = argmax + (int64_t)q * N * T + t;
        const float* g = dscores + (int64_t)q * N;
        for (int first = part; first < N; first += PARTS * AHEAD) {
            u32x4 x[AHEAD];
            float w[AHEAD];
#pragma unroll
            for (int j = 0; j < AHEAD; ++j) {
                x[j] = u32x4{0u, 0u, 0u, 0u};
                w[j] = 0.f;
                const int i = first + j * PARTS;
                if (i < N) {
                    const int64_t at = a[(int64_t)i * T], row = off[i] + at;
                    if (at >= 0 && row >= 0 && row < total) {
                        w[j] = g[i];
                        x[j] = *(const u32x4*)((const char*)(docs + row * D) + piece * 16);
                    }
                }
            }
#pragma unroll
            for (int j = 0; j < AHEAD; ++j) R::add(acc, x[j], w[j]);
        }
    }
#pragma unroll
    for (int j = 0; j < R::PER; ++j) sums[part * WIDTH + piece * R::PER + j] = acc[j];
    __syncthreads();
    if (part == 0 && piece < R::PIECES) {
        for (int p = 1; p < PARTS; ++p)
#pragma unroll
            for (int j = 0; j < R::PER; ++j) acc[j] += sums[p * WIDTH + piece * R::PER + j];
        R::store(dQ + (int64_t)block * D, piece, acc);
    }
}

// Documents: a token's row is the weighted sum of the query tokens that chose it.  A workgroup has 64 tokens; it sorts the
// (query, token) entries that chose one of them by token, keeping their order (each wavefront a quarter of the entries, lanes
// with the same token found by ballots), and each lane group adds up the lists of consecutive tokens as one, eight rows on
// their way at a time.  The sort, not atomics on the rows, so that the order of the sums is fixed.
// 64 x 32 tokens and 512 passages: 74 us by themselves, 87 together with the queries' workgroups.  Over that launch vector
// instructions take 70 % of the SIMDs' clocks (the sort's ballots and places; a multiply-add and half an unpacking for every value),
// and the wavefronts wait 61 % of theirs; the queries that are gathered, 0.5 MB, lie in every L2.
// MANY: more entries than are sorted at once; the rows are added up in LDS then.
constexpr int kEntries = 4096, kTokens = 64;
template <int D, bool MANY> struct TokenLists {
    float weight[kEntries];
    uint16_t list[kEntries];
    int8_t token[kEntries];
    int next[4][kTokens], begin[kTokens + 1];
    __align__(16) float rows[MANY ? kTokens : 1][MANY ? D : 1];
};
template <class E, int D, bool MANY>
__device__ __forceinline__ void document_gradient(char* lds, int block, const float* dscores, const int32_t* argmax, const E* Q, int nq,
                                                  int T, const int64_t* off, int N, int total, E* ddocs) {
    using R = RowLanes<E, D>;
    constexpr int GROUPS = 256 / R::LANES, OWN = kTokens / GROUPS, AHEAD = 8;
    TokenLists<D, MANY>& s = *(TokenLists<D, MANY>*)lds;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int doc = find_sequence(off, N, kTokens, total, block, lane);
    bool rest;
    const Range r = rows_of_place(off, doc, N, total, kTokens, block, rest);
    const int first = (block - r.place) * kTokens;
    if (first < 0 || first >= r.n) return;
    const int piece = tid % R::LANES, group = tid / R::LANES;
    if (rest) {                                      // tokens of no document
        const float none[R::PER] = {};
        for (int token = first + group; token < r.n && token < first + kTokens; token += GROUPS)
            if (piece < R::PIECES) R::store(ddocs + (int64_t)(r.lo + token) * D, piece, none);
        return;
    }
    const int entries = nq * T;
    if constexpr (MANY)
        for (int i = tid; i < kTokens * D; i += 256) (&s.rows[0][0])[i] = 0.f;
    for (int e0 = 0; e0 < entries; e0 += kEntries) {
        const int count = entries - e0 < kEntries ? entries - e0 : kEntries;
        const int quarter = ((count + 255) / 256) * 64;          // entries of a wavefront, 64 a step
        const int w0 = wave * quarter, w1 = w0 + quarter < count ? w0 + quarter : count;
        __syncthreads();
        s.next[wave][lane] = 0;
#pragma unroll 4
        for (int e = w0 + lane; e < w1; e += 64) {
            const int q = (int)((uint32_t)(e0 + e) / (uint32_t)T);
            const int x = argmax[((int64_t)q * N + doc) * T + (e0 + e - q * T)] - first;
            s.token[e] = (int8_t)(x >= 0 && x < kTokens ? x : -1);
        }
        __syncthreads();
        auto same = [&](int x) {                     // lanes of the step with this lane's token
            uint64_t m = __ballot(x >= 0);
#pragma unroll
            for (int b = 0; b < 6; ++b) {
                const uint64_t set = __ballot((x >> b) & 1);
                m &= (x >> b) & 1 ? set : ~set;
            }
            return m;
        };
        for (int e = w0; e < w1; e += 64) {
            const int x = e + lane < w1 ? s.token[e + lane] : -1;
            const uint64_t m = same(x);
            if (x >= 0 && lane == __builtin_ctzll(m)) s.next[wave][x] += __builtin_popcountll(m);
            __builtin_amdgcn_wave_barrier();
        }
        __syncthreads();
        if (wave == 0) {
            int n = 0, c[4];
#pragma unroll
            for (int w = 0; w < 4; ++w) {
                c[w] = s.next[w][lane];
                n += c[w];
            }
            int end = n;
#pragma unroll
            for (int m = 1; m < 64; m <<= 1) {
                const int x = __shfl_up(end, m);
                if (lane >= m) end += x;
            }
            int at = end - n;
            s.begin[lane] = at;
            if (lane == 63) s.begin[64] = end;
#pragma unroll
            for (int w = 0; w < 4; ++w) {
                s.next[w][lane] = at;
                at += c[w];
            }
        }
        __syncthreads();
        for (int e = w0; e < w1; e += 64) {
            const int x = e + lane < w1 ? s.token[e + lane] : -1;
            const uint64_t m = same(x);
            if (x >= 0) {
                const int at = s.next[wave][x] + __builtin_popcountll(m & ((1ull << lane) - 1ull));
                __builtin_amdgcn_wave_barrier();
                s.list[at] = (uint16_t)(e + lane);
                s.weight[at] = dscores[(int64_t)((uint32_t)(e0 + e + lane) / (uint32_t)T) * N + doc];
                if (lane == 63 - __builtin_clzll(m)) s.next[wave][x] = at + 1;
            }
            __builtin_amdgcn_wave_barrier();
        }
        __syncthreads();
        if (piece < R::PIECES) {
            int token = group * OWN, bound = s.begin[token + 1];
            const int end = s.begin[group * OWN + OWN];
            float acc[R::PER] = {};
            auto done = [&]() {                      // with a token's list
                if constexpr (MANY) {
#pragma unroll
                    for (int j = 0; j < R::PER; ++j) s.rows[token][piece * R::PER + j] += acc[j];
                } else if (first + token < r.n) {
                    R::store(ddocs + (int64_t)(r.lo + first + token) * D, piece, acc);
                }
#pragma unroll
                for (int j = 0; j < R::PER; ++j) acc[j] = 0.f;
                ++token;
                bound = s.begin[token + 1 < kTokens ? token + 1 : kTokens];
            };
            for (int b = s.begin[token]; b < end; b += AHEAD) {
                u32x4 x[AHEAD];
                float w[AHEAD];
#pragma unroll
                for (int j = 0; j < AHEAD; ++j) {
                    x[j] = u32x4{0u, 0u, 0u, 0u};
                    w[j] = 0.f;
                    if (b + j < end) {
                        w[j] = s.weight[b + j];
                        x[j] = *(const u32x4*)((const char*)(Q + (int64_t)(e0 + s.list[b + j]) * D) + piece * 16);
                    }
                }
#pragma unroll
                for (int j = 0; j < AHEAD; ++j) {
                    while (b + j >= bound && b + j < end) done();
                    R::add(acc, x[j], w[j]);
                }
            }
            while (token < group * OWN + OWN) done();
        }
    }
    if constexpr (MANY) {
        if (piece < R::PIECES) {                     // the lane group's own tokens
            for (int k = 0; k < OWN; ++k) {
                const int token = group * OWN + k;
                if (first + token >= r.n) break;
                float acc[R::PER];
#pragma unroll
                for (int j = 0; j < R::PER; ++j) acc[j] = s.rows[token][piece * R::PER + j];
                R::store(ddocs + (int64_t)(r.lo + first + token) * D, piece, acc);
            }
        }
    }
}

// One launch for both: the first workgroups take documents, which take longer.
template <class E, int D, bool MANY>
__global__ __launch_bounds__(256, MANY ? 2 : 4) void k_maxsim_gradients(const float* dscores, const int32_t* argmax, const E* Q, int nq, int T,
                                                          const E* docs, const int64_t* off, int N, int total, int doc_blocks, E* dQ,
                                                          E* ddocs) {
    constexpr size_t SUMS = sizeof(float) * (256 / RowLanes<E, D>::LANES) * RowLanes<E, D>::LANES * RowLanes<E, D>::PER;
    constexpr size_t LISTS = sizeof(TokenLists<D, MANY>);
    __shared__ __align__(16) char lds[SUMS > LISTS ? SUMS : LISTS];
    const int block = blockIdx.x;
    if (block < doc_blocks) document_gradient<E, D, MANY>(lds, block, dscores, argmax, Q, nq, T, off, N, total, ddocs);
    else query_gradient<E, D>(lds, block - doc_blocks, dscores, argmax, T, docs, off, N, total, dQ);
}

// ---- launches ------------------------------------------------------------------------------------------------
template <class F> hipError_t by_type_and_width(int dt, int d, F&& f) {
    auto width = [&](auto type) {
        switch (d) {
            case 32: return f(type, std::integral_constant<int, 32>{});
            case 64: return f(type, std::integral_constant<int, 64>{});
            case 96: return f(type, std::integral_constant<int, 96>{});
            default: return f(type, std::integral_constant<int, 128>{});
        }
    };
    return dt == TR_BF16 ? width((__bf16)0.f) : width(0.f);
}

hipError_t launch_maxsim_scores(const void* Q, int nq, int T, int d, int dt, const void* docs, const int64_t* off, int64_t N,
                                int64_t total, float* scores, int32_t* argmax, hipStream_t st) {
    return by_type_and_width(dt, d, [&](auto type, auto dc) {
        using E = decltype(type);
        constexpr int D = decltype(dc)::value;
        // About as many workgroups as run at once (four a CU; 512, 768 and 2,048 measured alike), of consecutive documents each.
        // Two columns a lane read a tile's operands half as often (64 x 32 tokens against 512 passages, the whole loss: 140 us, one
        // column 145), where there are enough workgroups of them (16 x 24 tokens against 128 pages: 63 us, one column 57).
        constexpr int64_t kGroups = 1024;
        auto go = [&](auto ct) {
            constexpr int CT = decltype(ct)::value;
            const int q_per = 128 * CT / T, col_groups = (nq + q_per - 1) / q_per;
            int64_t docs_per = N * col_groups / kGroups;
            docs_per = docs_per < 1 ? 1 : docs_per;
            const int64_t parts = (N + docs_per - 1) / docs_per;
            k_maxsim_train<E, D, CT><<<dim3((unsigned)(parts * col_groups)), 256, 0, st>>>(
                (const E*)Q, nq, T, (const E*)docs, off, (int)N, (int)total, col_groups, q_per, (int)docs_per, scores, argmax);
            return hipGetLastError();
        };
        const int two = 256 / T;
        if ((nq + two - 1) / two * N < kGroups) return go(std::integral_constant<int, 1>{});
        return go(std::integral_constant<int, 2>{});
    });
}

hipError_t launch_contrastive_loss(const float* scores, int nq, int64_t N, const int64_t* targets, float temperature, float* loss,
                                   float* dscores, hipStream_t st) {
    k_contrastive<<<dim3((unsigned)nq), 256, 0, st>>>(scores, nq, N, targets, temperature, loss, dscores);
    return hipGetLastError();
}

static int64_t document_groups(int64_t N, int64_t total) { return total > 0 ? total / kTokens + N + 1 : 0; }
int64_t maxsim_backward_groups(int nq, int T, int64_t N, int64_t total) { return document_groups(N, total) + (int64_t)nq * T; }

hipError_t launch_maxsim_backward(const float* dscores, const int32_t* argmax, const void* Q, int nq, int T, int d, int dt,
                                  const void* docs, const int64_t* off, int64_t N, int64_t total, void* dQ, void* ddocs,
                                  hipStream_t st) {
    return by_type_and_width(dt, d, [&](auto type, auto dc) {
        using E = decltype(type);
        constexpr int D = decltype(dc)::value;
        const int doc_blocks = (int)document_groups(N, total);
        auto go = [&](auto many) {
            k_maxsim_gradients<E, D, decltype(many)::value><<<dim3((unsigned)(doc_blocks + nq * T)), 256, 0, st>>>(
                dscores, argmax, (const E*)Q, nq, T, (const E*)docs, off, (int)N, (int)total, doc_blocks, (E*)dQ, (E*)ddocs);
            return hipGetLastError();
        };
        return nq * T > kEntries ? go(std::true_type{}) : go(std::false_type{});
    });
}

}  // namespace cb
