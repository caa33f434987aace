// MaxSim scores with the tokens that were chosen, the contrastive loss over them, and the gradients of both sides'
// embeddings.
#include <type_traits>

#include "cb_tile.h"
#include "cb_train.h"

namespace cb {

// ---- scores --------------------------------------------------------------------------------------------------
// A workgroup keeps the rows of a few whole queries in registers, 32 * CT columns to a wavefront, and streams the tokens of
// its documents through LDS.  A column's running maximum and its place stay in the column's two lanes.
template <class E, int D, int CT>
__global__ __launch_bounds__(256) void k_maxsim_train(const E* Q, int nq, int T, const E* docs, const int64_t* off, int N, int total,
                                                      int col_groups, int q_per, int docs_per, float* scores, int32_t* argmax) {
    using O = Oper<E>;
    using L = Tile<E, D>;
    constexpr int NB = L::ROWS / 32, PIECES = L::ROWS * L::PIECES / 256;
    __shared__ __align__(16) char tile[L::BYTES];
    __shared__ float cells[128 * CT];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, n = lane & 31, h = lane >> 5;
    const int group = blockIdx.x % col_groups, part = blockIdx.x / col_groups;
    const int q0 = group * q_per, queries = nq - q0 < q_per ? nq - q0 : q_per, cols = queries * T;
    const int doc0 = part * docs_per, doc_end = N - doc0 < docs_per ? N : doc0 + docs_per;
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
    for (int i = doc0; i < doc_end; ++i) {
        const Range r = sequence_rows(off, i, total);
        float best[CT];
        int where[CT];
#pragma unroll
        for (int ct = 0; ct < CT; ++ct) {
            best[ct] = -INFINITY;
            where[ct] = r.n ? 0 : -1;
        }
        u32x4 next[PIECES];
        auto fetch = [&](int base) {
#pragma unroll
            for (int p = 0; p < PIECES; ++p) {
                const int at = p * 256 + tid, row = base + at / L::PIECES;
                next[p] = u32x4{0u, 0u, 0u, 0u};
                if (row < r.n) next[p] = *(const u32x4*)((const char*)(docs + (int64_t)(r.lo + row) * D) + at % L::PIECES * 16);
            }
        };
        if (r.n) fetch(0);
        for (int base = 0; base < r.n; base += L::ROWS) {
            __syncthreads();
#pragma unroll
            for (int p = 0; p < PIECES; ++p) {
                const int at = p * 256 + tid;
                *(u32x4*)(tile + L::at(at / L::PIECES, at % L::PIECES)) = next[p];
            }
            __syncthreads();
            if (base + L::ROWS < r.n) fetch(base + L::ROWS);
            if (wave * CT * 32 >= cols) continue;
#pragma unroll
            for (int b = 0; b < NB; ++b) {
                if (base + 32 * b >= r.n) break;
                f32x16 s[CT] = {};
#pragma unroll
                for (int c = 0; c < D / 16; ++c) {
                    const typename O::Frag a = L::rows(tile, lane, b, c);
#pragma unroll
                    for (int ct = 0; ct < CT; ++ct) O::mma(s[ct], a, q[ct][c]);
                }
                const int first = base + 32 * b + 4 * h, room = r.n - first;
                const bool whole = base + 32 * b + 32 <= r.n;
#pragma unroll
                for (int ct = 0; ct < CT; ++ct)
#pragma unroll
                    for (int x = 0; x < 16; ++x) {
                        const int k = 8 * (x >> 2) + (x & 3);
                        const bool more = s[ct][x] > best[ct] && (whole || k < room);
                        best[ct] = more ? s[ct][x] : best[ct];
                        where[ct] = more ? first + k : where[ct];
                    }
            }
        }
#pragma unroll
        for (int ct = 0; ct < CT; ++ct) {
            const float b2 = __shfl_xor(best[ct], 32);
            const int w2 = __shfl_xor(where[ct], 32);
            const bool take = b2 > best[ct] || (b2 == best[ct] && w2 < where[ct]);
            if (take) {
                best[ct] = b2;
                where[ct] = w2;
            }
            const int col = (wave * CT + ct) * 32 + n;
            if (ct == 0) __syncthreads();            // the sums of the document before have been read
            if (h == 0) cells[col] = best[ct];
            if (h == 0 && col < cols) argmax[((int64_t)(q0 + col / T) * N + i) * T + col % T] = where[ct];
        }
        __syncthreads();
        if (tid < queries) {
            float sum = 0.f;
            for (int t = 0; t < T; ++t) sum += cells[tid * T + t];
            scores[(int64_t)(q0 + tid) * N + i] = sum;
        }
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

// One workgroup a query: two passes over its scores, statistics in 32 bits.
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

// Queries: a row is the weighted sum of one token of every document.  A workgroup has four tokens of a query; the documents
// are split over its lane groups, whose sums are added in their order.
template <class E, int D>
__global__ __launch_bounds__(256) void k_maxsim_dq(const float* dscores, const int32_t* argmax, int T, int t_groups, const E* docs,
                                                   const int64_t* off, int N, int total, E* dQ) {
    using R = RowLanes<E, D>;
    constexpr int GROUPS = 256 / R::LANES, TOKENS = 4, PARTS = GROUPS / TOKENS, AHEAD = 8;
    __shared__ float sums[PARTS][TOKENS][R::LANES * R::PER];
    const int tid = threadIdx.x, piece = tid % R::LANES, token = tid / R::LANES % TOKENS, part = tid / R::LANES / TOKENS;
    const int q = blockIdx.x / t_groups, t = blockIdx.x % t_groups * TOKENS + token;
    const int each = (N + PARTS - 1) / PARTS, i0 = part * each, i1 = N - i0 < each ? N : i0 + each;
    float acc[R::PER] = {};
    if (t < T && piece < R::PIECES) {
        const int32_t* a = argmax + (int64_t)q * N * T + t;
        const float* g = dscores + (int64_t)q * N;
        for (int i = i0; i < i1; i += AHEAD) {
            u32x4 x[AHEAD];
            float w[AHEAD];
#pragma unroll
            for (int j = 0; j < AHEAD; ++j) {
                x[j] = u32x4{0u, 0u, 0u, 0u};
                w[j] = 0.f;
                if (i + j < i1) {
                    const int64_t at = a[(int64_t)(i + j) * T], row = off[i + j] + at;
                    if (at >= 0 && row >= 0 && row < total) {
                        w[j] = g[i + j];
                        x[j] = *(const u32x4*)((const char*)(docs + row * D) + piece * 16);
                    }
                }
            }
#pragma unroll
            for (int j = 0; j < AHEAD; ++j) R::add(acc, x[j], w[j]);
        }
    }
#pragma unroll
    for (int j = 0; j < R::PER; ++j) sums[part][token][piece * R::PER + j] = acc[j];
    __syncthreads();
    if (part == 0 && t < T && piece < R::PIECES) {
        for (int p = 1; p < PARTS; ++p)
#pragma unroll
            for (int j = 0; j < R::PER; ++j) acc[j] += sums[p][token][piece * R::PER + j];
        R::store(dQ + ((int64_t)q * T + t) * D, piece, acc);
    }
}

// Documents: a token's row is the weighted sum of the query tokens that chose it.  A workgroup has 64 tokens; it sorts the
// (query, token) entries that chose one of them by token, keeping their order (each wavefront a quarter of the entries, lanes
// with the same token found by ballots), and lane groups add up a token's list each.  The sort, not atomics on the rows, so
// that the order of the sums is fixed.
constexpr int kEntries = 4096, kTokens = 64;
template <class E, int D>
__global__ __launch_bounds__(256) void k_maxsim_ddocs(const float* dscores, const int32_t* argmax, const E* Q, int nq, int T,
                                                      const int64_t* off, int N, int total, E* ddocs) {
    using R = RowLanes<E, D>;
    constexpr int GROUPS = 256 / R::LANES, OWN = kTokens / GROUPS, AHEAD = 4;
    __shared__ float weight[kEntries];
    __shared__ uint16_t list[kEntries];
    __shared__ int8_t token[kEntries];
    __shared__ int next[4][kTokens], begin[kTokens + 1];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int doc = find_sequence(off, N, kTokens, total, blockIdx.x, lane);
    const Range r = sequence_rows(off, doc, total, kTokens);
    const int first = ((int)blockIdx.x - r.place) * kTokens;
    if (first < 0 || first >= r.n) return;
    const int piece = tid % R::LANES, group = tid / R::LANES;
    const int entries = nq * T;
    float acc[OWN][R::PER] = {};
    for (int e0 = 0; e0 < entries; e0 += kEntries) {
        const int count = entries - e0 < kEntries ? entries - e0 : kEntries;
        const int quarter = ((count + 255) / 256) * 64;          // entries of a wavefront, 64 a step
        const int w0 = wave * quarter, w1 = w0 + quarter < count ? w0 + quarter : count;
        __syncthreads();
        next[wave][lane] = 0;
#pragma unroll 4
        for (int e = w0 + lane; e < w1; e += 64) {
            const int q = (int)((uint32_t)(e0 + e) / (uint32_t)T);
            const int x = argmax[((int64_t)q * N + doc) * T + (e0 + e - q * T)] - first;
            token[e] = (int8_t)(x >= 0 && x < kTokens ? x : -1);
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
            const int x = e + lane < w1 ? token[e + lane] : -1;
            const uint64_t m = same(x);
            if (x >= 0 && lane == __builtin_ctzll(m)) next[wave][x] += __builtin_popcountll(m);
            __builtin_amdgcn_wave_barrier();
        }
        __syncthreads();
        if (wave == 0) {
            int n = 0, c[4];
#pragma unroll
            for (int w = 0; w < 4; ++w) {
                c[w] = next[w][lane];
                n += c[w];
            }
            int end = n;
#pragma unroll
            for (int m = 1; m < 64; m <<= 1) {
                const int x = __shfl_up(end, m);
                if (lane >= m) end += x;
            }
            int at = end - n;
            begin[lane] = at;
            if (lane == 63) begin[64] = end;
#pragma unroll
            for (int w = 0; w < 4; ++w) {
                next[w][lane] = at;
                at += c[w];
            }
        }
        __syncthreads();
        for (int e = w0; e < w1; e += 64) {
            const int x = e + lane < w1 ? token[e + lane] : -1;
            const uint64_t m = same(x);
            if (x >= 0) {
                const int at = next[wave][x] + __builtin_popcountll(m & ((1ull << lane) - 1ull));
                __builtin_amdgcn_wave_barrier();
                list[at] = (uint16_t)(e + lane);
                weight[at] = dscores[(int64_t)((uint32_t)(e0 + e + lane) / (uint32_t)T) * N + doc];
                if (lane == 63 - __builtin_clzll(m)) next[wave][x] = at + 1;
            }
            __builtin_amdgcn_wave_barrier();
        }
        __syncthreads();
        if (piece < R::PIECES) {
#pragma unroll
            for (int k = 0; k < OWN; ++k) {
                const int tk = group + k * GROUPS, b1 = begin[tk + 1];
                for (int b = begin[tk]; b < b1; b += AHEAD) {
                    u32x4 x[AHEAD];
                    float w[AHEAD];
#pragma unroll
                    for (int j = 0; j < AHEAD; ++j) {
                        x[j] = u32x4{0u, 0u, 0u, 0u};
                        w[j] = 0.f;
                        if (b + j < b1) {
                            w[j] = weight[b + j];
                            x[j] = *(const u32x4*)((const char*)(Q + (int64_t)(e0 + list[b + j]) * D) + piece * 16);
                        }
                    }
#pragma unroll
                    for (int j = 0; j < AHEAD; ++j) R::add(acc[k], x[j], w[j]);
                }
            }
        }
    }
    if (piece < R::PIECES) {
#pragma unroll
        for (int k = 0; k < OWN; ++k) {
            const int row = first + group + k * GROUPS;
            if (row < r.n) R::store(ddocs + (int64_t)(r.lo + row) * D, piece, acc[k]);
        }
    }
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
        auto go = [&](auto ct) {
            constexpr int CT = decltype(ct)::value;
            const int q_per = 128 * CT / T, col_groups = (nq + q_per - 1) / q_per;
            int64_t docs_per = N * col_groups / 2048;
            docs_per = docs_per < 1 ? 1 : docs_per;
            const int64_t parts = (N + docs_per - 1) / docs_per;
            k_maxsim_train<E, D, CT><<<dim3((unsigned)(parts * col_groups)), 256, 0, st>>>(
                (const E*)Q, nq, T, (const E*)docs, off, (int)N, (int)total, col_groups, q_per, (int)docs_per, scores, argmax);
            return hipGetLastError();
        };
        if ((int64_t)nq * T <= 128) return go(std::integral_constant<int, 1>{});
        return go(std::integral_constant<int, 2>{});
    });
}

hipError_t launch_contrastive_loss(const float* scores, int nq, int64_t N, const int64_t* targets, float temperature, float* loss,
                                   float* dscores, hipStream_t st) {
    k_contrastive<<<dim3((unsigned)nq), 256, 0, st>>>(scores, nq, N, targets, temperature, loss, dscores);
    return hipGetLastError();
}

hipError_t launch_maxsim_backward(const float* dscores, const int32_t* argmax, const void* Q, int nq, int T, int d, int dt,
                                  const void* docs, const int64_t* off, int64_t N, int64_t total, void* dQ, void* ddocs,
                                  hipStream_t st) {
    return by_type_and_width(dt, d, [&](auto type, auto dc) {
        using E = decltype(type);
        constexpr int D = decltype(dc)::value;
        const int t_groups = (T + 3) / 4;
        k_maxsim_dq<E, D><<<dim3((unsigned)(nq * t_groups)), 256, 0, st>>>(dscores, argmax, T, t_groups, (const E*)docs, off, (int)N,
                                                                           (int)total, (E*)dQ);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess || total == 0) return e;
        k_maxsim_ddocs<E, D><<<dim3((unsigned)(total / kTokens + N)), 256, 0, st>>>(dscores, argmax, (const E*)Q, nq, T, off, (int)N,
                                                                                    (int)total, (E*)ddocs);
        return hipGetLastError();
    });
}

}  // namespace cb
