// Queries and keys of each head normalised by their root mean square, weighted, and rotated by their row's position, in one pass; and
// its gradients.
#include <type_traits>

#include "cb_train.h"

namespace cb {

namespace {

typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x8 __attribute__((ext_vector_type(8)));

// With x a head's d values: n = x / sqrt(mean x^2 + eps), y = n w, and of each pair (y_a, y_b) the outputs are y_a c - y_b s and
// y_b c + y_a s, where c, s are the cosine and sine of the row's position for that pair.  Gradients, u being that of y n's, i.e. the
// outputs' rotated back: dw = sum of u n over all rows and heads, e = u w, dx = (e - n mean(e n)) / sqrt(mean x^2 + eps).
// A lane has four pairs of a head: two runs of four values that lie half a head apart, or eight values in a row (neighbours).  Either
// way pairs are within the lane, and a lane's four cosines and sines are the same for all heads of its row, so they are read once.
template <class E, bool NEAR> struct Head {
    float a[4], b[4];                                // first and second values of the pairs
    __device__ __forceinline__ void load(const E* p, int l, int half) {
        if constexpr (NEAR) {
            f32x8 x;
            if constexpr (sizeof(E) == 2) {
                x = __builtin_convertvector(*(const bf16x8*)(p + 8 * l), f32x8);
            } else {
                const f32x4 lo = *(const f32x4*)(p + 8 * l), hi = *(const f32x4*)(p + 8 * l + 4);
                x = __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
            }
#pragma unroll
            for (int i = 0; i < 4; ++i) a[i] = x[2 * i], b[i] = x[2 * i + 1];
        } else {
            f32x4 x, y;
            if constexpr (sizeof(E) == 2) {
                x = __builtin_convertvector(*(const bf16x4*)(p + 4 * l), f32x4);
                y = __builtin_convertvector(*(const bf16x4*)(p + half + 4 * l), f32x4);
            } else {
                x = *(const f32x4*)(p + 4 * l);
                y = *(const f32x4*)(p + half + 4 * l);
            }
#pragma unroll
            for (int i = 0; i < 4; ++i) a[i] = x[i], b[i] = y[i];
        }
    }
    __device__ __forceinline__ void store(E* p, int l, int half) const {
        if constexpr (NEAR) {
            const f32x8 x = {a[0], b[0], a[1], b[1], a[2], b[2], a[3], b[3]};
            if constexpr (sizeof(E) == 2) {
                *(bf16x8*)(p + 8 * l) = __builtin_convertvector(x, bf16x8);
            } else {
                *(f32x4*)(p + 8 * l) = __builtin_shufflevector(x, x, 0, 1, 2, 3);
                *(f32x4*)(p + 8 * l + 4) = __builtin_shufflevector(x, x, 4, 5, 6, 7);
            }
        } else {
            const f32x4 x = {a[0], a[1], a[2], a[3]}, y = {b[0], b[1], b[2], b[3]};
            if constexpr (sizeof(E) == 2) {
                *(bf16x4*)(p + 4 * l) = __builtin_convertvector(x, bf16x4);
                *(bf16x4*)(p + half + 4 * l) = __builtin_convertvector(y, bf16x4);
            } else {
                *(f32x4*)(p + 4 * l) = x;
                *(f32x4*)(p + half + 4 * l) = y;
            }
        }
    }
};

// Lanes of a head: D / 8, in groups of a power of two.
template <int D> constexpr int kLanes = D == 96 ? 16 : D / 8;
template <int D> __device__ __forceinline__ float sum_of_head(float x) {
#pragma unroll
    for (int m = 1; m < kLanes<D>; m <<= 1) x += __shfl_xor(x, m);
    return x;
}
template <int D> __device__ __forceinline__ float inverse_norm(float squares, float eps) { return 1.f / sqrtf(squares * (1.f / D) + eps); }

constexpr int kThreads = 256;

// A group's lanes take `parts`-th heads of a row, queries' and then keys'.
template <class E, int D, bool NEAR, bool BACK>
__global__ __launch_bounds__(kThreads) void k_rotate(const RotateArgs A, int parts) {
    constexpr int L = kLanes<D>, GROUPS = kThreads / L, AHEAD = BACK ? 2 : 4;
    const int tid = threadIdx.x, l = tid % L, group = tid / L;
    const bool on = l < D / 8;                       // (96 wide: twelve lanes of sixteen)
    const int heads = A.heads + A.kv_heads;
    float w[2][2][4], sums[2][2][4] = {};            // weights of queries and keys, by pair; their gradients
#pragma unroll
    for (int x = 0; x < 2; ++x) {
        const float* p = x ? A.k_weight : A.q_weight;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            w[x][0][i] = p && on ? p[NEAR ? 8 * l + 2 * i : 4 * l + i] : 1.f;
            w[x][1][i] = p && on ? p[NEAR ? 8 * l + 2 * i + 1 : D / 2 + 4 * l + i] : 1.f;
        }
    }
    const int64_t all = A.rows * parts, step = (int64_t)gridDim.x * GROUPS;
    for (int64_t work = (int64_t)blockIdx.x * GROUPS + group; work < all; work += step) {
        const int64_t row = parts == 1 ? work : work / parts;
        const int part = parts == 1 ? 0 : (int)(work - row * parts);
        const int64_t position = A.table ? A.positions[row] : 0;
        const bool none = A.table && (uint64_t)position >= (uint64_t)A.n_positions;
        f32x4 cs[2] = {f32x4{1.f, 0.f, 1.f, 0.f}, f32x4{1.f, 0.f, 1.f, 0.f}};
        if (A.table && !none && on) {
            const f32x4* t = (const f32x4*)(A.table + position * D) + 2 * l;
            cs[0] = t[0];
            cs[1] = t[1];
        }
        auto cosine = [&](int i) { return cs[i >> 1][2 * (i & 1)]; };
        auto sine = [&](int i) { return cs[i >> 1][2 * (i & 1) + 1]; };
        for (int h0 = part; h0 < heads; h0 += parts * AHEAD) {
            Head<E, NEAR> x[AHEAD], g[BACK ? AHEAD : 1];
#pragma unroll
            for (int j = 0; j < AHEAD; ++j) {
                const int h = h0 + j * parts;
                if (h >= heads || !on) continue;
                const bool key = h >= A.heads;
                const E* p = key ? (const E*)A.k + row * A.k_row + (h - A.heads) * A.k_head : (const E*)A.q + row * A.q_row + h * A.q_head;
                x[j].load(p, l, D / 2);
                if constexpr (BACK) {
                    const E* o = key ? (const E*)A.dk_out + (row * A.kv_heads + h - A.heads) * D : (const E*)A.dq_out + (row * A.heads + h) * D;
                    g[j].load(o, l, D / 2);
                }
            }
#pragma unroll
            for (int j = 0; j < AHEAD; ++j) {
                const int h = h0 + j * parts;
                if (h >= heads) break;
                const bool key = h >= A.heads;
                Head<E, NEAR>& v = x[j];
                float squares = 0.f;
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    if (!on) v.a[i] = v.b[i] = 0.f;
                    squares += v.a[i] * v.a[i] + v.b[i] * v.b[i];
                }
                const float r = inverse_norm<D>(sum_of_head<D>(squares), A.eps);
                if constexpr (!BACK) {
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const float a = v.a[i] * r * (key ? w[1][0][i] : w[0][0][i]), b = v.b[i] * r * (key ? w[1][1][i] : w[0][1][i]);
                        v.a[i] = none ? 0.f : a * cosine(i) - b * sine(i);
                        v.b[i] = none ? 0.f : b * cosine(i) + a * sine(i);
                    }
                } else {
                    float dot = 0.f;
                    float e[2][4];
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const float ga = on && !none ? g[j].a[i] : 0.f, gb = on && !none ? g[j].b[i] : 0.f;
                        const float ua = ga * cosine(i) + gb * sine(i), ub = gb * cosine(i) - ga * sine(i);
                        v.a[i] *= r;
                        v.b[i] *= r;
                        if (!none) {
                            sums[0][0][i] += key ? 0.f : ua * v.a[i];
                            sums[0][1][i] += key ? 0.f : ub * v.b[i];
                            sums[1][0][i] += key ? ua * v.a[i] : 0.f;
                            sums[1][1][i] += key ? ub * v.b[i] : 0.f;
                        }
                        e[0][i] = ua * (key ? w[1][0][i] : w[0][0][i]);
                        e[1][i] = ub * (key ? w[1][1][i] : w[0][1][i]);
                        dot += e[0][i] * v.a[i] + e[1][i] * v.b[i];
                    }
                    dot = sum_of_head<D>(dot) * (1.f / D);
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        v.a[i] = none ? 0.f : r * (e[0][i] - v.a[i] * dot);
                        v.b[i] = none ? 0.f : r * (e[1][i] - v.b[i] * dot);
                    }
                }
                if (on) v.store(key ? (E*)A.k_to + (row * A.kv_heads + h - A.heads) * D : (E*)A.q_to + (row * A.heads + h) * D, l, D / 2);
            }
        }
    }
    if constexpr (BACK) {                            // the workgroup's sums for the weights, its groups in their order
        __shared__ float part_of[GROUPS][D + 1];
#pragma unroll
        for (int x = 0; x < 2; ++x) {
            __syncthreads();
            if (on)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    part_of[group][NEAR ? 8 * l + 2 * i : 4 * l + i] = sums[x][0][i];
                    part_of[group][NEAR ? 8 * l + 2 * i + 1 : D / 2 + 4 * l + i] = sums[x][1][i];
                }
            __syncthreads();
            if (tid < D) {
                float s = 0.f;
                for (int y = 0; y < GROUPS; ++y) s += part_of[y][tid];
                A.part[((int64_t)blockIdx.x * 2 + x) * D + tid] = s;
            }
        }
    }
}

// Adds up the workgroups' sums for the weights: 16 values a workgroup, 64 threads each.
constexpr int kJoinThreads = 1024, kJoinValues = 16;
__global__ __launch_bounds__(kJoinThreads) void k_rotate_join(const float* part, int parts, int d, float* dq_weight, float* dk_weight) {
    __shared__ float sums[kJoinThreads / kJoinValues][kJoinValues + 1];
    const int own = threadIdx.x % kJoinValues, from = threadIdx.x / kJoinValues, at = blockIdx.x * kJoinValues + own;
    float s = 0.f;
#pragma unroll 8
    for (int p = from; p < parts; p += kJoinThreads / kJoinValues) s += part[(int64_t)p * 2 * d + at];
    sums[from][own] = s;
    __syncthreads();
    if (from) return;
    s = 0.f;
    for (int p = 0; p < kJoinThreads / kJoinValues; ++p) s += sums[p][own];
    float* to = at < d ? dq_weight : dk_weight;
    if (to) to[at < d ? at : at - d] = s;
}

// Heads of a row are dealt to several groups where rows are few.
int parts_of(const RotateArgs& A, int lanes) {
    const int heads = A.heads + A.kv_heads;
    int parts = 1;
    while (parts < heads && A.rows * parts * lanes < 1 << 19) parts *= 2;
    return parts < heads ? parts : heads;
}
constexpr int64_t kMostGroups = 1024;                // of the backward pass
int64_t groups_of(const RotateArgs& A, int parts, int lanes, bool back) {
    const int64_t per = kThreads / lanes, groups = (A.rows * parts + per - 1) / per;
    return back && groups > kMostGroups ? kMostGroups : groups;
}
int lanes_of(int d) { return d == 96 ? 16 : d / 8; }

template <class F> hipError_t by_width(int d, F&& f) {
    switch (d) {
        case 32: return f(std::integral_constant<int, 32>{});
        case 64: return f(std::integral_constant<int, 64>{});
        case 96: return f(std::integral_constant<int, 96>{});
        default: return f(std::integral_constant<int, 128>{});
    }
}
template <bool BACK> hipError_t launch(const RotateArgs& A, int d, int dt, hipStream_t st) {
    const int parts = parts_of(A, lanes_of(d));
    const dim3 grid((unsigned)groups_of(A, parts, lanes_of(d), BACK));
    return by_width(d, [&](auto dc) {
        constexpr int D = decltype(dc)::value;
        auto go = [&](auto* e, auto near) {
            using E = std::remove_pointer_t<decltype(e)>;
            k_rotate<E, D, decltype(near)::value, BACK><<<grid, kThreads, 0, st>>>(A, parts);
            return hipGetLastError();
        };
        if (dt == TR_BF16) return A.near ? go((__bf16*)nullptr, std::true_type{}) : go((__bf16*)nullptr, std::false_type{});
        return A.near ? go((float*)nullptr, std::true_type{}) : go((float*)nullptr, std::false_type{});
    });
}

}  // namespace

int64_t rotate_groups(const RotateArgs& A, int d, bool back) { return groups_of(A, parts_of(A, lanes_of(d)), lanes_of(d), back); }
size_t rotate_workspace_bytes(const RotateArgs& A, int d) { return (size_t)(rotate_groups(A, d, true) * 2 * d * 4 + 255) / 256 * 256; }

hipError_t launch_rotate(const RotateArgs& A, int d, int dt, hipStream_t st) {
    return A.rows == 0 ? hipSuccess : launch<false>(A, d, dt, st);
}
hipError_t launch_rotate_backward(const RotateArgs& A, int d, int dt, float* dq_weight, float* dk_weight, hipStream_t st) {
    if (A.rows) {
        const hipError_t e = launch<true>(A, d, dt, st);
        if (e != hipSuccess) return e;
    }
    if (!dq_weight && !dk_weight) return hipSuccess;
    k_rotate_join<<<dim3((unsigned)(2 * d / kJoinValues)), kJoinThreads, 0, st>>>(A.part, A.rows ? (int)rotate_groups(A, d, true) : 0, d, dq_weight,
                                                                                  dk_weight);
    return hipGetLastError();
}

}  // namespace cb
