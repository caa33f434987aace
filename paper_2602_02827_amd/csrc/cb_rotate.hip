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
typedef float f32x4_any __attribute__((ext_vector_type(4), aligned(4)));       // at any value

// With x a head's d values: n = x / sqrt(mean x^2 + eps), y = n w, and of each pair (y_a, y_b) the outputs are y_a c - y_b s and
// y_b c + y_a s, where c, s are the cosine and sine of the row's position for that pair.  Gradients, u being that of y n's, i.e. the
// outputs' rotated back: dw = sum of u n over all rows and heads, e = u w, dx = (e - n mean(e n)) / sqrt(mean x^2 + eps).
// A lane has four pairs of a head: two runs of four values that lie half a head apart, or, of 16-bit neighbours, eight values in a row
// (sixteen bytes a load or store; of 32-bit ones two stores to every other sixteen bytes take memory two to three times as long).  Either
// way pairs are within the lane, and a lane's four cosines and sines are the same for all heads of its row, so they are read once.
template <class E, int HALF, bool NEAR> struct Head {      // pointers: to the lane's first value
    f32x4 a, b;                                      // first and second values of the pairs
    __device__ __forceinline__ void load(const E* p) {
        f32x4 x, y;                                  // the lane's two runs of four
        if constexpr (sizeof(E) == 4) {
            x = *(const f32x4*)p;
            y = *(const f32x4*)(p + HALF);
        } else if constexpr (NEAR) {
            const bf16x8 z = *(const bf16x8*)p;
            x = __builtin_convertvector(__builtin_shufflevector(z, z, 0, 1, 2, 3), f32x4);
            y = __builtin_convertvector(__builtin_shufflevector(z, z, 4, 5, 6, 7), f32x4);
        } else {
            x = __builtin_convertvector(*(const bf16x4*)p, f32x4);
            y = __builtin_convertvector(*(const bf16x4*)(p + HALF), f32x4);
        }
        a = NEAR ? __builtin_shufflevector(x, y, 0, 2, 4, 6) : x;
        b = NEAR ? __builtin_shufflevector(x, y, 1, 3, 5, 7) : y;
    }
    __device__ __forceinline__ void store(E* p) const {
        const f32x4 x = NEAR ? __builtin_shufflevector(a, b, 0, 4, 1, 5) : a, y = NEAR ? __builtin_shufflevector(a, b, 2, 6, 3, 7) : b;
        if constexpr (sizeof(E) == 4) {
            *(f32x4*)p = x;
            *(f32x4*)(p + HALF) = y;
        } else if constexpr (NEAR) {
            *(bf16x8*)p = __builtin_convertvector(__builtin_shufflevector(x, y, 0, 1, 2, 3, 4, 5, 6, 7), bf16x8);
        } else {
            *(bf16x4*)p = __builtin_convertvector(x, bf16x4);
            *(bf16x4*)(p + HALF) = __builtin_convertvector(y, bf16x4);
        }
    }
};

// Lanes of a head: D / 8, in groups of a power of two.
template <int D> constexpr int kLanes = D == 96 ? 16 : D / 8;
// Sum over a head's lanes: each adds its neighbour's, then the other pair's, the other four's, the other eight's.
template <int CTRL> __device__ __forceinline__ float of_lane(float x) {
    return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(x), CTRL, 0xf, 0xf, true));
}
template <int D> __device__ __forceinline__ float sum_of_head(float x) {
    x += of_lane<0xB1>(x);                           // lanes 1 0 3 2
    x += of_lane<0x4E>(x);                           // lanes 2 3 0 1
    if constexpr (kLanes<D> >= 8) x += of_lane<0x141>(x);        // of eight, from the other end
    if constexpr (kLanes<D> >= 16) x += of_lane<0x140>(x);       // of sixteen
    return x;
}

constexpr int kThreads = 256;

// A group's lanes take every 2^lg_parts-th head of a row, queries' and then keys'.  One pass, since a head fits its lanes: each value is
// read once (the backward pass computes the norms again, from the inputs that it needs anyway) and written once.  Several heads are under
// way at a time: four forward, two backward, where each is two loads.  Bound by memory: 54 thousand rows of 24 heads of 64, bf16, 69 us
// (332 MB, 4.8 TB/s) and, with gradients, 106 (498 MB, 4.7 TB/s).  5.6 thousand fp32 rows of 9 heads of 96, pairs of neighbours: 13 and 14 us;
// 16 single rows 3.4, of which a launch and two dependent loads (the position, then its cosines) are most.
template <class E, int D, bool NEAR, bool BACK>
__global__ __launch_bounds__(kThreads) void k_rotate(const RotateArgs A, int lg_parts) {
    constexpr int L = kLanes<D>, GROUPS = kThreads / L, AHEAD = BACK ? 2 : 4;
    using H = Head<E, D / 2, NEAR>;
    const int tid = threadIdx.x, l = tid % L, group = tid / L;
    const bool on = D != 96 || l < D / 8;            // (96 wide: twelve lanes of sixteen)
    constexpr bool RUN = NEAR && sizeof(E) == 2;     // eight values in a row
    constexpr int SECOND = RUN ? 4 : D / 2;          // where the lane's other four begin
    const int own = on ? (RUN ? 8 * l : 4 * l) : 0;  // the lane's first value
    const int pairs = on ? (NEAR ? own : 8 * l) : 0, more_pairs = NEAR ? SECOND : 4;      // and its cosines and sines
    f32x4 w[2][2], sums[2][2] = {};                  // weights of queries and keys, by pair; their gradients
#pragma unroll
    for (int x = 0; x < 2; ++x) {
        const float* p = x ? A.k_weight : A.q_weight;
        f32x4_any first = {1.f, 1.f, 1.f, 1.f}, second = first;
        if (p) {
            first = *(const f32x4_any*)(p + own);
            second = *(const f32x4_any*)(p + own + SECOND);
        }
        w[x][0] = NEAR ? f32x4{first[0], first[2], second[0], second[2]} : f32x4{first[0], first[1], first[2], first[3]};
        w[x][1] = NEAR ? f32x4{first[1], first[3], second[1], second[3]} : f32x4{second[0], second[1], second[2], second[3]};
    }
    const int parts = 1 << lg_parts;
    const int64_t all = A.rows << lg_parts, step = (int64_t)gridDim.x * GROUPS;
    for (int64_t work = (int64_t)blockIdx.x * GROUPS + group; work < all; work += step) {
        const int64_t row = work >> lg_parts;
        const int part = (int)work & (parts - 1);
        const int64_t position = A.table ? A.positions[row] : 0;
        bool none = false;
        f32x4 cosine = {1.f, 1.f, 1.f, 1.f}, sine = {0.f, 0.f, 0.f, 0.f};
        auto look_up = [&] {
            none = (uint64_t)position >= (uint64_t)A.n_positions;
            const float* t = A.table + (none ? 0 : position) * D + pairs;
            const f32x4 x = *(const f32x4*)t, y = *(const f32x4*)(t + more_pairs);
            cosine = __builtin_shufflevector(x, y, 0, 2, 4, 6);
            sine = __builtin_shufflevector(x, y, 1, 3, 5, 7);
        };
        auto turn = [&](auto kind) {                 // the row's heads of one kind
            constexpr int x = decltype(kind)::value;
            const int n = x ? A.kv_heads : A.heads, h0 = x ? (part - A.heads) & (parts - 1) : part;
            const int64_t in_step = (x ? A.k_head : A.q_head) << lg_parts, step = (int64_t)D << lg_parts, dense = (row * n + h0) * D + own;
            const E* in = x ? (const E*)A.k + row * A.k_row + h0 * A.k_head + own : (const E*)A.q + row * A.q_row + h0 * A.q_head + own;
            const E* grad = (const E*)(x ? A.dk_out : A.dq_out) + dense;
            E* to = (E*)(x ? A.k_to : A.q_to) + dense;
            H v[AHEAD], g[BACK ? AHEAD : 1];
            bool first = x == 0;
            for (int left = n - h0; left > 0; left -= parts * AHEAD) {
#pragma unroll
                for (int j = 0; j < AHEAD; ++j) {
                    if (j * parts < left) {
                        v[j].load(in);
                        if constexpr (BACK) g[j].load(grad);
                    }
                    in += in_step;
                    if constexpr (BACK) grad += step;
                }
                if (first && A.table) look_up();     // the first heads are asked for before the position has arrived
                first = false;
#pragma unroll
                for (int j = 0; j < AHEAD; ++j) {
                    if (j * parts >= left) break;
                    f32x4 &a = v[j].a, &b = v[j].b;
                    const f32x4 zero = {0.f, 0.f, 0.f, 0.f};
                    if (D == 96 && !on) a = b = zero;
                    const f32x4 squares = a * a + b * b;
                    const float r = rsqrtf(sum_of_head<D>((squares[0] + squares[1]) + (squares[2] + squares[3])) * (1.f / D) + A.eps);
                    if constexpr (!BACK) {
                        const f32x4 y = a * r * w[x][0], z = b * r * w[x][1];
                        a = y * cosine - z * sine;
                        b = z * cosine + y * sine;
                        if (none) a = b = zero;
                    } else {
                        f32x4 &ga = g[j].a, &gb = g[j].b;
                        if (none || (D == 96 && !on)) a = b = ga = gb = zero;
                        const float by = none ? 0.f : r;
                        const f32x4 ua = ga * cosine + gb * sine, ub = gb * cosine - ga * sine;
                        a *= by;
                        b *= by;
                        sums[x][0] += ua * a;
                        sums[x][1] += ub * b;
                        const f32x4 ea = ua * w[x][0], eb = ub * w[x][1], both = ea * a + eb * b;
                        const float dot = sum_of_head<D>((both[0] + both[1]) + (both[2] + both[3])) * (1.f / D);
                        a = by * (ea - a * dot);
                        b = by * (eb - b * dot);
                    }
                    if (on) v[j].store(to);
                    to += step;
                }
            }
            if (first && A.table) look_up();         // none of the queries' heads are this group's
        };
        turn(std::integral_constant<int, 0>{});
        turn(std::integral_constant<int, 1>{});
    }
    if constexpr (BACK) {                            // the workgroup's sums for the weights, its groups in their order
        __shared__ float part_of[GROUPS][D + 1];
#pragma unroll
        for (int x = 0; x < 2; ++x) {
            __syncthreads();
            if (on)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int at = own + (NEAR ? (i < 2 ? 2 * i : SECOND + 2 * i - 4) : i);
                    part_of[group][at] = sums[x][0][i];
                    part_of[group][at + (NEAR ? 1 : D / 2)] = sums[x][1][i];
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

// Adds up the workgroups' sums for the weights, in a fixed order and not by atomics: 16 values a workgroup, 64 threads each.  Of up to
// 1,024 workgroups, 4 to 5 us, a launch and two rounds of loads.
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

// Heads of a row are dealt to several groups where rows are few: until there are 2^19 lanes.  (Forward, bf16, us, with 2^17, 2^19 and 2^21:
// 11 thousand rows of 10 heads of 128 11.4, 13.7 and 16.0; 20 thousand of 24 heads of 64 22.1, 20.6 and 32.5; 54 thousand 75.6, 68.5 and
// 77.3; up to 2.7 thousand alike.)
int lg_parts_of(const RotateArgs& A, int lanes) {
    int lg = 0;
    while (2 << lg <= A.heads + A.kv_heads && (A.rows * lanes << lg) < 1 << 19) ++lg;
    return lg;
}
constexpr int64_t kMostGroups = 1024, kMostForward = 0xffffffffll / kThreads;        // of the backward pass; what a launch can have
int64_t groups_of(const RotateArgs& A, int lg_parts, int lanes, bool back) {
    const int64_t per = kThreads / lanes, groups = ((A.rows << lg_parts) + per - 1) / per, most = back ? kMostGroups : kMostForward;
    return groups > most ? most : groups;
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
    const int lg_parts = lg_parts_of(A, lanes_of(d));
    const dim3 grid((unsigned)groups_of(A, lg_parts, lanes_of(d), BACK));
    return by_width(d, [&](auto dc) {
        constexpr int D = decltype(dc)::value;
        auto go = [&](auto* e, auto near) {
            using E = std::remove_pointer_t<decltype(e)>;
            k_rotate<E, D, decltype(near)::value, BACK><<<grid, kThreads, 0, st>>>(A, lg_parts);
            return hipGetLastError();
        };
        if (dt == TR_BF16) return A.near ? go((__bf16*)nullptr, std::true_type{}) : go((__bf16*)nullptr, std::false_type{});
        return A.near ? go((float*)nullptr, std::true_type{}) : go((float*)nullptr, std::false_type{});
    });
}

}  // namespace

namespace {
int64_t parts_of(const RotateArgs& A, int d) { return groups_of(A, lg_parts_of(A, lanes_of(d)), lanes_of(d), true); }
}
size_t rotate_workspace_bytes(const RotateArgs& A, int d) { return (size_t)(parts_of(A, d) * 2 * d * 4 + 255) / 256 * 256; }

hipError_t launch_rotate(const RotateArgs& A, int d, int dt, hipStream_t st) {
    return A.rows == 0 ? hipSuccess : launch<false>(A, d, dt, st);
}
hipError_t launch_rotate_backward(const RotateArgs& A, int d, int dt, float* dq_weight, float* dk_weight, hipStream_t st) {
    if (A.rows) {
        const hipError_t e = launch<true>(A, d, dt, st);
        if (e != hipSuccess) return e;
    }
    if (!dq_weight && !dk_weight) return hipSuccess;
    k_rotate_join<<<dim3((unsigned)(2 * d / kJoinValues)), kJoinThreads, 0, st>>>(A.part, A.rows ? (int)parts_of(A, d) : 0, d, dq_weight,
                                                                                  dk_weight);
    return hipGetLastError();
}

}  // namespace cb
