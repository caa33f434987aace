// Matrices made nearly orthogonal by a quintic polynomial of their singular values, several steps of it.
#include <type_traits>

#include "cb_ortho.h"
#include "cb_tile.h"
#include "cb_train.h"

namespace cb {

namespace {

// X <- a X + B X, B = b A + c A^2, A = X X^T, with X of the smaller side's rows (a tall matrix is transposed as it comes in and as it
// goes out), divided by its Frobenius norm at first.  The polynomial raises small singular values by a factor of a each step, so what
// is lost of X or A at first is raised as well: products of single 16-bit values are 1e-3 off at the end, of two bf16 pieces 3e-5.
// Here X, A and B are held as two fp16 pieces each, 22 bits, a product is three products of pieces (the fourth is 2^-22 of it), and
// sums are in 32 bits: the result is as far from 64 bits (1.7e-6) as that of plain 32-bit products, at a third of the 16-bit rate
// instead of a sixteenth.  fp16 has few exponents: pieces are held times a power of two that puts the largest possible value (the
// host knows how far the polynomial can take a singular value) just below overflow, so that second pieces are normal numbers.
constexpr float kScaleX = 8192.f, kScaleA = 2048.f, kScaleB = 1024.f;

typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x4 __attribute__((ext_vector_type(4)));

// Pieces lie in lines of 128 bytes: 32 consecutive values of a row, all first pieces and then all second ones.
constexpr int kLine = 128;
__device__ __forceinline__ char* line_at(char* base, int row, int blocks, int block) {
    return base + ((int64_t)row * blocks + block) * kLine;
}
__device__ __forceinline__ const char* line_at(const char* base, int row, int blocks, int block) {
    return base + ((int64_t)row * blocks + block) * kLine;
}
__device__ __forceinline__ void split(const f32x4& x, f16x4& first, f16x4& second) {
    first = __builtin_convertvector(x, f16x4);
    second = __builtin_convertvector(x - __builtin_convertvector(first, f32x4), f16x4);
}
__device__ __forceinline__ void store_line(char* line, int at, const f32x4& x) {
    f16x4 first, second;
    split(x, first, second);
    *(f16x4*)(line + 2 * at) = first;
    *(f16x4*)(line + 64 + 2 * at) = second;
}
__device__ __forceinline__ f32x4 load_line(const char* line, int at) {
    return __builtin_convertvector(*(const f16x4*)(line + 2 * at), f32x4) + __builtin_convertvector(*(const f16x4*)(line + 64 + 2 * at), f32x4);
}

template <class F> __device__ __forceinline__ int find_matrix(const OrthoTable& t, uint32_t block, F&& first) {
    int lo = 0, hi = t.n;
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (first(mid) <= block) lo = mid; else hi = mid;
    }
    return lo;
}

constexpr int kThreads = 256;

// ---- in -------------------------------------------------------------------------------------------------------
constexpr int64_t kNormChunk = 8192;

template <class E> __device__ __forceinline__ double squares_of(const E* p, int count) {
    double sum = 0.0;
    for (int i = threadIdx.x; i < count; i += kThreads) {
        const double x = (double)(float)p[i];
        sum = fma(x, x, sum);
    }
    return sum;
}
__device__ __forceinline__ double block_total(double x) {
    __shared__ double s[kThreads / 64];
#pragma unroll
    for (int m = 1; m < 64; m <<= 1) x += __shfl_xor(x, m);
    __syncthreads();
    if ((threadIdx.x & 63) == 0) s[threadIdx.x >> 6] = x;
    __syncthreads();
    return (s[0] + s[1]) + (s[2] + s[3]);
}

// Sums of squares, in 64 bits, of chunks of each matrix.
__global__ __launch_bounds__(kThreads) void k_ortho_norm(const OrthoTable t, double* parts) {
    const int i = find_matrix(t, blockIdx.x, [&](int j) { return t.of[j].chunk0; });
    const OrthoMatrix& M = t.of[i];
    const int64_t size = (int64_t)M.m * M.n, first = (int64_t)(blockIdx.x - M.chunk0) * kNormChunk;
    const int count = (int)(size - first < kNormChunk ? size - first : kNormChunk);
    const double sum = block_total(M.bf16 ? squares_of((const __bf16*)M.in + first, count) : squares_of((const float*)M.in + first, count));
    if (threadIdx.x == 0) parts[blockIdx.x] = sum;
}

// Pieces of 64 x 64 values of X: of a row that is none, zeros.
constexpr int kSide = 64;
template <class E> __device__ __forceinline__ void load_side(const E* p, const OrthoMatrix& M, int i0, int j0, double by, float (*to)[kSide + 1]) {
    for (int x = threadIdx.x; x < kSide * kSide; x += kThreads) {
        const int r = x / kSide, c = x % kSide;
        if (!M.tall) {
            to[r][c] = i0 + r < M.m && j0 + c < M.n ? (float)((double)(float)p[(int64_t)(i0 + r) * M.n + j0 + c] * by) : 0.f;
        } else {
            to[c][r] = i0 + c < M.m && j0 + r < M.n ? (float)((double)(float)p[(int64_t)(j0 + r) * M.m + i0 + c] * by) : 0.f;
        }
    }
}
__global__ __launch_bounds__(kThreads) void k_ortho_in(const OrthoTable t, const double* parts, char* ws) {
    __shared__ float side[kSide][kSide + 1];
    const int i = find_matrix(t, blockIdx.x, [&](int j) { return t.of[j].side0; });
    const OrthoMatrix& M = t.of[i];
    const int chunks = (int)(((int64_t)M.m * M.n + kNormChunk - 1) / kNormChunk);
    double sum = 0.0;
    for (int c = threadIdx.x; c < chunks; c += kThreads) sum += parts[M.chunk0 + c];
    sum = block_total(sum);
    // a matrix of zeros stays one; one that is not finite is NaN everywhere, as its products would be
    const double by = sum == 0.0 ? 0.0 : sum < (double)INFINITY ? (double)kScaleX / sqrt(sum) : (double)NAN;
    const int blocks = M.np / 32, across = M.np / kSide, at = blockIdx.x - M.side0;
    const int i0 = at / across * kSide, j0 = at % across * kSide;
    if (M.bf16) load_side((const __bf16*)M.in, M, i0, j0, by, side);
    else load_side((const float*)M.in, M, i0, j0, by, side);
    __syncthreads();
    const int r = threadIdx.x / 4, c = threadIdx.x % 4 * 16;
    char* line = line_at(ws + M.x, i0 + r, blocks, (j0 + c) / 32);
#pragma unroll
    for (int q = 0; q < 4; ++q) {
        const float* x = &side[r][c + 4 * q];
        store_line(line, c % 32 + 4 * q, f32x4{x[0], x[1], x[2], x[3]});
    }
}

// ---- products ---------------------------------------------------------------------------------------------------
// C[i][j] = sum over k of P[i][k] Q[j][k], a tile of T x T by four wavefronts.  The wavefronts' accumulators have i in their columns,
// so that a lane's registers are runs of four j, which lie side by side in a line.
//   GRAM    A = X X^T                 P, Q: rows of X
//   SQUARE  B = b A + c A A           P, Q: rows of A, which is symmetric
//   APPLY   X' = a X + B X            P: rows of B; Q: columns of X, by transposing reads
// Symmetric products are made for tiles on and below the diagonal and stored twice.
// Tiles of 32 k of both operands pass through LDS, two of them, copied there by the memory unit.  A line's 16-byte pieces are turned
// by its row, so that sixteen rows' pieces (256 bytes, what LDS reads a clock) lie in different banks, and so do four rows' halves.
enum { GRAM, SQUARE, APPLY };

__device__ __forceinline__ int turn_of(int row) {
    const int x = row >> 1 & 7;
    return (x & 1) << 2 | x >> 1;
}
__device__ __forceinline__ f16x8 read_piece(lds_ptr p) { return *(const __attribute__((address_space(3))) f16x8*)(uintptr_t)p; }
__device__ __forceinline__ void mma(f32x16& acc, const f16x8& a, const f16x8& b) { acc = __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, acc, 0, 0, 0); }

template <int T, int STEP, bool LAST>
__global__ __launch_bounds__(kThreads, 2) void k_ortho_product(const OrthoTable t, char* ws, int odd, float a, float b, float c) {
    constexpr int NB = T / 64, BYTES = T * kLine;    // blocks of 32 of a wavefront's side; one operand's tile
    __shared__ __align__(256) char lds[2][2 * BYTES];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), n = lane & 31, h = lane >> 5;
    const int which = find_matrix(t, blockIdx.x, [&](int j) { return STEP == APPLY ? t.of[j].apply0 : t.of[j].square0; });
    const OrthoMatrix& M = t.of[which];
    const char* X = ws + (odd ? M.y : M.x);
    const int at = blockIdx.x - (STEP == APPLY ? M.apply0 : M.square0);
    int ti, tj;
    if constexpr (STEP == APPLY) {
        const int across = M.np / T;
        ti = at / across;
        tj = at - ti * across;
    } else {                                         // rows of the lower triangle, one after the other
        ti = (int)((sqrtf(8.f * (float)at + 1.f) - 1.f) * 0.5f);
        while ((ti + 1) * (ti + 2) / 2 <= at) ++ti;
        while (ti * (ti + 1) / 2 > at) --ti;
        tj = at - ti * (ti + 1) / 2;
    }
    const int i0 = ti * T, j0 = tj * T;
    const int x_blocks = M.np / 32, a_blocks = M.mp / 32;
    const char* P = STEP == GRAM ? X : ws + (STEP == SQUARE ? M.a : M.b);
    const int p_blocks = STEP == GRAM ? x_blocks : a_blocks, steps = p_blocks;
    auto issue = [&](int kb, int buf) {
#pragma unroll
        for (int x = 0; x < T / 32; ++x) {           // eight lines a wavefront
            const int line = x * 32 + wave * 8 + (lane >> 3), piece = (lane & 7) ^ turn_of(line);
            char* to = lds[buf] + (x * 32 + wave * 8) * kLine;
            copy_to_lds(line_at(P, i0 + line, p_blocks, kb) + piece * 16, to);
            const char* q = STEP == APPLY ? line_at(X, kb * 32 + (line & 31), x_blocks, j0 / 32 + (line >> 5)) : line_at(P, j0 + line, p_blocks, kb);
            copy_to_lds(q + piece * 16, to + BYTES);
        }
    };
    const int wi = (wave & 1) * (T / 2), wj = (wave >> 1) * (T / 2);
    const lds_ptr base = in_lds(lds[0]);
    // row operand: line `row`, eight values from 16 c + 8 h on; turned: sixteen lanes read four rows of sixteen values
    const lds_ptr p_place = base + (uint32_t)((wi + n) * kLine), q_place = base + (uint32_t)(BYTES + (wj + n) * kLine);
    const int t_row = 8 * h + ((lane & 15) >> 2), t_piece = ((lane >> 4) & 1) * 2 + ((lane & 3) >> 1);
    f32x16 acc[NB][NB] = {};                         // [j][i]
    issue(0, 0);
    wait_for_copies();
    __syncthreads();
    for (int kb = 0; kb < steps; ++kb) {
        const int buf = kb & 1;
        if (kb + 1 < steps) issue(kb + 1, buf ^ 1);
        const uint32_t from = (uint32_t)(buf * 2 * BYTES);
#pragma unroll
        for (int s = 0; s < 2; ++s) {
            f16x8 p[NB][2], q[NB][2];
#pragma unroll
            for (int x = 0; x < NB; ++x)
#pragma unroll
                for (int y = 0; y < 2; ++y) {
                    const uint32_t piece = (uint32_t)(((2 * s + h + 4 * y) ^ turn_of(n)) << 4);
                    p[x][y] = read_piece(p_place + from + (uint32_t)(x * 32 * kLine) + piece);
                    if constexpr (STEP != APPLY) {
                        q[x][y] = read_piece(q_place + from + (uint32_t)(x * 32 * kLine) + piece);
                    } else {
                        auto place = [&](int row) {
                            return base + from + (uint32_t)(BYTES + (wj + 32 * x + row) * kLine + (((t_piece + 4 * y) ^ turn_of(row)) << 4) + (lane & 1) * 8);
                        };
                        q[x][y] = __builtin_bit_cast(f16x8, read_turned(place(16 * s + t_row), place(16 * s + t_row + 4)));
                    }
                }
#pragma unroll
            for (int x = 0; x < NB; ++x)
#pragma unroll
                for (int y = 0; y < NB; ++y) {       // the smallest first
                    mma(acc[x][y], q[x][1], p[y][0]);
                    mma(acc[x][y], q[x][0], p[y][1]);
                    mma(acc[x][y], q[x][0], p[y][0]);
                }
        }
        wait_for_copies();
        __syncthreads();
    }
#pragma unroll
    for (int x = 0; x < NB; ++x)
#pragma unroll
        for (int y = 0; y < NB; ++y) {
            const int i = i0 + wi + 32 * y + n, jb = j0 + wj + 32 * x;
            f32x16& v = acc[x][y];
            if constexpr (STEP != APPLY) {
                char* to = ws + (STEP == GRAM ? M.a : M.b);
                if constexpr (STEP == GRAM) v *= kScaleA / (kScaleX * kScaleX);
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    const int j = 8 * r + 4 * h;
                    f32x4 z = {v[4 * r], v[4 * r + 1], v[4 * r + 2], v[4 * r + 3]};
                    if constexpr (STEP == SQUARE) {
                        z = z * (c * (kScaleB / (kScaleA * kScaleA))) + load_line(line_at(P, i, a_blocks, jb / 32), j) * (b * (kScaleB / kScaleA));
                    }
                    store_line(line_at(to, i, a_blocks, jb / 32), j, z);
                    if (ti != tj) {                  // its other half
                        f16x4 first, second;
                        split(z, first, second);
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            char* line = line_at(to, jb + j + e, a_blocks, i / 32);
                            *(_Float16*)(line + 2 * n) = first[e];
                            *(_Float16*)(line + 64 + 2 * n) = second[e];
                        }
                    }
                }
            } else {
                const float by = kScaleX / (kScaleB * kScaleX);
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    const int j = 8 * r + 4 * h;
                    f32x4 z = f32x4{v[4 * r], v[4 * r + 1], v[4 * r + 2], v[4 * r + 3]} * by + load_line(line_at(X, i, x_blocks, jb / 32), j) * a;
                    if constexpr (!LAST) {
                        store_line(line_at(ws + (odd ? M.x : M.y), i, x_blocks, jb / 32), j, z);
                    } else {
                        z *= 1.f / kScaleX;
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            if (i >= M.m || jb + j + e >= M.n) continue;
                            const int64_t place = M.tall ? (int64_t)(jb + j + e) * M.m + i : (int64_t)i * M.n + jb + j + e;
                            if (M.bf16) ((__bf16*)M.out)[place] = (__bf16)z[e]; else ((float*)M.out)[place] = z[e];
                        }
                    }
                }
            }
        }
}

int64_t round_up(int64_t x, int64_t to) { return (x + to - 1) / to * to; }

// The matrices from `first` on that one series of launches takes, and what it needs.
struct OrthoGroup { OrthoTable t; int64_t end, chunks, sides, squares, applies; size_t parts, bytes; int tile; };
OrthoGroup group_from(int64_t first, int64_t n, const int64_t* rows, const int64_t* cols, const void* const* in, void* const* out,
                      const int32_t* dts) {
    OrthoGroup G = {};
    G.end = first + kOrthoTable < n ? first + kOrthoTable : n;
    int64_t wide_tiles = 0;                          // of 128, in the products that have fewest
    for (int64_t i = first; i < G.end; ++i) {
        const int64_t m = rows[i] < cols[i] ? rows[i] : cols[i], across = (m + 127) / 128;
        wide_tiles += across * (across + 1) / 2;
    }
    G.tile = wide_tiles >= 256 ? 128 : 64;
    size_t at = 0;
    auto take = [&](int64_t bytes) {
        const size_t x = at;
        at += (size_t)round_up(bytes, 256);
        return x;
    };
    for (int64_t i = first; i < G.end; ++i) {
        if (!rows[i] || !cols[i]) continue;
        OrthoMatrix& M = G.t.of[G.t.n++];
        M.tall = rows[i] > cols[i];
        M.m = (int)(M.tall ? cols[i] : rows[i]);
        M.n = (int)(M.tall ? rows[i] : cols[i]);
        M.mp = (int)round_up(M.m, G.tile);
        M.np = (int)round_up(M.n, G.tile);
        M.in = in ? in[i] : nullptr;
        M.out = out ? out[i] : nullptr;
        M.bf16 = dts && dts[i] == TR_BF16;
        M.chunk0 = (uint32_t)G.chunks;
        M.side0 = (uint32_t)G.sides;
        M.square0 = (uint32_t)G.squares;
        M.apply0 = (uint32_t)G.applies;
        const int64_t ti = M.mp / G.tile, tj = M.np / G.tile;
        G.chunks += ((int64_t)M.m * M.n + kNormChunk - 1) / kNormChunk;
        G.sides += (int64_t)(M.mp / kSide) * (M.np / kSide);
        G.squares += ti * (ti + 1) / 2;
        G.applies += ti * tj;
        const int64_t x = (int64_t)M.mp * M.np * 4, a = (int64_t)M.mp * M.mp * 4;
        M.x = take(x);
        M.y = take(x);
        M.a = take(a);
        M.b = take(a);
    }
    G.parts = take(G.chunks * 8);
    G.bytes = at;
    return G;
}

template <int T> hipError_t launch_group(const OrthoGroup& G, char* ws, int steps, const float* k, hipStream_t st) {
    double* parts = (double*)(ws + G.parts);
    k_ortho_norm<<<dim3((unsigned)G.chunks), kThreads, 0, st>>>(G.t, parts);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    k_ortho_in<<<dim3((unsigned)G.sides), kThreads, 0, st>>>(G.t, parts, ws);
    e = hipGetLastError();
    for (int s = 0; s < steps && e == hipSuccess; ++s) {
        const int odd = s & 1;
        k_ortho_product<T, GRAM, false><<<dim3((unsigned)G.squares), kThreads, 0, st>>>(G.t, ws, odd, k[0], k[1], k[2]);
        if ((e = hipGetLastError()) != hipSuccess) break;
        k_ortho_product<T, SQUARE, false><<<dim3((unsigned)G.squares), kThreads, 0, st>>>(G.t, ws, odd, k[0], k[1], k[2]);
        if ((e = hipGetLastError()) != hipSuccess) break;
        if (s + 1 < steps) k_ortho_product<T, APPLY, false><<<dim3((unsigned)G.applies), kThreads, 0, st>>>(G.t, ws, odd, k[0], k[1], k[2]);
        else k_ortho_product<T, APPLY, true><<<dim3((unsigned)G.applies), kThreads, 0, st>>>(G.t, ws, odd, k[0], k[1], k[2]);
        e = hipGetLastError();
    }
    return e;
}

}  // namespace

size_t ortho_workspace_bytes(int64_t n, const int64_t* rows, const int64_t* cols) {
    size_t most = 0;
    for (int64_t i = 0; i < n;) {
        const OrthoGroup G = group_from(i, n, rows, cols, nullptr, nullptr, nullptr);
        if (G.bytes > most) most = G.bytes;
        i = G.end;
    }
    return most;
}

bool ortho_launchable(int64_t n, const int64_t* rows, const int64_t* cols) {
    constexpr int64_t most = 0xffffffffll / kThreads;
    for (int64_t i = 0; i < n;) {
        const OrthoGroup G = group_from(i, n, rows, cols, nullptr, nullptr, nullptr);
        if (G.chunks > most || G.sides > most || G.squares > most || G.applies > most) return false;
        i = G.end;
    }
    return true;
}

// Groups use the workspace one after the other.
hipError_t launch_ortho(int64_t n, const void* const* in, void* const* out, const int64_t* rows, const int64_t* cols, const int32_t* dts,
                        int steps, const float* coefficients, char* ws, hipStream_t st) {
    for (int64_t i = 0; i < n;) {
        const OrthoGroup G = group_from(i, n, rows, cols, in, out, dts);
        i = G.end;
        if (!G.t.n) continue;
        const hipError_t e = G.tile == 128 ? launch_group<128>(G, ws, steps, coefficients, st) : launch_group<64>(G, ws, steps, coefficients, st);
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

}  // namespace cb
