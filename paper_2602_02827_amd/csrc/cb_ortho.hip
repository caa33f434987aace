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
// host knows how far the polynomial can take a singular value) just below overflow.  Second pieces of what is more than 2^11 below that
// are no normal numbers any more: whatever a value's size, 2^-40 of the matrix' norm is lost of it.  In a matrix whose rows or columns
// are of very different sizes that is all there is of some, and each step raises it with them.  So that is the rule, by the steps'
// polynomial and the sizes: WIDE, where what is lost could be raised to more than kLost of the result, or where small values become
// smaller, X, A and B are held in 32 bits, and cut into three bf16 pieces as they are multiplied (six products of pieces, what is left
// out is 2^-26).  (128 x 512, rows that fall to 10^-8 of the first, twelve usual steps: 7.7e-5 off in pieces, 7e-7 so, plain 32-bit
// products 3e-6; five steps: 5e-7, 3e-7 and 1.4e-6.  An encoder's 25 matrices, five steps: 1,575 us in pieces, 3,280 WIDE; one of 768 x 128: 99 and
// 155.)
constexpr double kLost = 0x1p-19;
constexpr double kSmallest = 0x1p-24 / 3.4641016151377544;       // root mean square of a second piece's rounding, of which 2^-24 is the last place

typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x4 __attribute__((ext_vector_type(4)));

// Values lie in lines of 128 bytes: 32 consecutive ones of a row, all first pieces and then all second ones, or 32 bits each.  The lines of a block
// of 32 columns follow one another, so that what a tile reads at once lies side by side (with a row's lines side by side the rows of a
// tile lie a few KB apart, in a quarter of the L2's channels).
constexpr int kLine = 128;
__device__ __forceinline__ char* line_at(char* base, int row, int rows, int block) {
    return base + ((int64_t)block * rows + row) * kLine;
}
__device__ __forceinline__ const char* line_at(const char* base, int row, int rows, int block) {
    return base + ((int64_t)block * rows + row) * kLine;
}
__device__ __forceinline__ void split(const f32x4& x, f16x4& first, f16x4& second) {
    first = __builtin_convertvector(x, f16x4);
    second = __builtin_convertvector(x - __builtin_convertvector(first, f32x4), f16x4);
}
template <bool WIDE> __device__ __forceinline__ void store_line(char* line, int at, const f32x4& x) {
    if constexpr (WIDE) {
        *(f32x4*)(line + 4 * at) = x;
    } else {
        f16x4 first, second;
        split(x, first, second);
        *(f16x4*)(line + 2 * at) = first;
        *(f16x4*)(line + 64 + 2 * at) = second;
    }
}
__device__ __forceinline__ void split(const f32x8& x, f16x8& first, f16x8& second) {
    first = __builtin_convertvector(x, f16x8);
    second = __builtin_convertvector(x - __builtin_convertvector(first, f32x8), f16x8);
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

// Eight values at a time where they lie at a whole multiple of sixteen bytes.
__device__ __forceinline__ f32x8 load_eight(const float* p) {
    return __builtin_shufflevector(*(const f32x4*)p, *(const f32x4*)(p + 4), 0, 1, 2, 3, 4, 5, 6, 7);
}
__device__ __forceinline__ f32x8 load_eight(const __bf16* p) { return __builtin_convertvector(*(const bf16x8*)p, f32x8); }
template <class E> __device__ __forceinline__ double squares_of(const E* p, int count) {
    double sum = 0.0, more = 0.0;
    const int eights = ((uintptr_t)p & 15) ? 0 : count / 8;
#pragma unroll 4
    for (int i = threadIdx.x; i < eights; i += kThreads) {
        const f32x8 x = load_eight(p + 8 * i);
#pragma unroll
        for (int e = 0; e < 8; e += 2) {
            sum = fma((double)x[e], (double)x[e], sum);
            more = fma((double)x[e + 1], (double)x[e + 1], more);
        }
    }
    for (int i = 8 * eights + threadIdx.x; i < count; i += kThreads) {
        const double x = (double)(float)p[i];
        sum = fma(x, x, sum);
    }
    return sum + more;
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

// Sums of squares, in 64 bits (no matrix of finite values overflows or vanishes), of chunks of each matrix.  32 million bf16 values: 16 us,
// 4 TB/s; the next kernel's sums of a matrix's chunks, and its pieces, 38 us (64 MB read, 128 MB written).
__global__ __launch_bounds__(kThreads) void k_ortho_norm(const OrthoTable t, double* parts, OrthoTable* table) {
    // the others read the table from memory, where a second one finds it in L2 (the same nine matrices: 139 us from a kernel's arguments,
    // 131 so)
    if (blockIdx.x == 0)
        for (int i = threadIdx.x; i < (int)(sizeof t / 4); i += kThreads) ((uint32_t*)table)[i] = ((const uint32_t*)&t)[i];
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
    const int across = M.tall ? M.m : M.n, r0 = M.tall ? j0 : i0, c0 = M.tall ? i0 : j0;
    if (across % 8 == 0 && ((uintptr_t)p & 15) == 0) {
#pragma unroll
        for (int y = 0; y < kSide * kSide / 8 / kThreads; ++y) {
            const int x = y * kThreads + threadIdx.x, r = x / (kSide / 8), c = x % (kSide / 8) * 8;
            f32x8 v = {};
            if (r0 + r < (M.tall ? M.n : M.m) && c0 + c < across) v = load_eight(p + (int64_t)(r0 + r) * across + c0 + c);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const float z = (float)((double)v[e] * by);
                if (M.tall) to[c + e][r] = z; else to[r][c + e] = z;
            }
        }
        return;
    }
    for (int x = threadIdx.x; x < kSide * kSide; x += kThreads) {
        const int r = x / kSide, c = x % kSide;
        if (!M.tall) {
            to[r][c] = i0 + r < M.m && j0 + c < M.n ? (float)((double)(float)p[(int64_t)(i0 + r) * M.n + j0 + c] * by) : 0.f;
        } else {
            to[c][r] = i0 + c < M.m && j0 + r < M.n ? (float)((double)(float)p[(int64_t)(j0 + r) * M.m + i0 + c] * by) : 0.f;
        }
    }
}
template <bool WIDE>
__global__ __launch_bounds__(kThreads) void k_ortho_in(const OrthoTable* __restrict__ table, const double* parts, char* ws, float scale) {
    const OrthoTable& t = *table;
    __shared__ float side[kSide][kSide + 1];
    const int i = find_matrix(t, blockIdx.x, [&](int j) { return t.of[j].side0; });
    const OrthoMatrix& M = t.of[i];
    const int chunks = (int)(((int64_t)M.m * M.n + kNormChunk - 1) / kNormChunk);
    double sum = 0.0;
    for (int c = threadIdx.x; c < chunks; c += kThreads) sum += parts[M.chunk0 + c];
    sum = block_total(sum);
    // a matrix of zeros stays one; one that is not finite is NaN everywhere, as its products would be
    const double by = sum == 0.0 ? 0.0 : sum < (double)INFINITY ? (double)scale / sqrt(sum) : (double)NAN;
    const int across = M.np / kSide, at = blockIdx.x - M.side0;
    const int i0 = at / across * kSide, j0 = at % across * kSide;
    if (M.bf16) load_side((const __bf16*)M.in, M, i0, j0, by, side);
    else load_side((const float*)M.in, M, i0, j0, by, side);
    __syncthreads();
    const int r = threadIdx.x / 4, c = threadIdx.x % 4 * 16;
    char* line = line_at(ws + M.x, i0 + r, M.mp, (j0 + c) / 32);
#pragma unroll
    for (int q = 0; q < 4; ++q) {
        const float* x = &side[r][c + 4 * q];
        store_line<WIDE>(line, c % 32 + 4 * q, f32x4{x[0], x[1], x[2], x[3]});
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
// Each XCD has tiles that follow one another, of as much work as any other's: a matrix is then read into one L2 and not into eight.
// Launches go through the matrices there and back: what one wrote last, the next reads first, from the last-level cache.
// Bound by the matrix units and by memory in turn: of all matrices of six layers of 768 (32 million values, 422 GFLOP in five steps, three
// times that as products of pieces), one step's launches take 104, 46 and 155 us (830 TFLOP/s of pieces), of which the products alone 72,
// 22 and 74.  What is left is mostly the way of a finished tile to memory, 64 KB, through LDS and with what it is added to: a workgroup's
// products are 24 to 96 turns, too few to hide it behind those of the other workgroup on the CU, which ends at about the same time (to
// delay every second one made no difference).  A 768 x 128 matrix: 97 us for 17 launches that depend on each other, 4 to 9 us each.
enum { GRAM, SQUARE, APPLY };

__device__ __forceinline__ int turn_of(int row) {
    const int x = row >> 1 & 7;
    return (x & 1) << 2 | x >> 1;
}
__device__ __forceinline__ f16x8 read_piece(lds_ptr p) { return *(const __attribute__((address_space(3))) f16x8*)(uintptr_t)p; }
__device__ __forceinline__ void mma(f32x16& acc, const f16x8& a, const f16x8& b) { acc = __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, acc, 0, 0, 0); }
__device__ __forceinline__ f32x4 read_four(lds_ptr p) { return *(const __attribute__((address_space(3))) f32x4*)(uintptr_t)p; }
__device__ __forceinline__ float read_one(lds_ptr p) { return *(const __attribute__((address_space(3))) float*)(uintptr_t)p; }

// (WIDE) Eight values cut into three pieces, each rounded: what they leave is 2^-27 of a value.
struct Cut {
    bf16x8 p[3];
    __device__ __forceinline__ Cut() {}
    __device__ __forceinline__ explicit Cut(const f32x8& x) {
        p[0] = __builtin_convertvector(x, bf16x8);
        const f32x8 rest = x - __builtin_convertvector(p[0], f32x8);
        p[1] = __builtin_convertvector(rest, bf16x8);
        p[2] = __builtin_convertvector(rest - __builtin_convertvector(p[1], f32x8), bf16x8);
    }
};
__device__ __forceinline__ void mma(f32x16& acc, const bf16x8& a, const bf16x8& b) { acc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, acc, 0, 0, 0); }

// Eight values of a row of the output, which has the input's shape.
__device__ __forceinline__ void store_row(const OrthoMatrix& M, int row, int col, const f32x8& z) {
    const int rows = M.tall ? M.n : M.m, cols = M.tall ? M.m : M.n;
    if (row >= rows || col >= cols) return;
    const int64_t at = (int64_t)row * cols + col;
    if (cols % 8 == 0 && ((uintptr_t)M.out & 15) == 0) {
        if (M.bf16) {
            *(bf16x8*)((__bf16*)M.out + at) = __builtin_convertvector(z, bf16x8);
        } else {
            *(f32x4*)((float*)M.out + at) = __builtin_shufflevector(z, z, 0, 1, 2, 3);
            *(f32x4*)((float*)M.out + at + 4) = __builtin_shufflevector(z, z, 4, 5, 6, 7);
        }
        return;
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        if (col + e >= cols) continue;
        if (M.bf16) ((__bf16*)M.out)[at + e] = (__bf16)z[e]; else ((float*)M.out)[at + e] = z[e];
    }
}

struct Piece { int row, col; };                      // of a tile: eight values from here on
template <bool WIDE> __device__ __forceinline__ void store_piece(char* line, const Piece& p, const f32x8& z) {
    if constexpr (WIDE) {
        f32x4* to = (f32x4*)(line + p.col % 32 * 4);
        to[0] = __builtin_shufflevector(z, z, 0, 1, 2, 3);
        to[1] = __builtin_shufflevector(z, z, 4, 5, 6, 7);
    } else {
        f16x8 first, second;
        split(z, first, second);
        *(f16x8*)(line + p.col % 32 * 2) = first;
        *(f16x8*)(line + 64 + p.col % 32 * 2) = second;
    }
}
// One as it is stored.
template <bool WIDE> struct Stored {
    f16x8 x[2];
    __device__ __forceinline__ void load(const char* line, const Piece& p) {
        x[0] = *(const f16x8*)(line + p.col % 32 * 2);
        x[1] = *(const f16x8*)(line + p.col % 32 * 2 + 64);
    }
    __device__ __forceinline__ f32x8 value() const { return __builtin_convertvector(x[0], f32x8) + __builtin_convertvector(x[1], f32x8); }
};
template <> struct Stored<true> {
    f32x4 x[2];
    __device__ __forceinline__ void load(const char* line, const Piece& p) {
        x[0] = *(const f32x4*)(line + p.col % 32 * 4);
        x[1] = *(const f32x4*)(line + p.col % 32 * 4 + 16);
    }
    __device__ __forceinline__ f32x8 value() const { return __builtin_shufflevector(x[0], x[1], 0, 1, 2, 3, 4, 5, 6, 7); }
};

// DEEP: that many groups of four wavefronts share a tile, each with every DEEP-th tile of k; their sums are added in their order.
template <int T, int DEEP, int AHEAD, bool WIDE, int STEP, bool LAST>
__global__ __launch_bounds__(DEEP * kThreads, DEEP > 1 ? DEEP : 2) void k_ortho_product(const OrthoTable* __restrict__ table, char* ws, int odd,
                                                                                        int back, float scale, float more) {
    constexpr int NB = T / 64;                       // blocks of 32 of a wavefront's side
    constexpr int BYTES = 2 * T * kLine, COPIES = T / 16;
    __shared__ __align__(256) char lds[DEEP][AHEAD + 1][BYTES];
    static_assert(T * T * 4 <= (AHEAD + 1) * BYTES, "the tile goes through the same LDS");
    static_assert(DEEP == 1 || AHEAD == 1, "which copies are under way");
    const int tid = threadIdx.x, lane = tid & 63, n = lane & 31, h = lane >> 5;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6) % 4, deep = __builtin_amdgcn_readfirstlane(tid >> 6) / 4;
    const OrthoTable& t = *table;
    const OrthoEnds& ends = STEP == GRAM ? t.gram : STEP == SQUARE ? t.square : t.apply;
    const uint32_t first = ends.of[blockIdx.x % kXcds], behind = ends.of[blockIdx.x % kXcds + 1];
    if (blockIdx.x / kXcds >= behind - first) return;
    const uint32_t tile = back ? behind - 1 - blockIdx.x / kXcds : first + blockIdx.x / kXcds;
    const int which = find_matrix(t, tile, [&](int j) { return STEP == APPLY ? t.of[j].apply0 : t.of[j].square0; });
    const OrthoMatrix& M = t.of[which];
    const char* X = ws + (odd ? M.y : M.x);
    const int at = tile - (STEP == APPLY ? M.apply0 : M.square0);
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
    const int i0 = ti * T, j0 = tj * T, rows = M.mp;
    const char* P = STEP == GRAM ? X : ws + (STEP == SQUARE ? M.a : M.b);
    const int tiles = (STEP == GRAM ? M.np : M.mp) / 32, steps = (tiles + DEEP - 1) / DEEP;
    auto issue = [&](int s) {
        char* to = lds[deep][s % (AHEAD + 1)] + wave * 8 * kLine;      // eight lines a wavefront
        const int kb = s * DEEP + deep;
        if (DEEP > 1 && kb >= tiles) return;
        const char *p = line_at(P, i0, rows, kb), *q = STEP == APPLY ? line_at(X, kb * 32, rows, j0 / 32) : line_at(P, j0, rows, kb);
#pragma unroll
        for (int x = 0; x < COPIES / 2; ++x) {
            const int line = x * 32 + wave * 8 + (lane >> 3);
            const uint32_t piece = (uint32_t)((lane & 7) ^ turn_of(line)) * 16;
            copy_to_lds(p, (uint32_t)line * kLine + piece, to + x * 32 * kLine);
            copy_to_lds(q, (STEP == APPLY ? (uint32_t)(line >> 5) * (uint32_t)rows + (uint32_t)(line & 31) : (uint32_t)line) * kLine + piece,
                       to + (T + x * 32) * kLine);
        }
    };
    const int wi = (wave & 1) * (T / 2), wj = (wave >> 1) * (T / 2);
    const lds_ptr base = in_lds(lds[deep]);
    // row operand: line `row`, eight values from 16 c + 8 h on; turned: sixteen lanes read four rows of sixteen values
    const lds_ptr p_place = base + (uint32_t)((wi + n) * kLine), q_place = base + (uint32_t)((T + wj + n) * kLine);
    const int t_row = 8 * h + ((lane & 15) >> 2), t_piece = ((lane >> 4) & 1) * 2 + ((lane & 3) >> 1);
    // what the product is added to: a thread's pieces of eight values, a block's lines one after the other
    constexpr int ALL = T * T / 8, PIECES = (ALL + DEEP * kThreads - 1) / (DEEP * kThreads);
    const bool has = ALL % (DEEP * kThreads) == 0 || tid < ALL;
    auto piece_of = [&](int x) {
        const int p = x * DEEP * kThreads + tid;
        return Piece{(p >> 2) % T, (p >> 2) / T * 32 + (p & 3) * 8};
    };
    f32x16 acc[NB][NB] = {};                         // [j][i]
    // (WIDE) of all but the first pieces: small sums, which are rounded as such (12 usual steps of graded matrices: with one sum for all
    // of them 0.6 of plain 32-bit products' error, so 0.4)
    f32x16 more_acc[WIDE ? NB : 1][WIDE ? NB : 1] = {};
    for (int kb = 0; kb < AHEAD && kb < steps; ++kb) issue(kb);
    for (int kb = 0; kb < steps; ++kb) {
        // this tile's copies have arrived: those of AHEAD - 1 later ones may be under way
        if (kb + AHEAD - 1 < steps) wait_for_copies<(AHEAD - 1) * COPIES>(); else wait_for_copies();
        __syncthreads();                             // everyone's, and nobody reads the one before any more
        if (kb + AHEAD < steps) issue(kb + AHEAD);
        const uint32_t from = (uint32_t)(kb % (AHEAD + 1) * BYTES);
        if (DEEP > 1 && kb * DEEP + deep >= tiles) continue;
        if constexpr (WIDE) {
            auto row_operand = [&](lds_ptr line, int s) {
                const lds_ptr at = line + from + (uint32_t)(((4 * s + 2 * h) ^ turn_of(n)) << 4);
                return Cut(__builtin_shufflevector(read_four(at), read_four(at ^ 16), 0, 1, 2, 3, 4, 5, 6, 7));
            };
#pragma unroll
            for (int s = 0; s < 2; ++s) {
                Cut p[NB], q[NB];
#pragma unroll
                for (int x = 0; x < NB; ++x) {
                    p[x] = row_operand(p_place + (uint32_t)(x * 32 * kLine), s);
                    if constexpr (STEP != APPLY) {
                        q[x] = row_operand(q_place + (uint32_t)(x * 32 * kLine), s);
                    } else {                         // column n of eight rows
                        f32x8 z;
#pragma unroll
                        for (int e = 0; e < 8; ++e) {
                            const int row = 16 * s + 8 * h + e;
                            z[e] = read_one(base + from + (uint32_t)((T + wj + 32 * x + row) * kLine + (((n >> 2) ^ turn_of(row)) << 4) + (n & 3) * 4));
                        }
                        q[x] = Cut(z);
                    }
                }
                constexpr int X[6] = {2, 0, 1, 1, 0, 0}, Y[6] = {0, 2, 1, 0, 1, 0};      // the smallest first
#pragma unroll
                for (int z = 0; z < 6; ++z)
#pragma unroll
                    for (int x = 0; x < NB; ++x)
#pragma unroll
                        for (int y = 0; y < NB; ++y) mma(z < 5 ? more_acc[x][y] : acc[x][y], q[x].p[X[z]], p[y].p[Y[z]]);
            }
            continue;
        }
        // all operands are asked for first: the products begin with the first ones while the others arrive
        f16x8 p[2][NB][2], q[2][NB][2];
#pragma unroll
        for (int s = 0; s < 2; ++s)
#pragma unroll
            for (int y = 1; y >= 0; --y) {
                const uint32_t piece = (uint32_t)(((2 * s + h + 4 * y) ^ turn_of(n)) << 4);
#pragma unroll
                for (int x = 0; x < NB; ++x) {
                    if constexpr (STEP != APPLY) {
                        q[s][x][y] = read_piece(q_place + from + (uint32_t)(x * 32 * kLine) + piece);
                    } else {
                        auto place = [&](int row) {
                            return base + from + (uint32_t)((T + wj + 32 * x + row) * kLine + (((t_piece + 4 * y) ^ turn_of(row)) << 4) + (lane & 1) * 8);
                        };
                        q[s][x][y] = __builtin_bit_cast(f16x8, read_turned(place(16 * s + t_row), place(16 * s + t_row + 4)));
                    }
                }
#pragma unroll
                for (int x = 0; x < NB; ++x) p[s][x][1 - y] = read_piece(p_place + from + (uint32_t)(x * 32 * kLine) + (piece ^ 64));
            }
        phase();
#pragma unroll
        for (int s = 0; s < 2; ++s)
#pragma unroll
            for (int z = 0; z < 3; ++z)              // the smallest first
#pragma unroll
                for (int x = 0; x < NB; ++x)
#pragma unroll
                    for (int y = 0; y < NB; ++y) mma(acc[x][y], q[s][x][z == 0], p[s][y][z == 1]);
    }
    if constexpr (WIDE)
#pragma unroll
        for (int x = 0; x < NB; ++x)
#pragma unroll
            for (int y = 0; y < NB; ++y) acc[x][y] += more_acc[x][y];
    // (before the products the first copies would be waited for together with it: 1,600 us instead of 1,576 for an encoder's matrices)
    Stored<WIDE> add[STEP == GRAM ? 1 : PIECES] = {};
    if constexpr (STEP != GRAM)
#pragma unroll
        for (int x = 0; x < PIECES; ++x) {
            if (!has) break;
            const Piece p = piece_of(x);
            add[x].load(line_at(STEP == SQUARE ? P : X, i0 + p.row, rows, (j0 + p.col) / 32), p);
        }
    __syncthreads();
    // The tile goes through LDS once more, in 32 bits, so that lines are read and written whole (from the accumulators a lane would
    // have eight bytes of each: twice as many requests to L2 as the products' operands).  Four values' places are turned by the row.
    float* tile_of = (float*)lds;
    auto place = [&](int i, int j) { return i * T + (((j >> 2) ^ (i & (T / 4 - 1))) << 2 | (j & 3)); };
#pragma unroll
    for (int x = 0; x < NB; ++x)
#pragma unroll
        for (int y = 0; y < NB; ++y)
#pragma unroll
            for (int r = 0; r < 4; ++r)
                *(f32x4*)(tile_of + deep * T * T + place(wi + 32 * y + n, wj + 32 * x + 8 * r + 4 * h)) =
                    f32x4{acc[x][y][4 * r], acc[x][y][4 * r + 1], acc[x][y][4 * r + 2], acc[x][y][4 * r + 3]};
    char* to = ws + (STEP == GRAM ? M.a : STEP == SQUARE ? M.b : odd ? M.x : M.y);
    const float by = STEP == GRAM ? (WIDE ? 1.f : kGramScale) : scale;
    constexpr bool AGAIN = STEP != GRAM || DEEP > 1;              // the transpose is stored from what was stored
    const bool mirrored = STEP != APPLY && ti != tj, again = STEP == APPLY ? LAST && M.tall : mirrored;
    __syncthreads();
#pragma unroll
    for (int x = 0; x < PIECES; ++x) {
        if (!has) break;
        const Piece p = piece_of(x);
        f32x8 z;
#pragma unroll
        for (int q = 0; q < 2; ++q) {
            f32x4 v = *(const f32x4*)(tile_of + place(p.row, p.col + 4 * q));
#pragma unroll
            for (int d = 1; d < DEEP; ++d) v += *(const f32x4*)(tile_of + d * T * T + place(p.row, p.col + 4 * q));
#pragma unroll
            for (int e = 0; e < 4; ++e) z[4 * q + e] = v[e] * by;
        }
        if constexpr (STEP != GRAM) z += add[x].value() * more;
        if constexpr (!LAST) store_piece<WIDE>(line_at(to, i0 + p.row, rows, (j0 + p.col) / 32), p, z);
        else if (!M.tall) store_row(M, i0 + p.row, j0 + p.col, z);
        if constexpr (AGAIN) {
            if (again)                               // each thread's own places
#pragma unroll
                for (int q = 0; q < 2; ++q)
                    *(f32x4*)(tile_of + place(p.row, p.col + 4 * q)) = f32x4{z[4 * q], z[4 * q + 1], z[4 * q + 2], z[4 * q + 3]};
        }
    }
    if (!again) return;                              // the tile is also, or only, stored as its transpose
    if constexpr (AGAIN) __syncthreads();
#pragma unroll 2
    for (int x = 0; x < PIECES; ++x) {
        if (!has) break;
        const Piece p = piece_of(x);                 // of the transpose
        f32x8 z;
#pragma unroll
        for (int e = 0; e < 8; ++e) z[e] = tile_of[place(p.col + e, p.row)] * (AGAIN ? 1.f : by);
        if constexpr (STEP == APPLY) store_row(M, j0 + p.row, i0 + p.col, z);
        else store_piece<WIDE>(line_at(to, j0 + p.row, rows, (i0 + p.col) / 32), p, z);
    }
}

int64_t round_up(int64_t x, int64_t to) { return (x + to - 1) / to * to; }

// Tiles of all matrices in eight runs of about the same work, a matrix's being tiles of `depth`.
template <class Depth> void share_out(const OrthoTable& t, OrthoEnds& ends, int64_t tiles, uint32_t OrthoMatrix::*first, Depth&& depth) {
    auto tiles_of = [&](int i) { return (i + 1 < t.n ? (int64_t)(t.of[i + 1].*first) : tiles) - (int64_t)(t.of[i].*first); };
    double all = 0.0, before = 0.0;
    for (int i = 0; i < t.n; ++i) all += (double)tiles_of(i) * depth(t.of[i]);
    int x = 1;
    for (int i = 0; i < t.n; ++i) {
        const double own = (double)tiles_of(i) * depth(t.of[i]);
        while (x < kXcds && before + own >= all * x / kXcds) {
            const int64_t at = (int64_t)((all * x / kXcds - before) / depth(t.of[i]) + 0.5);
            ends.of[x++] = (uint32_t)((int64_t)(t.of[i].*first) + (at < tiles_of(i) ? at : tiles_of(i)));
        }
        before += own;
    }
    while (x <= kXcds) ends.of[x++] = (uint32_t)tiles;
}

// The matrices from `first` on that one series of launches takes, and what it needs.
struct OrthoGroup { OrthoTable t; int64_t end, chunks, sides, squares, applies; size_t parts, table, bytes; int tile; };
OrthoGroup group_from(int64_t first, int64_t n, const int64_t* rows, const int64_t* cols, const void* const* in, void* const* out,
                      const int32_t* dts) {
    OrthoGroup G = {};
    G.end = first + kOrthoTable < n ? first + kOrthoTable : n;
    int64_t half = 0;                                // tiles of 128, in the products that have fewest
    for (int64_t i = first; i < G.end; ++i) {
        const int64_t m = rows[i] < cols[i] ? rows[i] : cols[i], across = (m + 127) / 128;
        half += across * (across + 1) / 2;
    }
    // Large tiles where they fill the CUs.  (Five steps, us, with 128 and 64: 16 matrices of 768 x 768, 336 such tiles, 705 and 740; 8 of
    // 1,024, 288, 730 and 834; 4 of 768, 84, 362 and 270; 24 of 384, 144, 266 and 225.  Some long sums gain below that too: 4 of 1,024,
    // 144, 472 and 505.)
    G.tile = half >= 256 ? 128 : 64;
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
    G.table = take(sizeof(OrthoTable));
    G.bytes = at;
    share_out(G.t, G.t.gram, G.squares, &OrthoMatrix::square0, [](const OrthoMatrix& M) { return M.np; });
    share_out(G.t, G.t.square, G.squares, &OrthoMatrix::square0, [](const OrthoMatrix& M) { return M.mp; });
    share_out(G.t, G.t.apply, G.applies, &OrthoMatrix::apply0, [](const OrthoMatrix& M) { return M.mp; });
    return G;
}

unsigned groups_of(const OrthoEnds& ends) {
    uint32_t most = 0;
    for (int x = 0; x < kXcds; ++x) most = ends.of[x + 1] - ends.of[x] > most ? ends.of[x + 1] - ends.of[x] : most;
    return most * kXcds;
}

// Tiles of 128 x 128 leave room for two workgroups a CU, one storing while the other multiplies, with copies one k tile ahead; of
// small matrices, in tiles of 64 x 64, the copies' latency is all there is: three ahead, or, where there is no more than one tile for
// each CU, four groups of wavefronts at a tile (nine fp32 matrices of up to 640 x 256: 152 us without, 139 so, 155 with them also
// where tiles are more).
template <bool WIDE, int STEP, bool LAST = false>
hipError_t launch_product(const OrthoGroup& G, const OrthoEnds& ends, char* ws, int odd, int back, const OrthoPolynomial& K, hipStream_t st) {
    const dim3 grid(groups_of(ends));
    const OrthoTable* t = (const OrthoTable*)(ws + G.table);
    // what a tile is multiplied by as it is stored, and what it is added to; the pieces' scales among them (the last step's are taken out)
    const float last = LAST ? 1.f / K.scale_x : 1.f;
    const float by = STEP == SQUARE ? K.c * (K.scale_b / (K.scale_a * K.scale_a)) : last / K.scale_b;       // (GRAM: a constant)
    const float more = STEP == SQUARE ? K.b * (K.scale_b / K.scale_a) : K.a * last;
    if (G.tile == 128) k_ortho_product<128, 1, 1, WIDE, STEP, LAST><<<grid, kThreads, 0, st>>>(t, ws, odd, back, by, more);
    else if (grid.x <= 256) k_ortho_product<64, 4, 1, WIDE, STEP, LAST><<<grid, 4 * kThreads, 0, st>>>(t, ws, odd, back, by, more);
    else k_ortho_product<64, 1, 3, WIDE, STEP, LAST><<<grid, kThreads, 0, st>>>(t, ws, odd, back, by, more);
    return hipGetLastError();
}

// Whether two pieces hold all matrices' values well enough for the polynomial's steps.
bool pieces_hold(const OrthoGroup& G, const OrthoPolynomial& K) {
    for (int i = 0; i < G.t.n; ++i)
        if (!(sqrt((double)G.t.of[i].m * G.t.of[i].n) * (kSmallest / K.scale_x) * K.raised <= kLost)) return false;
    return true;
}

template <bool WIDE> hipError_t launch_group(const OrthoGroup& G, char* ws, int steps, const OrthoPolynomial& K, hipStream_t st) {
    double* parts = (double*)(ws + G.parts);
    k_ortho_norm<<<dim3((unsigned)G.chunks), kThreads, 0, st>>>(G.t, parts, (OrthoTable*)(ws + G.table));
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    k_ortho_in<WIDE><<<dim3((unsigned)G.sides), kThreads, 0, st>>>((const OrthoTable*)(ws + G.table), parts, ws, K.scale_x);
    e = hipGetLastError();
    for (int s = 0; s < steps && e == hipSuccess; ++s) {
        const int odd = s & 1;
        if ((e = launch_product<WIDE, GRAM>(G, G.t.gram, ws, odd, s & 1, K, st)) != hipSuccess) break;
        if ((e = launch_product<WIDE, SQUARE>(G, G.t.square, ws, odd, ~s & 1, K, st)) != hipSuccess) break;
        e = s + 1 < steps ? launch_product<WIDE, APPLY>(G, G.t.apply, ws, odd, s & 1, K, st)
                          : launch_product<WIDE, APPLY, true>(G, G.t.apply, ws, odd, s & 1, K, st);
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
        if (G.chunks > most || G.sides > most || 8 * G.squares > most || 8 * G.applies > most) return false;
        i = G.end;
    }
    return true;
}

// Groups use the workspace one after the other.
hipError_t launch_ortho(int64_t n, const void* const* in, void* const* out, const int64_t* rows, const int64_t* cols, const int32_t* dts,
                        int steps, const OrthoPolynomial& polynomial, char* ws, hipStream_t st) {
    OrthoPolynomial whole = polynomial;
    whole.scale_x = whole.scale_a = whole.scale_b = 1.f;
    for (int64_t i = 0; i < n;) {
        const OrthoGroup G = group_from(i, n, rows, cols, in, out, dts);
        i = G.end;
        if (!G.t.n) continue;
        const hipError_t e = pieces_hold(G, polynomial) ? launch_group<false>(G, ws, steps, polynomial, st)
                                                        : launch_group<true>(G, ws, steps, whole, st);
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

}  // namespace cb
