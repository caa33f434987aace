// Device-side building blocks of the training kernels: tiles of matrix rows in LDS and the operands of the
// 32x32 matrix instructions that are read from them.  Written for gfx950 (64-lane wavefronts).
//
// Lane l of a wavefront has n = l & 31 and h = l >> 5.  An operand of one 16-deep step is eight values a lane:
//   row operand    row n (of A) or column n (of B), elements 16c + 8h .. +7 of the contracted axis
//   accumulator    column n, register r: row 8 * (r / 4) + 4 * h + r % 4
// A product of accumulators, as P V after S = Q K^T, contracts over the accumulator's rows.  Registers 8c .. 8c+7
// then are the B operand of step c as they are, if the A operand takes its eight elements in the same order: 16c + 4h
// .. +3 and 16c + 8 + 4h .. +3 (turned operand).  So probabilities never leave the registers they were computed in.
//   bf16   one v_mfma_f32_32x32x16_bf16 a step; turned operands by two transposing LDS reads of four rows each
//   fp32   eight v_mfma_f32_32x32x2_f32 a step, element e of both operands in the e-th
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace cb {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
typedef short i16x4 __attribute__((ext_vector_type(4)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x8 __attribute__((ext_vector_type(8)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

constexpr float LOG2E = 1.4426950408889634f, LN2 = 0.6931471805599453f;

__device__ __forceinline__ float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); }

template <class E> struct Oper;
template <> struct Oper<__bf16> {
    using Frag = bf16x8;
    static constexpr int ROWS = 64;                  // of a staged tile
    static __device__ __forceinline__ void mma(f32x16& acc, const Frag& a, const Frag& b) {
        acc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, acc, 0, 0, 0);
    }
    static __device__ __forceinline__ Frag round(const f32x8& x) { return __builtin_convertvector(x, bf16x8); }
    static __device__ __forceinline__ f32x8 wide(const Frag& x) { return __builtin_convertvector(x, f32x8); }
    static __device__ __forceinline__ Frag load(const void* p) { return *(const bf16x8*)p; }
    static __device__ __forceinline__ void store4(__bf16* p, const f32x4& x) { *(bf16x4*)p = __builtin_convertvector(x, bf16x4); }
};
template <> struct Oper<float> {
    using Frag = f32x8;
    static constexpr int ROWS = 32;
    static __device__ __forceinline__ void mma(f32x16& acc, const Frag& a, const Frag& b) {
#pragma unroll
        for (int e = 0; e < 8; ++e) acc = __builtin_amdgcn_mfma_f32_32x32x2f32(a[e], b[e], acc, 0, 0, 0);
    }
    static __device__ __forceinline__ Frag round(const f32x8& x) { return x; }
    static __device__ __forceinline__ f32x8 wide(const Frag& x) { return x; }
    static __device__ __forceinline__ Frag load(const void* p) {
        const f32x4 a = *(const f32x4*)p, b = *((const f32x4*)p + 1);
        return __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7);
    }
    static __device__ __forceinline__ void store4(float* p, const f32x4& x) { *(f32x4*)p = x; }
};

// ROWS rows of D values in LDS, as 16-byte pieces.  A piece's place in its row is turned by the row's low bits.  256 bytes are
// read a clock: sixteen rows' pieces of one column (row operands) lie in different banks, and so do the four rows of 64 bytes
// that half a wavefront takes of a turned operand in 16 bits (128-byte and 256-byte rows: by the turn's upper bits; the others
// by their pitch).
template <class E, int D> struct Tile {
    using Frag = typename Oper<E>::Frag;
    static constexpr int ROWS = Oper<E>::ROWS, PITCH = D * (int)sizeof(E), PIECES = PITCH / 16;
    static constexpr int BYTES = ROWS * PITCH;
    static __device__ __forceinline__ int turn(int row) {
        if constexpr (sizeof(E) == 4 && PIECES % 16 == 0) return (row & 3) | ((row >> 1) & 4) | ((row << 1) & 8);
        if constexpr (PIECES % 16 == 0) return ((row & 3) << 2) | ((row >> 2) & 3);
        if constexpr (PIECES % 8 == 0) return ((row & 2) << 1) | ((row >> 2) & 3);
        return (row >> 2) & 3;
    }
    static __device__ __forceinline__ int at(int row, int piece) { return row * PITCH + ((piece ^ turn(row)) << 4); }
    // rows 32b .. 32b+31, elements 16c .. 16c+15 of each
    static __device__ __forceinline__ Frag rows(const char* t, int lane, int b, int c) {
        const int n = lane & 31, h = lane >> 5;
        if constexpr (sizeof(E) == 2) {
            return *(const bf16x8*)(t + at(32 * b + n, 2 * c + h));
        } else {
            const f32x4 x = *(const f32x4*)(t + at(32 * b + n, 4 * c + 2 * h));
            const f32x4 y = *(const f32x4*)(t + at(32 * b + n, 4 * c + 2 * h + 1));
            return __builtin_shufflevector(x, y, 0, 1, 2, 3, 4, 5, 6, 7);
        }
    }
    // columns 32db .. 32db+31 of the rows 32b + 16c .. +15, in the accumulators' order
    static __device__ __forceinline__ Frag turned(const char* t, int lane, int b, int c, int db) {
        const int h = lane >> 5;
        if constexpr (sizeof(E) == 2) {
            // sixteen lanes read four rows of sixteen values and get a column of four each
            const int row = 32 * b + 16 * c + 4 * h + ((lane & 15) >> 2);
            const int piece = 4 * db + ((lane >> 4) & 1) * 2 + ((lane & 3) >> 1);
            const char* p = t + at(row, piece) + (lane & 1) * 8;
            using L = __attribute__((address_space(3))) i16x4;
            const i16x4 x = __builtin_amdgcn_ds_read_tr16_b64_v4i16((L*)p);
            const char* p8 = t + at(row + 8, piece) + (lane & 1) * 8;
            const i16x4 y = __builtin_amdgcn_ds_read_tr16_b64_v4i16((L*)p8);
            const auto both = __builtin_shufflevector(x, y, 0, 1, 2, 3, 4, 5, 6, 7);
            return __builtin_bit_cast(bf16x8, both);
        } else {
            const int col = 32 * db + (lane & 31);
            f32x8 r;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const int row = 32 * b + 16 * c + 8 * (e >> 2) + 4 * h + (e & 3);
                r[e] = *(const float*)(t + at(row, col >> 2) + (col & 3) * 4);
            }
            return r;
        }
    }
};

// The two halves of a column's rows are in lanes n and n + 32.
__device__ __forceinline__ float max_of_halves(float x) {
    const uint32_t u = __builtin_bit_cast(uint32_t, x);
    const auto s = __builtin_amdgcn_permlane32_swap(u, u, false, false);
    const uint32_t a = s[0], b = s[1];
    return fmaxf(__uint_as_float(a), __uint_as_float(b));
}
__device__ __forceinline__ float sum_of_halves(float x) {
    const uint32_t u = __builtin_bit_cast(uint32_t, x);
    const auto s = __builtin_amdgcn_permlane32_swap(u, u, false, false);
    const uint32_t a = s[0], b = s[1];
    return __uint_as_float(a) + __uint_as_float(b);
}

// The same value, but one that the compiler works out what depends on it from where it stands: addresses that a loop needs
// once a turn then take no registers over the whole of it.
__device__ __forceinline__ int here(int x) {
    asm volatile("" : "+v"(x));
    return x;
}

// The compiler moves nothing across: operands of the next products are not read while the registers are needed for these.
__device__ __forceinline__ void phase() { __builtin_amdgcn_sched_barrier(0); }

// Sixteen bytes a lane from memory to LDS without registers: lane i's go to dst + 16 i (dst: the same for the wavefront).
__device__ __forceinline__ void copy_to_lds(const void* src, char* dst) {
    using G = const __attribute__((address_space(1))) void;
    using L = __attribute__((address_space(3))) void;
    __builtin_amdgcn_global_load_lds((G*)src, (L*)dst, 16, 0, 0);
}
__device__ __forceinline__ void wait_for_copies() { asm volatile("s_waitcnt vmcnt(0)" ::: "memory"); }

// Tiles of ragged sequences: sequence i begins at place off[i] / per + i, which leaves room for all its tiles of `per` rows
// and needs no table.  Finds the sequence of a place (all lanes of a wavefront together), 64 offsets at a time.
__device__ __forceinline__ int place_of(int64_t x, int i, int per, int total) {
    x = x < 0 ? 0 : x > total ? total : x;
    return (int)((uint32_t)x / (uint32_t)per) + i;
}
__device__ __forceinline__ int find_sequence(const int64_t* off, int n, int per, int total, int place, int lane) {
    int lo = 0, hi = n;
    while (hi - lo > 1) {
        const int step = (hi - lo + 63) / 64;
        const int i = lo + lane * step;
        const unsigned long long le = __ballot(i < hi && place_of(off[i], i, per, total) <= place);
        const int c = le == ~0ull ? 64 : __builtin_ctzll(~le);   // of the first ones: also for offsets that are out of order
        if (c == 0) break;
        lo += (c - 1) * step;
        hi = lo + step < hi ? lo + step : hi;
    }
    return __builtin_amdgcn_readfirstlane(lo);
}
// Rows of sequence i (the same in all lanes), and the place of its first tile.
struct Range { int lo, n, place; };
__device__ __forceinline__ Range sequence_rows(const int64_t* off, int i, int total, int per = 1) {
    int64_t a = off[i], b = off[i + 1];
    a = a < 0 ? 0 : a > total ? total : a;
    b = b < a ? a : b > total ? total : b;
    return {(int)a, (int)(b - a), place_of(a, i, per, total)};
}

}  // namespace cb
