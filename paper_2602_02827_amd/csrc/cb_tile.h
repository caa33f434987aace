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
//   fp32   the same instruction, whose rate is sixteen times that of the 32-bit ones, on three bf16 pieces of eight bits of every
//          value: six products of pieces a step, the three smallest (2^-22 of a product together) left out
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
    template <bool TURNED = false> static __device__ __forceinline__ void mma(f32x16& acc, const Frag& a, const Frag& b) {
        acc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, acc, 0, 0, 0);
    }
    static __device__ __forceinline__ Frag round(const f32x8& x) { return __builtin_convertvector(x, bf16x8); }
    static __device__ __forceinline__ f32x8 wide(const Frag& x) { return __builtin_convertvector(x, f32x8); }
    static __device__ __forceinline__ Frag load(const void* p) { return *(const bf16x8*)p; }
    static __device__ __forceinline__ void store4(__bf16* p, const f32x4& x) { *(bf16x4*)p = __builtin_convertvector(x, bf16x4); }
};
template <> struct Oper<float> {
    // The first piece is cut off, so that it never overflows, the others are rounded; their sum is the value.
    struct Frag {
        bf16x8 p[3];
        __device__ __forceinline__ Frag operator-() const { return {{-p[0], -p[1], -p[2]}}; }
    };
    static constexpr int ROWS = 32;
    // TURNED: the operands are in each other's place; the result is the same to the last bit.
    template <bool TURNED = false> static __device__ __forceinline__ void mma(f32x16& acc, const Frag& a, const Frag& b) {
        constexpr int X[6] = {2, 0, 1, 1, 0, 0}, Y[6] = {0, 2, 1, 0, 1, 0};       // the smallest first
#pragma unroll
        for (int i = 0; i < 6; ++i)
            acc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a.p[TURNED ? Y[i] : X[i]], b.p[TURNED ? X[i] : Y[i]], acc, 0, 0, 0);
    }
    static __device__ __forceinline__ Frag round(const f32x8& x) {
        f32x8 first;
#pragma unroll
        for (int i = 0; i < 8; ++i) first[i] = __uint_as_float(__float_as_uint(x[i]) & 0xffff0000u);
        Frag f;
        f.p[0] = __builtin_convertvector(first, bf16x8);
        const f32x8 rest = x - first;
        f.p[1] = __builtin_convertvector(rest, bf16x8);
        f.p[2] = __builtin_convertvector(rest - __builtin_convertvector(f.p[1], f32x8), bf16x8);
        return f;
    }
    static __device__ __forceinline__ f32x8 wide(const Frag& x) {
        return __builtin_convertvector(x.p[0], f32x8) + (__builtin_convertvector(x.p[1], f32x8) + __builtin_convertvector(x.p[2], f32x8));
    }
    static __device__ __forceinline__ Frag load(const void* p) {
        const f32x4 a = *(const f32x4*)p, b = *((const f32x4*)p + 1);
        return round(__builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7));
    }
    static __device__ __forceinline__ void store4(float* p, const f32x4& x) { *(f32x4*)p = x; }
};

// ROWS rows of D values in LDS, as 16-byte pieces of bf16.  A piece's place in its row is turned by the row's low bits.  256 bytes
// are read a clock: sixteen rows' pieces of one column (row operands) lie in different banks, and so do the four rows of 64 bytes
// that half a wavefront takes of a turned operand (128-byte and 256-byte rows: by the turn's upper bits; the others by their pitch).
// All that a lane's places differ by is then a constant, added or (below 256, tiles are aligned to that) toggled.
template <int ROWS, int D> struct Plane {
    static constexpr int PITCH = 2 * D, PIECES = PITCH / 16, BYTES = ROWS * PITCH;
    static constexpr bool POWER = (PIECES & (PIECES - 1)) == 0;
    static __device__ __forceinline__ int turn(int row) {
        if constexpr (PIECES % 16 == 0) return ((row & 3) << 2) | ((row >> 2) & 3);
        if constexpr (PIECES % 8 == 0) return ((row & 2) << 1) | ((row >> 2) & 3);
        return (row >> 2) & 3;
    }
    static __device__ __forceinline__ int at(int row, int piece) { return row * PITCH + ((piece ^ turn(row)) << 4); }
    // row operands: row n, piece 2c + h
    static __device__ __forceinline__ uint32_t row_place(int lane) { return (uint32_t)at(lane & 31, lane >> 5); }
    static __device__ __forceinline__ uint32_t row_place(uint32_t p, int b, int c) {
        return (p ^ (uint32_t)((POWER ? c : c & 1) << 5)) + (uint32_t)(32 * b * PITCH + (POWER ? 0 : (c >> 1) * 64));
    }
    // turned operands: sixteen lanes read four rows of sixteen values and get a column of four each; eight rows on for the other four
    static __device__ __forceinline__ uint32_t turned_place(int lane) {
        return (uint32_t)(at(4 * (lane >> 5) + ((lane & 15) >> 2), ((lane >> 4) & 1) * 2 + ((lane & 3) >> 1)) + (lane & 1) * 8);
    }
    static __device__ __forceinline__ uint32_t turned_place(uint32_t p, int b, int c, int db, int half) {
        return (p ^ (uint32_t)((half << 5) | (POWER ? db << 6 : 0))) + (uint32_t)((32 * b + 16 * c + 8 * half) * PITCH + (POWER ? 0 : db * 64));
    }
};
using lds_ptr = uint32_t;                             // an address in LDS
__device__ __forceinline__ lds_ptr in_lds(const void* p) { return (lds_ptr)(uintptr_t)(const __attribute__((address_space(3))) char*)p; }
__device__ __forceinline__ bf16x8 read_row(lds_ptr p) { return *(const __attribute__((address_space(3))) bf16x8*)(uintptr_t)p; }
__device__ __forceinline__ bf16x8 read_turned(lds_ptr p, lds_ptr q) {
    using L = __attribute__((address_space(3))) i16x4;
    const i16x4 a = __builtin_amdgcn_ds_read_tr16_b64_v4i16((L*)(uintptr_t)p), b = __builtin_amdgcn_ds_read_tr16_b64_v4i16((L*)(uintptr_t)q);
    const auto both = __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7);
    return __builtin_bit_cast(bf16x8, both);
}

// A tile: one plane, or one of each piece.  R rows of it.
template <class E, int D, int R = Oper<E>::ROWS> struct Tile {
    using O = Oper<E>;
    using Frag = typename O::Frag;
    static constexpr int ROWS = R, PLANES = sizeof(E) == 2 ? 1 : 3;
    using P = Plane<ROWS, D>;
    static constexpr int PIECES = P::PIECES, BYTES = PLANES * P::BYTES;
    // a lane's places in a tile
    struct At {
        lds_ptr row, turned;
        __device__ __forceinline__ At(const char* t, int lane) : row(in_lds(t) + P::row_place(lane)), turned(in_lds(t) + P::turned_place(lane)) {}
        __device__ __forceinline__ At(lds_ptr r, lds_ptr u) : row(r), turned(u) {}
        __device__ __forceinline__ At operator+(int bytes) const { return At(row + bytes, turned + bytes); }
    };
    // rows 32b .. 32b+31, elements 16c .. 16c+15 of each
    static __device__ __forceinline__ Frag rows(const At& t, int b, int c) {
        const lds_ptr p = P::row_place(t.row, b, c);
        if constexpr (PLANES == 1) return read_row(p);
        else return {{read_row(p), read_row(p + P::BYTES), read_row(p + 2 * P::BYTES)}};
    }
    // columns 32db .. 32db+31 of the rows 32b + 16c .. +15, in the accumulators' order
    static __device__ __forceinline__ Frag turned(const At& t, int b, int c, int db) {
        const lds_ptr x = P::turned_place(t.turned, b, c, db, 0), y = P::turned_place(t.turned, b, c, db, 1);
        if constexpr (PLANES == 1) return read_turned(x, y);
        else return {{read_turned(x, y), read_turned(x + P::BYTES, y + P::BYTES), read_turned(x + 2 * P::BYTES, y + 2 * P::BYTES)}};
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
// Matrix instructions and LDS accesses stay on their side, others may move across.
__device__ __forceinline__ void in_turn() { __builtin_amdgcn_sched_barrier(0x406); }

// Sixteen bytes a lane from memory to LDS without registers: lane i's, from base + offset, go to dst + 16 i (base, dst: the same for
// the wavefront).  Every copy is waited for, and followed by a barrier, before its bytes are read and before the wavefront ends.
// The instruction is written out because the compiler, for its own builtin, waits for all copies under way before the next read of any
// LDS, which it cannot tell from theirs, so that nothing would be a tile ahead.
__device__ __forceinline__ void copy_to_lds(const void* base, uint32_t offset, char* dst) {
    const uint32_t to = __builtin_amdgcn_readfirstlane((uint32_t)(uintptr_t)dst);      // (LDS begins at a whole multiple of 4 GiB)
    const uint64_t at = (uint64_t)(uintptr_t)base;
    const uint64_t from = (uint64_t)(uint32_t)__builtin_amdgcn_readfirstlane((uint32_t)(at >> 32)) << 32 |
                          (uint32_t)__builtin_amdgcn_readfirstlane((uint32_t)at);
    uint32_t before;                                 // m0 is left as it was
    asm volatile("s_mov_b32 %0, m0\n\ts_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %2, %3\n\ts_mov_b32 m0, %0"
                 : "=&s"(before) : "s"(to), "v"(offset), "s"(from) : "memory");
}
// All but the last N of the wavefront's copies and loads have arrived.  By the builtin, which the compiler counts: loads from before a
// loop, were their wait not known to it, would be waited for in every turn, and the copies under way with them.
template <int N = 0> __device__ __forceinline__ void wait_for_copies() {
    static_assert(N < 64, "a count of six bits");
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_waitcnt((N & 15) | (N >> 4) << 14 | 0xf70);       // the other counters: any
    asm volatile("" ::: "memory");
}

// Where tiles are copied by the memory unit: said at the top of a loop over tiles, where nothing is under way, for the compiler, which
// else finds ways around the waits that are never gone, and waits for the copies in the middle of the turn.
template <class E> __device__ __forceinline__ void settle() {
    if constexpr (sizeof(E) == 2) wait_for_copies();
}

// A matrix's rows on their way to a tile in LDS, a tile ahead of its use, rows past the end as the last row again.  16 bits: by the
// memory unit itself.  32 bits: they wait in registers, and are cut into their pieces as they are written.
// at(row): byte offset of a row; whole(i): whether the i-th piece of this thread is kept (zeros otherwise).
template <class E, int D, int THREADS, int R = Oper<E>::ROWS> struct Rows {
    using T = Tile<E, D, R>;
    static constexpr int ALL = T::ROWS * T::PIECES, N = (ALL + THREADS - 1) / THREADS;
    static constexpr bool DIRECT = sizeof(E) == 2;
    f32x4 x[DIRECT ? 1 : N][2];
    static __device__ __forceinline__ int row(int i, int tid) { return (i * THREADS + tid) / T::PIECES; }
    static __device__ __forceinline__ uint32_t piece(int i, int tid) {
        return (uint32_t)(((i * THREADS + tid) % T::PIECES ^ T::P::turn(row(i, tid))) * 8 * (int)sizeof(E));
    }
    template <class At> __device__ __forceinline__ void issue(const char* a, char* lds, int rows, int tid, int wave, At&& at) {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            if (ALL % THREADS && i * THREADS + wave * 64 >= ALL) break;          // of the wavefront
            const int place = row(i, tid);
            const uint32_t offset = at(place < rows ? place : rows - 1) + piece(i, tid);
            if constexpr (DIRECT) {
                copy_to_lds(a, offset, lds + (i * THREADS + wave * 64) * 16);
            } else {
                const char* src = a + offset;
                x[i][0] = *(const f32x4*)src;
                x[i][1] = *((const f32x4*)src + 1);
            }
        }
    }
    template <class Whole> __device__ __forceinline__ void finish(char* lds, int tid, Whole&& whole) const {
        if constexpr (DIRECT) wait_for_copies();
#pragma unroll
        for (int i = 0; i < N; ++i) {
            if (ALL % THREADS && i * THREADS + tid >= ALL) break;
            char* to = lds + (i * THREADS + tid) * 16;
            if constexpr (DIRECT) {
                if (!whole(i)) *(u32x4*)to = u32x4{0u, 0u, 0u, 0u};      // its own pieces have arrived
            } else {
                const f32x8 v = __builtin_shufflevector(x[i][0], x[i][1], 0, 1, 2, 3, 4, 5, 6, 7);
                const auto f = Oper<E>::round(whole(i) ? v : f32x8{0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f});
#pragma unroll
                for (int p = 0; p < 3; ++p) *(bf16x8*)(to + p * T::P::BYTES) = f.p[p];
            }
        }
    }
};

// Tiles of ragged sequences: sequence i begins at place off[i] / per + i, which leaves room for all its tiles of `per` rows
// and needs no table.  Rows behind the last sequence follow as one more.  Finds the sequence of a place (all lanes of a wavefront together), 64 offsets at a time.
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
// The same for the sequence of a place, of n; rest: the place is one of the rows behind the last sequence, and these are meant.
__device__ __forceinline__ Range rows_of_place(const int64_t* off, int i, int n, int total, int per, int place, bool& rest) {
    const Range r = sequence_rows(off, i, total, per);
    const int end = r.lo + r.n, after = place_of(end, n, per, total);
    rest = i == n - 1 && place >= after;
    return rest ? Range{end, total - end, after} : r;
}

}  // namespace cb
