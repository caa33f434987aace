// Rows of a token table, scaled, and the table's gradient by sorted tokens.
#include <type_traits>

#include "cb_train.h"

namespace cb {

namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));

// V consecutive values in 32 bits: eight where one side has 16 bits, four where both have 32 (sixteen bytes a lane), and one where rows
// do not lie so.  (54 thousand rows of 768, a 32-bit table of 32,000 under 16-bit rows, with the gradient: pieces of eight 108 us, of four
// 115; 2,700 rows of 256 in 32 bits: 14.4 and 13.7.)
template <int V> struct Piece { float v[V]; };
template <int V> __device__ __forceinline__ Piece<V> load_piece(const float* p) {
    Piece<V> x;
    if constexpr (V > 1) {
#pragma unroll
        for (int q = 0; q < V / 4; ++q) {
            const f32x4 a = *((const f32x4*)p + q);
#pragma unroll
            for (int i = 0; i < 4; ++i) x.v[4 * q + i] = a[i];
        }
    } else {
        x.v[0] = *p;
    }
    return x;
}
template <int V> __device__ __forceinline__ Piece<V> load_piece(const __bf16* p) {
    Piece<V> x;
    if constexpr (V == 8) {
        const f32x8 a = __builtin_convertvector(*(const bf16x8*)p, f32x8);
#pragma unroll
        for (int i = 0; i < 8; ++i) x.v[i] = a[i];
    } else {
        x.v[0] = (float)*p;
    }
    return x;
}
template <int V> __device__ __forceinline__ void store_piece(float* p, const Piece<V>& x) {
    if constexpr (V == 8) {
        *(f32x4*)p = f32x4{x.v[0], x.v[1], x.v[2], x.v[3]};
        *((f32x4*)p + 1) = f32x4{x.v[4], x.v[5], x.v[6], x.v[7]};
    } else if constexpr (V == 4) {
        *(f32x4*)p = f32x4{x.v[0], x.v[1], x.v[2], x.v[3]};
    } else {
        *p = x.v[0];
    }
}
template <int V> __device__ __forceinline__ void store_piece(__bf16* p, const Piece<V>& x) {
    if constexpr (V == 8) {
        bf16x8 a;
#pragma unroll
        for (int i = 0; i < 8; ++i) a[i] = (__bf16)x.v[i];
        *(bf16x8*)p = a;
    } else {
        *p = (__bf16)x.v[0];
    }
}
template <class W, class O> constexpr int kMostPiece = sizeof(W) + sizeof(O) == 8 ? 4 : 8;

// Pieces of all rows are dealt to threads one after the other, so that no lane is left over whatever a row's width is.
struct Place { uint64_t row; uint32_t piece; };
__device__ __forceinline__ Place place_of_piece(uint64_t first, uint32_t more, uint32_t pieces) {
    const uint64_t row0 = first >> 32 ? first / pieces : (uint32_t)first / pieces;         // of the workgroup
    const uint32_t at = (uint32_t)(first - row0 * pieces) + more, r = at / pieces;
    return {row0 + r, at - r * pieces};
}

constexpr int kThreads = 256;

// out[i] = scale * table[tokens[i]], in 32 bits, rounded once.  Bound by memory: 54 thousand rows of 768, a 32-bit table under 16-bit rows,
// 35 us (83 MB written, and a table's rows read that come again from the last-level cache); one query of 32 tokens 2.5 us, a launch and
// two dependent loads.
template <class W, class O, int V, int U>
__global__ __launch_bounds__(kThreads) void k_embed(const W* table, int64_t table_row, const int64_t* tokens, uint64_t vocab, uint64_t n,
                                                    uint32_t pieces, float scale, O* out) {
    const uint64_t first = (uint64_t)blockIdx.x * (kThreads * U);
    Place at[U];
    uint64_t token[U];
    Piece<V> x[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
        at[u] = place_of_piece(first, u * kThreads + threadIdx.x, pieces);
        token[u] = at[u].row < n ? (uint64_t)tokens[at[u].row] : ~0ull;
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
        x[u] = {};
        if (token[u] < vocab) x[u] = load_piece<V>(table + (int64_t)token[u] * table_row + (int64_t)at[u].piece * V);
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
        if (at[u].row >= n) continue;
#pragma unroll
        for (int i = 0; i < V; ++i) x[u].v[i] = token[u] < vocab ? x[u].v[i] * scale : 0.f;
        store_piece<V>(out + (at[u].row * pieces + at[u].piece) * V, x[u]);
    }
}

// ---- gradient ------------------------------------------------------------------------------------------------
// dtable[v] = scale * sum of dout[i] over the i whose token is v, in the order of i: the same inputs give the same bits.
// First tokens are sorted, each workgroup having a range of the table's rows: it goes over all tokens, counts those below its range
// (which is where its part of the sorted list begins) and those of each row, and then puts its own into their places.  A wavefront
// has a run of consecutive tokens, so that the order of equal ones is that of the list.  It notes its own tokens as it comes by, and
// only goes over its run again where there are more of them than it has room for.  All workgroups read all tokens, from L2: 256 of them,
// so that this is done at once on all CUs; one sort by all of them together would be several dependent launches, of 3.6 us each.  54
// thousand tokens, 32,000 rows: 17 us; 2,700 tokens, 800 rows: 6 us.
constexpr int kSortThreads = 1024, kSortWaves = kSortThreads / 64, kMostRange = 960, kNoted = 512;

// A token in 32 bits, which rows are counted in.
constexpr uint32_t kNoToken = 0xffffffffu;
__device__ __forceinline__ uint32_t in_32_bits(int64_t token) { return (uint64_t)token >> 32 ? kNoToken : (uint32_t)token; }

__global__ __launch_bounds__(kSortThreads) void k_embed_sort(const int64_t* tokens, int n, int vocab, int range, int* starts, int* order) {
    extern __shared__ int place[];                   // [wavefront][row of the range]: counts, then next places
    __shared__ int below_of[kSortWaves], sums[kSortWaves];
    __shared__ int noted[kSortWaves][kNoted];
    __shared__ uint16_t noted_row[kSortWaves][kNoted];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int lo = blockIdx.x * range, rows = vocab - lo < range ? vocab - lo : range;
    int* own = place + wave * range;
    for (int i = tid; i < kSortWaves * range; i += kSortThreads) place[i] = 0;
    __syncthreads();
    const int each = ((n + kSortWaves - 1) / kSortWaves + 63) / 64 * 64;
    const int64_t run = (int64_t)wave * each;        // (n is below 2^31, a run's end may not be)
    const int begin = run < n ? (int)run : n, end = run + each < n ? (int)(run + each) : n;
    const uint64_t before_me = (1ull << lane) - 1ull;
    int below = 0, notes = 0;
    constexpr int AHEAD = 8;
    for (int i0 = begin; i0 < end; i0 += 64 * AHEAD) {
        int64_t t[AHEAD];                            // past the end: the last token, and none below
#pragma unroll
        for (int j = 0; j < AHEAD; ++j) t[j] = tokens[i0 + 64 * j + lane < end ? i0 + 64 * j + lane : end - 1];
#pragma unroll
        for (int j = 0; j < AHEAD; ++j) {
            const uint32_t x = i0 + 64 * j + lane < end ? in_32_bits(t[j]) : kNoToken, r = x - (uint32_t)lo;
            below += __popcll(__ballot(x < (uint32_t)lo));
            const bool mine = r < (uint32_t)rows;
            const uint64_t all = __ballot(mine);
            if (!all) continue;
            const int at = notes + __popcll(all & before_me);
            if (mine) {
                atomicAdd(own + r, 1);
                if (at < kNoted) {
                    noted[wave][at] = i0 + 64 * j + lane;
                    noted_row[wave][at] = (uint16_t)r;
                }
            }
            notes += __popcll(all);
        }
    }
    if (lane == 0) below_of[wave] = below;
    __syncthreads();
    // a row's tokens of all wavefronts, then those of the rows before it
    int count = 0;
    if (tid < rows)
        for (int w = 0; w < kSortWaves; ++w) {
            const int c = place[w * range + tid];
            place[w * range + tid] = count;
            count += c;
        }
    int upto = count;
#pragma unroll
    for (int m = 1; m < 64; m <<= 1) {
        const int x = __shfl_up(upto, m);
        upto += lane >= m ? x : 0;
    }
    if (lane == 63) sums[wave] = upto;
    __syncthreads();
    int first = upto - count;
    for (int w = 0; w < kSortWaves; ++w) first += below_of[w] + (w < wave ? sums[w] : 0);
    if (tid < rows) {
        starts[lo + tid] = first;
        if (lo + tid == vocab - 1) starts[vocab] = first + count;
        for (int w = 0; w < kSortWaves; ++w) place[w * range + tid] += first;
    }
    __syncthreads();
    // sixty-four of its tokens: row by row, a row's lanes in their order (r: -1 in lanes that have none)
    auto put = [&](int r, int position) {
        uint64_t left = __ballot(r >= 0);
        while (left) {
            const int row = __shfl(r, __builtin_ctzll(left));
            const uint64_t same = __ballot(r == row);
            if (r == row) {
                const int before = __popcll(same & before_me);
                const int at = own[row];
                order[at + before] = position;
                if (before == 0) own[row] = at + __popcll(same);
            }
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
            left &= ~same;
        }
    };
    if (notes <= kNoted) {
        for (int i = lane; i - lane < notes; i += 64) put(i < notes ? (int)noted_row[wave][i] : -1, i < notes ? noted[wave][i] : 0);
        return;
    }
    for (int i = begin; i < end; i += 64) {
        const uint32_t r = (end - i > lane ? in_32_bits(tokens[i + lane]) : kNoToken) - (uint32_t)lo;
        put(r < (uint32_t)rows ? (int)r : -1, i + lane);
    }
}

// Then rows are added up.  A row of up to kLong tokens, or of none, is one thread's sum for each piece.  The sorted list is cut into
// chunks of kLong, and what a chunk has of longer rows (at most of two: one that began before and one that goes on) is a sum of its
// own, joined by a second launch.
// Bound by memory, or by the most frequent tokens' rows (a row's additions are one after the other): 54 thousand rows of 768 in 16 bits,
// 49 us (83 MB read, 98 MB of the table written, 3.7 TB/s) and 6 us to join.  2,700 rows of 256 in 32 bits, 800 tokens: 3.5 and 2 us.
// (32-bit tables of 16-bit rows' gradients, us, with kLong 32, 64 and 128: 54 thousand tokens of 32,000, all alike, rows of 768, 50.8, 48.4
// and 47.4; of 300, rows of 256, 29.1, 35.9 and 52.1; the most frequent of 32,000 a tenth of all 205, 206 and 221.)
constexpr int kLong = 64;

// A piece as it is stored, so that many are under way in few registers.
template <class O, int V> struct Raw;
template <> struct Raw<__bf16, 8> { bf16x8 x; };
template <> struct Raw<float, 4> { f32x4 x; };
template <> struct Raw<float, 8> { f32x4 x[2]; };
template <class O> struct Raw<O, 1> { O x[1]; };

template <class O, int V>
__device__ __forceinline__ Piece<V> sum_of_tokens(const O* dout, int64_t dout_row, uint32_t piece, const int* order, int begin, int end) {
    constexpr int AHEAD = 8;
    Piece<V> sum = {};
#pragma unroll 1
    for (int i = begin; i < end; i += AHEAD) {
        Raw<O, V> x[AHEAD];
        int at[AHEAD];
#pragma unroll
        for (int j = 0; j < AHEAD; ++j) at[j] = i + j < end ? order[i + j] : -1;
#pragma unroll
        for (int j = 0; j < AHEAD; ++j) {
            x[j] = {};
            if (at[j] >= 0) x[j] = *(const Raw<O, V>*)(dout + at[j] * dout_row + (int64_t)piece * V);
        }
#pragma unroll
        for (int j = 0; j < AHEAD; ++j) {
            const Piece<V> y = load_piece<V>((const O*)&x[j]);
#pragma unroll
            for (int e = 0; e < V; ++e) sum.v[e] += y.v[e];
        }
    }
    return sum;
}

template <class W, class O, int V>
__global__ __launch_bounds__(kThreads) void k_embed_sum(const O* dout, int64_t dout_row, const int64_t* tokens, int vocab, uint32_t pieces,
                                                        const int* starts, const int* order, uint32_t chunk_groups, int chunks, float scale,
                                                        W* dtable, float* part) {
    if (blockIdx.x < chunk_groups) {
        const Place at = place_of_piece((uint64_t)blockIdx.x * kThreads, threadIdx.x, pieces);
        const int all = starts[vocab];
        if (at.row >= (uint64_t)chunks || (int64_t)at.row * kLong >= all) return;
        const int begin = (int)at.row * kLong, end = begin + kLong < all ? begin + kLong : all;
        const int64_t a = tokens[order[begin]], b = tokens[order[end - 1]];
        auto sum_part = [&](int64_t t, int slot) {
            const int from = starts[t], to = starts[t + 1];
            if (to - from <= kLong) return;
            const Piece<V> x = sum_of_tokens<O, V>(dout, dout_row, at.piece, order, from > begin ? from : begin, to < end ? to : end);
            store_piece<V>(part + ((int64_t)(2 * at.row + slot) * pieces + at.piece) * V, x);
        };
        sum_part(a, 0);
        if (b != a) sum_part(b, 1);
        return;
    }
    const Place at = place_of_piece((uint64_t)(blockIdx.x - chunk_groups) * kThreads, threadIdx.x, pieces);
    if (at.row >= (uint64_t)vocab) return;
    const int begin = starts[at.row], end = starts[at.row + 1];
    if (end - begin > kLong) return;
    Piece<V> x = sum_of_tokens<O, V>(dout, dout_row, at.piece, order, begin, end);
#pragma unroll
    for (int e = 0; e < V; ++e) x.v[e] *= scale;
    store_piece<V>(dtable + ((int64_t)at.row * pieces + at.piece) * V, x);
}

// Joins the chunks of long rows: a workgroup for kJoinPieces pieces of the long row that begins in a chunk, the chunks dealt to its
// other threads, whose sums are added in their order.
constexpr int kJoinPieces = 16, kJoinParts = kThreads / kJoinPieces;
template <class W, int V>
__global__ __launch_bounds__(kThreads) void k_embed_join(const int64_t* tokens, int vocab, uint32_t pieces, const int* starts, const int* order,
                                                         int groups, float scale, const float* part, W* dtable) {
    __shared__ Piece<V> sums[kJoinParts][kJoinPieces];
    const int chunk = blockIdx.x / groups, begin = chunk * kLong, all = starts[vocab];
    if (begin >= all) return;
    const int end = begin + kLong < all ? begin + kLong : all;
    const int64_t t = tokens[order[end - 1]];
    const int from = starts[t], to = starts[t + 1];
    if (to - from <= kLong || from < begin) return;
    const int last = (to - 1) / kLong, mine = threadIdx.x / kJoinPieces;
    const uint32_t piece = blockIdx.x % groups * kJoinPieces + threadIdx.x % kJoinPieces;
    Piece<V> sum = {};
    if (piece < pieces) {
#pragma unroll 4
        for (int c = chunk + mine; c <= last; c += kJoinParts) {
            const Raw<float, V> x = *(const Raw<float, V>*)(part + ((int64_t)(2 * (int64_t)c + (c == chunk && from > begin)) * pieces + piece) * V);
#pragma unroll
            for (int e = 0; e < V; ++e) sum.v[e] += ((const float*)&x)[e];
        }
    }
    sums[mine][threadIdx.x % kJoinPieces] = sum;
    __syncthreads();
    if (mine || piece >= pieces) return;
    for (int p = 1; p < kJoinParts; ++p)
#pragma unroll
        for (int e = 0; e < V; ++e) sum.v[e] += sums[p][threadIdx.x].v[e];
#pragma unroll
    for (int e = 0; e < V; ++e) sum.v[e] *= scale;
    store_piece<V>(dtable + (t * pieces + piece) * V, sum);
}

int64_t round_up(int64_t x) { return (x + 255) / 256 * 256; }
struct EmbedPlan { int range, groups, chunks; size_t order, part, bytes; };
EmbedPlan plan_embed(int64_t n, int64_t vocab, int64_t width) {
    EmbedPlan P = {};
    P.range = (int)((vocab + 255) / 256);
    if (P.range > kMostRange) P.range = kMostRange;
    P.groups = (int)((vocab + P.range - 1) / P.range);
    P.chunks = n > kLong ? (int)((n + kLong - 1) / kLong) : 0;           // (no row is long otherwise)
    P.order = (size_t)round_up((vocab + 1) * 4);
    P.part = P.order + (size_t)round_up(n * 4);
    P.bytes = P.part + (size_t)round_up(2 * (int64_t)P.chunks * width * 4);
    return P;
}

template <class F> hipError_t by_types(int w, int o, F&& f) {
    if (w == TR_F32) return o == TR_F32 ? f((float*)nullptr, (float*)nullptr) : f((float*)nullptr, (__bf16*)nullptr);
    return o == TR_F32 ? f((__bf16*)nullptr, (float*)nullptr) : f((__bf16*)nullptr, (__bf16*)nullptr);
}
int size_of(int dt) { return dt == TR_BF16 ? 2 : 4; }
}  // namespace

// Values of a piece; `rows` and `dense` are the two sides.
int embedding_piece(const void* rows, int rows_dt, int64_t row, const void* dense, int dense_dt, int64_t width) {
    const int v = rows_dt == TR_F32 && dense_dt == TR_F32 ? 4 : 8;
    auto lie = [&](const void* p, int64_t r, int dt) { return (uintptr_t)p % 16 == 0 && r * size_of(dt) % 16 == 0; };
    return width % v == 0 && lie(rows, row, rows_dt) && lie(dense, width, dense_dt) ? v : 1;
}
bool embedding_launchable(int64_t n, int64_t vocab, int64_t width, int piece, bool backward) {
    const int64_t pieces = width / piece, most = 0xffffffffll / kThreads;
    if (!backward) return (n * pieces + 4 * kThreads - 1) / (4 * kThreads) <= most;
    const EmbedPlan P = plan_embed(n, vocab, width);
    return (P.chunks * pieces + kThreads - 1) / kThreads + (vocab * pieces + kThreads - 1) / kThreads <= most &&
           P.chunks * ((pieces + kJoinPieces - 1) / kJoinPieces) <= most && P.groups <= 0xffffffffll / kSortThreads;
}

hipError_t launch_embedding(const void* table, int table_dt, int64_t table_row, const int64_t* tokens, int64_t n, int64_t vocab, int64_t width,
                            float scale, void* out, int out_dt, hipStream_t st) {
    if (n == 0) return hipSuccess;
    const bool wide = embedding_piece(table, table_dt, table_row, out, out_dt, width) > 1;
    return by_types(table_dt, out_dt, [&](auto* w, auto* o) {
        using W = std::remove_pointer_t<decltype(w)>;
        using O = std::remove_pointer_t<decltype(o)>;
        auto go = [&](auto vc, auto uc) {
            constexpr int V = decltype(vc)::value, U = decltype(uc)::value;
            const int64_t pieces = width / V, per = kThreads * U;
            k_embed<W, O, V, U><<<dim3((unsigned)((n * pieces + per - 1) / per)), kThreads, 0, st>>>(
                (const W*)table, table_row, tokens, (uint64_t)vocab, (uint64_t)n, (uint32_t)pieces, scale, (O*)out);
            return hipGetLastError();
        };
        using one = std::integral_constant<int, 1>;
        using four = std::integral_constant<int, 4>;
        using wide_piece = std::integral_constant<int, kMostPiece<W, O>>;
        // few pieces: a thread each, so that all are asked for at once; many: four, whose loads are under way together (us, a piece and four
        // pieces a thread: 340 rows of 768 in bf16, 2^15 pieces, 2.4 and 3.4; 54 thousand rows of 256 in fp32, 2^22, 17.7 and 17.3; in between
        // a piece is faster up to 2^19: 1,360 rows of 768 2.6 and 3.6, 5,400 4.2 and 4.7, 13 thousand 7.7 and 7.7)
        const bool few = n * (width / (wide ? wide_piece::value : 1)) <= 1 << 16;
        if (wide) return few ? go(wide_piece{}, one{}) : go(wide_piece{}, four{});
        return few ? go(one{}, one{}) : go(one{}, four{});
    });
}

size_t embedding_workspace_bytes(int64_t n, int64_t vocab, int64_t width) { return plan_embed(n, vocab, width).bytes; }

hipError_t launch_embedding_backward(const void* dout, int dout_dt, int64_t dout_row, const int64_t* tokens, int64_t n, int64_t vocab,
                                     int64_t width, float scale, void* dtable, int table_dt, char* ws, hipStream_t st) {
    const EmbedPlan P = plan_embed(n, vocab, width);
    int *starts = (int*)ws, *order = (int*)(ws + P.order);
    float* part = (float*)(ws + P.part);
    k_embed_sort<<<dim3((unsigned)P.groups), kSortThreads, kSortWaves * P.range * 4, st>>>(tokens, (int)n, (int)vocab, P.range, starts, order);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    const bool wide = embedding_piece(dout, dout_dt, dout_row, dtable, table_dt, width) > 1;
    return by_types(table_dt, dout_dt, [&](auto* w, auto* o) {
        using W = std::remove_pointer_t<decltype(w)>;
        using O = std::remove_pointer_t<decltype(o)>;
        auto go = [&](auto vc) {
            constexpr int V = decltype(vc)::value;
            const int64_t pieces = width / V, chunk_groups = (P.chunks * pieces + kThreads - 1) / kThreads,
                          row_groups = (vocab * pieces + kThreads - 1) / kThreads;
            k_embed_sum<W, O, V><<<dim3((unsigned)(chunk_groups + row_groups)), kThreads, 0, st>>>(
                (const O*)dout, dout_row, tokens, (int)vocab, (uint32_t)pieces, starts, order, (uint32_t)chunk_groups, P.chunks, scale, (W*)dtable,
                part);
            const hipError_t e = hipGetLastError();
            if (e != hipSuccess || !P.chunks) return e;
            const int groups = (int)((pieces + kJoinPieces - 1) / kJoinPieces);
            k_embed_join<W, V><<<dim3((unsigned)(P.chunks * (int64_t)groups)), kThreads, 0, st>>>(tokens, (int)vocab, (uint32_t)pieces, starts,
                                                                                               order, groups, scale, part, (W*)dtable);
            return hipGetLastError();
        };
        return wide ? go(std::integral_constant<int, kMostPiece<W, O>>{}) : go(std::integral_constant<int, 1>{});
    });
}

}  // namespace cb
