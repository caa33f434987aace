// Global gradient norm over many tensors, and the tensors clipped to it.
#include "cb_train.h"

namespace cb {

// Two launches for up to kTable tensors: squares into one partial sum a workgroup, then every workgroup of the second adds up the
// partial sums itself, in their order (they are few and in L2), and scales its share.  What is read last by the first is read
// first by the second, from the last-level cache where it fits.  Bound by memory: 57 million fp32 values, 48 us for the norm (4.7
// TB/s) and 78 us for the scaling (226 MB in and out, 5.8 TB/s); a single small matrix by its two launches (5 us each).
// Four workgroups a CU: 133 us in a row and 135 with cold caches, with eight 132 and 139, with two 169; chunks of half and twice the
// size 134 and 137.
constexpr int kTable = 128, kThreads = 256, kMostParts = 1024;
constexpr int64_t kChunk = 8192;                     // values of a chunk; a chunk has one tensor

struct ClipTable {
    const void* in[kTable];
    void* out[kTable];
    int64_t size[kTable];
    uint32_t chunk0[kTable + 1];                     // first chunk of each tensor
    uint8_t bf16[kTable];
    int n;
};

struct Chunk { int tensor; int64_t first; int count; };
__device__ __forceinline__ Chunk find_chunk(const ClipTable& t, uint32_t c) {
    int lo = 0, hi = t.n;
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (t.chunk0[mid] <= c) lo = mid; else hi = mid;
    }
    const int64_t first = (int64_t)(c - t.chunk0[lo]) * kChunk, left = t.size[lo] - first;
    return {lo, first, (int)(left < kChunk ? left : kChunk)};
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

__device__ __forceinline__ float bf16_low(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float bf16_high(uint32_t w) { return __uint_as_float(w & 0xffff0000u); }
__device__ __forceinline__ uint16_t to_bf16(float x) { return __builtin_bit_cast(uint16_t, (__bf16)x); }

// Squares are summed in 64 bits: no finite gradient overflows, and the card's 64-bit rate is far above what memory feeds.
__global__ __launch_bounds__(kThreads) void k_clip_norm(const ClipTable t, uint32_t chunks, double* parts) {
    double sum = 0.0;
    for (uint32_t c = blockIdx.x; c < chunks; c += gridDim.x) {
        const Chunk k = find_chunk(t, c);
        auto add = [&](float x) { sum = fma((double)x, (double)x, sum); };
        if (t.bf16[k.tensor]) {
            const uint16_t* p = (const uint16_t*)t.in[k.tensor] + k.first;
            const int vec = ((uintptr_t)p & 15) ? 0 : k.count / 8;
            for (int i = threadIdx.x; i < vec; i += kThreads) {
                const uint4 x = ((const uint4*)p)[i];
                add(bf16_low(x.x)); add(bf16_high(x.x)); add(bf16_low(x.y)); add(bf16_high(x.y));
                add(bf16_low(x.z)); add(bf16_high(x.z)); add(bf16_low(x.w)); add(bf16_high(x.w));
            }
            for (int i = vec * 8 + threadIdx.x; i < k.count; i += kThreads) add(bf16_low(p[i]));
        } else {
            const float* p = (const float*)t.in[k.tensor] + k.first;
            const int vec = ((uintptr_t)p & 15) ? 0 : k.count / 4;
            for (int i = threadIdx.x; i < vec; i += kThreads) {
                const float4 x = ((const float4*)p)[i];
                add(x.x); add(x.y); add(x.z); add(x.w);
            }
            for (int i = vec * 4 + threadIdx.x; i < k.count; i += kThreads) add(p[i]);
        }
    }
    sum = block_total(sum);
    if (threadIdx.x == 0) parts[blockIdx.x] = sum;
}

__global__ __launch_bounds__(kThreads) void k_clip_scale(const ClipTable t, uint32_t chunks, const double* parts, int n_parts,
                                                         float max_norm, float* norm) {
    double sum = 0.0;
    for (int i = threadIdx.x; i < n_parts; i += kThreads) sum += parts[i];
    sum = block_total(sum);
    const double total = sqrt(sum), ratio = max_norm / (total + 1e-6);
    const float by = ratio > 1.0 ? 1.f : (float)ratio;   // a NaN stays one
    if (norm && blockIdx.x == 0 && threadIdx.x == 0) *norm = (float)total;
    for (uint32_t c = blockIdx.x; c < chunks; c += gridDim.x) {
        const Chunk k = find_chunk(t, chunks - 1 - c);
        if (t.in[k.tensor] == t.out[k.tensor] && by == 1.f) continue;
        if (t.bf16[k.tensor]) {
            const uint16_t* p = (const uint16_t*)t.in[k.tensor] + k.first;
            uint16_t* o = (uint16_t*)t.out[k.tensor] + k.first;
            const int vec = (((uintptr_t)p | (uintptr_t)o) & 15) ? 0 : k.count / 8;
            auto two = [&](uint32_t w) { return (uint32_t)to_bf16(bf16_low(w) * by) | (uint32_t)to_bf16(bf16_high(w) * by) << 16; };
            for (int i = threadIdx.x; i < vec; i += kThreads) {
                const uint4 x = ((const uint4*)p)[i];
                ((uint4*)o)[i] = make_uint4(two(x.x), two(x.y), two(x.z), two(x.w));
            }
            for (int i = vec * 8 + threadIdx.x; i < k.count; i += kThreads) o[i] = to_bf16(bf16_low(p[i]) * by);
        } else {
            const float* p = (const float*)t.in[k.tensor] + k.first;
            float* o = (float*)t.out[k.tensor] + k.first;
            const int vec = (((uintptr_t)p | (uintptr_t)o) & 15) ? 0 : k.count / 4;
            for (int i = threadIdx.x; i < vec; i += kThreads) {
                const float4 x = ((const float4*)p)[i];
                ((float4*)o)[i] = make_float4(x.x * by, x.y * by, x.z * by, x.w * by);
            }
            for (int i = vec * 4 + threadIdx.x; i < k.count; i += kThreads) o[i] = p[i] * by;
        }
    }
}

namespace {
int64_t chunks_of(int64_t size) { return (size + kChunk - 1) / kChunk; }
// partial sums of one launch's tensors
int64_t parts_of(int64_t chunks, int64_t launches) {
    const int64_t most = kMostParts / launches < 64 ? 64 : kMostParts / launches;
    return chunks < most ? chunks : most;
}
template <class F> void by_table(int64_t n, const int64_t* sizes, F&& f) {
    for (int64_t first = 0; first < n; first += kTable) {
        const int64_t end = first + kTable < n ? first + kTable : n;
        int64_t chunks = 0;
        for (int64_t i = first; i < end; ++i) chunks += chunks_of(sizes[i]);
        f(first, end, chunks);
    }
}
}  // namespace

size_t clip_workspace_bytes(int64_t n, const int64_t* sizes) {
    const int64_t launches = (n + kTable - 1) / kTable;
    int64_t parts = 0;
    by_table(n, sizes, [&](int64_t, int64_t, int64_t chunks) { parts += parts_of(chunks, launches); });
    return (size_t)(parts * 8 + 255) / 256 * 256 + 256;
}

hipError_t launch_clip(int64_t n, const void* const* grads, void* const* out, const int64_t* sizes, const int32_t* dts,
                       float max_norm, float* norm, void* ws, hipStream_t st) {
    const int64_t launches = (n + kTable - 1) / kTable;
    hipError_t e = hipSuccess;
    int64_t parts = 0;
    auto each = [&](auto&& f) {
        by_table(n, sizes, [&](int64_t first, int64_t end, int64_t chunks) {
            if (e != hipSuccess) return;
            ClipTable t = {};
            uint32_t c = 0;
            for (int64_t i = first; i < end; ++i) {
                t.in[i - first] = grads[i];
                t.out[i - first] = out ? out[i] : nullptr;
                t.size[i - first] = sizes[i];
                t.chunk0[i - first] = c;
                t.bf16[i - first] = dts[i] == TR_BF16;
                c += (uint32_t)chunks_of(sizes[i]);
            }
            t.n = (int)(end - first);
            t.chunk0[t.n] = c;
            f(t, (uint32_t)chunks, first == 0);
            e = hipGetLastError();
        });
    };
    each([&](const ClipTable& t, uint32_t chunks, bool) {
        const int64_t p = parts_of(chunks, launches);
        if (p) k_clip_norm<<<dim3((unsigned)p), kThreads, 0, st>>>(t, chunks, (double*)ws + parts);
        parts += p;
    });
    each([&](const ClipTable& t, uint32_t chunks, bool first) {
        const uint32_t work = out ? chunks : 0;
        if (work || first)
            k_clip_scale<<<dim3(work < 1 ? 1 : work < kMostParts ? work : kMostParts), kThreads, 0, st>>>(t, work, (const double*)ws, (int)parts,
                                                                                               max_norm, first ? norm : nullptr);
    });
    return e;
}

}  // namespace cb
