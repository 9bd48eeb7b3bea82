// grad_clip.cu -- the global norm of many gradient tensors, and their clipping:
//
//     n = sqrt(sum over tensors and elements of g^2),  c = n > max_norm ? max_norm / n : 1,  out = c g
//
// Bound by memory: one read for the norm, then one read and one write, of which the second read finds in L2 what fits
// there.  The tensors are cut into chunks (16384 elements, or a larger power of two that keeps their number near 4096).
// One cooperative launch: each block sums the squares of its chunks in fp32 and writes one fp64 partial per chunk; after a
// barrier over the grid every block adds all partials in the same fixed order, so the norm does not depend on the grid, and
// scales its chunks, the last read first.  The table of the tensors is a kernel argument; more of them than it holds take a
// launch per table for the norm and one per table for the scaling.
// A chunk whose fp32 sum left the range in which it is exact to fp32's precision (overflow, or so small that
// squares were lost below 2^-126) is summed again with its elements scaled by a power of two.
#include <cooperative_groups.h>
#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include "dtp_common.cuh"
#include "layer_common.cuh"

namespace dtp {
namespace clip {

using layer::from_f32;
using layer::to_f32;

constexpr int kThreads = 512;
constexpr int kWarps = kThreads / 32;
constexpr int64_t kMinChunk = 16384;   // elements
constexpr int64_t kManyChunks = 4096;
constexpr int kBlocksPerSm = 2;

template <int CAP>
struct Table {
    const void* src[CAP];
    void* dst[CAP];
    int64_t numel[CAP];
    int first[CAP + 1];                // first chunk of the tensor
    uint8_t f32[CAP];
    int count;
    int chunks;                        // of this table
    int chunk0;                        // the table's first partial
    int all_chunks;                    // of all tables
    int64_t chunk;                     // elements
    float max_norm;
    double* partial;
    float* norm;
    int* status;
};
constexpr int kSmallTable = 64, kLargeTable = 1024;
static_assert(sizeof(Table<kLargeTable>) <= 32000, "kernel arguments");

// the tensor of chunk c: the last one whose first chunk is <= c (empty tensors are not in the table)
template <int CAP>
__device__ __forceinline__ int tensor_of(const Table<CAP>& t, int c) {
    int lo = 0, hi = t.count;
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (t.first[mid] <= c) lo = mid;
        else hi = mid;
    }
    return lo;
}

template <typename V>
__device__ __forceinline__ V block_sum(V v, V* red) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xFFFFFFFFu, v, o);
    __syncthreads();
    if (lane == 0) red[warp] = v;
    __syncthreads();
    V s = 0;
#pragma unroll
    for (int w = 0; w < kWarps; ++w) s += red[w];
    return s;
}

// The 16-byte words of n elements from p, and the elements before and after them.
template <typename E>
struct Span {
    static constexpr int kPer = 16 / sizeof(E);
    int head;
    int64_t words;
    __device__ __forceinline__ Span(const void* p, int64_t n) {
        const int64_t lead = ((16 - (reinterpret_cast<uintptr_t>(p) & 15)) & 15) / sizeof(E);
        head = static_cast<int>(lead < n ? lead : n);
        words = (n - head) / kPer;
    }
};

template <typename E>
__device__ __forceinline__ void unpack(const uint4& q, float (&v)[16 / sizeof(E)]) {
    const uint32_t w[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if constexpr (sizeof(E) == 4) {
            v[i] = __uint_as_float(w[i]);
        } else {
            v[2 * i] = __uint_as_float(w[i] << 16);
            v[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
        }
    }
}

template <typename E>
__device__ __forceinline__ uint4 pack(const float (&v)[16 / sizeof(E)]) {
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if constexpr (sizeof(E) == 4) {
            w[i] = __float_as_uint(v[i]);
        } else {
            const __nv_bfloat162 b = __floats2bfloat162_rn(v[2 * i], v[2 * i + 1]);
            w[i] = *reinterpret_cast<const uint32_t*>(&b);
        }
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
}

// This thread's share of sum (scale p[i])^2: a round of four words at a time, each round's sum added to the total.
template <typename E>
__device__ __forceinline__ float sum_squares(const E* p, int64_t n, float scale) {
    const Span<E> s(p, n);
    const uint4* words = reinterpret_cast<const uint4*>(p + s.head);
    auto square = [&](float x, float& to) { x *= scale; to = fmaf(x, x, to); };
    auto word = [&](const uint4& q, float& to) {
        float v[Span<E>::kPer];
        unpack<E>(q, v);
#pragma unroll
        for (int i = 0; i < Span<E>::kPer; ++i) square(v[i], to);
    };
    float total = 0.0f;
    int64_t i = threadIdx.x;
    for (; i + 3 * kThreads < s.words; i += 4 * kThreads) {
        uint4 q[4];
        float r[4] = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
        for (int j = 0; j < 4; ++j) q[j] = words[i + j * kThreads];
#pragma unroll
        for (int j = 0; j < 4; ++j) word(q[j], r[j]);
        total += (r[0] + r[1]) + (r[2] + r[3]);
    }
    for (; i < s.words; i += kThreads) {
        float r = 0.0f;
        word(words[i], r);
        total += r;
    }
    if (static_cast<int>(threadIdx.x) < s.head) square(to_f32(p[threadIdx.x]), total);
    const int64_t tail = s.head + s.words * Span<E>::kPer + threadIdx.x;
    if (tail < n) square(to_f32(p[tail]), total);
    return total;
}

constexpr float kTiny = 8.271806e-25f;         // 2^-80
constexpr float kUp = 1.2676506e30f;           // 2^100
constexpr float kDown = 7.888609e-31f;         // 2^-100

template <typename E>
__device__ __forceinline__ double chunk_squares(const E* p, int64_t n, float* red) {
    float s = block_sum(sum_squares(p, n, 1.0f), red);
    if (s >= kTiny && s <= 3.0e38f) return static_cast<double>(s);      // the same value in every thread
    const float scale = s < kTiny ? kUp : kDown;                        // (a NaN stays one either way)
    s = block_sum(sum_squares(p, n, scale), red);
    return static_cast<double>(s) / (static_cast<double>(scale) * static_cast<double>(scale));
}

// dst = c src.  Words where both are equally aligned; c == 1 copies bit for bit, NaNs too.
template <typename E>
__device__ __forceinline__ void scale_chunk(const E* src, E* dst, int64_t n, float c) {
    const bool copy = c == 1.0f;
    if (copy && src == dst) return;
    auto one = [&](int64_t i) { dst[i] = copy ? src[i] : from_f32<E>(to_f32(src[i]) * c); };
    if ((reinterpret_cast<uintptr_t>(src) ^ reinterpret_cast<uintptr_t>(dst)) & 15) {
        for (int64_t i = threadIdx.x; i < n; i += kThreads) one(i);
        return;
    }
    const Span<E> s(src, n);
    const uint4* from = reinterpret_cast<const uint4*>(src + s.head);
    uint4* to = reinterpret_cast<uint4*>(dst + s.head);
    auto word = [&](const uint4& q) {
        if (copy) return q;
        float v[Span<E>::kPer];
        unpack<E>(q, v);
#pragma unroll
        for (int i = 0; i < Span<E>::kPer; ++i) v[i] *= c;
        return pack<E>(v);
    };
    int64_t i = threadIdx.x;
    for (; i + 3 * kThreads < s.words; i += 4 * kThreads) {
        uint4 q[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) q[j] = from[i + j * kThreads];
#pragma unroll
        for (int j = 0; j < 4; ++j) __stcs(to + i + j * kThreads, word(q[j]));
    }
    for (; i < s.words; i += kThreads) __stcs(to + i, word(from[i]));
    if (static_cast<int>(threadIdx.x) < s.head) one(threadIdx.x);
    const int64_t tail = s.head + s.words * Span<E>::kPer + threadIdx.x;
    if (tail < n) one(tail);
}

enum Mode { kBoth = 0, kNorm = 1, kScale = 2 };

template <int CAP, int MODE>
__global__ void __launch_bounds__(kThreads, kBlocksPerSm) clip_kernel(const __grid_constant__ Table<CAP> t) {
    __shared__ float red[kWarps];
    __shared__ double red64[kWarps];
    auto chunk_of = [&](int c, int& i, int64_t& at, int64_t& n) {
        i = tensor_of(t, c);
        at = (c - t.first[i]) * t.chunk;
        n = t.numel[i] - at < t.chunk ? t.numel[i] - at : t.chunk;
    };
    if (blockIdx.x == 0 && threadIdx.x == 0) *t.status = DTP_OK;     // nothing here can give up
    if constexpr (MODE != kScale) {
        for (int c = blockIdx.x; c < t.chunks; c += gridDim.x) {
            int i;
            int64_t at, n;
            chunk_of(c, i, at, n);
            const double s = t.f32[i] ? chunk_squares(static_cast<const float*>(t.src[i]) + at, n, red)
                                      : chunk_squares(static_cast<const __nv_bfloat16*>(t.src[i]) + at, n, red);
            if (threadIdx.x == 0) t.partial[t.chunk0 + c] = s;
        }
    }
    if constexpr (MODE == kBoth) cooperative_groups::this_grid().sync();
    if constexpr (MODE != kNorm) {
        double s = 0.0;
        for (int c = threadIdx.x; c < t.all_chunks; c += kThreads) s += __ldcg(t.partial + c);
        const double r = sqrt(block_sum(s, red64));
        // a norm that is not finite leaves the gradients as they are
        const float f = isfinite(r) && r > static_cast<double>(t.max_norm) ? static_cast<float>(t.max_norm / r) : 1.0f;
        if (blockIdx.x == 0 && threadIdx.x == 0) *t.norm = static_cast<float>(r);
        const int last = t.chunks - 1 - static_cast<int>(blockIdx.x);
        for (int c = static_cast<int>(blockIdx.x) + (last < 0 ? 0 : last / static_cast<int>(gridDim.x) * static_cast<int>(gridDim.x));
             c >= 0 && c < t.chunks; c -= gridDim.x) {
            int i;
            int64_t at, n;
            chunk_of(c, i, at, n);
            if (t.f32[i])
                scale_chunk(static_cast<const float*>(t.src[i]) + at, static_cast<float*>(t.dst[i]) + at, n, f);
            else
                scale_chunk(static_cast<const __nv_bfloat16*>(t.src[i]) + at,
                            static_cast<__nv_bfloat16*>(t.dst[i]) + at, n, f);
        }
    }
}

// ------------------------------------------------------------------------------------ host

static int64_t chunk_elements(int count, const int64_t* numel) {
    int64_t total = 0, chunk = kMinChunk;
    for (int i = 0; i < count; ++i) total += numel[i];
    while (total / chunk > kManyChunks) chunk *= 2;
    return chunk;
}

// Chunks of all tensors; -1 for a negative size or too many of them.
int64_t chunk_count(int count, const int64_t* numel) {
    int64_t total = 0;
    for (int i = 0; i < count; ++i) {
        if (numel[i] < 0 || numel[i] > (int64_t(1) << 46)) return -1;
        total += numel[i];
        if (total > (int64_t(1) << 46)) return -1;
    }
    const int64_t chunk = chunk_elements(count, numel);
    int64_t chunks = 0;
    for (int i = 0; i < count; ++i) chunks += (numel[i] + chunk - 1) / chunk;
    return chunks;
}

size_t workspace_bytes(int64_t chunks) {
    return kWorkspaceHeader + align_up(static_cast<size_t>(chunks) * sizeof(double), 256);
}

template <int CAP, int MODE>
static int launch_table(const Table<CAP>& t, int sms, cudaStream_t stream) {
    auto kernel = clip_kernel<CAP, MODE>;
    cudaLaunchConfig_t cfg = {};
    const int most = kBlocksPerSm * sms;
    cfg.gridDim = dim3(static_cast<unsigned>(t.chunks < 1 ? 1 : t.chunks < most ? t.chunks : most));
    cfg.blockDim = dim3(kThreads);
    cfg.stream = stream;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeCooperative;
    attr[0].val.cooperative = 1;
    cfg.attrs = attr;
    cfg.numAttrs = MODE == kBoth ? 1 : 0;
    DTP_CUDA_TRY(cudaLaunchKernelEx(&cfg, kernel, t));
    return DTP_OK;
}

// Tables of at most CAP non-empty tensors (one, perhaps empty, if there are none), each passed to fn.
template <int CAP, typename F>
static int each_table(const void* const* grads, void* const* out, const int64_t* numel, const int* dtype, int count,
                      Table<CAP>& t, F fn) {
    t.count = 0, t.chunk0 = 0;
    int chunks = 0, launched = 0;
    auto flush = [&]() {
        t.chunks = chunks;
        t.first[t.count] = chunks;
        const int st = fn();
        t.chunk0 += chunks;
        t.count = 0, chunks = 0;
        ++launched;
        return st;
    };
    for (int i = 0; i < count; ++i) {
        if (numel[i] == 0) continue;
        if (t.count == CAP) {
            const int st = flush();
            if (st != DTP_OK) return st;
        }
        t.src[t.count] = grads[i];
        t.dst[t.count] = out ? out[i] : const_cast<void*>(grads[i]);
        t.numel[t.count] = numel[i];
        t.first[t.count] = chunks;
        t.f32[t.count] = dtype[i] == DTP_F32;
        ++t.count;
        chunks += static_cast<int>((numel[i] + t.chunk - 1) / t.chunk);
    }
    return t.count || !launched ? flush() : static_cast<int>(DTP_OK);
}

template <int CAP>
static int launch_capacity(const void* const* grads, void* const* out, const int64_t* numel, const int* dtype,
                           int count, bool one, float max_norm, float* norm, void* workspace, int sms,
                           cudaStream_t stream) {
    Table<CAP> t;
    t.chunk = chunk_elements(count, numel);
    t.all_chunks = static_cast<int>(chunk_count(count, numel));
    t.max_norm = max_norm;
    t.norm = norm;
    t.status = static_cast<int*>(workspace);
    t.partial = reinterpret_cast<double*>(static_cast<uint8_t*>(workspace) + kWorkspaceHeader);
    if (one)
        return each_table(grads, out, numel, dtype, count, t,
                          [&] { return launch_table<CAP, kBoth>(t, sms, stream); });
    const int st = each_table(grads, out, numel, dtype, count, t,
                              [&] { return launch_table<CAP, kNorm>(t, sms, stream); });
    if (st != DTP_OK) return st;
    return each_table(grads, out, numel, dtype, count, t, [&] { return launch_table<CAP, kScale>(t, sms, stream); });
}

int launch(const void* const* grads, void* const* out, const int64_t* numel, const int* dtype, int count,
           float max_norm, float* norm, void* workspace, cudaStream_t stream) {
    int dev = 0, sms = 0;
    DTP_CUDA_TRY(cudaGetDevice(&dev));
    DTP_CUDA_TRY(cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev));
    int filled = 0;
    for (int i = 0; i < count; ++i) filled += numel[i] != 0;
    if (filled <= kSmallTable)
        return launch_capacity<kSmallTable>(grads, out, numel, dtype, count, true, max_norm, norm, workspace, sms, stream);
    return launch_capacity<kLargeTable>(grads, out, numel, dtype, count, filled <= kLargeTable, max_norm, norm, workspace,
                                        sms, stream);
}

}  // namespace clip
}  // namespace dtp
