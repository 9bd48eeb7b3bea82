// grad_clip.cu -- the global norm of many gradient tensors, and their clipping:
//
//     n = sqrt(sum over tensors and elements of g^2),  c = n > max_norm ? max_norm / n : 1,  out = c g
//
// The tensors are cut into chunks of 16384 elements.  A block sums a chunk's squares in fp32 and writes one
// fp64 partial per chunk; the partials are added in a fixed order, so the norm does not depend on the grid.
// A chunk whose fp32 sum left the range in which it is exact to fp32's precision (overflow, or so small that
// squares were lost below 2^-126) is summed again with its elements scaled by a power of two.
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
constexpr int kChunk = 16384;     // elements
constexpr int kMaxTensors = 512;  // per launch: the table is a kernel argument

struct Table {
    int count;
    int chunks;                        // of this launch
    int64_t chunk0;                    // of the launch's first partial
    const void* src[kMaxTensors];
    void* dst[kMaxTensors];
    int64_t numel[kMaxTensors];
    int first[kMaxTensors + 1];        // first chunk of the tensor
    uint8_t f32[kMaxTensors];
};

// the tensor of chunk c: the last one whose first chunk is <= c (empty tensors have no chunk)
__device__ __forceinline__ int tensor_of(const Table& t, int c) {
    int lo = 0, hi = t.count;
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (t.first[mid] <= c) lo = mid;
        else hi = mid;
    }
    return lo;
}

__device__ __forceinline__ float block_sum(float v, float* red) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xFFFFFFFFu, v, o);
    __syncthreads();
    if (lane == 0) red[warp] = v;
    __syncthreads();
    float s = 0.0f;
#pragma unroll
    for (int w = 0; w < kThreads / 32; ++w) s += red[w];
    return s;
}

template <typename E>
__device__ __forceinline__ float sum_squares(const E* p, int n, float scale) {
    float s = 0.0f;
    for (int i = threadIdx.x; i < n; i += kThreads) {
        const float v = to_f32(p[i]) * scale;
        s = fmaf(v, v, s);
    }
    return s;
}

constexpr float kTiny = 8.271806e-25f;         // 2^-80
constexpr float kUp = 1.2676506e30f;           // 2^100
constexpr float kDown = 7.888609e-31f;         // 2^-100

template <typename E>
__device__ __forceinline__ double chunk_squares(const E* p, int n, float* red) {
    float s = block_sum(sum_squares(p, n, 1.0f), red);
    if (s >= kTiny && s <= 3.0e38f) return static_cast<double>(s);      // the same value in every thread
    const float scale = s < kTiny ? kUp : kDown;                        // (a NaN stays one either way)
    s = block_sum(sum_squares(p, n, scale), red);
    return static_cast<double>(s) / (static_cast<double>(scale) * static_cast<double>(scale));
}

__global__ void __launch_bounds__(kThreads) norm_kernel(const __grid_constant__ Table t, double* partial) {
    __shared__ float red[kThreads / 32];
    for (int c = blockIdx.x; c < t.chunks; c += gridDim.x) {
        const int i = tensor_of(t, c);
        const int64_t at = static_cast<int64_t>(c - t.first[i]) * kChunk;
        const int n = static_cast<int>(t.numel[i] - at < kChunk ? t.numel[i] - at : kChunk);
        const double s = t.f32[i] ? chunk_squares(static_cast<const float*>(t.src[i]) + at, n, red)
                                  : chunk_squares(static_cast<const __nv_bfloat16*>(t.src[i]) + at, n, red);
        if (threadIdx.x == 0) partial[t.chunk0 + c] = s;
    }
}

// norm and coefficient from the partials, in a fixed order: one block.
__global__ void __launch_bounds__(kThreads)
finish_kernel(const double* __restrict__ partial, int64_t n, float max_norm, float* norm, float* coef) {
    __shared__ double red[kThreads];
    double s = 0.0;
    for (int64_t i = threadIdx.x; i < n; i += kThreads) s += partial[i];
    red[threadIdx.x] = s;
    __syncthreads();
    for (int o = kThreads / 2; o > 0; o >>= 1) {
        if (threadIdx.x < o) red[threadIdx.x] += red[threadIdx.x + o];
        __syncthreads();
    }
    if (threadIdx.x == 0) {
        const double r = sqrt(red[0]);
        *norm = static_cast<float>(r);
        // a norm that is not finite leaves the gradients as they are
        *coef = isfinite(r) && r > static_cast<double>(max_norm) ? static_cast<float>(max_norm / r) : 1.0f;
    }
}

template <typename E>
__device__ __forceinline__ void scale_chunk(const E* src, E* dst, int n, float c) {
    if (c == 1.0f) {
        if (src == dst) return;
        for (int i = threadIdx.x; i < n; i += kThreads) dst[i] = src[i];      // bit for bit, NaNs too
    } else {
        for (int i = threadIdx.x; i < n; i += kThreads) dst[i] = from_f32<E>(to_f32(src[i]) * c);
    }
}

__global__ void __launch_bounds__(kThreads) scale_kernel(const __grid_constant__ Table t, const float* coef) {
    const float f = *coef;
    for (int c = blockIdx.x; c < t.chunks; c += gridDim.x) {
        const int i = tensor_of(t, c);
        const int64_t at = static_cast<int64_t>(c - t.first[i]) * kChunk;
        const int n = static_cast<int>(t.numel[i] - at < kChunk ? t.numel[i] - at : kChunk);
        if (t.f32[i])
            scale_chunk(static_cast<const float*>(t.src[i]) + at, static_cast<float*>(t.dst[i]) + at, n, f);
        else
            scale_chunk(static_cast<const __nv_bfloat16*>(t.src[i]) + at,
                        static_cast<__nv_bfloat16*>(t.dst[i]) + at, n, f);
    }
}

static int64_t chunks_of(int64_t numel) { return (numel + kChunk - 1) / kChunk; }

// Chunks of all tensors; -1 for a negative size or too many of them.
int64_t chunk_count(int count, const int64_t* numel) {
    int64_t chunks = 0;
    for (int i = 0; i < count; ++i) {
        if (numel[i] < 0 || numel[i] > (int64_t(1) << 46)) return -1;
        chunks += chunks_of(numel[i]);
        if (chunks > 0x7FFFFFFF) return -1;
    }
    return chunks;
}

size_t workspace_bytes(int64_t chunks) {
    return kWorkspaceHeader + align_up(static_cast<size_t>(chunks) * sizeof(double), 256);
}

// Tables of at most kMaxTensors non-empty tensors, each passed to fn with the number of its chunks.
template <typename F>
static int each_table(const void* const* grads, void* const* out, const int64_t* numel, const int* dtype, int count,
                      F fn) {
    Table t;
    t.count = 0, t.chunks = 0, t.chunk0 = 0;
    int64_t chunks = 0;
    auto flush = [&]() {
        if (t.count == 0) return static_cast<int>(DTP_OK);
        t.chunks = static_cast<int>(chunks);
        t.first[t.count] = t.chunks;
        const int st = fn(t);
        t.chunk0 += chunks;
        t.count = 0, chunks = 0;
        return st;
    };
    for (int i = 0; i < count; ++i) {
        if (numel[i] == 0) continue;
        const int64_t c = chunks_of(numel[i]);
        if (t.count == kMaxTensors) {
            const int st = flush();
            if (st != DTP_OK) return st;
        }
        t.src[t.count] = grads[i];
        t.dst[t.count] = out ? out[i] : const_cast<void*>(grads[i]);
        t.numel[t.count] = numel[i];
        t.first[t.count] = static_cast<int>(chunks);
        t.f32[t.count] = dtype[i] == DTP_F32;
        ++t.count;
        chunks += c;
    }
    return flush();
}

int launch(const void* const* grads, void* const* out, const int64_t* numel, const int* dtype, int count,
           float max_norm, float* norm, void* workspace, cudaStream_t stream) {
    int dev = 0, sms = 0;
    DTP_CUDA_TRY(cudaGetDevice(&dev));
    DTP_CUDA_TRY(cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev));
    uint8_t* ws = static_cast<uint8_t*>(workspace);
    float* coef = reinterpret_cast<float*>(ws + 128);       // in the header, behind the status word
    double* partial = reinterpret_cast<double*>(ws + kWorkspaceHeader);
    const int64_t total = chunk_count(count, numel);
    DTP_CUDA_TRY(cudaMemsetAsync(ws, 0, kWorkspaceHeader, stream));
    int st = each_table(grads, out, numel, dtype, count, [&](const Table& t) -> int {
        const int grid = t.chunks < 4 * sms ? t.chunks : 4 * sms;
        norm_kernel<<<grid, kThreads, 0, stream>>>(t, partial);
        DTP_CUDA_TRY(cudaGetLastError());
        return DTP_OK;
    });
    if (st != DTP_OK) return st;
    finish_kernel<<<1, kThreads, 0, stream>>>(partial, total, max_norm, norm, coef);
    DTP_CUDA_TRY(cudaGetLastError());
    return each_table(grads, out, numel, dtype, count, [&](const Table& t) -> int {
        const int grid = t.chunks < 4 * sms ? t.chunks : 4 * sms;
        scale_kernel<<<grid, kThreads, 0, stream>>>(t, coef);
        DTP_CUDA_TRY(cudaGetLastError());
        return DTP_OK;
    });
}

}  // namespace clip
}  // namespace dtp
