// rms_norm.cu -- the RMS norm of rows and its gradients:
//
//     rms_t = sqrt(mean_i x_ti^2 + eps),  y = gamma n,  n = x / rms
//     dx = (dn - n mean_i(dn n)) / rms + dresidual,  dn = gamma dy,   dgamma_i = sum_t dy_ti n_ti
//
// Bound by memory.  Sums in fp32 (a row's in 256 threads' parts); dgamma's in runs of at most kRun rows, which are added in fp64.
#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include "dtp_common.cuh"
#include "layer_common.cuh"
#include "layer_host.cuh"

namespace dtp {
namespace norm {

using layer::from_f32;
using layer::grid_release;
using layer::grid_wait;
using layer::to_f32;

constexpr int kThreads = 256;
constexpr int kRun = 256;              // rows of a partial sum of dgamma
constexpr float kDown = 5.4210109e-20f;      // 2^-64: a row whose squares leave fp32's range is summed again at this scale

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
__global__ void __launch_bounds__(kThreads)
forward_kernel(const E* X, const float* gamma, int64_t T, int d, float eps, E* Y, float* rms) {
    __shared__ float red[kThreads / 32];
    grid_wait();
    grid_release();
    for (int64_t t = blockIdx.x; t < T; t += gridDim.x) {
        const E* x = X + t * d;
        auto squares = [&](float scale) {
            float s = 0.0f;
            for (int i = threadIdx.x; i < d; i += kThreads) {
                const float v = to_f32(x[i]) * scale;
                s = fmaf(v, v, s);
            }
            return block_sum(s, red) / static_cast<float>(d);
        };
        const float s = squares(1.0f);
        const float r = s <= 3.0e38f ? sqrtf(s + eps) : sqrtf(squares(kDown)) / kDown;
        if (threadIdx.x == 0) rms[t] = r;
        for (int i = threadIdx.x; i < d; i += kThreads) Y[t * d + i] = from_f32<E>(to_f32(x[i]) / r * gamma[i]);
    }
}

// dX by rows
template <typename E>
__global__ void __launch_bounds__(kThreads)
rows_kernel(const E* dY, const E* X, const float* gamma, const float* rms, const E* dres, int64_t T, int d, E* dX) {
    __shared__ float red[kThreads / 32];
    grid_wait();
    grid_release();
    for (int64_t t = blockIdx.x; t < T; t += gridDim.x) {
        const float r = rms[t];
        float s = 0.0f;
        for (int i = threadIdx.x; i < d; i += kThreads)
            s = fmaf(to_f32(dY[t * d + i]) * gamma[i], to_f32(X[t * d + i]) / r, s);
        s = block_sum(s, red) / static_cast<float>(d);
        for (int i = threadIdx.x; i < d; i += kThreads) {
            float v = (to_f32(dY[t * d + i]) * gamma[i] - to_f32(X[t * d + i]) / r * s) / r;
            if (dres) v += to_f32(dres[t * d + i]);
            dX[t * d + i] = from_f32<E>(v);
        }
    }
}

// partial[run][i] = sum over the run's rows of dy n, in order
template <typename E>
__global__ void __launch_bounds__(kThreads)
columns_kernel(const E* dY, const E* X, const float* rms, int64_t T, int d, float* partial) {
    grid_wait();
    grid_release();
    const int blocks = (d + kThreads - 1) / kThreads;
    const int64_t run = blockIdx.x / blocks, t1 = run * kRun + kRun < T ? run * kRun + kRun : T;
    const int i = static_cast<int>(blockIdx.x % blocks) * kThreads + threadIdx.x;
    if (i >= d) return;
    float s = 0.0f;
    for (int64_t t = run * kRun; t < t1; ++t) s = fmaf(to_f32(dY[t * d + i]), to_f32(X[t * d + i]) / rms[t], s);
    partial[run * d + i] = s;
}

__global__ void __launch_bounds__(256) join_kernel(const float* partial, int64_t runs, int d, float* dgamma) {
    __shared__ double red[8][32];
    grid_wait();
    grid_release();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, i = blockIdx.x * 32 + lane;
    double s = 0.0;
    if (i < d)
        for (int64_t r = warp; r < runs; r += 8) s += partial[r * d + i];
    red[warp][lane] = s;
    __syncthreads();
    if (warp == 0 && i < d) {
        double v = 0.0;
#pragma unroll
        for (int w = 0; w < 8; ++w) v += red[w][lane];
        dgamma[i] = static_cast<float>(v);
    }
}

static int64_t runs_of(int64_t T) { return (T + kRun - 1) / kRun; }

size_t backward_workspace_bytes(int64_t T, int d) {
    layer::Carver c(nullptr);
    c.take(static_cast<size_t>(runs_of(T)) * d * sizeof(float));
    return c.used;
}

template <typename E>
static int forward(const void* X, const float* gamma, int64_t T, int d, float eps, void* Y, float* rms, cudaStream_t stream) {
    return layer::launch_after(forward_kernel<E>, T < 8192 ? T : 8192, stream, static_cast<const E*>(X), gamma, T, d, eps,
                               static_cast<E*>(Y), rms);
}

template <typename E>
static int backward(const void* dY, const void* X, const float* gamma, const float* rms, const void* dres, int64_t T, int d,
                    void* dX, float* dgamma, void* workspace, cudaStream_t stream) {
    int st = DTP_OK;
    if (dX && T > 0)
        st = layer::launch_after(rows_kernel<E>, T < 8192 ? T : 8192, stream, static_cast<const E*>(dY), static_cast<const E*>(X),
                                 gamma, rms, static_cast<const E*>(dres), T, d, static_cast<E*>(dX));
    if (st != DTP_OK || !dgamma) return st;
    layer::Carver c(workspace);
    auto* partial = static_cast<float*>(c.take(static_cast<size_t>(runs_of(T)) * d * sizeof(float)));
    if (T > 0)
        st = layer::launch_after(columns_kernel<E>, runs_of(T) * ((d + kThreads - 1) / kThreads), stream,
                                 static_cast<const E*>(dY), static_cast<const E*>(X), rms, T, d, partial);
    if (st != DTP_OK) return st;
    return layer::launch_after(join_kernel, (d + 31) / 32, stream, static_cast<const float*>(partial), runs_of(T), d, dgamma);
}

int launch_forward(const void* X, const float* gamma, int64_t T, int d, float eps, int dtype, void* Y, float* rms,
                   cudaStream_t stream) {
    return dtype == DTP_BF16 ? forward<__nv_bfloat16>(X, gamma, T, d, eps, Y, rms, stream)
                             : forward<float>(X, gamma, T, d, eps, Y, rms, stream);
}

int launch_backward(const void* dY, const void* X, const float* gamma, const float* rms, const void* dres, int64_t T, int d,
                    int dtype, void* dX, float* dgamma, void* workspace, cudaStream_t stream) {
    return dtype == DTP_BF16 ? backward<__nv_bfloat16>(dY, X, gamma, rms, dres, T, d, dX, dgamma, workspace, stream)
                             : backward<float>(dY, X, gamma, rms, dres, T, d, dX, dgamma, workspace, stream);
}

}  // namespace norm
}  // namespace dtp
