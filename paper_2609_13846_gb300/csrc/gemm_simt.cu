// gemm_simt.cu -- the matrix products of the layer operators on the CUDA cores: any sizes, any of the four
// operand orders, fp32 sums.
#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include "dtp_common.cuh"
#include "layer_common.cuh"

namespace dtp {
namespace simt {

using namespace layer;

constexpr int TM = 64, TN = 64, TK = 16;
constexpr int kThreads = 256;

// A block computes a 64 x 64 tile, a thread 4 x 4 of it, over k blocks of 16 staged in shared memory.
template <typename E, int KIND>
__global__ void __launch_bounds__(kThreads) gemm_kernel(const Product p, int tiles_n) {
    constexpr int kAcc = KIND == kEpiGated ? 2 : 1;
    __shared__ float as[TK][TM + 4];
    __shared__ float bs[kAcc][TK][TN + 4];
    const int tid = threadIdx.x, tx = tid & 15, ty = tid >> 4;
    const int64_t m0 = static_cast<int64_t>(blockIdx.x / tiles_n) * TM;
    const int n0 = static_cast<int>(blockIdx.x % tiles_n) * TN;
    float acc[kAcc][4][4];
#pragma unroll
    for (int a = 0; a < kAcc; ++a)
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int j = 0; j < 4; ++j) acc[a][i][j] = 0.0f;
    // element x of a 64 x 16 tile: neighbouring threads take neighbours along the contiguous axis
    auto stage = [&](const Mat& a, int64_t r0, int64_t rows, int64_t k0, float* to) {
        const E* src = reinterpret_cast<const E*>(a.p);
        for (int x = tid; x < TM * TK; x += kThreads) {
            const int r = a.ks == 1 ? x / TK : x % TM, k = a.ks == 1 ? x % TK : x / TM;
            const bool in = r0 + r < rows && k0 + k < p.K;
            to[k * (TM + 4) + r] = in ? to_f32(src[(r0 + r) * a.rs + (k0 + k) * a.ks]) : 0.0f;
        }
    };
    for (int s = 0; s < p.segments; ++s)
        for (int64_t k0 = 0; k0 < p.K; k0 += TK) {
            stage(p.A[s], m0, p.M, k0, &as[0][0]);
            if constexpr (kAcc == 1) {
                stage(p.B[s], n0, p.N, k0, &bs[0][0][0]);
            } else {
                stage(p.B[0], n0, p.N, k0, &bs[0][0][0]);
                stage(p.B[1], n0, p.N, k0, &bs[1][0][0]);
            }
            __syncthreads();
#pragma unroll
            for (int k = 0; k < TK; ++k) {
                const float4 a = *reinterpret_cast<const float4*>(&as[k][4 * ty]);
                const float av[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
                for (int q = 0; q < kAcc; ++q) {
                    const float4 b = *reinterpret_cast<const float4*>(&bs[q][k][4 * tx]);
                    const float bv[4] = {b.x, b.y, b.z, b.w};
#pragma unroll
                    for (int i = 0; i < 4; ++i)
#pragma unroll
                        for (int j = 0; j < 4; ++j) acc[q][i][j] = fmaf(av[i], bv[j], acc[q][i][j]);
                }
            }
            __syncthreads();
        }
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int64_t m = m0 + 4 * ty + i;
            const int n = n0 + 4 * tx + j;
            if (m < p.M && n < p.N) epilogue_element<E, KIND>(p.epi, m, n, acc[0][i][j], acc[kAcc - 1][i][j]);
        }
}

template <typename E>
static int launch_typed(const Product& p, cudaStream_t stream) {
    const int64_t tiles_n = (p.N + TN - 1) / TN, tiles = (p.M + TM - 1) / TM * tiles_n;
    if (tiles > 0x7FFFFFFF) return DTP_ERR_UNSUPPORTED;
    auto kernel = p.epi.kind == kEpiLinear  ? gemm_kernel<E, kEpiLinear>
                  : p.epi.kind == kEpiGated ? gemm_kernel<E, kEpiGated>
                                            : gemm_kernel<E, kEpiGatedGrad>;
    kernel<<<static_cast<unsigned>(tiles), kThreads, 0, stream>>>(p, static_cast<int>(tiles_n));
    DTP_CUDA_TRY(cudaGetLastError());
    return DTP_OK;
}

int launch(const Product& p, int dtype, cudaStream_t stream) {
    return dtype == DTP_BF16 ? launch_typed<__nv_bfloat16>(p, stream) : launch_typed<float>(p, stream);
}

}  // namespace simt
}  // namespace dtp
