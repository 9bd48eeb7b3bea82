// few_loss_f32.cu -- the fp32 products of the softmax cross entropy for up to 32 tokens, on the CUDA cores:
//
//     Z [T, V] = X W^T,   dX [T, d] = dZ W,   dW [V, d] = dZ^T X
//
// The vocabulary is long and the tokens are few, so tiles of 64 tokens would be half empty or worse, and dX has one or two of
// them with a sum over the whole vocabulary.  Here the tokens lie in registers or shared memory, and W is streamed once (dW
// written once).  18 tokens, 65536 x 768 (201 MB): Z 114 us (tiles 185), bound by shared memory and FMAs alike, 43 us of each with
// the tokens padded to 32; dX 122 and dW 92 (120 and 290 in tiles).  5 tokens, 32768 x 1024: 45, 48 and 34 us of 134 MB.
#include <cuda_runtime.h>
#include <stdint.h>

#include "dtp_common.cuh"
#include "layer_common.cuh"
#include "layer_host.cuh"

namespace dtp {
namespace fewl {

using layer::grid_release;
using layer::grid_wait;

constexpr int kThreads = 256;
constexpr int kMost = 32;              // tokens

// --------------------------------------------------------------------------- Z

constexpr int kSums = 64;              // of a lane: rows of W that a warp takes at once x tokens of a pass over them
constexpr int kStep = 128;             // k of a step: four consecutive ones a lane
constexpr int kShared = 96 * 1024;     // bytes of X in shared memory, two blocks per SM

// TOK tokens a pass; a second pass finds the rows in L1.  kWide: rows on 16-byte boundaries.
template <int TOK, bool kWide>
__global__ void __launch_bounds__(kThreads, 2)
logits_kernel(const float* X, const float* W, int T, int64_t V, int d, float* Z) {
    constexpr int ROWS = kSums / TOK;
    extern __shared__ __align__(16) float xs[];            // [token][pitch]
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int pitch = (d + kStep - 1) / kStep * kStep, padded = (T + TOK - 1) / TOK * TOK;
    grid_wait();
    grid_release();
    for (int i = threadIdx.x; i < padded * pitch; i += kThreads) {
        const int t = i / pitch, k = i - t * pitch;
        xs[i] = t < T && k < d ? X[static_cast<int64_t>(t) * d + k] : 0.0f;
    }
    __syncthreads();
    constexpr int kBlockRows = ROWS * kThreads / 32;
    for (int64_t v = static_cast<int64_t>(blockIdx.x) * kBlockRows + warp * ROWS; v < V; v += static_cast<int64_t>(gridDim.x) * kBlockRows) {
        auto load = [&](int k, float4 (&w)[ROWS]) {
#pragma unroll
            for (int r = 0; r < ROWS; ++r) {
                const float* row = W + (v + r) * d + k;
                if constexpr (kWide) {
                    w[r] = v + r < V && k < d ? *reinterpret_cast<const float4*>(row) : make_float4(0.f, 0.f, 0.f, 0.f);
                } else {
                    auto at = [&](int j) { return v + r < V && k + j < d ? row[j] : 0.0f; };
                    w[r] = make_float4(at(0), at(1), at(2), at(3));
                }
            }
        };
        for (int p0 = 0; p0 < padded; p0 += TOK) {
            float acc[kSums];
#pragma unroll
            for (int i = 0; i < kSums; ++i) acc[i] = 0.0f;
            float4 w[ROWS];
            load(4 * lane, w);
            for (int k = 4 * lane; k < pitch; k += kStep) {        // the same turns for every lane
                float4 next[ROWS];
                load(k + kStep, next);                              // beyond the row: zeros
#pragma unroll
                for (int t = 0; t < TOK; ++t) {
                    const float4 x = *reinterpret_cast<const float4*>(xs + (p0 + t) * pitch + k);
#pragma unroll
                    for (int r = 0; r < ROWS; ++r) {
                        float& s = acc[r * TOK + t];
                        s = fmaf(w[r].x, x.x, s), s = fmaf(w[r].y, x.y, s), s = fmaf(w[r].z, x.z, s), s = fmaf(w[r].w, x.w, s);
                    }
                }
#pragma unroll
                for (int r = 0; r < ROWS; ++r) w[r] = next[r];
            }
            // the lanes' sums: at each exchange a lane keeps half of the values, and ends with two consecutive ones
#pragma unroll
            for (int o = 16; o > 0; o >>= 1) {
                const bool high = lane & o;
#pragma unroll
                for (int i = 0; i < kSums / 2; ++i) {
                    if (i >= 2 * o) continue;
                    const float give = high ? acc[i] : acc[i + 2 * o], keep = high ? acc[i + 2 * o] : acc[i];
                    acc[i] = keep + __shfl_xor_sync(0xFFFFFFFFu, give, o);
                }
            }
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const int at = 2 * lane + i, t = p0 + at % TOK;
                const int64_t row = v + at / TOK;
                if (t < T && row < V) Z[static_cast<int64_t>(t) * V + row] = acc[i];
            }
        }
    }
}

static size_t shared_bytes(int64_t T, int d) {
    const int64_t tok = T <= 8 ? 8 : 16;
    return static_cast<size_t>((T + tok - 1) / tok * tok) * ((d + kStep - 1) / kStep * kStep) * sizeof(float);
}
bool takes_logits(int64_t T, int d) { return T <= kMost && shared_bytes(T, d) <= kShared; }

int launch_logits(const float* X, const float* W, int64_t T, int64_t V, int d, float* Z, cudaStream_t stream) {
    const bool wide = d % 4 == 0 && aligned16(W);
    auto kernel = T <= 8 ? (wide ? logits_kernel<8, true> : logits_kernel<8, false>)
                         : (wide ? logits_kernel<16, true> : logits_kernel<16, false>);
    DTP_CUDA_TRY(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kShared));
    const int64_t rows = (T <= 8 ? 8 : 4) * kThreads / 32, groups = (V + rows - 1) / rows;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(static_cast<unsigned>(groups < 304 ? groups : 304));
    cfg.blockDim = dim3(kThreads);
    cfg.dynamicSmemBytes = shared_bytes(T, d);
    cfg.stream = stream;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    DTP_CUDA_TRY(cudaLaunchKernelEx(&cfg, kernel, X, W, static_cast<int>(T), V, d, Z));
    return DTP_OK;
}

// --------------------------------------------------------------------- dX and dW

constexpr int kCols = 2 * kThreads;    // columns of a block, two a thread
constexpr int kChunk = 64;             // rows of the vocabulary at once in shared memory
constexpr int kAtOnce = 8;             // of them at once in registers

// dZ's rows v0 .. as [row][token], TP tokens
template <int TP>
__device__ __forceinline__ void fill_dz(const float* dZ, int T, int64_t V, int64_t v0, int64_t v1, float (&s)[kChunk][TP]) {
    for (int i = threadIdx.x; i < kChunk * TP; i += kThreads) {
        const int t = i / kChunk, r = i % kChunk;
        s[r][t] = t < T && v0 + r < v1 ? dZ[static_cast<int64_t>(t) * V + v0 + r] : 0.0f;
    }
}

// kInput: parts[block's range][t][c] = sum over the range's rows of dZ W; else dW[v][c] = sum over the tokens of dZ X.
template <int TP, bool kInput>
__global__ void __launch_bounds__(kThreads, 2)
gradient_kernel(const float* dZ, const float* from, int T, int64_t V, int d, int ranges, float* to) {
    __shared__ __align__(16) float dz[kChunk][TP];
    grid_wait();
    grid_release();
    const int blocks = (d + kCols - 1) / kCols;
    const int range = static_cast<int>(blockIdx.x) / blocks, c = static_cast<int>(blockIdx.x) % blocks * kCols + 2 * threadIdx.x;
    const int64_t first = V * range / ranges, last = V * (range + 1) / ranges;
    const bool pair = d % 2 == 0 && (reinterpret_cast<uintptr_t>(from) & 7) == 0 && (reinterpret_cast<uintptr_t>(to) & 7) == 0;
    auto load = [&](const float* p) {
        if (c >= d) return make_float2(0.0f, 0.0f);
        if (pair) return *reinterpret_cast<const float2*>(p);
        return make_float2(p[0], c + 1 < d ? p[1] : 0.0f);
    };
    auto store = [&](float* p, float2 v) {
        if (c >= d) return;
        if (pair) {
            *reinterpret_cast<float2*>(p) = v;
        } else {
            p[0] = v.x;
            if (c + 1 < d) p[1] = v.y;
        }
    };
    float2 own[TP];            // kInput: the sums; else X
#pragma unroll
    for (int t = 0; t < TP; ++t)
        own[t] = !kInput && t < T ? load(from + static_cast<int64_t>(t) * d + c) : make_float2(0.0f, 0.0f);
    for (int64_t v0 = first; v0 < last; v0 += kChunk) {
        __syncthreads();
        fill_dz<TP>(dZ, T, V, v0, last, dz);
        __syncthreads();
        const int rows = last - v0 < kChunk ? static_cast<int>(last - v0) : kChunk;
        for (int r0 = 0; r0 < rows; r0 += kAtOnce) {       // their loads in flight together
            float2 w[kAtOnce];
#pragma unroll
            for (int j = 0; j < kAtOnce; ++j)
                w[j] = kInput && r0 + j < rows ? load(from + (v0 + r0 + j) * d + c) : make_float2(0.0f, 0.0f);
#pragma unroll
            for (int j = 0; j < kAtOnce; ++j) {
#pragma unroll
                for (int t = 0; t < TP; t += 4) {
                    const float4 q = *reinterpret_cast<const float4*>(&dz[r0 + j][t]);
                    const float g[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        float2& s = kInput ? own[t + i] : w[j];
                        const float2 f = kInput ? w[j] : own[t + i];
                        s.x = fmaf(g[i], f.x, s.x), s.y = fmaf(g[i], f.y, s.y);
                    }
                }
                if (!kInput && r0 + j < rows) store(to + (v0 + r0 + j) * d + c, w[j]);
            }
        }
    }
    if constexpr (kInput) {
#pragma unroll
        for (int t = 0; t < TP; ++t)
            if (t < T) store(to + (static_cast<int64_t>(range) * T + t) * d + c, own[t]);
    }
}

// Ranges of a vocabulary of V for d columns: blocks for 152 SMs, two each, of at least one chunk.
int ranges_of(int64_t V, int d) {
    const int64_t blocks = (d + kCols - 1) / kCols, n = (304 + blocks - 1) / blocks, most = (V + kChunk - 1) / kChunk;
    return static_cast<int>(n < most ? n : most);
}

template <bool kInput>
static int launch_gradient(const float* dZ, const float* from, int64_t T, int64_t V, int d, int ranges, float* to, cudaStream_t stream) {
    auto kernel = T <= 8 ? gradient_kernel<8, kInput> : T <= 16 ? gradient_kernel<16, kInput> : T <= 24 ? gradient_kernel<24, kInput> : gradient_kernel<32, kInput>;
    return layer::launch_after(kernel, static_cast<int64_t>(ranges) * ((d + kCols - 1) / kCols), stream, dZ, from, static_cast<int>(T), V,
                               d, ranges, to);
}

// parts [ranges][T, d]
int launch_dx(const float* dZ, const float* W, int64_t T, int64_t V, int d, int ranges, float* parts, cudaStream_t stream) {
    return launch_gradient<true>(dZ, W, T, V, d, ranges, parts, stream);
}
int launch_dw(const float* dZ, const float* X, int64_t T, int64_t V, int d, float* dW, cudaStream_t stream) {
    // more ranges than for dX: nothing is added up behind them
    const int64_t blocks = (d + kCols - 1) / kCols, n = (1216 + blocks - 1) / blocks, most = (V + kChunk - 1) / kChunk;
    return launch_gradient<false>(dZ, X, T, V, d, static_cast<int>(n < most ? n : most), dW, stream);
}

}  // namespace fewl
}  // namespace dtp
