// vocab_loss.cu -- softmax cross entropy over a vocabulary from the hidden states, and its gradients:
//
//     z_t = W x_t,  lse_t = log sum_v exp z_tv,  loss_t = lse_t - z_t[y_t]
//     dz_t = dloss_t (exp(z_t - lse_t) - onehot(y_t)),  dX = dZ W,  dW = dZ^T X
//
// in pieces of the vocabulary, so that no more than a piece of the logits exists at a time.  Forward, each row's maximum and
// sum of exponentials of every chunk of columns meet in a last launch.  Backward, a piece of the logits is made again, turned into dZ,
// and multiplied both ways; dX is added up over the pieces in fp32.
#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include "dtp_common.cuh"
#include "layer_common.cuh"
#include "layer_host.cuh"

namespace dtp {
namespace layer {

constexpr int kChunk = 8192;                         // columns of a partial sum
constexpr size_t kPieceBytes = size_t(256) << 20;    // of a piece of the logits

// A row's maximum and its sum of exp(z - maximum).
struct Part { float top, sum; };
__device__ __forceinline__ Part join(const Part& a, const Part& b) {
    const float top = fmaxf(a.top, b.top);
    // a part that holds nothing, or only -inf, counts for nothing
    const float u = a.top == top ? a.sum : a.sum * expf(a.top - top), v = b.top == top ? b.sum : b.sum * expf(b.top - top);
    return Part{top, u + v};
}

// Z [T, cols] in fp32, columns v0 .. of the vocabulary: parts[chunk][t], and the target's logit where it is among them.
__global__ void __launch_bounds__(256)
parts_kernel(const float* Z, int64_t T, int cols, int v0, const int64_t* targets, Part* parts, float* hit) {
    __shared__ Part red[8];
    grid_wait();
    grid_release();
    const int chunks = (cols + kChunk - 1) / kChunk;
    for (int64_t i = blockIdx.x; i < T * chunks; i += gridDim.x) {
        const int64_t t = i / chunks;
        const int c = static_cast<int>(i - t * chunks), c1 = (c + 1) * kChunk < cols ? (c + 1) * kChunk : cols;
        const float* z = Z + t * cols;
        Part p{-INFINITY, 0.0f};
        bool nan = false;
        for (int j = c * kChunk + threadIdx.x; j < c1; j += 256) {
            nan |= isnan(z[j]);
            p = join(p, Part{z[j], 1.0f});
        }
        if (nan) p.sum = NAN;
#pragma unroll
        for (int o = 16; o > 0; o >>= 1)
            p = join(p, Part{__shfl_xor_sync(0xFFFFFFFFu, p.top, o), __shfl_xor_sync(0xFFFFFFFFu, p.sum, o)});
        __syncthreads();
        if ((threadIdx.x & 31) == 0) red[threadIdx.x >> 5] = p;
        __syncthreads();
        if (threadIdx.x == 0) {
            for (int w = 1; w < 8; ++w) p = join(p, red[w]);
            parts[c * T + t] = p;
            const int64_t y = targets[t] - v0;
            if (c == 0 && y >= 0 && y < cols) hit[t] = z[y];
        }
    }
}

// The parts of each token joined in their order: a warp takes every eighth part of 32 tokens.  A target that is no token's sets the status.
__global__ void __launch_bounds__(256)
loss_kernel(const Part* parts, int64_t count, const float* hit, const int64_t* targets, int64_t T, int V, int64_t ignore,
            float* loss, float* lse, int* status) {
    __shared__ Part red[8][32];
    grid_wait();
    grid_release();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int64_t t = blockIdx.x * 32ll + lane;
    Part p{-INFINITY, 0.0f};
    if (t < T)
        for (int64_t c = warp; c < count; c += 8) p = join(p, parts[c * T + t]);
    red[warp][lane] = p;
    __syncthreads();
    if (warp != 0 || t >= T) return;
    for (int w = 1; w < 8; ++w) p = join(p, red[w][lane]);
    const float l = p.top + logf(p.sum);
    lse[t] = l;
    const int64_t y = targets[t];
    const bool bad = y != ignore && (y < 0 || y >= V);
    loss[t] = y == ignore ? 0.0f : bad ? NAN : l - hit[t];
    if (bad) atomicCAS(status, static_cast<int>(DTP_OK), static_cast<int>(DTP_ERR_ARG));
}

// X at an aligned pitch, with zeros in the rows of tokens without a target: whatever stands there must not reach dW.
template <typename E>
__global__ void __launch_bounds__(256)
live_rows_kernel(const E* X, int64_t T, int d, int64_t pitch, const int64_t* targets, int64_t ignore, int V, E* out, int* status) {
    grid_wait();
    grid_release();
    if (blockIdx.x == 0 && threadIdx.x == 0) *status = DTP_OK;
    for (int64_t t = blockIdx.x; t < T; t += gridDim.x) {
        const int64_t y = targets[t];
        const bool live = y != ignore && y >= 0 && y < V;
        for (int i = threadIdx.x; i < d; i += 256) out[t * pitch + i] = live ? X[t * d + i] : from_f32<E>(0.0f);
    }
}

template <typename E>
__global__ void __launch_bounds__(256)
dz_kernel(const float* Z, int64_t T, int cols, int v0, const int64_t* targets, int64_t ignore, int V, const float* dloss,
          const float* lse, E* dZ, int64_t ld, int* status) {
    grid_wait();
    grid_release();
    for (int64_t t = blockIdx.x; t < T; t += gridDim.x) {
        const int64_t y = targets[t];
        const bool bad = y != ignore && (y < 0 || y >= V), live = y != ignore && !bad;
        if (bad && threadIdx.x == 0) atomicCAS(status, static_cast<int>(DTP_OK), static_cast<int>(DTP_ERR_ARG));
        const float g = dloss[t], l = lse[t];
        for (int j = threadIdx.x; j < cols; j += 256) {
            const float p = expf(Z[t * cols + j] - l) - (y - v0 == j ? 1.0f : 0.0f);
            dZ[t * ld + j] = from_f32<E>(live ? p * g : 0.0f);
        }
    }
}

// sum += part, and the last time the sum in its type
template <typename E>
__global__ void __launch_bounds__(256) add_kernel(const float* part, int64_t n, int first, float* sum, E* out) {
    grid_wait();
    grid_release();
    for (int64_t i = blockIdx.x * 256ll + threadIdx.x; i < n; i += gridDim.x * 256ll) {
        const float v = first ? part[i] : sum[i] + part[i];
        if (out) out[i] = from_f32<E>(v);
        else sum[i] = v;
    }
}

static int64_t grid_of(int64_t blocks) { return blocks < 8192 ? blocks : 8192; }

// Columns of a piece of T tokens' logits.
static int piece_cols(int64_t T, int V) {
    int64_t n = static_cast<int64_t>(kPieceBytes / sizeof(float)) / T / 128 * 128;
    if (n < 128) n = 128;
    return static_cast<int>(n < V ? n : V);
}
static int64_t parts_of(int64_t T, int V) {
    const int piece = piece_cols(T, V);
    const int64_t whole = V / piece, rest = V % piece;
    return whole * ((piece + kChunk - 1) / kChunk) + (rest + kChunk - 1) / kChunk;
}

// What a call takes from its workspace.
struct LossSpace {
    float* Z;
    void* dz;            // also what the products make of Z in their type
    Part* parts;
    float* hit;
    void* x;
    float *part, *sum;
};
static LossSpace carve(Carver& c, int64_t T, int d, int V, int dtype, int backward) {
    LossSpace s{};
    const int piece = piece_cols(T, V);
    s.Z = static_cast<float*>(c.take(static_cast<size_t>(T) * piece * sizeof(float)));
    s.dz = c.take(static_cast<size_t>(T) * padded(piece) * elem(dtype));
    s.parts = static_cast<Part*>(c.take(static_cast<size_t>(T) * parts_of(T, V) * sizeof(Part)));
    s.hit = static_cast<float*>(c.take(static_cast<size_t>(T) * sizeof(float)));
    if (backward) {
        s.x = c.take(static_cast<size_t>(T) * padded(d) * elem(dtype));
        s.part = static_cast<float*>(c.take(static_cast<size_t>(T) * d * sizeof(float)));
        s.sum = static_cast<float*>(c.take(static_cast<size_t>(T) * d * sizeof(float)));
    }
    return s;
}

size_t loss_workspace_bytes(int64_t T, int d, int V, int dtype, int backward) {
    if (T == 0) return kWorkspaceHeader;
    Carver c(nullptr);
    carve(c, T, d, V, dtype, backward);
    c.take(repitch_bytes(T, d, dtype));
    c.take(repitch_bytes(V, d, dtype));
    if (backward) c.take(runs_bytes(T, piece_cols(T, V), d));
    return c.used;
}

// Z = X W_piece^T in fp32
static int logits(Call& call, const Rows& x, const Rows& w, int64_t T, int d, int v0, int cols, const LossSpace& s) {
    Product p;
    p.A[0] = by_row(x.p, x.ld);
    p.B[0] = by_row(static_cast<const uint8_t*>(w.p) + static_cast<size_t>(v0) * w.ld * elem(call.dtype), w.ld);
    p.M = T, p.N = cols, p.K = d;
    p.epi.out = call.dtype == DTP_F32 ? static_cast<void*>(s.Z) : s.dz;
    p.epi.ldo = call.dtype == DTP_F32 ? cols : padded(cols);
    p.epi.Z = call.dtype == DTP_F32 ? nullptr : s.Z;
    p.epi.M = T, p.epi.N = cols;
    return call.run(p);
}

int loss_forward(const void* X, const void* W, const int64_t* targets, int64_t T, int d, int V, int64_t ignore, int dtype,
                 float* loss, float* lse, void* workspace, cudaStream_t stream) {
    Call call{dtype, workspace, stream};
    Carver c(workspace);
    const LossSpace s = carve(c, T, d, V, dtype, 0);
    const int piece = piece_cols(T, V);
    Rows x, w;
    int st = aligned_rows(X, T, d, dtype, c, stream, &x);
    if (st == DTP_OK) st = aligned_rows(W, V, d, dtype, c, stream, &w);
    Part* at = s.parts;
    for (int v0 = 0; st == DTP_OK && v0 < V; v0 += piece) {
        const int cols = V - v0 < piece ? V - v0 : piece;
        st = logits(call, x, w, T, d, v0, cols, s);
        const int64_t chunks = (cols + kChunk - 1) / kChunk;
        if (st == DTP_OK)
            st = launch_after(parts_kernel, grid_of(T * chunks), stream, static_cast<const float*>(s.Z), T, cols, v0, targets, at,
                              s.hit);
        at += chunks * T;
    }
    if (st != DTP_OK) return st;
    return launch_after(loss_kernel, (T + 31) / 32, stream, static_cast<const Part*>(s.parts), parts_of(T, V),
                        static_cast<const float*>(s.hit), targets, T, V, ignore, loss, lse, static_cast<int*>(workspace));
}

template <typename E>
static int backward(const float* dloss, const void* X, const void* W, const int64_t* targets, const float* lse, int64_t T, int d,
                    int V, int64_t ignore, int dtype, void* dX, void* dW, void* workspace, cudaStream_t stream) {
    Call call{dtype, workspace, stream};
    Carver c(workspace);
    const LossSpace s = carve(c, T, d, V, dtype, 1);
    const int piece = piece_cols(T, V);
    int* status = static_cast<int*>(workspace);
    const int64_t ld = padded(d);
    int st = launch_after(live_rows_kernel<E>, grid_of(T), stream, static_cast<const E*>(X), T, d, ld, targets, ignore, V,
                          static_cast<E*>(s.x), status);
    call.fresh = false;
    const Rows x{s.x, ld};
    Rows w;
    if (st == DTP_OK) st = aligned_rows(W, V, d, dtype, c, stream, &w);
    auto* runs = static_cast<float*>(c.take(runs_bytes(T, piece, d)));
    const int64_t values = T * d, add_blocks = grid_of((values + 255) / 256);
    for (int v0 = 0; st == DTP_OK && v0 < V; v0 += piece) {
        const int cols = V - v0 < piece ? V - v0 : piece;
        const int64_t ldz = padded(cols);
        st = logits(call, x, w, T, d, v0, cols, s);
        if (st == DTP_OK)
            st = launch_after(dz_kernel<E>, grid_of(T), stream, static_cast<const float*>(s.Z), T, cols, v0, targets, ignore, V,
                              dloss, lse, static_cast<E*>(s.dz), ldz, status);
        if (st == DTP_OK && dX) {
            const bool last = cols == V - v0;
            Product p;
            p.A[0] = by_row(s.dz, ldz);
            p.B[0] = by_col(static_cast<const uint8_t*>(w.p) + static_cast<size_t>(v0) * w.ld * sizeof(E), w.ld);
            p.M = T, p.N = d, p.K = cols;
            p.epi.out = dX, p.epi.ldo = d, p.epi.M = T, p.epi.N = d;
            const bool one = last && v0 == 0;
            if (!one) {
                if (dtype == DTP_F32) p.epi.out = s.part;
                else p.epi.Z = s.part;
            }
            st = call.run(p);
            if (st == DTP_OK && !one)
                st = launch_after(add_kernel<E>, add_blocks, stream, static_cast<const float*>(s.part), values,
                                  static_cast<int>(v0 == 0), s.sum, last ? static_cast<E*>(dX) : nullptr);
        }
        if (st == DTP_OK && dW)
            st = weight_gradient(call, Also{by_col(s.dz, ldz), by_col(x.p, x.ld), cols, d, static_cast<E*>(dW) + static_cast<int64_t>(v0) * d, d},
                                 T, runs);
    }
    return st;
}

int loss_backward(const float* dloss, const void* X, const void* W, const int64_t* targets, const float* lse, int64_t T, int d,
                  int V, int64_t ignore, int dtype, void* dX, void* dW, void* workspace, cudaStream_t stream) {
    if (T == 0) {
        const size_t bytes = static_cast<size_t>(V) * d * elem(dtype);
        DTP_CUDA_TRY(cudaMemsetAsync(workspace, 0, sizeof(int), stream));
        if (dW) DTP_CUDA_TRY(cudaMemsetAsync(dW, 0, bytes, stream));
        return DTP_OK;
    }
    auto go = dtype == DTP_BF16 ? backward<__nv_bfloat16> : backward<float>;
    return go(dloss, X, W, targets, lse, T, d, V, ignore, dtype, dX, dW, workspace, stream);
}

}  // namespace layer
}  // namespace dtp
