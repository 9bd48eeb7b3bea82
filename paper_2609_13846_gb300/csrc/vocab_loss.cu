// vocab_loss.cu -- softmax cross entropy over a vocabulary from the hidden states, and its gradients:
//
//     z_t = W x_t,  lse_t = log sum_v exp z_tv,  loss_t = lse_t - z_t[y_t]
//     dz_t = dloss_t (exp(z_t - lse_t) - onehot(y_t)),  dX = dZ W,  dW = dZ^T X
//
// in pieces of the vocabulary, so that no more than a piece of the logits exists at a time.  Forward, each row's maximum and
// sum of exponentials of every chunk of columns meet in a last launch; bf16 products of more than 32 tokens take them from the
// accumulators (kEpiParts), and their logits are never stored.  Backward, a piece of the logits is made again and turned into
// dZ, in the product's epilogue (kEpiProb) or by a kernel of its own, and multiplied both ways; dX is added up over the
// pieces in fp32.
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

__device__ __forceinline__ Part join(const Part& a, const Part& b) {
    const float top = fmaxf(a.top, b.top);
    // a part that holds nothing, or only -inf, counts for nothing
    const float u = a.top == top ? a.sum : a.sum * exp2_fast(a.top - top), v = b.top == top ? b.sum : b.sum * exp2_fast(b.top - top);
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
            p = join(p, Part{z[j] * kLog2e, 1.0f});
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
            if (c == 0 && y >= 0 && y < cols) hit[t] = z[y];      // of one piece
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
    const float l = kLn2 * (p.top + log2f(p.sum));
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

// dZ of Z [T, cols], columns v0 .. of the vocabulary; a block takes kChunk columns of a token.  dZ may be Z.
template <typename E>
__global__ void __launch_bounds__(256)
dz_kernel(const float* Z, int64_t T, int cols, Vocab e, E* dZ, int64_t ld, int* status) {
    grid_wait();
    grid_release();
    const int chunks = (cols + kChunk - 1) / kChunk;
    for (int64_t i = blockIdx.x; i < T * chunks; i += gridDim.x) {
        const int64_t t = i / chunks;
        const int c = static_cast<int>(i - t * chunks), c1 = (c + 1) * kChunk < cols ? (c + 1) * kChunk : cols;
        const int64_t y = e.targets[t];
        if (c == 0 && threadIdx.x == 0 && e.bad(y)) atomicCAS(status, static_cast<int>(DTP_OK), static_cast<int>(DTP_ERR_ARG));
        const bool live = e.live(y);
        const float g = live ? e.dloss[t] : 0.0f, lse2 = e.lse[t] * kLog2e;
#pragma unroll 4
        for (int j = c * kChunk + threadIdx.x; j < c1; j += 256) {
            const float p = exp2_fast(fmaf(Z[t * cols + j], kLog2e, -lse2)) - (y - e.v0 == j ? 1.0f : 0.0f);
            dZ[t * ld + j] = from_f32<E>(live ? p * g : 0.0f);
        }
    }
}

// dX from its sums
__global__ void __launch_bounds__(256) round_kernel(const float* sum, int64_t n, __nv_bfloat16* out) {
    grid_wait();
    grid_release();
    const int64_t words = n / 4;
    for (int64_t i = blockIdx.x * 256ll + threadIdx.x; i < words; i += gridDim.x * 256ll) {
        const float4 v = reinterpret_cast<const float4*>(sum)[i];
        const __nv_bfloat162 a = __floats2bfloat162_rn(v.x, v.y), b = __floats2bfloat162_rn(v.z, v.w);
        reinterpret_cast<uint2*>(out)[i] = make_uint2(*reinterpret_cast<const uint32_t*>(&a), *reinterpret_cast<const uint32_t*>(&b));
    }
    const int64_t rest = 4 * words + threadIdx.x;
    if (blockIdx.x == 0 && rest < n) out[rest] = __float2bfloat16_rn(sum[rest]);
}

static int64_t grid_of(int64_t blocks) { return blocks < 8192 ? blocks : 8192; }

// Whether a product's epilogue takes the softmax.  Up to 32 tokens the products are the few-token kernels', which stream the
// weights at the memory's rate; their logits are small beside those.
static bool fused(int64_t T, int dtype) { return dtype == DTP_BF16 && T > 32; }

// Tokens of a forward run: its parts, and the logits' pieces where there are any, stay within 256 MB.
static int64_t forward_rows(int64_t T, int V, int dtype) {
    int64_t n = 16384;
    if (fused(T, dtype)) n = static_cast<int64_t>(kPieceBytes / sizeof(Part)) / gtc::most_chunks(V) / 256 * 256;
    if (n < 256) n = 256;
    return n < T ? n : T;
}
// Columns of a piece of T tokens' logits.
static int piece_cols(int64_t T, int V, size_t bytes) {
    int64_t n = static_cast<int64_t>(bytes) / T / 256 * 256;
    if (n < 256) n = 256;
    return static_cast<int>(n < V ? n : V);
}
static int forward_piece(int64_t rows, int V, int dtype) {
    return fused(rows, dtype) ? V : piece_cols(rows, V, kPieceBytes / sizeof(float));
}
static int backward_piece(int64_t T, int V, int dtype) { return piece_cols(T, V, kPieceBytes / elem(dtype)); }
static int64_t parts_of(int64_t rows, int V, int dtype) {
    if (fused(rows, dtype)) return gtc::most_chunks(V);
    const int piece = forward_piece(rows, V, dtype);
    const int64_t whole = V / piece, rest = V % piece;
    return whole * ((piece + kChunk - 1) / kChunk) + (rest + kChunk - 1) / kChunk;
}

// What a call takes from its workspace.
struct ForwardSpace {
    float* Z;            // a piece of the logits, where they are stored
    Part* parts;
    float* hit;
};
static ForwardSpace carve_forward(Carver& c, int64_t rows, int V, int dtype) {
    ForwardSpace s{};
    if (!fused(rows, dtype)) s.Z = static_cast<float*>(c.take(static_cast<size_t>(rows) * forward_piece(rows, V, dtype) * sizeof(float)));
    s.parts = static_cast<Part*>(c.take(static_cast<size_t>(rows) * parts_of(rows, V, dtype) * sizeof(Part)));
    s.hit = static_cast<float*>(c.take(static_cast<size_t>(rows) * sizeof(float)));
    return s;
}
struct BackwardSpace {
    float* Z;            // the same; in fp32 dZ takes its place
    void* dz;
    void* x;
    float *sum, *runs;
};
static BackwardSpace carve_backward(Carver& c, int64_t T, int d, int V, int dtype) {
    BackwardSpace s{};
    const int piece = backward_piece(T, V, dtype);
    if (!fused(T, dtype)) s.Z = static_cast<float*>(c.take(static_cast<size_t>(T) * piece * sizeof(float)));
    s.dz = dtype == DTP_F32 ? s.Z : c.take(static_cast<size_t>(T) * padded(piece) * elem(dtype));
    s.x = c.take(static_cast<size_t>(T) * padded(d) * elem(dtype));
    s.sum = static_cast<float*>(c.take(dtype == DTP_BF16 && piece < V ? static_cast<size_t>(T) * d * sizeof(float) : 0));
    s.runs = static_cast<float*>(c.take(runs_bytes(T, piece, d)));
    return s;
}

size_t loss_workspace_bytes(int64_t T, int d, int V, int dtype, int backward) {
    if (T == 0) return kWorkspaceHeader;
    Carver f(nullptr);
    f.take(repitch_bytes(V, d, dtype));
    Carver b = f;
    f.take(repitch_bytes(T, d, dtype));
    const int64_t rows = forward_rows(T, V, dtype);
    carve_forward(f, rows, V, dtype);
    // the last run may be one of few tokens
    if (T % rows) {
        Carver last = f;
        last.used = f.used;
        carve_forward(last, T % rows, V, dtype);
        f.used = last.used;
    }
    if (!backward) return f.used;
    carve_backward(b, T, d, V, dtype);
    return f.used > b.used ? f.used : b.used;
}

// The product of T tokens with columns v0 .. of the vocabulary.
static Product logits(const Rows& x, int64_t t0, const Rows& w, int64_t T, int d, int v0, int cols, int dtype) {
    auto from = [&](const Rows& r, int64_t row) {
        return by_row(static_cast<const uint8_t*>(r.p) + static_cast<size_t>(row) * r.ld * elem(dtype), r.ld);
    };
    Product p;
    p.A[0] = from(x, t0);
    p.B[0] = from(w, v0);
    p.M = T, p.N = cols, p.K = d;
    p.epi.M = T, p.epi.N = cols, p.epi.ldo = cols;
    return p;
}

// Stored logits: Z [T, cols] in fp32.
static int store_logits(Call& call, Product& p, float* Z) {
    if (call.dtype == DTP_F32) p.epi.out = Z;
    else p.epi.Z = Z;
    return call.run(p);
}

int loss_forward(const void* X, const void* W, const int64_t* targets, int64_t T, int d, int V, int64_t ignore, int dtype,
                 float* loss, float* lse, void* workspace, cudaStream_t stream) {
    Call call{dtype, workspace, stream};
    Carver c(workspace);
    Rows x, w;
    int st = aligned_rows(W, V, d, dtype, c, stream, &w);
    if (st == DTP_OK) st = aligned_rows(X, T, d, dtype, c, stream, &x);
    int* status = static_cast<int*>(workspace);
    const int64_t most = forward_rows(T, V, dtype);
    ForwardSpace s = carve_forward(c, most, V, dtype);
    for (int64_t t0 = 0; st == DTP_OK && t0 < T; t0 += most) {
        const int64_t rows = T - t0 < most ? T - t0 : most;
        if (rows < most) s = carve_forward(c, rows, V, dtype);
        Vocab e;
        e.targets = targets + t0, e.ignore = ignore, e.V = V, e.parts = s.parts, e.hit = s.hit;
        int64_t count = 0;
        if (fused(rows, dtype)) {
            Product p = logits(x, t0, w, rows, d, 0, V, dtype);
            p.epi.kind = kEpiParts, p.epi.vocab = e;
            st = gtc::launch(p, status, call.fresh, stream, &count);
            call.fresh = false;
        }
        const int piece = forward_piece(rows, V, dtype);
        for (int v0 = 0; st == DTP_OK && s.Z && v0 < V; v0 += piece) {
            const int cols = V - v0 < piece ? V - v0 : piece;
            Product p = logits(x, t0, w, rows, d, v0, cols, dtype);
            st = store_logits(call, p, s.Z);
            const int64_t chunks = (cols + kChunk - 1) / kChunk;
            if (st == DTP_OK)
                st = launch_after(parts_kernel, grid_of(rows * chunks), stream, static_cast<const float*>(s.Z), rows, cols, v0,
                                  e.targets, s.parts + count * rows, s.hit);
            count += chunks;
        }
        if (st == DTP_OK)
            st = launch_after(loss_kernel, (rows + 31) / 32, stream, static_cast<const Part*>(s.parts), count,
                              static_cast<const float*>(s.hit), e.targets, rows, V, ignore, loss + t0, lse + t0, status);
    }
    return st;
}

template <typename E>
static int backward(const float* dloss, const void* X, const void* W, const int64_t* targets, const float* lse, int64_t T, int d,
                    int V, int64_t ignore, int dtype, void* dX, void* dW, void* workspace, cudaStream_t stream) {
    Call call{dtype, workspace, stream};
    Carver c(workspace);
    Rows w;
    int st = aligned_rows(W, V, d, dtype, c, stream, &w);
    const BackwardSpace s = carve_backward(c, T, d, V, dtype);
    const int piece = backward_piece(T, V, dtype);
    int* status = static_cast<int*>(workspace);
    const Rows x{s.x, padded(d)};
    Vocab e;
    e.targets = targets, e.ignore = ignore, e.V = V, e.lse = lse, e.dloss = dloss;
    if (st == DTP_OK)
        st = launch_after(live_rows_kernel<E>, grid_of(T), stream, static_cast<const E*>(X), T, d, x.ld, targets, ignore, V,
                          static_cast<E*>(s.x), status);
    call.fresh = false;
    for (int v0 = 0; st == DTP_OK && v0 < V; v0 += piece) {
        const int cols = V - v0 < piece ? V - v0 : piece;
        const int64_t ldz = dtype == DTP_F32 ? cols : padded(cols);
        e.v0 = v0;
        Product p = logits(x, 0, w, T, d, v0, cols, dtype);
        if (fused(T, dtype)) {
            p.epi.kind = kEpiProb, p.epi.vocab = e, p.epi.out = s.dz, p.epi.ldo = ldz;
            st = gtc::launch(p, status, 0, stream);
        } else {
            st = store_logits(call, p, s.Z);
            if (st == DTP_OK)
                st = launch_after(dz_kernel<E>, grid_of(T * ((cols + kChunk - 1) / kChunk)), stream, static_cast<const float*>(s.Z),
                                  T, cols, e, static_cast<E*>(s.dz), ldz, status);
        }
        if (st == DTP_OK && dX) {
            Product q;
            q.A[0] = by_row(s.dz, ldz);
            q.B[0] = by_col(static_cast<const uint8_t*>(w.p) + static_cast<size_t>(v0) * w.ld * sizeof(E), w.ld);
            q.M = T, q.N = d, q.K = cols;
            q.epi.ldo = d, q.epi.M = T, q.epi.N = d;
            if (dtype == DTP_F32) q.epi.out = dX, q.epi.residual = v0 > 0 ? dX : nullptr;
            else if (piece >= V) q.epi.out = dX;
            else q.epi.Z = s.sum, q.epi.add = v0 > 0;
            st = call.run(q);
        }
        if (st == DTP_OK && dW)
            st = weight_gradient(call, Also{by_col(s.dz, ldz), by_col(x.p, x.ld), cols, d, static_cast<E*>(dW) + static_cast<int64_t>(v0) * d, d},
                                 T, s.runs);
    }
    if (st == DTP_OK && dX && dtype == DTP_BF16 && piece < V)
        st = launch_after(round_kernel, grid_of((T * d / 4 + 255) / 256 + 1), stream, static_cast<const float*>(s.sum), T * d,
                          static_cast<__nv_bfloat16*>(dX));
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
