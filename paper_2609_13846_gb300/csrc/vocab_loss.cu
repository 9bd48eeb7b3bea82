// vocab_loss.cu -- softmax cross entropy over a vocabulary from the hidden states, and its gradients:
//
//     z_t = W x_t,  lse_t = log sum_v exp z_tv,  loss_t = lse_t - z_t[y_t]
//     dz_t = dloss_t (exp(z_t - lse_t) - onehot(y_t)),  dX = dZ W,  dW = dZ^T X
//
// in pieces of the vocabulary, so that no more than a piece of the logits exists at a time.  Forward, each row's maximum and
// sum of exponentials of every chunk of columns meet in a last launch; bf16 products take them from the accumulators
// (kEpiParts), and their logits are never stored.  Backward, a piece of the logits is made again and turned into
// dZ, in the product's epilogue (kEpiProb) or by a kernel of its own, and multiplied both ways; dX is added up over the
// pieces in fp32.
// The price of not keeping the logits is their product again: 8 T d V operations a training step and not 6.  8192 x 131072 of 1024, a
// tenth of the tokens without a target: 4.9 to 5.2 ms, at the power cap; 4096 x 65536 of 4096 4.8 to 4.9.  One token through 131072 x
// 1024: 51 us, of which 44 stream W.
#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include "dtp_common.cuh"
#include "layer_common.cuh"
#include "layer_host.cuh"

namespace dtp {
namespace layer {

constexpr int kChunk = 8192;                         // columns of a partial sum
constexpr size_t kPieceBytes = size_t(256) << 20;    // of a piece of the logits, or of a run's parts
// of a piece of dZ in bf16 (8192 x 131072 x 1024, forward and backward: 4.84 ms; with 256 MB 4.88, with 64, which L2 would hold, 5.58: the
// launches' ends and the rounds left unfilled cost more than the traffic)
constexpr size_t kDzBytes = size_t(512) << 20;

// Parts joined at their largest logit.  Where that is infinite the terms are taken from 0: parts that hold nothing, or -inf alone, have no
// sum, and one with an infinity has an infinite one.  The exponentials do not wait for one another (one part at a time, 1003 tokens
// of 782 parts: 177 us in all, 172 so).
template <int N>
__device__ __forceinline__ Part join(const Part& a, const Part (&b)[N]) {
    float top = a.top;
#pragma unroll
    for (int j = 0; j < N; ++j) top = fmaxf(top, b[j].top);
    const float from = isinf(top) ? 0.0f : top;
    float sum = a.sum * exp2_fast((a.top - from) * kLog2e);
#pragma unroll
    for (int j = 0; j < N; ++j) sum = fmaf(b[j].sum, exp2_fast((b[j].top - from) * kLog2e), sum);
    return Part{top, sum};
}
__device__ __forceinline__ Part join(const Part& a, const Part& b) {
    const Part one[1] = {b};
    return join(a, one);
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
            if (c == 0 && y >= 0 && y < cols) hit[t] = z[y];      // of one piece
        }
    }
}

// The parts of each token joined: each of 32 warps takes every 32nd part of 32 tokens, eight in flight, and the first one joins the
// warps' in order (a vocabulary of 131072 has 1024 parts from 256-wide tiles, 2048 from the 128-wide ones that a few tokens get; with 8 warps
// and one part at a time one token took 65 us).  A target that is no token's sets the status.
constexpr int kLossWarps = 32;
__global__ void __launch_bounds__(32 * kLossWarps)
loss_kernel(const Part* parts, int64_t count, const float* hit, const int64_t* targets, int64_t T, int V, int64_t ignore,
            float* loss, float* lse, int* status) {
    __shared__ Part red[kLossWarps][32];
    grid_wait();
    grid_release();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int64_t t = blockIdx.x * 32ll + lane;
    Part p{-INFINITY, 0.0f};
    if (t < T) {
        for (int64_t c = warp; c < count; c += 8 * kLossWarps) {
            Part q[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) q[j] = c + j * kLossWarps < count ? parts[(c + j * kLossWarps) * T + t] : Part{-INFINITY, 0.0f};
            p = join(p, q);
        }
    }
    red[warp][lane] = p;
    __syncthreads();
    if (warp != 0 || t >= T) return;
    for (int w = 0; w < kLossWarps; w += 8) {
        Part q[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) q[j] = w + j > 0 ? red[w + j][lane] : Part{-INFINITY, 0.0f};        // p is the first
        p = join(p, q);
    }
    const float rest = kLn2 * log2f(p.sum);
    lse[t] = p.top + rest;
    const int64_t y = targets[t];
    const bool bad = y != ignore && (y < 0 || y >= V);
    // the largest logit first: it takes the target's out exactly where that leads, and the sum beside it is at least 1, so that no
    // loss is negative
    loss[t] = y == ignore ? 0.0f : bad ? NAN : (p.top - hit[t]) + rest;
    if (bad) atomicCAS(status, static_cast<int>(DTP_OK), static_cast<int>(DTP_ERR_ARG));
}

// Which tokens count, for the backward pass (bf16): place[t] is token t's row among them, or -1, and what its row needs is put there; live[0]
// is the rows that the products take, padded to 64 and at least that many, live[1] the tokens.  Tokens that do not count then cost
// nothing, and whatever stands in their rows reaches nothing.  Also dZ's unit, the largest finite size of dloss among them (at least
// 2^-126; else 1): rounding dloss (p - onehot) to bf16 would round dloss of a mean, the same in all rows, and the error would not average
// out.  One block, 4096 tokens at a time.  compact 0: all tokens keep their rows.
struct Compact {
    int* place;
    int* live;
    int64_t* targets;
    float *lse, *dloss, *unit;
};
constexpr int kIndexThreads = 1024;
__global__ void __launch_bounds__(kIndexThreads)
index_kernel(const int64_t* targets, const float* lse, const float* dloss, int64_t T, int64_t ignore, int V, int compact, const Compact to,
             int* status) {
    __shared__ int sums[2][kIndexThreads / 32];
    __shared__ float tops[kIndexThreads / 32];
    grid_wait();
    grid_release();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    int base = 0, turn = 0;
    float top = 0.0f;
    bool bad = false;
    for (int64_t t0 = 0; t0 < T; t0 += 4 * kIndexThreads, ++turn) {
        const int64_t t = t0 + 4 * threadIdx.x;
        int64_t y[4];
        int count = 0;
        bool live[4], counts[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            y[j] = t + j < T ? targets[t + j] : ignore;
            const bool in = y[j] >= 0 && y[j] < V;
            bad |= y[j] != ignore && !in;
            counts[j] = t + j < T && y[j] != ignore && in;
            live[j] = t + j < T && (!compact || counts[j]);
            count += live[j];
        }
        int before = count;          // of the lanes up to this one
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int v = __shfl_up_sync(0xFFFFFFFFu, before, o);
            if (lane >= o) before += v;
        }
        if (lane == 31) sums[turn & 1][warp] = before;
        __syncthreads();
        const int mine = sums[turn & 1][lane];
        int warps = mine;            // of the warps up to `lane`
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int v = __shfl_up_sync(0xFFFFFFFFu, warps, o);
            if (lane >= o) warps += v;
        }
        const int all = __shfl_sync(0xFFFFFFFFu, warps, 31), earlier = __shfl_sync(0xFFFFFFFFu, warps - mine, warp);
        int at = base + earlier + before - count;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            if (t + j >= T) continue;
            to.place[t + j] = live[j] ? at : -1;
            if (!live[j]) continue;
            const float g = dloss[t + j];
            to.targets[at] = y[j], to.lse[at] = lse[t + j], to.dloss[at] = g;
            if (counts[j] && isfinite(g)) top = fmaxf(top, fabsf(g));
            ++at;
        }
        base += all;
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xFFFFFFFFu, top, o));
    if (lane == 0) tops[warp] = top;
    const bool any = __syncthreads_or(bad);
    if (threadIdx.x == 0) {
        for (int w = 1; w < kIndexThreads / 32; ++w) top = fmaxf(top, tops[w]);
        *to.unit = top >= 1.1754944e-38f ? top : 1.0f;
        const int rows = (base + 63) / 64 * 64;
        to.live[0] = rows > 64 ? rows : 64;
        to.live[1] = base;
        *status = any ? static_cast<int>(DTP_ERR_ARG) : static_cast<int>(DTP_OK);
    }
}

// X's rows at an aligned pitch.  With `place` at their places, and zeros in the rows behind the last; rows that have a place but do not count
// are zeros too.  Without, zeros in the rows from T to `rows`.
template <typename E>
__global__ void __launch_bounds__(256)
place_rows_kernel(const E* X, int64_t T, int64_t rows, int d, int64_t pitch, const int64_t* targets, int64_t ignore, int V,
                  const int* place, const int* live, E* out) {
    grid_wait();
    grid_release();
    constexpr int kPer = 16 / sizeof(E);
    const bool wide = d % kPer == 0 && pitch % kPer == 0 && (reinterpret_cast<uintptr_t>(X) & 15) == 0;
    auto row = [&](const E* from, E* to) {            // from NULL: zeros
        if (wide) {
#pragma unroll 4
            for (int i = threadIdx.x; i < d / kPer; i += 256)
                reinterpret_cast<uint4*>(to)[i] = from ? reinterpret_cast<const uint4*>(from)[i] : make_uint4(0, 0, 0, 0);
        } else {
#pragma unroll 4
            for (int i = threadIdx.x; i < d; i += 256) to[i] = from ? from[i] : from_f32<E>(0.0f);
        }
    };
    auto counts = [&](int64_t t) {
        if (!targets) return true;
        const int64_t y = targets[t];
        return y != ignore && y >= 0 && y < V;
    };
    const int64_t held = live ? live[1] : T, all = live ? live[0] : rows;
    for (int64_t t = blockIdx.x; t < T; t += gridDim.x) {
        const int64_t at = place ? place[t] : t;
        if (at >= 0) row(counts(t) ? X + t * d : nullptr, out + at * pitch);
    }
    for (int64_t t = held + blockIdx.x; t < all; t += gridDim.x) row(nullptr, out + t * pitch);
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
        const float g = live ? e.dloss[t] : 0.0f, lse = e.lse[t];
#pragma unroll 4
        for (int j = c * kChunk + threadIdx.x; j < c1; j += 256) {
            const float p = exp2_fast((Z[t * cols + j] - lse) * kLog2e) - (y - e.v0 == j ? 1.0f : 0.0f);
            dZ[t * ld + j] = from_f32<E>(live ? p * g : 0.0f);
        }
    }
}

// fp32: dX (+)= the sums of its parts
__global__ void __launch_bounds__(256) add_parts_kernel(const float* sums, int parts, int64_t n, int add, float* out) {
    grid_wait();
    grid_release();
    for (int64_t i = blockIdx.x * 256ll + threadIdx.x; i < n; i += gridDim.x * 256ll) {
        float v = add ? out[i] : 0.0f;
#pragma unroll 8
        for (int p = 0; p < parts; ++p) v += sums[p * n + i];
        out[i] = v;
    }
}

// fp32: zeros for the tokens that do not count, whose sums are 0 times what stands in W.
__global__ void __launch_bounds__(256) clear_rows_kernel(int64_t T, int d, const Vocab e, float* dX) {
    grid_wait();
    grid_release();
    for (int64_t t = blockIdx.x; t < T; t += gridDim.x) {
        if (e.live(e.targets[t])) continue;
        for (int i = threadIdx.x; i < d; i += 256) dX[t * d + i] = 0.0f;
    }
}

// dX from its sums, in dZ's unit: `parts` of them, `stride` values apart, each token's at its place; zeros for those that do not count.  A
// warp takes 512 columns of a token.
__global__ void __launch_bounds__(256)
round_kernel(const float* sum, int parts, int64_t stride, int64_t T, int d, const int64_t* targets, int64_t ignore, int V,
             const int* place, const float* unit, __nv_bfloat16* out) {
    grid_wait();
    grid_release();
    const float u = *unit;
    const int pieces = (d + 511) / 512, lane = threadIdx.x & 31;
    const bool wide = d % 4 == 0;          // the binding's and the C ABI's tensors start on 16 bytes
    for (int64_t i = blockIdx.x * 8ll + (threadIdx.x >> 5); i < T * pieces; i += gridDim.x * 8ll) {
        const int64_t t = i / pieces;
        const int64_t y = targets[t];
        const int c0 = static_cast<int>(i - t * pieces) * 512, at = y != ignore && y >= 0 && y < V ? place[t] : -1;
        const float* from = sum + static_cast<int64_t>(at) * d;
        __nv_bfloat16* to = out + t * d;
        if (wide) {
            float4 v[4];
#pragma unroll
            for (int q = 0; q < 4; ++q) v[q] = make_float4(0.f, 0.f, 0.f, 0.f);
            for (int p = 0; p < (at >= 0 ? parts : 0); ++p) {
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    const int c = c0 + 128 * q + 4 * lane;
                    if (c >= d) continue;
                    const float4 w = *reinterpret_cast<const float4*>(from + p * stride + c);
                    v[q].x += w.x, v[q].y += w.y, v[q].z += w.z, v[q].w += w.w;
                }
            }
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const int c = c0 + 128 * q + 4 * lane;
                if (c >= d) continue;
                const __nv_bfloat162 a = __floats2bfloat162_rn(u * v[q].x, u * v[q].y), b = __floats2bfloat162_rn(u * v[q].z, u * v[q].w);
                *reinterpret_cast<uint2*>(to + c) = make_uint2(*reinterpret_cast<const uint32_t*>(&a), *reinterpret_cast<const uint32_t*>(&b));
            }
        } else {
            const int c1 = c0 + 512 < d ? c0 + 512 : d;
            for (int c = c0 + lane; c < c1; c += 32) {
                float v = 0.0f;
                for (int p = 0; p < (at >= 0 ? parts : 0); ++p) v += from[p * stride + c];
                to[c] = __float2bfloat16_rn(u * v);
            }
        }
    }
}

static int64_t grid_of(int64_t blocks) { return blocks < 8192 ? blocks : 8192; }

// bf16: a product's epilogue takes the softmax, and two launches a piece make the gradients, of rows padded to 64, the products' k block.
constexpr int64_t kRowPad = 64;
static int64_t padded_rows(int64_t T) { return (T + kRowPad - 1) / kRowPad * kRowPad; }

// Tokens of a forward run: its parts, and the logits' pieces where there are any, stay within kPieceBytes.
static int64_t forward_rows(int64_t T, int V, int dtype) {
    int64_t n = 16384;
    if (dtype == DTP_BF16) n = static_cast<int64_t>(kPieceBytes / sizeof(Part)) / gtc::most_chunks(V) / 256 * 256;
    if (n < 256) n = 256;
    return n < T ? n : T;
}
constexpr int64_t kFew = 32;          // tokens of the fp32 kernels for few of them
// Columns of a piece of T tokens' logits (fp32), forward or backward.
static int stored_cols(int64_t T, int V) {
    int64_t n = static_cast<int64_t>(kPieceBytes / sizeof(float)) / T / 256 * 256;
    if (n < 256) n = 256;
    return static_cast<int>(n < V ? n : V);
}
static int64_t parts_of(int64_t rows, int V, int dtype) {
    if (dtype == DTP_BF16) return gtc::most_chunks(V);
    const int piece = stored_cols(rows, V);
    const int64_t whole = V / piece, rest = V % piece;
    return whole * ((piece + kChunk - 1) / kChunk) + (rest + kChunk - 1) / kChunk;
}

// The pieces of the backward pass: columns of each but the last, and the parts in which dX is summed.  bf16: of the numbers of pieces that
// keep dZ within kDzBytes, up to twice the least, the one whose tiles leave the fewest rounds of pairs unfilled; sizes near
// 8192 x 131072 x 1024 differ by 10% in that.
// fp32: few tokens have few tiles, and dX a sum over the whole piece: as many parts of it as blocks of 64 x 128 leave the chip's 608
// places empty after the tiles are split in eight, with at least 512 columns for each (64 tokens, 32768 x 1024: 570 us in one), or those
// of the few tokens' kernel.
struct Pieces { int cols, parts; };
static Pieces backward_pieces(int64_t T, int d, int V, int dtype) {
    if (dtype == DTP_F32) {
        const int cols = stored_cols(T, V);
        if (T <= kFew) return Pieces{cols, fewl::ranges_of(cols, d)};
        const int64_t tiles = (T + 63) / 64 * ((d + 127) / 128), room = 608 / (8 * tiles), most = cols / 512;
        const int64_t parts = room < most ? room : most;
        return Pieces{cols, static_cast<int>(parts > 1 ? parts : 1)};
    }
    const int64_t rows = padded_rows(T);
    int64_t most = static_cast<int64_t>(kDzBytes / 2) / rows / 256 * 256;
    if (most < 256) most = 256;
    if (most >= V) most = (V + 255) / 256 * 256;
    const int64_t least = (V + most - 1) / most;
    Pieces best{};
    int64_t best_clocks = 0, seen = 0;
    for (int64_t n = least; n <= 2 * least + 1 && n < least + 64; ++n) {
        const int64_t cols = ((V + n - 1) / n + 255) / 256 * 256;
        if (cols == seen) continue;
        seen = cols;
        auto clocks = [&](int64_t c, int* parts) {
            const int64_t tiles = (rows + 255) / 256 * ((c + 255) / 256), blocks = (d + 63) / 64;
            return (tiles + 75) / 76 * (blocks > 5 ? blocks + 1 : 6) + gtc::pair_clocks(rows, static_cast<int>(c), d, parts) + 30;
        };
        int parts = 1, other = 1;
        const int64_t whole = V / cols, rest = V % cols;
        const int64_t total = (whole ? whole * clocks(cols, &parts) : 0) + (rest ? clocks(rest, whole ? &other : &parts) : 0);
        if (best.cols == 0 || total < best_clocks - best_clocks / 100)
            best = Pieces{static_cast<int>(cols < V ? cols : V), parts}, best_clocks = total;
    }
    return best;
}

// What a call takes from its workspace.
struct ForwardSpace {
    float* Z;            // a piece of the logits (fp32)
    Part* parts;
    float* hit;
};
static ForwardSpace carve_forward(Carver& c, int64_t rows, int V, int dtype) {
    ForwardSpace s{};
    if (dtype == DTP_F32) s.Z = static_cast<float*>(c.take(static_cast<size_t>(rows) * stored_cols(rows, V) * sizeof(float)));
    s.parts = static_cast<Part*>(c.take(static_cast<size_t>(rows) * parts_of(rows, V, dtype) * sizeof(Part)));
    s.hit = static_cast<float*>(c.take(static_cast<size_t>(rows) * sizeof(float)));
    return s;
}
// whether the forward pass copies X to an aligned pitch
static bool copies_x(int d, int dtype) { return repitch_bytes(1, d, dtype) > 0; }
struct BackwardSpace {
    void* dz;            // in fp32 the logits before
    void* x;
    float *sum, *runs;
    Compact compact;     // bf16
};
static int64_t sum_rows(int64_t T) { return (padded_rows(T) + 255) / 256 * 256; }
static BackwardSpace carve_backward(Carver& c, int64_t T, int d, int V, int dtype, const Pieces& pieces) {
    BackwardSpace s{};
    const int64_t rows = dtype == DTP_BF16 ? padded_rows(T) : T;
    s.dz = c.take(static_cast<size_t>(rows) * (dtype == DTP_BF16 ? padded(pieces.cols) : pieces.cols) * elem(dtype));
    s.x = c.take(static_cast<size_t>(rows) * padded(d) * elem(dtype));
    const int64_t summed = dtype == DTP_BF16 ? sum_rows(T) : pieces.parts > 1 || T <= kFew ? T : 0;
    s.sum = static_cast<float*>(c.take(static_cast<size_t>(summed) * pieces.parts * d * sizeof(float)));
    s.runs = static_cast<float*>(c.take(runs_bytes(rows, pieces.cols, d)));
    if (dtype == DTP_BF16) {
        const size_t n = static_cast<size_t>(T);
        s.compact.place = static_cast<int*>(c.take(n * sizeof(int)));
        s.compact.live = static_cast<int*>(c.take(2 * sizeof(int)));
        s.compact.targets = static_cast<int64_t*>(c.take(n * sizeof(int64_t)));
        s.compact.lse = static_cast<float*>(c.take(n * sizeof(float)));
        s.compact.dloss = static_cast<float*>(c.take(n * sizeof(float)));
        s.compact.unit = static_cast<float*>(c.take(sizeof(float)));
    }
    return s;
}

size_t loss_workspace_bytes(int64_t T, int d, int V, int dtype, int backward) {
    if (T == 0) return kWorkspaceHeader;
    Carver f(nullptr);
    f.take(repitch_bytes(V, d, dtype));
    Carver b = f;
    if (copies_x(d, dtype)) f.take(static_cast<size_t>(padded_rows(T)) * padded(d) * elem(dtype));
    const int64_t rows = forward_rows(T, V, dtype);
    carve_forward(f, rows, V, dtype);
    if (T % rows) carve_forward(f, T % rows, V, dtype);
    if (!backward) return f.used;
    carve_backward(b, T, d, V, dtype, backward_pieces(T, d, V, dtype));
    return f.used > b.used ? f.used : b.used;
}

// The product of T tokens with columns v0 .. of the vocabulary; x has `rows_x` rows.
static Product logits(const Rows& x, int64_t rows_x, int64_t t0, const Rows& w, int64_t T, int d, int v0, int cols, int dtype) {
    auto from = [&](const Rows& r, int64_t row) {
        return by_row(static_cast<const uint8_t*>(r.p) + static_cast<size_t>(row) * r.ld * elem(dtype), r.ld);
    };
    Product p;
    p.A[0] = from(x, t0);
    p.B[0] = from(w, v0);
    p.M = T, p.N = cols, p.K = d, p.rows_a = rows_x - t0;
    p.epi.M = T, p.epi.N = cols, p.epi.ldo = cols;
    return p;
}

// Stored logits (fp32): few tokens have kernels of their own.
static int store_logits(Call& call, const Product& p) {
    if (p.M <= kFew && !fewl::takes_logits(p.M, static_cast<int>(p.K))) return call.run(p);
    int* status = call.fresh ? static_cast<int*>(call.workspace) : nullptr;
    if (p.M > kFew) {
        call.fresh = false;
        return simt::launch(p, call.dtype, status, call.stream);
    }
    if (status) DTP_CUDA_TRY(cudaMemsetAsync(status, 0, sizeof(int), call.stream));
    call.fresh = false;
    return fewl::launch_logits(static_cast<const float*>(p.A[0].p), static_cast<const float*>(p.B[0].p), p.M, p.N, static_cast<int>(p.K),
                               static_cast<float*>(p.epi.out), call.stream);
}

int loss_forward(const void* X, const void* W, const int64_t* targets, int64_t T, int d, int V, int64_t ignore, int dtype,
                 float* loss, float* lse, void* workspace, cudaStream_t stream) {
    Call call{dtype, workspace, stream};
    Carver c(workspace);
    Rows x{X, d}, w;
    int64_t rows_x = T;
    int st = aligned_rows(W, V, d, dtype, c, stream, &w);
    int* status = static_cast<int*>(workspace);
    if (st == DTP_OK && copies_x(d, dtype)) {
        rows_x = padded_rows(T);
        void* to = c.take(static_cast<size_t>(rows_x) * padded(d) * elem(dtype));
        x = Rows{to, padded(d)};
        st = launch_after(place_rows_kernel<__nv_bfloat16>, grid_of(rows_x), stream, static_cast<const __nv_bfloat16*>(X), T, rows_x, d,
                          x.ld, static_cast<const int64_t*>(nullptr), int64_t(0), 0, static_cast<const int*>(nullptr),
                          static_cast<const int*>(nullptr), static_cast<__nv_bfloat16*>(to));
    }
    const int64_t most = forward_rows(T, V, dtype);
    ForwardSpace s = carve_forward(c, most, V, dtype);
    for (int64_t t0 = 0; st == DTP_OK && t0 < T; t0 += most) {
        const int64_t rows = T - t0 < most ? T - t0 : most;
        if (rows < most) s = carve_forward(c, rows, V, dtype);
        Vocab e;
        e.targets = targets + t0, e.ignore = ignore, e.T = rows, e.V = V, e.parts = s.parts, e.hit = s.hit;
        int64_t count = 0;
        if (dtype == DTP_BF16) {
            Product p = logits(x, rows_x, t0, w, rows, d, 0, V, dtype);
            p.epi.kind = kEpiParts, p.epi.vocab = e;
            st = gtc::launch(p, status, call.fresh, stream, &count);
            call.fresh = false;
        } else {
            const int piece = stored_cols(rows, V);
            for (int v0 = 0; st == DTP_OK && v0 < V; v0 += piece) {
                const int cols = V - v0 < piece ? V - v0 : piece;
                Product p = logits(x, rows_x, t0, w, rows, d, v0, cols, dtype);
                p.epi.out = s.Z;
                st = store_logits(call, p);
                const int64_t chunks = (cols + kChunk - 1) / kChunk;
                if (st == DTP_OK)
                    st = launch_after(parts_kernel, grid_of(rows * chunks), stream, static_cast<const float*>(s.Z), rows, cols, v0,
                                      e.targets, s.parts + count * rows, s.hit);
                count += chunks;
            }
        }
        if (st == DTP_OK)
            st = launch_blocks(loss_kernel, (rows + 31) / 32, 32 * kLossWarps, stream, static_cast<const Part*>(s.parts), count,
                               static_cast<const float*>(s.hit), e.targets, rows, V, ignore, loss + t0, lse + t0, status);
    }
    return st;
}

template <typename E>
static int backward(const float* dloss, const void* X, const void* W, const int64_t* targets, const float* lse, int64_t T, int d,
                    int V, int64_t ignore, int dtype, void* dX, void* dW, void* workspace, cudaStream_t stream) {
    constexpr bool kBf16 = sizeof(E) == 2;
    Call call{dtype, workspace, stream};
    Carver c(workspace);
    Rows w;
    int st = aligned_rows(W, V, d, dtype, c, stream, &w);
    const Pieces pieces = backward_pieces(T, d, V, dtype);
    const BackwardSpace s = carve_backward(c, T, d, V, dtype, pieces);
    int* status = static_cast<int*>(workspace);
    const int64_t rows = kBf16 ? padded_rows(T) : T;
    const Rows x{s.x, kBf16 || T > kFew ? padded(d) : d};
    Vocab e;
    e.targets = targets, e.ignore = ignore, e.T = T, e.V = V, e.lse = lse, e.dloss = dloss;
    const bool in_runs = rows > kRun && dW;          // dW's sums over so many tokens are made in runs of a known length
    const Compact& k = s.compact;
    if constexpr (kBf16) {
        if (st == DTP_OK)
            st = launch_blocks(index_kernel, 1, kIndexThreads, stream, targets, lse, dloss, T, ignore, V, static_cast<int>(!in_runs), k, status);
        e.targets = k.targets, e.lse = k.lse, e.dloss = k.dloss, e.unit = k.unit, e.count = k.live + 1;
    } else if (st == DTP_OK) {
        DTP_CUDA_TRY(cudaMemsetAsync(status, 0, sizeof(int), stream));
    }
    if (st == DTP_OK)
        st = launch_after(place_rows_kernel<E>, grid_of(rows), stream, static_cast<const E*>(X), T, rows, d, x.ld, targets, ignore, V,
                          static_cast<const int*>(kBf16 ? k.place : nullptr), static_cast<const int*>(kBf16 ? k.live : nullptr),
                          static_cast<E*>(s.x));
    call.fresh = false;
    for (int v0 = 0; st == DTP_OK && v0 < V; v0 += pieces.cols) {
        const int cols = V - v0 < pieces.cols ? V - v0 : pieces.cols;
        const int64_t ldz = kBf16 ? padded(cols) : cols;
        const void* w_at = static_cast<const E*>(w.p) + static_cast<int64_t>(v0) * w.ld;
        E* dw_at = dW ? static_cast<E*>(dW) + static_cast<int64_t>(v0) * d : nullptr;
        e.v0 = v0;
        Product p = logits(x, rows, 0, w, rows, d, v0, cols, dtype);
        p.epi.out = s.dz, p.epi.ldo = ldz;
        if constexpr (kBf16) {
            p.epi.kind = kEpiProb, p.epi.vocab = e, p.live = k.live;
            st = gtc::launch(p, status, 0, stream);
            GradPair g{s.dz, s.x, w_at, ldz, x.ld, w.ld, rows, k.live, cols, d, pieces.parts, v0 > 0, k.unit, dX ? s.sum : nullptr,
                       in_runs ? nullptr : dw_at};
            if (g.parts > (cols + 63) / 64) g.parts = (cols + 63) / 64;       // a short last piece leaves the others' sums as they are
            if (st == DTP_OK) st = gtc::launch_pair(g, status, stream);
            if (st == DTP_OK && in_runs)
                st = weight_gradient(call, Also{by_col(s.dz, ldz), by_col(x.p, x.ld), cols, d, dw_at, d}, rows, s.runs, k.unit);
        } else {
            st = store_logits(call, p);
            if (st == DTP_OK)
                st = launch_after(dz_kernel<E>, grid_of(T * ((cols + kChunk - 1) / kChunk)), stream, static_cast<const float*>(s.dz),
                                  T, cols, e, static_cast<E*>(s.dz), ldz, status);
            if (st == DTP_OK && dX) {
                Product q;
                q.A[0] = by_row(s.dz, ldz);
                q.B[0] = by_col(w_at, w.ld);
                q.M = T, q.N = d, q.K = cols;
                q.epi.ldo = d, q.epi.M = T, q.epi.N = d;
                q.parts = pieces.parts;
                const bool few = T <= kFew;
                if (few) {
                    q.parts = fewl::ranges_of(cols, d);
                    st = fewl::launch_dx(static_cast<const float*>(s.dz), static_cast<const float*>(w_at), T, cols, d, q.parts, s.sum, stream);
                } else if (q.parts == 1) q.epi.out = dX, q.epi.residual = v0 > 0 ? dX : nullptr;
                else q.epi.out = s.sum;
                if (!few) st = simt::launch(q, dtype, nullptr, stream);
                if (st == DTP_OK && (few || q.parts > 1))
                    st = launch_after(add_parts_kernel, grid_of((T * d + 255) / 256), stream, static_cast<const float*>(s.sum), q.parts,
                                      T * d, static_cast<int>(v0 > 0), static_cast<float*>(dX));
            }
            if (st == DTP_OK && dW && T <= kFew)
                st = fewl::launch_dw(static_cast<const float*>(s.dz), static_cast<const float*>(x.p), T, cols, d,
                                     reinterpret_cast<float*>(dw_at), stream);
            else if (st == DTP_OK && dW)
                st = weight_gradient(call, Also{by_col(s.dz, ldz), by_col(x.p, x.ld), cols, d, dw_at, d}, T, s.runs);
        }
    }
    if (kBf16 && st == DTP_OK && dX)
        st = launch_after(round_kernel, grid_of((T * ((d + 511) / 512) + 7) / 8), stream, static_cast<const float*>(s.sum), pieces.parts,
                          sum_rows(T) * d, T, d, targets, ignore, V, static_cast<const int*>(k.place),
                          static_cast<const float*>(k.unit), static_cast<__nv_bfloat16*>(dX));
    if (!kBf16 && st == DTP_OK && dX) st = launch_after(clear_rows_kernel, grid_of(T), stream, T, d, e, static_cast<float*>(dX));
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
