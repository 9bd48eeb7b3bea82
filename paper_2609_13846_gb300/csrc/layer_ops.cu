// layer_ops.cu -- the linear layer and the gated feed-forward block, forward and backward, as sequences of
// matrix products with fused epilogues, and the elementwise kernels between them.
#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include <type_traits>

#include "dtp_common.cuh"
#include "layer_common.cuh"
#include "layer_host.cuh"

namespace dtp {
namespace layer {

constexpr int kRowChunk = 32;     // tokens per partial sum of the bias gradient
constexpr int kPer = 4;           // columns per thread

// dZ = dY act'(Z), rounded once, and the partial sums over kRowChunk tokens of the unrounded values (the bias
// gradient).  Bound by memory: 8192 x 4096 in bf16 50 us, 5.4 TB/s (a column of 32 and single elements: 84 us).  A block takes 128 columns x kRowChunk tokens, a thread 4 columns of every eighth token, two
// tokens in flight; each of the 8 warps sums its tokens in order.  kWide: rows on 16-byte boundaries.
template <typename E, bool kWide>
__global__ void __launch_bounds__(256)
act_grad_kernel(const E* dY, const float* Z, int64_t T, int N, int64_t ldz, int act, E* dZ, float* partial) {
    __shared__ float red[8][32 * kPer + 1];
    grid_wait();
    grid_release();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int wide_blocks = (N + 32 * kPer - 1) / (32 * kPer);
    const int block = static_cast<int>(blockIdx.x) % wide_blocks;
    const int64_t chunk = blockIdx.x / wide_blocks;
    const int n0 = (block * 32 + lane) * kPer;
    const int64_t t0 = chunk * kRowChunk;
    const int64_t t1 = t0 + kRowChunk < T ? t0 + kRowChunk : T;
    const bool full = kWide && n0 + kPer <= N;
    using W = std::conditional_t<sizeof(E) == 2, uint2, uint4>;       // the thread's columns of a token
    union Row { W q; E e[kPer]; };
    float sum[kPer];
#pragma unroll
    for (int j = 0; j < kPer; ++j) sum[j] = 0.0f;
    auto load = [&](int64_t t, Row& g, float (&z)[kPer]) {
        if (full) {
            g.q = *reinterpret_cast<const W*>(dY + t * N + n0);
            if (act != DTP_ACT_NONE) {
#pragma unroll
                for (int j = 0; j < kPer / 4; ++j) {
                    const float4 v = reinterpret_cast<const float4*>(Z + t * N + n0)[j];
                    z[4 * j] = v.x, z[4 * j + 1] = v.y, z[4 * j + 2] = v.z, z[4 * j + 3] = v.w;
                }
            }
        } else {
#pragma unroll
            for (int j = 0; j < kPer; ++j) {
                const bool in = n0 + j < N;
                g.e[j] = in ? dY[t * N + n0 + j] : from_f32<E>(0.0f);
                z[j] = in && act != DTP_ACT_NONE ? Z[t * N + n0 + j] : 0.0f;
            }
        }
    };
    auto store = [&](int64_t t, const Row& g, const float (&z)[kPer]) {
        Row o;
#pragma unroll
        for (int j = 0; j < kPer; ++j) {
            float x = to_f32(g.e[j]);
            if (act != DTP_ACT_NONE) {
                float v, s;
                act_both<IsFast<E>::value>(act, z[j], v, s);
                x *= s;
            }
            sum[j] += x;
            o.e[j] = from_f32<E>(x);
        }
        if (!dZ) return;
        if (full) {
            *reinterpret_cast<W*>(dZ + t * ldz + n0) = o.q;
        } else {
#pragma unroll
            for (int j = 0; j < kPer; ++j)
                if (n0 + j < N) dZ[t * ldz + n0 + j] = o.e[j];
        }
    };
    if (n0 < N) {
        int64_t t = t0 + warp;
        for (; t + 8 < t1; t += 16) {
            Row a, b;
            float za[kPer], zb[kPer];
            load(t, a, za);
            load(t + 8, b, zb);
            store(t, a, za);
            store(t + 8, b, zb);
        }
        if (t < t1) {
            Row a;
            float za[kPer];
            load(t, a, za);
            store(t, a, za);
        }
    }
    if (!partial) return;
#pragma unroll
    for (int j = 0; j < kPer; ++j) red[warp][lane * kPer + j] = sum[j];
    __syncthreads();
    const int n = block * 32 * kPer + threadIdx.x;
    if (threadIdx.x < 32 * kPer && n < N) {
        float s = 0.0f;
#pragma unroll
        for (int w = 0; w < 8; ++w) s += red[w][threadIdx.x];
        partial[chunk * N + n] = s;
    }
}

// out[n] = sum over the chunks: each of 8 warps sums every eighth in order, then the warps' sums in order.
template <typename E>
__global__ void __launch_bounds__(256)
bias_reduce_kernel(const float* partial, int64_t chunks, int N, E* out) {
    __shared__ float red[8][32];
    grid_wait();
    grid_release();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int n = blockIdx.x * 32 + lane;
    float s = 0.0f;
    if (n < N)
#pragma unroll 8
        for (int64_t c = warp; c < chunks; c += 8) s += partial[c * N + n];
    red[warp][lane] = s;
    __syncthreads();
    if (warp == 0 && n < N) {
        float v = 0.0f;
#pragma unroll
        for (int w = 0; w < 8; ++w) v += red[w][lane];
        out[n] = from_f32<E>(v);
    }
}

// relu has a kink where its gradient jumps: the gradient's mask wants the sign of the sum, and a sum near zero may come out on
// the wrong side.  How near goes by the terms, not by the sum.  An MMA of 16 k aligns its products and the accumulator to
// the largest of them, cuts each of the 17 off at 2^-25 of it and their sum at 2^-23 (measured: 1 + p - 1 with p in the same step and
// in others), and while a sum of terms of sizes S and a bias b comes back to zero no partial sum is above (S + |b|) / 2: 21/16 2^-22
// (S + |b|) for every 16 k.  S is at most |x| |w|, the norms of the two rows.  So every saved value below kSignShare (K + 64)
// (|x| |w| + |b|) is summed again, computed zeros too (64: the partial sums of a split range).
constexpr float kSignShare = 1.9557774e-8f;      // 21/16 2^-26

// Upper bounds of the 2-norms of T rows of X, then of N rows of W: a warp per row, fp32 sums of squares, with a power of two taken
// out where they leave fp32's range; a 128th covers their roundings (K / 32 additions a lane, K to 2^20, and the root halves
// the error).  Two bytes a row, rounded up.  A row of zeros gives 0, one with an infinity an infinity, a NaN a NaN.
__global__ void __launch_bounds__(256)
row_norms_kernel(const __nv_bfloat16* X, int64_t ldx, int64_t T, const __nv_bfloat16* W, int64_t ldw, int N, int K,
                 __nv_bfloat16* norms) {
    grid_wait();
    grid_release();
    const int lane = threadIdx.x & 31;
    for (int64_t i = blockIdx.x * 8ll + (threadIdx.x >> 5); i < T + N; i += gridDim.x * 8ll) {
        const int64_t ld = i < T ? ldx : ldw;
        const __nv_bfloat16* row = i < T ? X + i * ldx : W + (i - T) * ldw;
        const int words = (ld & 7) == 0 ? K / 8 : 0;
        auto squares = [&](float scale) {
            float s = 0.0f;
            auto add = [&](float v) { v *= scale, s = fmaf(v, v, s); };
#pragma unroll 4
            for (int k = lane; k < words; k += 32) {
                const uint4 a = reinterpret_cast<const uint4*>(row)[k];
                const uint32_t w[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
                for (int q = 0; q < 4; ++q) add(__uint_as_float(w[q] << 16)), add(__uint_as_float(w[q] & 0xFFFF0000u));
            }
            for (int k = 8 * words + lane; k < K; k += 32) add(to_f32(row[k]));
#pragma unroll
            for (int o = 16; o > 0; o >>= 1) s += __shfl_xor_sync(0xFFFFFFFFu, s, o);
            return s;
        };
        float s = squares(1.0f), back = 1.0f;
        if (!(s >= 8.271806e-25f && s <= 3.0e38f)) {                             // 2^-80
            back = s < 8.271806e-25f ? 7.888609e-31f : 1.2676506e30f;            // 2^-100, 2^100
            s = squares(1.0f / back);
        }
        if (lane == 0) norms[i] = __float2bfloat16_ru(1.0078125f * sqrtf(s) * back);
    }
}

// The product of two rows by a whole warp, in up to three steps, until the sum is larger than the step's error: fp32 in eight sums a lane;
// products in fp32 (exact) with each lane carrying its additions' errors along and the lanes meeting in fp64; and fp64, which is
// the result whatever it is (it may be zero).  `size` bounds the sum of the terms' sizes and the bias.
struct Dot {
    int K, words;            // words of eight that may be loaded at once
    float fp32, carried, least;
    __device__ __forceinline__ Dot(int K, bool wide) : K(K), words(wide ? K / 8 : 0) {
        const float most = (K + 31) / 32 + 8;                                // a lane's terms, of which a word has eight
        fp32 = (K / (wide ? 256 : 32) + 24.0f) * 5.9604645e-8f;              // 2^-24: a sum's additions, then the tree's
        carried = most * most * 3.5527137e-15f;                              // 2^-48: the errors' own roundings
        least = K * 1.4012985e-45f;                                          // among fp32's subnormal numbers
    }
    template <typename V>
    __device__ __forceinline__ static V lanes(V s) {
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) s += __shfl_xor_sync(0xFFFFFFFFu, s, o);
        return s;
    }
    template <typename F>
    __device__ __forceinline__ void each(const __nv_bfloat16* x, const __nv_bfloat16* w, F add) const {
        const int lane = threadIdx.x & 31;
#pragma unroll 4
        for (int k = lane; k < words; k += 32) {
            const uint4 a = reinterpret_cast<const uint4*>(x)[k], c = reinterpret_cast<const uint4*>(w)[k];
            const uint32_t aw[4] = {a.x, a.y, a.z, a.w}, cw[4] = {c.x, c.y, c.z, c.w};
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                add(2 * q, __uint_as_float(aw[q] << 16), __uint_as_float(cw[q] << 16));
                add(2 * q + 1, __uint_as_float(aw[q] & 0xFFFF0000u), __uint_as_float(cw[q] & 0xFFFF0000u));
            }
        }
        for (int k = 8 * words + lane; k < K; k += 32) add(0, to_f32(x[k]), to_f32(w[k]));
    }
    __device__ __forceinline__ float operator()(const __nv_bfloat16* x, const __nv_bfloat16* w, float bias, float size) const {
        float s[8] = {0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f};
        each(x, w, [&](int i, float a, float c) { s[i] = fmaf(a, c, s[i]); });
        const float plain = lanes(((s[0] + s[1]) + (s[2] + s[3])) + ((s[4] + s[5]) + (s[6] + s[7]))) + bias;
        if (fabsf(plain) > fmaxf(fp32 * size, least) && isfinite(plain)) return plain;
        float hi = 0.0f, lo = 0.0f;
        each(x, w, [&](int, float a, float c) {      // hi + lo is the sum: the error of each addition, exactly
            const float p = a * c, t = hi + p, b = t - hi;
            lo += (hi - (t - b)) + (p - b);
            hi = t;
        });
        double sum = lanes(static_cast<double>(hi) + static_cast<double>(lo)) + static_cast<double>(bias);
        if (!(fabs(sum) > fmaxf(carried * size, least)) || isinf(sum)) {
            sum = 0.0;
            each(x, w, [&](int, float a, float c) { sum = fma(static_cast<double>(a), static_cast<double>(c), sum); });
            sum = lanes(sum) + static_cast<double>(bias);
        }
        return static_cast<float>(sum);
    }
};

// The saved values that may have the wrong sign, summed again.  A warp reads 128 columns of four tokens, or where they are the block's
// saved gate (kPre) 16 neurons of 32 tokens, and takes its lanes' candidates one by one.  Where the terms are all zero the sum
// is, and nothing is a candidate; where a norm is infinite everything finite is, and beside a NaN nothing.  Candidates go
// with K sqrt(K) (random rows: 0.05% of the values at K = 1024, 0.4% at 4096, 1.2% at 8192), the rows that they read with K times
// that.  With the norms, 8192 x 4096 values of K = 1024: 69 us, reading Z and the candidates' latency (8192 x 3072 of the gate 71); 4096
// x 4096: 118 us at K = 4096, 453 at 8192, their rows from L2.
template <bool kPre>
__global__ void __launch_bounds__(256, 4)
relu_sign_kernel(const __nv_bfloat16* X, int64_t ldx, const __nv_bfloat16* W, int64_t ldw, const __nv_bfloat16* bias,
                 const __nv_bfloat16* norms, int64_t T, int K, int N, float* values) {
    grid_wait();
    grid_release();
    const int lane = threadIdx.x & 31;
    constexpr int kTokens = kPre ? 32 : 4, kCols = kPre ? 16 : 128;      // of a warp; 16 values a lane
    const int per_row = (N + kCols - 1) / kCols;
    const int64_t pieces = (T + kTokens - 1) / kTokens * per_row;
    const float share = kSignShare * (K + 64.0f);
    const Dot dot(K, (ldx & 7) == 0 && (ldw & 7) == 0);
    for (int64_t i = blockIdx.x * 8ll + (threadIdx.x >> 5); i < pieces; i += gridDim.x * 8ll) {
        const int64_t g = i / per_row, t0 = g * kTokens;
        const int n0 = static_cast<int>(i - g * per_row) * kCols;
        // of value j of lane l
        auto token = [&](int j, int l) { return kPre ? t0 + l : t0 + (j >> 2); };
        auto column = [&](int j, int l) { return kPre ? n0 + j : n0 + 32 * (j & 3) + l; };
        auto inside = [&](int j) { return column(j, lane) < N && token(j, lane) < T; };
        const float kNone = __int_as_float(0x7FC00000);      // beyond the edges: a NaN is no candidate
        float z[16];
        if constexpr (kPre) {                                // groups of four neurons; beyond the edges there is room
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                float4 v = make_float4(kNone, kNone, kNone, kNone);
                if (inside(4 * q)) v = *reinterpret_cast<const float4*>(values + pre_index(t0 + lane, n0 + 4 * q, N));
                z[4 * q] = v.x, z[4 * q + 1] = inside(4 * q + 1) ? v.y : kNone;
                z[4 * q + 2] = inside(4 * q + 2) ? v.z : kNone, z[4 * q + 3] = inside(4 * q + 3) ? v.w : kNone;
            }
        } else {
#pragma unroll
            for (int j = 0; j < 16; ++j) z[j] = inside(j) ? values[token(j, lane) * N + column(j, lane)] : kNone;
        }
        constexpr int kX = kPre ? 1 : 4, kW = kPre ? 16 : 4;      // the lane's tokens and columns: value j is of j / kW and j % kW
        float nx[kX], nw[kW], nb[kW];
#pragma unroll
        for (int j = 0; j < kX; ++j) nx[j] = token(kW * j, lane) < T ? to_f32(norms[token(kW * j, lane)]) : 0.0f;
#pragma unroll
        for (int j = 0; j < kW; ++j) {
            const int n = column(j, lane);
            nw[j] = n < N ? to_f32(norms[T + n]) : 0.0f;
            nb[j] = n < N && bias ? fabsf(to_f32(bias[n])) : 0.0f;
        }
        unsigned mine = 0;                                   // the lane's candidates
        float top = 0.0f;
#pragma unroll
        for (int j = 0; j < 16; ++j) {
            const float s = fmaf(nx[j / kW], nw[j % kW], nb[j % kW]), a = fabsf(z[j]);
            mine |= (a < share * s || (a < dot.least && s > 0.0f) ? 1u : 0u) << j;
            top = fmaxf(top, s);
        }
        if (!__any_sync(0xFFFFFFFFu, mine != 0)) continue;
#pragma unroll 1
        for (int j = 0; j < 16; ++j) {
            unsigned todo = __ballot_sync(0xFFFFFFFFu, (mine >> j) & 1u);
            while (todo) {
                const int at = __ffs(todo) - 1, n = column(j, at);
                const int64_t t = token(j, at);
                todo &= todo - 1;
                const float sum = dot(X + t * ldx, W + n * ldw, bias ? to_f32(bias[n]) : 0.0f, __shfl_sync(0xFFFFFFFFu, top, at));
                if (lane == at) values[kPre ? pre_index(t, n, N) : t * N + n] = sum;
            }
        }
    }
}

// Rows copied to a pitch of whole 16 bytes, for the tensor cores' loads; the pitch's spare entries stay unwritten
// (the loads' extents end before them).
__global__ void __launch_bounds__(256)
repitch_kernel(const uint16_t* src, int64_t rows, int cols, int64_t pitch, uint16_t* dst) {
    grid_wait();
    grid_release();
    // a warp per 512 entries of a row, all of them in flight (3162 x 3854: 10 us; a warp per row 13, and 12 for 640 rows, now 5)
    const int lane = threadIdx.x & 31, parts = (cols + 511) / 512;
    const int64_t pieces = rows * parts;
    for (int64_t i = blockIdx.x * 8ll + (threadIdx.x >> 5); i < pieces; i += gridDim.x * 8ll) {
        const int64_t r = i / parts;
        const int c0 = static_cast<int>(i - r * parts) * 512 + lane;
        const uint16_t* from = src + r * cols;
        uint16_t* to = dst + r * pitch;
        uint16_t v[16];
#pragma unroll
        for (int j = 0; j < 16; ++j) v[j] = c0 + 32 * j < cols ? from[c0 + 32 * j] : 0;
#pragma unroll
        for (int j = 0; j < 16; ++j)
            if (c0 + 32 * j < cols) to[c0 + 32 * j] = v[j];
    }
}

// The runs' sums of a weight gradient (see kRun), added in their order.
template <typename E>
__global__ void __launch_bounds__(256)
sum_runs_kernel(const float* runs, int64_t count, int64_t values, const float* unit, E* out) {
    grid_wait();
    grid_release();
    const double u = unit ? static_cast<double>(*unit) : 1.0;
    for (int64_t i = blockIdx.x * 256ll + threadIdx.x; i < values; i += gridDim.x * 256ll) {
        double s = 0.0;
#pragma unroll 4
        for (int64_t r = 0; r < count; ++r) s += static_cast<double>(runs[r * values + i]);
        out[i] = from_f32<E>(static_cast<float>(s * u));
    }
}

static int64_t chunks_of(int64_t T) { return (T + kRowChunk - 1) / kRowChunk; }

size_t repitch_bytes(int64_t rows, int cols, int dtype) {
    return dtype == DTP_BF16 && cols % 8 ? static_cast<size_t>(rows) * padded(cols) * 2 : 0;
}
// the row norms for relu's signs
static size_t norms_bytes(int64_t T, int N, int dtype) {
    return dtype == DTP_BF16 ? static_cast<size_t>(T + N) * sizeof(__nv_bfloat16) : 0;
}
int aligned_rows(const void* p, int64_t rows, int cols, int dtype, Carver& c, cudaStream_t stream, Rows* out) {
    const size_t bytes = repitch_bytes(rows, cols, dtype);
    if (bytes == 0) {
        *out = Rows{p, cols};
        return DTP_OK;
    }
    void* to = c.take(bytes);
    *out = Rows{to, padded(cols)};
    const int64_t blocks = (rows * ((cols + 511) / 512) + 7) / 8;
    return launch_after(repitch_kernel, blocks < 8192 ? blocks : 8192, stream, static_cast<const uint16_t*>(p), rows, cols,
                        padded(cols), static_cast<uint16_t*>(to));
}

size_t runs_bytes(int64_t T, int64_t rows, int64_t cols) {
    return T > kRun ? static_cast<size_t>((T + kRun - 1) / kRun) * rows * cols * sizeof(float) : 0;
}

int weight_gradient(Call& call, const Also& w, int64_t T, float* runs, const float* unit) {
    const int64_t values = w.M * w.N, count = T > kRun ? (T + kRun - 1) / kRun : 1;
    for (int64_t r = 0; r < count; ++r) {
        const int64_t t0 = r * kRun;
        auto from = [&](const Mat& m) {
            return by_col(static_cast<const uint8_t*>(m.p) + static_cast<size_t>(t0 * m.ks) * elem(call.dtype), m.ks);
        };
        Product p;
        p.A[0] = count > 1 ? from(w.A) : w.A;
        p.B[0] = count > 1 ? from(w.B) : w.B;
        p.M = w.M, p.N = w.N, p.K = count > 1 && T - t0 > kRun ? kRun : T - t0;
        p.epi.out = w.out, p.epi.ldo = w.ldo, p.epi.M = w.M, p.epi.N = w.N;
        if (count > 1) p.epi.Z = runs + r * values;
        const int st = call.run(p);
        if (st != DTP_OK) return st;
    }
    if (count == 1) return DTP_OK;
    const int64_t blocks = (values + 255) / 256 < 8192 ? (values + 255) / 256 : 8192;
    return call.dtype == DTP_BF16 ? launch_after(sum_runs_kernel<__nv_bfloat16>, blocks, call.stream, static_cast<const float*>(runs),
                                                 count, values, unit, static_cast<__nv_bfloat16*>(w.out))
                                  : launch_after(sum_runs_kernel<float>, blocks, call.stream, static_cast<const float*>(runs), count,
                                                 values, unit, static_cast<float*>(w.out));
}

// ------------------------------------------------------------------------------- linear layer

size_t linear_workspace_bytes(int64_t T, int K, int N, int dtype, int backward) {
    Carver c(nullptr);
    c.take(repitch_bytes(T, K, dtype));
    c.take(repitch_bytes(N, K, dtype));
    c.take(norms_bytes(T, N, dtype));
    if (backward) {
        c.take(static_cast<size_t>(T) * padded(N) * elem(dtype));
        c.take(static_cast<size_t>(chunks_of(T)) * N * sizeof(float));
        c.take(runs_bytes(T, N, K));
    }
    return c.used;
}

// The saved values of a bf16 product with relu (Z, or the block's gate) get the sums' signs.
template <bool kPre>
static int relu_signs(const Product& p, const __nv_bfloat16* bias, float* values, Carver& c, cudaStream_t stream) {
    const auto* X = static_cast<const __nv_bfloat16*>(p.A[0].p);
    const auto* W = static_cast<const __nv_bfloat16*>(p.B[0].p);
    const int K = static_cast<int>(p.K);
    auto* norms = static_cast<__nv_bfloat16*>(c.take(norms_bytes(p.M, p.N, DTP_BF16)));
    const int64_t rows = (p.M + p.N + 7) / 8;
    const int64_t warps = kPre ? (p.M + 31) / 32 * ((p.N + 15) / 16) : (p.M + 3) / 4 * ((p.N + 127) / 128), blocks = (warps + 7) / 8;
    const int st = launch_after(row_norms_kernel, rows < 8192 ? rows : 8192, stream, X, p.A[0].rs, p.M, W, p.B[0].rs, p.N, K, norms);
    if (st != DTP_OK) return st;
    return launch_after(relu_sign_kernel<kPre>, blocks < 8192 ? blocks : 8192, stream, X, p.A[0].rs, W, p.B[0].rs, bias,
                        static_cast<const __nv_bfloat16*>(norms), p.M, K, p.N, values);
}

int linear_forward(const void* X, const void* W, const void* bias, const void* residual, int64_t T, int K, int N,
                   int act, int dtype, void* Y, float* Z, void* workspace, cudaStream_t stream) {
    Call call{dtype, workspace, stream};
    Carver c(workspace);
    int st = DTP_OK;
    Product p;
    p.A[0] = by_row(X, K);
    p.B[0] = by_row(W, K);
    p.M = T, p.N = N, p.K = K;
    if (!fews::takes(p, dtype)) {            // which reads rows at any pitch
        Rows x, w;
        if ((st = aligned_rows(X, T, K, dtype, c, stream, &x)) != DTP_OK) return st;
        if ((st = aligned_rows(W, N, K, dtype, c, stream, &w)) != DTP_OK) return st;
        p.A[0] = by_row(x.p, x.ld);
        p.B[0] = by_row(w.p, w.ld);
    }
    p.epi.act = act, p.epi.bias = bias, p.epi.residual = residual, p.epi.out = Y, p.epi.ldo = N, p.epi.Z = Z;
    p.epi.M = T, p.epi.N = N;
    if ((st = call.run(p)) != DTP_OK) return st;
    if (dtype == DTP_BF16 && act == DTP_ACT_RELU && Z)
        st = relu_signs<false>(p, static_cast<const __nv_bfloat16*>(bias), Z, c, stream);
    if (st != DTP_OK) return st;
    return call.done();
}

template <typename E>
static int launch_act_grad(const void* dY, const float* Z, int64_t T, int N, int act, void* dZ, int64_t ldz,
                           float* partial, void* dbias, cudaStream_t stream) {
    if (T > 0) {
        const int64_t blocks = chunks_of(T) * ((N + 32 * kPer - 1) / (32 * kPer));
        auto kernel = N % kPer == 0 ? act_grad_kernel<E, true> : act_grad_kernel<E, false>;
        const int st = launch_after(kernel, blocks, stream, static_cast<const E*>(dY), Z, T, N, ldz, act,
                                    static_cast<E*>(dZ), dbias ? partial : nullptr);
        if (st != DTP_OK) return st;
    }
    if (!dbias) return DTP_OK;
    return launch_after(bias_reduce_kernel<E>, (N + 31) / 32, stream, static_cast<const float*>(partial), chunks_of(T), N,
                        static_cast<E*>(dbias));
}

int linear_backward(const void* dY, const void* X, const void* W, const float* Z, int64_t T, int K, int N, int act,
                    int dtype, void* dX, void* dW, void* dbias, void* workspace, cudaStream_t stream) {
    Call call{dtype, workspace, stream};
    Carver c(workspace);
    void* dz = c.take(static_cast<size_t>(T) * padded(N) * elem(dtype));
    float* partial = static_cast<float*>(c.take(static_cast<size_t>(chunks_of(T)) * N * sizeof(float)));
    // dY itself serves as dZ where nothing changes it and the tensor cores can load its rows
    const bool own_dz = act != DTP_ACT_NONE || repitch_bytes(T, N, dtype) > 0;
    const int64_t ldz = own_dz ? padded(N) : N;
    int st = DTP_OK;
    if (own_dz || dbias) {
        auto go = dtype == DTP_BF16 ? launch_act_grad<__nv_bfloat16> : launch_act_grad<float>;
        st = go(dY, Z, T, N, act, own_dz ? dz : nullptr, ldz, partial, dbias, stream);
        if (st != DTP_OK) return st;
    }
    const void* g = own_dz ? dz : dY;
    if (dX && T > 0) {
        Rows w;
        if ((st = aligned_rows(W, N, K, dtype, c, stream, &w)) != DTP_OK) return st;
        Product p;
        p.A[0] = by_row(g, ldz);
        p.B[0] = by_col(w.p, w.ld);
        p.M = T, p.N = K, p.K = N;
        p.epi.out = dX, p.epi.ldo = K, p.epi.M = T, p.epi.N = K;
        if ((st = call.run(p)) != DTP_OK) return st;
    }
    if (dW) {
        Rows x;
        if ((st = aligned_rows(X, T, K, dtype, c, stream, &x)) != DTP_OK) return st;
        auto* runs = static_cast<float*>(c.take(runs_bytes(T, N, K)));
        st = weight_gradient(call, Also{by_col(g, ldz), by_col(x.p, x.ld), N, K, dW, K}, T, runs);
        if (st != DTP_OK) return st;
    }
    return call.done();
}

// ------------------------------------------------------------------------- gated feed-forward

size_t gated_workspace_bytes(int64_t T, int d, int N, int dtype, int backward) {
    Carver c(nullptr);
    c.take(static_cast<size_t>(T) * padded(N) * elem(dtype));
    for (int64_t rows : {T, static_cast<int64_t>(N), static_cast<int64_t>(N)}) c.take(repitch_bytes(rows, d, dtype));
    c.take(repitch_bytes(d, N, dtype));
    c.take(norms_bytes(T, N, dtype));
    if (backward) {
        c.take(static_cast<size_t>(T) * padded(N) * elem(dtype));
        c.take(repitch_bytes(T, d, dtype));
        c.take(runs_bytes(T, N, d));
    }
    return c.used;
}

size_t gated_saved_bytes(int64_t T, int N) { return static_cast<size_t>(pre_floats(T, N)) * sizeof(float); }

int gated_forward(const void* X, const void* Wg, const void* Wu, const void* Wd, const void* residual, int64_t T,
                  int d, int N, int act, int dtype, void* Y, void* H, float* pre, void* workspace,
                  cudaStream_t stream) {
    Call call{dtype, workspace, stream};
    Carver c(workspace);
    void* h = H ? H : c.take(static_cast<size_t>(T) * padded(N) * elem(dtype));
    int st = DTP_OK;
    Product p;
    p.A[0] = by_row(X, d);
    p.B[0] = by_row(Wg, d), p.B[1] = by_row(Wu, d);
    p.M = T, p.N = N, p.K = d;
    Rows wd{Wd, N};
    if (!fews::takes(p, dtype)) {            // which reads rows at any pitch
        Rows x, wg, wu;
        st = aligned_rows(X, T, d, dtype, c, stream, &x);
        if (st == DTP_OK) st = aligned_rows(Wg, N, d, dtype, c, stream, &wg);
        if (st == DTP_OK) st = aligned_rows(Wu, N, d, dtype, c, stream, &wu);
        if (st == DTP_OK) st = aligned_rows(Wd, d, N, dtype, c, stream, &wd);
        if (st != DTP_OK) return st;
        p.A[0] = by_row(x.p, x.ld);
        p.B[0] = by_row(wg.p, wg.ld), p.B[1] = by_row(wu.p, wu.ld);
    }
    p.epi.kind = kEpiGated, p.epi.act = act, p.epi.out = h, p.epi.ldo = padded(N), p.epi.pre = pre;
    p.epi.M = T, p.epi.N = N;
    if ((st = call.run(p)) != DTP_OK) return st;
    Product q;
    q.A[0] = by_row(h, padded(N));
    q.B[0] = by_row(wd.p, wd.ld);
    q.M = T, q.N = d, q.K = N;
    q.epi.residual = residual, q.epi.out = Y, q.epi.ldo = d, q.epi.M = T, q.epi.N = d;
    if ((st = call.run(q)) != DTP_OK) return st;
    if (dtype == DTP_BF16 && act == DTP_ACT_RELU && pre) st = relu_signs<true>(p, nullptr, pre, c, stream);
    if (st != DTP_OK) return st;
    return call.done();
}

int gated_backward(const void* dY, const void* X, const void* Wg, const void* Wu, const void* Wd, const void* H,
                   const float* pre, int64_t T, int d, int N, int act, int dtype, void* dX, void* dWg, void* dWu,
                   void* dWd, void* workspace, cudaStream_t stream) {
    Call call{dtype, workspace, stream};
    Carver c(workspace);
    const int64_t ld = padded(N);
    void* dg = c.take(static_cast<size_t>(T) * ld * elem(dtype));
    void* du = c.take(static_cast<size_t>(T) * ld * elem(dtype));
    int st = DTP_OK;
    Rows x{}, wg{}, wu{}, wd{}, dy{};
    if (T > 0) {                             // without tokens no input is read, and they may be NULL
        st = aligned_rows(X, T, d, dtype, c, stream, &x);
        if (st == DTP_OK) st = aligned_rows(Wg, N, d, dtype, c, stream, &wg);
        if (st == DTP_OK) st = aligned_rows(Wu, N, d, dtype, c, stream, &wu);
        if (st == DTP_OK) st = aligned_rows(Wd, d, N, dtype, c, stream, &wd);
        if (st == DTP_OK) st = aligned_rows(dY, T, d, dtype, c, stream, &dy);
        if (st != DTP_OK) return st;
        Product p;
        p.A[0] = by_row(dy.p, dy.ld);
        p.B[0] = by_col(wd.p, wd.ld);
        p.M = T, p.N = N, p.K = d;
        p.epi.kind = kEpiGatedGrad, p.epi.act = act, p.epi.out = dg, p.epi.out2 = du, p.epi.ldo = ld;
        p.epi.pre = const_cast<float*>(pre), p.epi.M = T, p.epi.N = N;
        if ((st = call.run(p)) != DTP_OK) return st;
    }
    if (dX && T > 0) {
        Product p;
        p.segments = 2;
        p.A[0] = by_row(dg, ld), p.A[1] = by_row(du, ld);
        p.B[0] = by_col(wg.p, wg.ld), p.B[1] = by_col(wu.p, wu.ld);
        p.M = T, p.N = d, p.K = N;
        p.epi.out = dX, p.epi.ldo = d, p.epi.M = T, p.epi.N = d;
        if ((st = call.run(p)) != DTP_OK) return st;
    }
    Also w[3];
    int count = 0;
    auto weight = [&](const void* a, int64_t lda, int64_t rows, const void* b, int64_t ldb, int cols, void* out) {
        if (out) w[count++] = Also{by_col(a, lda), by_col(b, ldb), rows, cols, out, cols};
    };
    weight(dg, ld, N, x.p, x.ld, d, dWg);
    weight(du, ld, N, x.p, x.ld, d, dWu);
    weight(dy.p, dy.ld, d, H, ld, N, dWd);
    // they share their K: one launch for all that are wanted (bf16), so that their tiles fill the rounds
    if (dtype == DTP_BF16 && T > 0 && T <= kRun && count > 0) {
        Product p;
        p.A[0] = w[0].A;
        p.B[0] = w[0].B;
        p.M = w[0].M, p.N = w[0].N, p.K = T;
        p.epi.out = w[0].out, p.epi.ldo = w[0].ldo, p.epi.M = w[0].M, p.epi.N = w[0].N;
        p.batch = count;
        for (int j = 1; j < count; ++j) p.also[j - 1] = w[j];
        if ((st = call.run(p)) != DTP_OK) return st;
        return call.done();
    }
    auto* runs = static_cast<float*>(c.take(runs_bytes(T, N, d)));
    for (int i = 0; i < count; ++i)
        if ((st = weight_gradient(call, w[i], T, runs)) != DTP_OK) return st;
    return call.done();
}

}  // namespace layer
}  // namespace dtp
