// rms_norm.cu -- the RMS norm of rows and its gradients:
//
//     rms_t = sqrt(mean_i x_ti^2 + eps),  y = gamma n,  n = x / rms
//     dx = (dn - n mean_i(dn n)) / rms + dresidual,  dn = gamma dy,   dgamma_i = sum_t dy_ti n_ti
//
// Bound by memory: each value is read and written once.  A row lies in the registers of a warp (to 512 columns, forward 1024) or
// of a block of 128 to 512 threads (to 8192), eight consecutive columns to a thread at a time, so that its sum and what is made
// of it need one read.  Backward, a thread keeps its columns' sums for dgamma over the rows that its group takes, at most kRun;
// the groups of a block add theirs in shared memory, and the blocks' are added by a last launch.  Wider rows go through memory
// again (from L2).  Rows that are not on 16-byte boundaries are read element by element in the same places, with the same
// results bit for bit.  16384 x 4096 in bf16: 48 us forward (5.6 TB/s), 84 backward with a residual's gradient (6.4), 6 for the
// last launch; 4096 x 16384 both ways, through memory, 648.
#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <stdint.h>
#include <string.h>

#include <type_traits>

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
constexpr int kWidest = 8192;          // columns of a row in registers
constexpr int kSms = 152;              // for which the backward pass's blocks are counted

// Threads of a block whose rows take TPR threads each.
__host__ __device__ constexpr int block_threads(int tpr) { return tpr > 32 ? tpr : kThreads; }
// A row whose mean square and eps leave fp32's range is summed again at this scale.  Their sum is at least 2^127.8, so that what counts
// stays far above the least number (2^-149), and 2^20 squares of numbers below 2^128 sum to no more than 2^84.
constexpr float kDown = 0x1p-96f;

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

// Sums over the threads of a row: 32 of them, or the block.  kRows values at once; `red` is used in turns, so that one barrier is
// enough: who writes it again has passed the barrier of the turn between.
template <int TPR, int kRows>
__device__ __forceinline__ void row_sums(float (&v)[kRows], float (&red)[2][kRows][TPR / 32], int turn) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
#pragma unroll
    for (int r = 0; r < kRows; ++r)
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) v[r] += __shfl_xor_sync(0xFFFFFFFFu, v[r], o);
    if constexpr (TPR > 32) {
#pragma unroll
        for (int r = 0; r < kRows; ++r)
            if (lane == 0) red[turn & 1][r][warp] = v[r];
        __syncthreads();
#pragma unroll
        for (int r = 0; r < kRows; ++r) {
            v[r] = 0.0f;
#pragma unroll
            for (int w = 0; w < TPR / 32; w += 4) {
                const float4 a = *reinterpret_cast<const float4*>(red[turn & 1][r] + w);
                v[r] += (a.x + a.y) + (a.z + a.w);
            }
        }
    }
}

// Blocks of the forward pass on an SM.
__host__ __device__ constexpr int forward_blocks(int tpr) { return tpr == 512 ? 2 : 768 / block_threads(tpr); }

// How a thread's columns lie: octets of consecutive ones in words; the same element by element, where rows start on other
// boundaries; or, in rows whose length is no multiple of eight and which have no aligned form to agree with, every TPR-th column, so that a
// warp's elements are consecutive (4095 columns: 2.5 times the octets' rate).
enum Map { kWords, kOctets, kStrided };

// Column of element j of octet k.
template <int TPR, Map kMap>
__device__ __forceinline__ int column(int k, int j) {
    const int me = threadIdx.x % TPR;
    return kMap == kStrided ? (8 * k + j) * TPR + me : (TPR * k + me) * 8 + j;
}

// Eight columns of a row of d.
template <typename E, int TPR, Map kMap>
struct Octet {
    uint4 q[sizeof(E) == 2 ? 1 : 2];
    __device__ __forceinline__ void load(const E* row, int k, int d, bool in) {
        if constexpr (kMap == kWords) {
            const int c = column<TPR, kMap>(k, 0);
#pragma unroll
            for (int i = 0; i < static_cast<int>(sizeof(q) / 16); ++i)
                q[i] = in && c < d ? reinterpret_cast<const uint4*>(row + c)[i] : make_uint4(0, 0, 0, 0);
        } else {
            E e[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const int c = column<TPR, kMap>(k, j);
                e[j] = in && c < d ? row[c] : from_f32<E>(0.0f);
            }
            memcpy(q, e, sizeof(q));
        }
    }
    __device__ __forceinline__ void store(E* row, int k, int d) const {
        if constexpr (kMap == kWords) {
            const int c = column<TPR, kMap>(k, 0);
#pragma unroll
            for (int i = 0; i < static_cast<int>(sizeof(q) / 16); ++i)
                if (c < d) reinterpret_cast<uint4*>(row + c)[i] = q[i];
        } else {
            E e[8];
            memcpy(e, q, sizeof(q));
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const int c = column<TPR, kMap>(k, j);
                if (c < d) row[c] = e[j];
            }
        }
    }
    __device__ __forceinline__ void get(float (&v)[8]) const {
        const uint32_t* w = reinterpret_cast<const uint32_t*>(q);
#pragma unroll
        for (int j = 0; j < 8; ++j)
            v[j] = sizeof(E) == 4 ? __uint_as_float(w[j])
                                  : __uint_as_float(j & 1 ? w[j / 2] & 0xFFFF0000u : w[j / 2] << 16);
    }
    __device__ __forceinline__ void set(const float (&v)[8]) {
        E e[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) e[j] = from_f32<E>(v[j]);
        memcpy(q, e, sizeof(q));
    }
};

// Rows t .. t + rows - 1 on their way to L2, by one thread; in whole 16-byte words, the first and last of which they may share.
template <typename E>
__device__ __forceinline__ void prefetch_rows(const E* p, int64_t t, int rows, int64_t T, int d) {
    if (t >= T) return;
    const int64_t n = T - t < rows ? T - t : rows;
    const uintptr_t a = reinterpret_cast<uintptr_t>(p + t * d), from = a & ~uintptr_t(15), to = (a + n * d * sizeof(E) + 15) & ~uintptr_t(15);
    asm volatile("cp.async.bulk.prefetch.L2.global [%0], %1;" ::"l"(from), "r"(static_cast<uint32_t>(to - from)) : "memory");
}
constexpr int kAhead = 1;              // turns of a block by which its rows are prefetched (16384 x 4096: 138 us both ways, 148 with 2, 152 without)

// OCT octets to a thread.  kWords: every row and gamma on 16-byte boundaries.
template <typename E, int TPR, int OCT, int kRows, Map kMap>
__global__ void __launch_bounds__(block_threads(TPR), forward_blocks(TPR)) forward_rows_kernel(const E* X, const float* gamma, int64_t T, int d, float eps, E* Y,
                                                                float* rms) {
    __shared__ __align__(16) float red[2][kRows][TPR / 32];
    grid_wait();
    grid_release();
    constexpr int kGroups = block_threads(TPR) / TPR;
    const int me = threadIdx.x % TPR;
    const int64_t stride = static_cast<int64_t>(gridDim.x) * kGroups * kRows;
    const float width = static_cast<float>(d);
    int turn = 0;
    // groups of a block stay together: their rows are first .. first + kGroups * kRows - 1
    for (int64_t first = static_cast<int64_t>(blockIdx.x) * kGroups * kRows; first < T; first += stride) {
        const int64_t t0 = first + threadIdx.x / TPR * kRows;
        if (threadIdx.x == 0) prefetch_rows(X, first + kAhead * stride, kGroups * kRows, T, d);
        Octet<E, TPR, kMap> x[kRows][OCT];
        float s[kRows];
#pragma unroll
        for (int r = 0; r < kRows; ++r)
#pragma unroll
            for (int k = 0; k < OCT; ++k) x[r][k].load(X + (t0 + r) * d, k, d, t0 + r < T);
        auto squares = [&](float scale) {
#pragma unroll
            for (int r = 0; r < kRows; ++r) {
                s[r] = 0.0f;
#pragma unroll
                for (int k = 0; k < OCT; ++k) {
                    float v[8];
                    x[r][k].get(v);
#pragma unroll
                    for (int j = 0; j < 8; ++j) v[j] *= scale, s[r] = fmaf(v[j], v[j], s[r]);
                }
            }
            row_sums<TPR, kRows>(s, red, turn++);
        };
        squares(1.0f);
        float root[kRows];
        bool again = false;
#pragma unroll
        for (int r = 0; r < kRows; ++r) {
            root[r] = sqrtf(s[r] / width + eps);
            again |= !(s[r] / width + eps <= 3.0e38f);
        }
        if (TPR > 32 ? again : __any_sync(0xFFFFFFFFu, again)) {       // the same for all threads of a row
            squares(kDown);
#pragma unroll
            for (int r = 0; r < kRows; ++r)
                if (!(root[r] <= 1.7e19f)) root[r] = sqrtf(s[r] / width + eps * kDown * kDown) / kDown;
        }
#pragma unroll
        for (int r = 0; r < kRows; ++r) {
            if (t0 + r >= T) continue;
            if (me == 0 && rms) rms[t0 + r] = root[r];
            const float inv = 1.0f / root[r];
            const bool tiny = !(root[r] <= 8.0e37f);       // its reciprocal would be among fp32's subnormal numbers
#pragma unroll
            for (int k = 0; k < OCT; ++k) {
                Octet<float, TPR, kMap> g;
                g.load(gamma, k, d, true);
                float v[8], w[8];
                x[r][k].get(v);
                g.get(w);
#pragma unroll
                for (int j = 0; j < 8; ++j) v[j] = (tiny ? v[j] / root[r] : v[j] * inv) * w[j];
                Octet<E, TPR, kMap> y;
                y.set(v);
                y.store(Y + (t0 + r) * d, k, d);
            }
        }
    }
}

// dX, and the block's part of dgamma in partial[block] [d].
template <typename E, int TPR, int OCT, int kRows, Map kMap>
__global__ void __launch_bounds__(block_threads(TPR), 512 / block_threads(TPR))
backward_rows_kernel(const E* dY, const E* X, const float* gamma, const float* rms, const E* dres, int64_t T, int d, E* dX,
                     float* partial) {
    constexpr int kGroups = block_threads(TPR) / TPR;
    __shared__ __align__(16) float red[2][kRows][TPR / 32];
    __shared__ float sums[kGroups > 1 ? kGroups : 1][kGroups > 1 ? TPR * 8 + 4 : 1];
    grid_wait();
    grid_release();
    const int me = threadIdx.x % TPR;
    float g[OCT][8], acc[OCT][8];
#pragma unroll
    for (int k = 0; k < OCT; ++k) {
        Octet<float, TPR, kMap> q;
        q.load(gamma, k, d, gamma != nullptr);
        q.get(g[k]);
#pragma unroll
        for (int j = 0; j < 8; ++j) acc[k][j] = 0.0f;
    }
    const float width = static_cast<float>(d);
    int turn = 0;
    const int64_t stride = static_cast<int64_t>(gridDim.x) * kGroups * kRows;
    for (int64_t first = static_cast<int64_t>(blockIdx.x) * kGroups * kRows; first < T; first += stride) {
        const int64_t t0 = first + threadIdx.x / TPR * kRows;
        if (threadIdx.x == 0) {
            prefetch_rows(X, first + kAhead * stride, kGroups * kRows, T, d);
            prefetch_rows(dY, first + kAhead * stride, kGroups * kRows, T, d);
            if (dres) prefetch_rows(dres, first + kAhead * stride, kGroups * kRows, T, d);
        }
        Octet<E, TPR, kMap> x[kRows][OCT], y[kRows][OCT], z[kRows][OCT];
        float root[kRows], s[kRows];
#pragma unroll
        for (int r = 0; r < kRows; ++r) {
            const bool in = t0 + r < T;
            root[r] = in ? rms[t0 + r] : 1.0f;
#pragma unroll
            for (int k = 0; k < OCT; ++k) {
                const int64_t at = (t0 + r) * d;
                x[r][k].load(X + at, k, d, in);
                y[r][k].load(dY + at, k, d, in);
                z[r][k].load(dres + at, k, d, in && dres);
            }
        }
#pragma unroll
        for (int r = 0; r < kRows; ++r) {
            const float inv = 1.0f / root[r];
            s[r] = 0.0f;
#pragma unroll
            for (int k = 0; k < OCT; ++k) {
                float n[8], v[8];
                x[r][k].get(n);
                y[r][k].get(v);
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    n[j] *= inv;
                    acc[k][j] = fmaf(v[j], n[j], acc[k][j]);
                    s[r] = fmaf(v[j] * g[k][j], n[j], s[r]);
                }
            }
        }
        if (!dX) continue;
        row_sums<TPR, kRows>(s, red, turn++);
#pragma unroll
        for (int r = 0; r < kRows; ++r) {
            if (t0 + r >= T) continue;
            const float inv = 1.0f / root[r], mean = s[r] / width;
#pragma unroll
            for (int k = 0; k < OCT; ++k) {
                float n[8], v[8], w[8];
                x[r][k].get(n);
                y[r][k].get(v);
                z[r][k].get(w);
#pragma unroll
                for (int j = 0; j < 8; ++j) v[j] = fmaf(fmaf(-n[j] * inv, mean, v[j] * g[k][j]), inv, w[j]);
                Octet<E, TPR, kMap> o;
                o.set(v);
                o.store(dX + (t0 + r) * d, k, d);
            }
        }
    }
    if (!partial) return;
#pragma unroll
    for (int k = 0; k < OCT; ++k) {
        if constexpr (kGroups > 1) {               // the groups' sums in order, a chunk of columns at a time
            __syncthreads();
#pragma unroll
            for (int j = 0; j < 8; ++j) sums[threadIdx.x / TPR][column<TPR, kMap>(0, j)] = acc[k][j];
            __syncthreads();
            for (int i = threadIdx.x; i < TPR * 8; i += block_threads(TPR)) {
                float v = 0.0f;
#pragma unroll
                for (int q = 0; q < kGroups; ++q) v += sums[q][i];
                const int c = TPR * 8 * k + i;
                if (c < d) partial[static_cast<int64_t>(blockIdx.x) * d + c] = v;
            }
        } else {
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const int c = column<TPR, kMap>(k, j);
                if (c < d) partial[static_cast<int64_t>(blockIdx.x) * d + c] = acc[k][j];
            }
        }
    }
}

// Rows wider than kWidest.
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
            return block_sum(s, red) / static_cast<float>(d) + eps * scale * scale;
        };
        const float s = squares(1.0f);
        const float r = s <= 3.0e38f ? sqrtf(s) : sqrtf(squares(kDown)) / kDown;
        if (threadIdx.x == 0 && rms) rms[t] = r;
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

// A sum of many fp32 terms with the rounding errors of the additions carried along.
struct Total {
    float sum = 0.0f, lost = 0.0f;
    __device__ __forceinline__ void add(float x) {
        const float t = sum + x, b = t - sum;
        lost += (sum - (t - b)) + (x - b);
        sum = t;
    }
    // the errors of infinite sums are no numbers
    __device__ __forceinline__ float value() const { return isfinite(sum) ? sum + lost : sum; }
};

// dgamma from the partial sums: each of 32 warps adds every 32nd in order, then the warps' sums in order, with their errors (in fp64, whose
// additions are slow here: 40 us for 304 sums of 1537 columns).
constexpr int kJoinWarps = 32;
__global__ void __launch_bounds__(32 * kJoinWarps) join_kernel(const float* partial, int64_t runs, int d, float* dgamma) {
    __shared__ Total red[kJoinWarps][32];
    grid_wait();
    grid_release();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, i = blockIdx.x * 32 + lane;
    Total s;
    if (i < d)
#pragma unroll 8
        for (int64_t r = warp; r < runs; r += kJoinWarps) s.add(partial[r * d + i]);
    red[warp][lane] = s;
    __syncthreads();
    if (warp == 0 && i < d) {
#pragma unroll
        for (int w = 1; w < kJoinWarps; ++w) s.add(red[w][lane].sum), s.lost += red[w][lane].lost;
        dgamma[i] = s.value();
    }
}

// The form for rows of d columns: threads of a row, octets of a thread, rows of a group at a time (so that loads of 64 to 128 bytes a
// thread are in flight without spilling the backward pass's registers).
template <int TPR_, int OCT_, int ROWS_>
struct Form {
    static constexpr int TPR = TPR_, OCT = OCT_, ROWS = ROWS_, kBlock = block_threads(TPR), kPerBlock = kBlock / TPR * ROWS;
};
template <int kHalf, typename F>
static int64_t with_form(int d, F fn) {
    if (d <= 256) return fn(Form<32, 1, 2 / kHalf>());
    if (d <= 512) return fn(Form<32, 2, 1>());
    if (d <= 1024) return fn(Form<128, 1, 4 / kHalf>());
    if (d <= 2048) return fn(Form<256, 1, 4 / kHalf>());
    if (d <= 4096) return fn(Form<256, 2, 2 / kHalf>());
    return fn(Form<512, 2, 2 / kHalf>());
}
template <typename E, typename F>
static int64_t with_form_of(int d, F fn) { return with_form<sizeof(E) / 2>(d, fn); }      // fp32 takes half the rows

// The forward pass holds one tensor's rows and no sums: a warp takes a row up to 1024 columns, without a barrier (65536 x 1024: 44 us,
// 54 with 128 threads; 2048 columns 62 us, 58 with 256 threads, and a single row 4.6 and 2.9).
template <typename E, typename F>
static int64_t with_forward_form(int d, F fn) {
    constexpr int kHalf = sizeof(E) / 2;
    if (d <= 256) return fn(Form<32, 1, 2 / kHalf>());
    if (d <= 512) return fn(Form<32, 2, 1>());
    if (d <= 1024) return fn(Form<32, 4, 1>());
    if (d <= 2048) return fn(Form<256, 1, 4 / kHalf>());
    if (d <= 4096) return fn(Form<256, 2, 2 / kHalf>());
    return fn(Form<512, 2, 2 / kHalf>());
}

// Blocks of the backward pass, each with a partial sum of dgamma: as many as run at once, but no more than kRun rows for a group.
template <typename E>
static int64_t backward_blocks(int64_t T, int d) {
    if (d > kWidest) return (T + kRun - 1) / kRun;
    return with_form_of<E>(d, [&](auto form) -> int64_t {
        using F = decltype(form);
        const int64_t tiles = (T + F::kPerBlock - 1) / F::kPerBlock;
        const int64_t least = (tiles * F::ROWS + kRun - 1) / kRun, once = kSms * (512 / F::kBlock);
        const int64_t n = least > once ? least : once;
        return n < tiles ? n : tiles;
    });
}

size_t backward_workspace_bytes(int64_t T, int d) {
    layer::Carver c(nullptr);
    const int64_t a = backward_blocks<float>(T, d), b = backward_blocks<__nv_bfloat16>(T, d);
    c.take(static_cast<size_t>(a > b ? a : b) * d * sizeof(float));
    return c.used;
}

static Map map_of(int d, const void* a, const void* b, const void* c, const void* e, const void* gamma) {
    const uintptr_t all = reinterpret_cast<uintptr_t>(a) | reinterpret_cast<uintptr_t>(b) | reinterpret_cast<uintptr_t>(c) |
                          reinterpret_cast<uintptr_t>(e) | reinterpret_cast<uintptr_t>(gamma);
    return d % 8 != 0 ? kStrided : (all & 15) == 0 ? kWords : kOctets;
}

template <typename E>
static int forward(const void* X, const float* gamma, int64_t T, int d, float eps, void* Y, float* rms, cudaStream_t stream) {
    const E* x = static_cast<const E*>(X);
    E* y = static_cast<E*>(Y);
    if (d > kWidest)
        return layer::launch_blocks(forward_kernel<E>, T < 8192 ? T : 8192, kThreads, stream, x, gamma, T, d, eps, y, rms);
    return static_cast<int>(with_forward_form<E>(d, [&](auto form) -> int64_t {
        using F = decltype(form);
        const int64_t tiles = (T + F::kPerBlock - 1) / F::kPerBlock, most = kSms * forward_blocks(F::TPR), blocks = tiles < most ? tiles : most;
        const Map map = map_of(d, X, Y, nullptr, nullptr, gamma);
        auto kernel = map == kWords    ? forward_rows_kernel<E, F::TPR, F::OCT, F::ROWS, kWords>
                      : map == kOctets ? forward_rows_kernel<E, F::TPR, F::OCT, F::ROWS, kOctets>
                                       : forward_rows_kernel<E, F::TPR, F::OCT, F::ROWS, kStrided>;
        return layer::launch_blocks(kernel, blocks, F::kBlock, stream, x, gamma, T, d, eps, y, rms);
    }));
}

template <typename E>
static int backward(const void* dY, const void* X, const float* gamma, const float* rms, const void* dres, int64_t T, int d,
                    void* dX, float* dgamma, void* workspace, cudaStream_t stream) {
    const E *dy = static_cast<const E*>(dY), *x = static_cast<const E*>(X), *dr = static_cast<const E*>(dres);
    E* dx = static_cast<E*>(dX);
    layer::Carver c(workspace);
    const int64_t blocks = backward_blocks<E>(T, d);
    auto* partial = static_cast<float*>(c.take(static_cast<size_t>(blocks) * d * sizeof(float)));
    int st = DTP_OK;
    if (T > 0 && d > kWidest) {
        if (dgamma)                        // first: dX may take the place of dY
            st = layer::launch_blocks(columns_kernel<E>, blocks * ((d + kThreads - 1) / kThreads), kThreads, stream, dy, x, rms, T, d, partial);
        if (st == DTP_OK && dX)
            st = layer::launch_blocks(rows_kernel<E>, T < 8192 ? T : 8192, kThreads, stream, dy, x, gamma, rms, dr, T, d, dx);
    } else if (T > 0 && (dX || dgamma)) {
        st = static_cast<int>(with_form_of<E>(d, [&](auto form) -> int64_t {
            using F = decltype(form);
            const Map map = map_of(d, dY, X, dres, dX, gamma);
            auto kernel = map == kWords    ? backward_rows_kernel<E, F::TPR, F::OCT, F::ROWS, kWords>
                          : map == kOctets ? backward_rows_kernel<E, F::TPR, F::OCT, F::ROWS, kOctets>
                                           : backward_rows_kernel<E, F::TPR, F::OCT, F::ROWS, kStrided>;
            return layer::launch_blocks(kernel, blocks, F::kBlock, stream, dy, x, gamma, rms, dr, T, d, dx, dgamma ? partial : nullptr);
        }));
    }
    if (st != DTP_OK || !dgamma) return st;
    return layer::launch_blocks(join_kernel, (d + 31) / 32, 32 * kJoinWarps, stream, static_cast<const float*>(partial), T > 0 ? blocks : 0, d, dgamma);
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
