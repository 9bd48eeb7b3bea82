// few_tokens_simt.cu -- the forward products of the layer operators for few tokens on the CUDA cores (bf16: one or two, fp32: up
// to 32, in groups of eight):
//
//     acc[t, n] = sum_k X[t, k] W[n, k]     (fp32), then the epilogue at (t, n)
//
// Bound by streaming the weights once.  A block takes eight weight rows (or four neurons' gate and up rows); its 256 threads
// share the k axis, each with one 16-byte word of every row in flight, and multiply it with all tokens' words, which come from
// L2.  The block's sums go over the lanes by halves (a butterfly that leaves each lane the values it finishes), then over the
// warps in order.  Eight rows: with T tokens the blocks read T / 8 times the weights' bytes from L2, and a thread's 8 T sums
// stay in registers.  Up to two tokens a thread holds the next words while it multiplies; with more, two blocks per SM hide
// the loads.  The groups of the same rows run side by side, so that HBM gives the weights once.
#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include "dtp_common.cuh"
#include "layer_common.cuh"

namespace dtp {
namespace fews {

using namespace layer;

constexpr int kThreads = 256;
constexpr int kWarps = kThreads / 32;
constexpr int R = 8;                   // weight rows per block

struct Args {
    const void* X;
    const void* W[2];
    int64_t ldx, ldw;
    int64_t K;
    int groups;      // of tokens
    int second;      // X was written by the launch before this one
    int* status;     // set: this launch clears it
    Epilogue epi;
};

// Coherent loads, not those of the read-only path: this kernel starts while the launch before it may still be writing the tokens (or, in
// a call of its own, the weights), and what that path reads must not change while the kernel lives.  The weights, read once,
// take no place in L1: 4096 x 4096 and one token 8.6 us with weights from HBM, 9.0 where they do.
__device__ __forceinline__ uint4 load_once(const void* p) {
    uint4 q;
    asm volatile("ld.global.L1::no_allocate.v4.u32 {%0, %1, %2, %3}, [%4];"
                 : "=r"(q.x), "=r"(q.y), "=r"(q.z), "=r"(q.w)
                 : "l"(p)
                 : "memory");
    return q;
}

// PER consecutive elements from k, zero beyond K.
template <typename E, bool kWide>
struct Word {
    static constexpr int PER = kWide ? 16 / static_cast<int>(sizeof(E)) : 1;
    uint4 q;
    template <bool kOnce>
    __device__ __forceinline__ void load(const E* row, int64_t k, int64_t K) {
        if constexpr (kWide) {
            q = make_uint4(0, 0, 0, 0);
            if (k < K) q = kOnce ? load_once(row + k) : *reinterpret_cast<const uint4*>(row + k);
        } else {
            const float v = k < K ? to_f32(row[k]) : 0.0f;
            q.x = __float_as_uint(v);
        }
    }
    __device__ __forceinline__ void get(float (&v)[PER]) const {
        if constexpr (!kWide) {
            v[0] = __uint_as_float(q.x);
        } else {
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
    }
};

// v[i] summed over the lanes, in a fixed order.  V >= 32: lane l ends with values 32 g + l in v[g]; below, lane l with value
// l / (32 / V) in v[0].
template <int V>
__device__ __forceinline__ void lane_sums(float (&v)[V], int lane) {
    if constexpr (V > 32) {
        float lo[V / 2], hi[V / 2];
#pragma unroll
        for (int i = 0; i < V / 2; ++i) lo[i] = v[i], hi[i] = v[V / 2 + i];
        lane_sums<V / 2>(lo, lane);
        lane_sums<V / 2>(hi, lane);
#pragma unroll
        for (int g = 0; g < V / 64; ++g) v[g] = lo[g], v[V / 64 + g] = hi[g];
    } else {
        int o = 16;
#pragma unroll
        for (int m = V / 2; m >= 1; m /= 2, o /= 2) {
            const bool upper = (lane & o) != 0;
#pragma unroll
            for (int i = 0; i < m; ++i) {
                const float send = upper ? v[i] : v[i + m];
                const float keep = upper ? v[i + m] : v[i];
                v[i] = keep + __shfl_xor_sync(0xFFFFFFFFu, send, o);
            }
        }
        for (; o >= 1; o /= 2) v[0] += __shfl_xor_sync(0xFFFFFFFFu, v[0], o);
    }
}

template <typename E, int TT, int KIND, bool kWide>
__global__ void __launch_bounds__(kThreads, 2) few_simt_kernel(const __grid_constant__ Args p) {
    constexpr bool kGated = KIND == kEpiGated;
    constexpr int kCols = kGated ? R / 2 : R;              // outputs per block
    constexpr int PER = Word<E, kWide>::PER, V = R * TT;
    __shared__ float red[kWarps][V];
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    constexpr bool kAhead = TT <= 2;
    const int n0 = static_cast<int>(blockIdx.x) / p.groups * kCols;
    const int t0 = static_cast<int>(blockIdx.x) % p.groups * TT;
    const int T = static_cast<int>(p.epi.M) - t0 < TT ? static_cast<int>(p.epi.M) - t0 : TT;
    const int64_t K = p.K;
    if (!p.second) grid_wait();
    // rows beyond the last read the last one's (their sums are not used)
    const E* row[R];
#pragma unroll
    for (int r = 0; r < R; ++r) {
        const int n = n0 + (kGated ? r % kCols : r);
        row[r] = static_cast<const E*>(p.W[kGated && r >= kCols]) + (n < p.epi.N ? n : p.epi.N - 1) * p.ldw;
    }
    float acc[V];
#pragma unroll
    for (int i = 0; i < V; ++i) acc[i] = 0.0f;
    Word<E, kWide> w[R];
    int64_t k = static_cast<int64_t>(tid) * PER;
    if constexpr (kAhead) {
#pragma unroll
        for (int r = 0; r < R; ++r) w[r].template load<true>(row[r], k, K);
    }
    if (p.second) grid_wait();                             // the weights do not come from the launch before
    grid_release();
    if (p.status && blockIdx.x == 0 && tid == 0) *p.status = DTP_OK;     // nothing here can give up
    const E* X = static_cast<const E*>(p.X) + t0 * p.ldx;
    for (; k < K; k += kThreads * PER) {
        float wv[R][PER];
        if constexpr (kAhead) {
#pragma unroll
            for (int r = 0; r < R; ++r) w[r].get(wv[r]);
#pragma unroll
            for (int r = 0; r < R; ++r) w[r].template load<true>(row[r], k + kThreads * PER, K);      // the next words
        } else {
#pragma unroll
            for (int r = 0; r < R; ++r) w[r].template load<true>(row[r], k, K);
#pragma unroll
            for (int r = 0; r < R; ++r) w[r].get(wv[r]);
        }
#pragma unroll
        for (int t = 0; t < TT; ++t) {
            Word<E, kWide> x;
            x.template load<false>(X + (t < T ? t : 0) * p.ldx, k, K);
            float xv[PER];
            x.get(xv);
#pragma unroll
            for (int r = 0; r < R; ++r)
#pragma unroll
                for (int i = 0; i < PER; ++i) acc[t * R + r] = fmaf(xv[i], wv[r][i], acc[t * R + r]);
        }
    }
    lane_sums<V>(acc, lane);
    if constexpr (V >= 32) {
#pragma unroll
        for (int g = 0; g < V / 32; ++g) red[warp][32 * g + lane] = acc[g];
    } else if (lane % (32 / V) == 0) {
        red[warp][lane / (32 / V)] = acc[0];
    }
    __syncthreads();
    for (int i = tid; i < TT * kCols; i += kThreads) {
        const int t = i / kCols, r = i % kCols;
        if (t >= T || n0 + r >= p.epi.N) continue;
        float a0 = 0.0f, a1 = 0.0f;
#pragma unroll
        for (int s = 0; s < kWarps; ++s) {
            a0 += red[s][t * R + r];
            if constexpr (kGated) a1 += red[s][t * R + kCols + r];
        }
        epilogue_element<E, KIND>(p.epi, t0 + t, n0 + r, a0, a1);
    }
}

template <typename E, int TT>
static int launch_tokens(const Product& p, Args& a, bool wide, cudaStream_t stream) {
    a.groups = static_cast<int>((p.M + TT - 1) / TT);
    const bool gated = p.epi.kind == kEpiGated;
    auto kernel = wide ? (gated ? few_simt_kernel<E, TT, kEpiGated, true> : few_simt_kernel<E, TT, kEpiLinear, true>)
                       : (gated ? few_simt_kernel<E, TT, kEpiGated, false> : few_simt_kernel<E, TT, kEpiLinear, false>);
    const int cols = gated ? R / 2 : R;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(static_cast<unsigned>((p.N + cols - 1) / cols * a.groups));
    cfg.blockDim = dim3(kThreads);
    cfg.stream = stream;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    DTP_CUDA_TRY(cudaLaunchKernelEx(&cfg, kernel, a));
    return DTP_OK;
}

template <typename E>
static int launch_typed(const Product& p, int* status, int second, cudaStream_t stream) {
    Args a;
    a.X = p.A[0].p;
    a.W[0] = p.B[0].p, a.W[1] = p.B[1].p;
    a.ldx = p.A[0].rs, a.ldw = p.B[0].rs;
    a.K = p.K;
    a.second = second;
    a.status = status;
    a.epi = p.epi;
    constexpr int64_t per = 16 / sizeof(E);
    // K a multiple of a word: no word has elements of the next row, or beyond the matrix
    const bool wide = p.K % per == 0 && a.ldx % per == 0 && a.ldw % per == 0;
    if (p.M == 1) return launch_tokens<E, 1>(p, a, wide, stream);
    if (p.M == 2) return launch_tokens<E, 2>(p, a, wide, stream);
    if constexpr (sizeof(E) == 4) {
        if (p.M <= 4) return launch_tokens<E, 4>(p, a, wide, stream);
        return launch_tokens<E, 8>(p, a, wide, stream);
    }
    return DTP_ERR_UNSUPPORTED;
}

// Whether this kernel takes the product: both operands with k contiguous, and few tokens.  bf16, one token and two, this kernel and the
// tensor cores: the block of 1024 x 3072 8.5 and 9.3 us for one (weights in L2 6.7 and 7.5), 7.4 and 7.7 for two (in L2);
// a layer of 4096 x 4096 by itself 5.3 and 6.0 us for one with the weights in L2, 8.3 and 7.8 from HBM, for two 6.1 and 6.0, 8.7
// and 8.0; odd widths are read here as they are, without a copy.  From three tokens on the tensor cores win.  fp32, up to 32:
// 4096 x 4096 12.6 us for one token (5.3 TB/s), 49 for 32, 62 in the tiles for 33.
bool takes(const Product& p, int dtype) {
    return p.M <= (dtype == DTP_BF16 ? 2 : 32) && p.segments == 1 && p.A[0].ks == 1 && p.B[0].ks == 1 &&
           p.epi.kind != kEpiGatedGrad;
}

// status: set when this launch clears it; second: X was written by the launch before this one on the stream, whose own
// predecessors' results are there when this one begins.
int launch(const Product& p, int dtype, int* status, int second, cudaStream_t stream) {
    return dtype == DTP_BF16 ? launch_typed<__nv_bfloat16>(p, status, second, stream)
                             : launch_typed<float>(p, status, second, stream);
}

}  // namespace fews
}  // namespace dtp
