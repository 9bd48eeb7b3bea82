// gemm_simt.cu -- the fp32 matrix products of the layer operators on the CUDA cores (and the empty sums of
// either type): any sizes, any of the four operand orders, fp32 sums, epilogues fused.
//
// Bound by the FMA pipe.  A thread owns 8 x 8 outputs and multiplies with packed fma.rn.f32x2 (each half rounds as a
// scalar fma): per k four float4 shared loads for 32 packed FMAs.  A block is 128 x 128 outputs (256 threads, two blocks
// per SM) or 64 x 128 (128 threads, four per SM), the smaller one unless there are four rounds of the larger.  k blocks of
// 16 come into a ring of shared-memory stages by cp.async: 4 bytes at a time, which takes any row pitch and lays rows of k
// down as columns on the way, or 16 where the operand's rows are contiguous and aligned.  The gated kind puts two gate
// columns beside the two up columns of the same neurons, so that a thread holds both.  Where there are fewer tiles than
// the chip holds blocks, a cluster shares a tile, each block with its own range of k; the partial sums meet in shared
// memory and are added in the order of the ranges.
// 4096 x 4096 x 4096 on a GB300: 52 to 58 TFLOP/s by operand order; 515 x 1536 x 1001 51 us, 31 TFLOP/s (64 x 64 tiles of
// 4 x 4 a thread: 73 us).
#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include "dtp_common.cuh"
#include "layer_common.cuh"

namespace dtp {
namespace simt {

using namespace layer;

constexpr int TK = 16;
constexpr int STAGES = 4;
constexpr int kMaxSplit = 8;
constexpr int PT = 8;                            // rows and columns per thread
constexpr int TN = 16 * PT;                      // columns per tile
constexpr int SB = TN + 4;                       // floats per k: 16-byte rows, start moving by 4 banks

template <int TY>                                // rows of 16 threads
struct Tile {
    static constexpr int TM = TY * PT;
    static constexpr int kThreads = 16 * TY;
    static constexpr int kBlocks = 32 / TY;      // per SM
    static constexpr int SA = TM + 4;
    static constexpr int kStage = TK * (SA + SB);
    static constexpr size_t kSmem = sizeof(float) * STAGES * kStage;
    // The partial sums of a split tile take the stages' place: up to TM / split rows, rounded up, from each block.
    static constexpr bool kSplits = STAGES * kStage >= (TM + kMaxSplit - 1) * TN;
    static_assert(kBlocks * (kSmem + 1024) <= 227 * 1024, "shared memory");
};

struct Args {
    Product p;
    int tiles_n;
    int split;
    int wide_a, wide_b;      // rows contiguous and on 16-byte boundaries
    int* status;             // set: this launch clears it (nothing here can give up)
};

__device__ __forceinline__ void fma2(uint64_t& d, uint64_t a, uint64_t b) {
    asm("fma.rn.f32x2 %0, %1, %2, %0;" : "+l"(d) : "l"(a), "l"(b));
}
__device__ __forceinline__ uint64_t twice(float v) {
    uint64_t r;
    asm("mov.b64 %0, {%1, %1};" : "=l"(r) : "f"(v));
    return r;
}
__device__ __forceinline__ float2 unpack2(uint64_t v) {
    float2 r;
    asm("mov.b64 {%0, %1}, %2;" : "=f"(r.x), "=f"(r.y) : "l"(v));
    return r;
}
// bytes beyond `valid` are written as zero
__device__ __forceinline__ void copy4(uint32_t dst, const float* src, int valid) {
    asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;" ::"r"(dst), "l"(src), "r"(valid) : "memory");
}
__device__ __forceinline__ void copy16(uint32_t dst, const float* src, int valid) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(valid) : "memory");
}
__device__ __forceinline__ void copies_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void copies_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }

__device__ __forceinline__ void st_shared_cluster_f32x4(uint32_t cluster_addr, float4 v) {
    asm volatile("st.shared::cluster.v4.f32 [%0], {%1, %2, %3, %4};" ::"r"(cluster_addr), "f"(v.x), "f"(v.y), "f"(v.z),
                 "f"(v.w)
                 : "memory");
}

// A thread's share of an operand's ROWS x TK blocks, laid down as [k][row].
template <int ROWS, int THREADS>
struct Copies {
    static constexpr int SR = ROWS + 4;
    const float *at0, *at1;  // the thread's first element of k block 0, per segment
    int64_t ks;
    int64_t step;            // elements between the thread's copies
    int mode;                // 0: k contiguous, 1: rows contiguous, 2: the same on 16-byte boundaries
    int k, rows_in, to;      // first k; copies (mode 0) or elements of a copy whose rows exist; place in the stage

    // rows r0 .. of `rows`; `gated`: every four tile rows are two of m[0] and the same two of m[1]
    __device__ __forceinline__ Copies(const Mat (&m)[2], int segments, int64_t r0, int64_t rows, bool wide, bool gated) {
        const int tid = threadIdx.x;
        const int64_t rs = m[0].rs;
        ks = m[0].ks;
        mode = ks == 1 ? 0 : wide ? 2 : 1;
        int r;
        at0 = static_cast<const float*>(m[0].p);
        at1 = static_cast<const float*>(segments == 2 ? m[1].p : m[0].p);
        if (mode == 0) {
            k = tid & 15, r = tid >> 4, to = k * SR + r;
            int64_t per = THREADS / 16;
            const int copies = ROWS * 16 / THREADS;
            if (gated) {
                if (r & 2) at0 = static_cast<const float*>(m[1].p);
                r = (r >> 2) * 2 + (r & 1);
                per /= 2;
            }
            step = per * rs;
            const int64_t left = (rows - r0 - r + per - 1) / per;
            rows_in = rows <= r0 + r ? 0 : static_cast<int>(left < copies ? left : copies);
        } else {
            const int width = mode == 2 ? 4 : 1;
            r = tid % (ROWS / width) * width, k = tid / (ROWS / width), to = k * SR + r;
            step = THREADS / (ROWS / width) * ks;
            const int64_t left = rows - r0 - r;
            rows_in = left <= 0 ? 0 : left < width ? static_cast<int>(left) : width;
        }
        const int64_t off = rows_in ? (r0 + r) * rs + k * ks : 0;
        at0 += off;
        at1 += off;
    }

    __device__ __forceinline__ void block(bool second, int64_t k0, int64_t K, float* stage) const {
        const uint32_t dst = smem_u32(stage + to);
        const float* base = second ? at1 : at0;            // a place that exists where nothing is read
        const float* src = base + k0 * ks;
        const int64_t left = K - k0 - k;                   // from the thread's first k
        if (mode == 0) {
            const int in = left > 0 ? rows_in : 0;
#pragma unroll
            for (int i = 0; i < ROWS * 16 / THREADS; ++i, src += step)
                copy4(dst + THREADS / 16 * 4 * i, i < in ? src : base, i < in ? 4 : 0);
        } else if (mode == 1) {
            constexpr int per = THREADS / ROWS;
            const int in = rows_in ? static_cast<int>(left < TK ? left : TK) : 0;
#pragma unroll
            for (int i = 0; i < TK / per; ++i, src += step)
                copy4(dst + per * SR * 4 * i, i * per < in ? src : base, i * per < in ? 4 : 0);
        } else {
            constexpr int per = THREADS / (ROWS / 4);
            const int in = static_cast<int>(left < TK ? left : TK);
#pragma unroll
            for (int i = 0; i < TK / per; ++i, src += step)
                copy16(dst + per * SR * 4 * i, i * per < in ? src : base, i * per < in ? rows_in * 4 : 0);
        }
    }
};

template <int TY, int KIND>
__global__ void __launch_bounds__(Tile<TY>::kThreads, Tile<TY>::kBlocks) gemm_f32_kernel(const __grid_constant__ Args g) {
    using S = Tile<TY>;
    constexpr int TM = S::TM, SA = S::SA;
    constexpr bool kGated = KIND == kEpiGated;
    constexpr int kCols = kGated ? TN / 2 : TN;           // outputs per tile
    extern __shared__ __align__(16) float stages[];
    const Product& p = g.p;
    const int tid = threadIdx.x, tx = tid & 15, ty = tid >> 4;
    const int part = static_cast<int>(blockIdx.x) % g.split;
    const int64_t tile = blockIdx.x / g.split;
    const int64_t m0 = tile / g.tiles_n * TM;
    const int n0 = static_cast<int>(tile % g.tiles_n) * kCols;
    const int64_t blocks = (p.K + TK - 1) / TK;           // per segment
    const int64_t b0 = p.segments * blocks * part / g.split, b1 = p.segments * blocks * (part + 1) / g.split;

    const Copies<TM, S::kThreads> ca(p.A, p.segments, m0, p.M, g.wide_a, false);
    const Copies<TN, S::kThreads> cb(p.B, p.segments, n0, p.N, g.wide_b, kGated);
    if (g.status && blockIdx.x == 0 && tid == 0) *g.status = DTP_OK;
    auto fetch = [&](int64_t b) {
        if (b < b1) {
            float* st = stages + (b % STAGES) * S::kStage;
            const bool second = b >= blocks;
            const int64_t k0 = (second ? b - blocks : b) * TK;
            ca.block(second, k0, p.K, st);
            cb.block(second, k0, p.K, st + TK * SA);
        }
        copies_commit();
    };

    uint64_t acc[PT][PT / 2];
#pragma unroll
    for (int i = 0; i < PT; ++i)
#pragma unroll
        for (int j = 0; j < PT / 2; ++j) acc[i][j] = 0;
    for (int s = 0; s < STAGES - 1; ++s) fetch(b0 + s);
    for (int64_t b = b0; b < b1; ++b) {
        copies_wait<STAGES - 2>();       // this thread's copies of block b have landed,
        __syncthreads();                 // everybody's have, and everybody is past block b - 1
        fetch(b + STAGES - 1);           // into the stage of block b - 1
        const float* as = stages + (b % STAGES) * S::kStage + PT * ty;
        const float* bs = stages + (b % STAGES) * S::kStage + TK * SA + 4 * tx;
#pragma unroll
        for (int k = 0; k < TK; ++k) {
            uint64_t a[PT], w[PT / 2];
#pragma unroll
            for (int i = 0; i < PT; i += 4) {
                const float4 v = *reinterpret_cast<const float4*>(as + k * SA + i);
                a[i] = twice(v.x), a[i + 1] = twice(v.y), a[i + 2] = twice(v.z), a[i + 3] = twice(v.w);
            }
#pragma unroll
            for (int q = 0; q < PT / 4; ++q) {
                const ulonglong2 v = *reinterpret_cast<const ulonglong2*>(bs + k * SB + 64 * q);
                w[2 * q] = v.x, w[2 * q + 1] = v.y;
            }
#pragma unroll
            for (int i = 0; i < PT; ++i)
#pragma unroll
                for (int j = 0; j < PT / 2; ++j) fma2(acc[i][j], a[i], w[j]);
        }
    }
    copies_wait<0>();

    // four tile columns c .. c + 3 of row m: outputs, or two neurons' gate and up sums
    auto finish = [&](int64_t m, int c, const float4& v) {
        if (m >= p.M) return;
        if constexpr (kGated) {
            const int n = n0 + c / 2;
            if (n < p.N) epilogue_element<float, KIND>(p.epi, m, n, v.x, v.z);
            if (n + 1 < p.N) epilogue_element<float, KIND>(p.epi, m, n + 1, v.y, v.w);
        } else {
            const float e[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if (n0 + c + i < p.N) epilogue_element<float, KIND>(p.epi, m, n0 + c + i, e[i], 0.0f);
        }
    };
    auto sums = [&](int i, int q) {
        const float2 x = unpack2(acc[i][2 * q]), y = unpack2(acc[i][2 * q + 1]);
        return make_float4(x.x, x.y, y.x, y.y);
    };
    if (g.split == 1) {
#pragma unroll
        for (int i = 0; i < PT; ++i)
#pragma unroll
            for (int q = 0; q < PT / 4; ++q) finish(m0 + PT * ty + i, 64 * q + 4 * tx, sums(i, q));
        return;
    }
    // block r of the cluster finishes rows r TM / split ..: every block sends it its sums of them
    const int split = g.split;
    auto first_row = [&](int r) { return TM * r / split; };
    cluster_sync();                      // nobody computes from its stages any more
#pragma unroll
    for (int i = 0; i < PT; ++i) {
        const int row = PT * ty + i, dst = ((row + 1) * split - 1) / TM;
        const int r0 = first_row(dst), own = first_row(dst + 1) - r0;
        const uint32_t to = mapa_shared(smem_u32(stages + (part * own + row - r0) * TN), static_cast<uint32_t>(dst));
#pragma unroll
        for (int q = 0; q < PT / 4; ++q) st_shared_cluster_f32x4(to + (64 * q + 4 * tx) * 4, sums(i, q));
    }
    cluster_sync();
    const int r0 = first_row(part), own = first_row(part + 1) - r0;
    for (int x = tid; x < own * (TN / 4); x += S::kThreads) {
        const int row = x / (TN / 4), c = x % (TN / 4) * 4;
        float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
        for (int s = 0; s < split; ++s) {
            const float4 w = *reinterpret_cast<const float4*>(stages + (s * own + row) * TN + c);
            v.x += w.x, v.y += w.y, v.z += w.z, v.w += w.w;
        }
        finish(m0 + r0 + row, c, v);
    }
}

template <int TY>
static int launch_tiles(const Product& p, int* status, int sms, cudaStream_t stream) {
    using S = Tile<TY>;
    const int cols = p.epi.kind == kEpiGated ? TN / 2 : TN;
    Args g;
    g.p = p;
    g.status = status;
    g.tiles_n = (p.N + cols - 1) / cols;
    const int64_t tiles = (p.M + S::TM - 1) / S::TM * g.tiles_n;
    // blocks per tile: as many as the chip holds of them, with at least 64 k for each
    const int64_t room = S::kBlocks * static_cast<int64_t>(sms) / tiles, most = p.K * p.segments / 64;
    const int64_t split = !S::kSplits ? 1 : room < most ? room : most;
    g.split = static_cast<int>(split < 1 ? 1 : split < kMaxSplit ? split : kMaxSplit);
    if (tiles * g.split > 0x7FFFFFFF) return DTP_ERR_UNSUPPORTED;
    auto wide = [](const Mat& m) { return m.ks != 1 && m.ks % 4 == 0 && aligned16(m.p); };
    g.wide_a = wide(p.A[0]) && (p.segments == 1 || wide(p.A[1]));
    g.wide_b = wide(p.B[0]) && (p.segments == 1 || wide(p.B[1])) && p.epi.kind != kEpiGated;
    auto kernel = p.epi.kind == kEpiLinear  ? gemm_f32_kernel<TY, kEpiLinear>
                  : p.epi.kind == kEpiGated ? gemm_f32_kernel<TY, kEpiGated>
                                            : gemm_f32_kernel<TY, kEpiGatedGrad>;
    DTP_CUDA_TRY(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                      static_cast<int>(S::kSmem)));
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(static_cast<unsigned>(tiles * g.split));
    cfg.blockDim = dim3(S::kThreads);
    cfg.dynamicSmemBytes = S::kSmem;
    cfg.stream = stream;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = static_cast<unsigned>(g.split);
    attr[0].val.clusterDim.y = 1;
    attr[0].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    DTP_CUDA_TRY(cudaLaunchKernelEx(&cfg, kernel, g));
    return DTP_OK;
}

// An empty sum (no tokens): out = 0, the only epilogue that such a product has.
template <typename E>
__global__ void zero_kernel(E* out, int64_t rows, int64_t cols, int64_t ld) {
    for (int64_t i = blockIdx.x * static_cast<int64_t>(blockDim.x) + threadIdx.x; i < rows * cols;
         i += static_cast<int64_t>(gridDim.x) * blockDim.x)
        out[i / cols * ld + i % cols] = from_f32<E>(0.0f);
}

// status: set when this launch clears it.
int launch(const Product& p, int dtype, int* status, cudaStream_t stream) {
    if (p.K == 0) {
        if (dtype == DTP_BF16)
            zero_kernel<<<256, 256, 0, stream>>>(static_cast<__nv_bfloat16*>(p.epi.out), p.M, p.N, p.epi.ldo);
        else
            zero_kernel<<<256, 256, 0, stream>>>(static_cast<float*>(p.epi.out), p.M, p.N, p.epi.ldo);
        DTP_CUDA_TRY(cudaGetLastError());
        return DTP_OK;
    }
    if (dtype != DTP_F32) return DTP_ERR_UNSUPPORTED;
    int dev = 0, sms = 0;
    DTP_CUDA_TRY(cudaGetDevice(&dev));
    DTP_CUDA_TRY(cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev));
    const int64_t cols = p.epi.kind == kEpiGated ? TN / 2 : TN;
    const int64_t large = (p.M + 127) / 128 * ((p.N + cols - 1) / cols);
    return large >= 8 * sms ? launch_tiles<16>(p, status, sms, stream) : launch_tiles<8>(p, status, sms, stream);
}

}  // namespace simt
}  // namespace dtp
