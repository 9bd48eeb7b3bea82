// few_tokens_tc.cu -- the forward products of the layer operators for few tokens (single-token serving, small
// batches up to 64), bf16, on the tcgen05 tensor cores:
//
//     acc[n, t] = sum_k W[n, k] X[t, k]     (fp32 in TMEM), then the epilogue at (t, n)
//
// Bound by streaming the weights once.  The operands change places: 128 weight rows are the MMA's rows and up to
// TN = 16, 32 or 64 tokens its columns, so no tensor work is spent on absent tokens beyond TN.  A tile is 128 outputs,
// or 64 neurons with their gate rows above their up rows.  To have enough loads in flight on the whole chip, a
// cluster of up to 8 CTAs shares a tile, each with its own range of k; the partial sums meet in shared memory
// (each CTA sends every peer the rows that the peer finishes) and are added in the order of the ranges, so the
// result does not depend on timing.
//
// Six warps: warp 4 loads 64-wide k blocks by TMA, two a stage up to 32 tokens (256 bytes of a row at a time, and half the
// barriers), warp 5 issues the MMAs, warps 0 to 3 send the partial sums, and all of them run the epilogue.  In a sequence of two products the second one starts early and loads its weights
// while the first finishes; it waits for the first before it touches the tokens.
#include <cuda.h>
#include <cudaTypedefs.h>
#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include "dtp_common.cuh"
#include "layer_common.cuh"

namespace dtp {
namespace few {

using namespace layer;

constexpr int BM = 128;       // weight rows per tile
constexpr int BK = 64;
constexpr int UK = 16;
constexpr int kThreads = 192;
constexpr int kMaxSplit = 8;  // CTAs of a portable cluster

template <int TN>
struct Form {
    static constexpr int kBoxes = TN <= 32 ? 2 : 1;                       // k blocks per stage
    static constexpr uint32_t kBoxBytes = (BM + TN) * BK * 2;
    static constexpr uint32_t kStageBytes = kBoxes * kBoxBytes;
    static constexpr size_t kSums = static_cast<size_t>(BM) * TN * 4;     // partial sums from all CTAs of the cluster
    static constexpr int STAGES = static_cast<int>((112 * 1024 - kSums - 1536) / kStageBytes);     // two CTAs per SM
    static constexpr uint32_t kTmemCols = TN < 32 ? 32 : TN;
    static constexpr size_t kSmemBytes = 1024 + STAGES * kStageBytes + kSums + 256;
};
static_assert(Form<16>::STAGES >= 2 && Form<32>::STAGES >= 2 && Form<64>::STAGES >= 3, "");
static_assert(Form<16>::kSmemBytes <= 113 * 1024 && Form<32>::kSmemBytes <= 113 * 1024 &&
                  Form<64>::kSmemBytes <= 113 * 1024, "two CTAs per SM");

struct Args {
    CUtensorMap w[2], x;
    int KB;          // k blocks of 64
    int split;       // CTAs per tile
    int second;      // this product reads what the launch before it wrote
    int reset;       // this launch clears the status word
    int* status;
    Epilogue epi;
};

__device__ __forceinline__ void st_shared_cluster_f32(uint32_t cluster_addr, float v) {
    asm volatile("st.shared::cluster.f32 [%0], %1;" ::"r"(cluster_addr), "f"(v) : "memory");
}

template <int TN, int KIND>
__global__ void __launch_bounds__(kThreads) few_tokens_kernel(const __grid_constant__ Args p) {
    using F = Form<TN>;
    constexpr int STAGES = F::STAGES;
    extern __shared__ uint8_t smem_raw[];
    // the same offset in every CTA of the cluster, so that a peer's buffer is found at this one's address
    uint8_t* smem = smem_raw + ((1024u - (smem_u32(smem_raw) & 1023u)) & 1023u);
    uint8_t* tiles = smem;
    float* sums = reinterpret_cast<float*>(smem + STAGES * F::kStageBytes);   // [source CTA][token][own row]
    uint64_t* bars = reinterpret_cast<uint64_t*>(smem + STAGES * F::kStageBytes + F::kSums);
    uint64_t* full_bar = bars;
    uint64_t* empty_bar = bars + STAGES;
    uint64_t* acc_full = bars + 2 * STAGES;
    uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(acc_full + 1);
    volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);

    const int warp = __shfl_sync(0xFFFFFFFFu, static_cast<int>(threadIdx.x >> 5), 0), lane = threadIdx.x & 31;
    const int S = p.split;
    const int rank = static_cast<int>(blockIdx.x) % S, tile = static_cast<int>(blockIdx.x) / S;
    constexpr int kCols = KIND == kEpiGated ? BM / 2 : BM;      // outputs per tile
    const int n0 = tile * kCols;
    const int kb0 = static_cast<int>(static_cast<int64_t>(p.KB) * rank / S);
    const int kb1 = static_cast<int>(static_cast<int64_t>(p.KB) * (rank + 1) / S);

    if (threadIdx.x == 0) {
        for (int s = 0; s < STAGES; ++s) {
            mbar_init(smem_u32(&full_bar[s]), 1);
            mbar_init(smem_u32(&empty_bar[s]), 1);
        }
        mbar_init(smem_u32(acc_full), 1);
        *abort_flag = 0;
        fence_mbar_init();
    }
    if (warp == 5) {
        tmem_alloc(smem_u32(tmem_slot), F::kTmemCols);
        tmem_relinquish();
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = *tmem_slot;
    asm volatile("barrier.cluster.arrive.relaxed;" ::: "memory");    // this CTA runs

    constexpr int kBoxes = F::kBoxes;
    // Before any bounded wait of this launch begins, the launch before it is over: it may run longer than their limit.
    if (warp != 4) grid_wait();
    if (warp == 4) {
        // -------------------------------------------------------------------- producer: one lane issues
        const bool issuer = elect_one();
        const uint32_t full0 = smem_u32(full_bar), empty0 = smem_u32(empty_bar), tiles0 = smem_u32(tiles);
        const CUtensorMap* lower = KIND == kEpiGated ? &p.w[1] : &p.w[0];
        const int lower_row = KIND == kEpiGated ? n0 : n0 + BM / 2;
        if (issuer) {
            tma_prefetch_desc(&p.w[0]);
            tma_prefetch_desc(&p.x);
        }
        auto boxes_at = [&](int kb) { return kb1 - kb < kBoxes ? kb1 - kb : kBoxes; };
        auto load_w = [&](int kb, int s) {
            const uint32_t fb = full0 + s * 8u;
            const int boxes = boxes_at(kb);
            if (!issuer) return;
            mbar_arrive_expect_tx(fb, boxes * F::kBoxBytes);
            for (int x = 0; x < boxes; ++x) {
                const uint32_t st = tiles0 + s * F::kStageBytes + x * F::kBoxBytes;
                tma_load_2d(st, &p.w[0], fb, (kb + x) * BK, n0);
                tma_load_2d(st + BM / 2 * BK * 2, lower, fb, (kb + x) * BK, lower_row);
            }
        };
        auto load_x = [&](int kb, int s) {
            const int boxes = boxes_at(kb);
            if (!issuer) return;
            for (int x = 0; x < boxes; ++x)
                tma_load_2d(tiles0 + s * F::kStageBytes + x * F::kBoxBytes + BM * BK * 2, &p.x, full0 + s * 8u,
                            (kb + x) * BK, 0);
        };
        const int filled = (kb1 - kb0 + kBoxes - 1) / kBoxes;
        const int first = filled < STAGES ? filled : STAGES;
        // the second product's weights do not come from the first
        if (!p.second) grid_wait();
        for (int i = 0; i < first; ++i) load_w(kb0 + i * kBoxes, i);
        if (p.second) grid_wait();
        grid_release();
        asm volatile("fence.proxy.async;" ::: "memory");
        // Clears the status of earlier calls.  A wait of this launch gives up two seconds after it began, long after
        // block 0, which starts first, has passed here.
        if (p.reset && blockIdx.x == 0 && issuer) *reinterpret_cast<volatile int*>(p.status) = DTP_OK;
        for (int i = 0; i < first; ++i) load_x(kb0 + i * kBoxes, i);
        int stage = 0;
        uint32_t phase = 0;                      // of the stage's reuse
        for (int kb = kb0 + first * kBoxes; kb < kb1; kb += kBoxes) {
            if (!warp_wait(empty0 + stage * 8u, phase, abort_flag)) break;
            load_w(kb, stage);
            load_x(kb, stage);
            if (++stage == STAGES) { stage = 0; phase ^= 1u; }
        }
    } else if (warp == 5) {
        // ------------------------------------------------------------------ MMA issuer
        const bool issuer = elect_one();
        constexpr uint32_t kIdesc = idesc_bf16_f32(BM, TN);
        const uint32_t full0 = smem_u32(full_bar), empty0 = smem_u32(empty_bar);
        const uint32_t low_w = desc_low(smem_u32(tiles), false);
        int stage = 0;
        uint32_t phase = 0;
        for (int kb = kb0; kb < kb1; kb += kBoxes) {
            if (!warp_wait(full0 + stage * 8u, phase, abort_flag)) break;
            tc_fence_after();
            const int boxes = kb1 - kb < kBoxes ? kb1 - kb : kBoxes;
            if (issuer) {
#pragma unroll
                for (int x = 0; x < kBoxes; ++x) {
                    if (x >= boxes) break;
                    const uint32_t w = low_w + ((stage * F::kStageBytes + x * F::kBoxBytes) >> 4);
#pragma unroll
                    for (int kk = 0; kk < BK / UK; ++kk) {
                        const uint32_t at = w + ((kk * UK * 2) >> 4);
                        umma_bf16(tmem, desc(at), desc(at + ((BM * BK * 2) >> 4)), kIdesc,
                                  (kb > kb0 || x > 0 || kk > 0) ? 1u : 0u);
                    }
                }
                umma_commit(empty0 + stage * 8u);
            }
            __syncwarp();
            if (++stage == STAGES) { stage = 0; phase ^= 1u; }
        }
        if (issuer) umma_commit(smem_u32(acc_full));
    }
    __syncwarp();
    asm volatile("barrier.cluster.wait;" ::: "memory");              // every peer runs: its memory may be written

    const int T = static_cast<int>(p.epi.M);
    // outputs that this CTA finishes: n0 + rank * own .., own a power of two
    const int own_log = (KIND == kEpiGated ? 6 : 7) - (31 - __clz(S)), own = 1 << own_log;
    if (warp < 4) {
        // ------------------------------------------------- partial sums to the CTAs that finish them
        const bool ok = warp_wait(smem_u32(acc_full), 0, abort_flag);
        tc_fence_after();
        if (ok) {
            const int row = warp * 32 + lane;            // of the tile
            const int j = KIND == kEpiGated ? row & (BM / 2 - 1) : row;
            const int dst = j >> own_log;
            // [rank][token][gate rows, then up rows, of the destination's outputs]
            const int pitch = KIND == kEpiGated ? 2 * own : own;
            const int at = rank * TN * pitch + (j & (own - 1)) + (KIND == kEpiGated && row >= BM / 2 ? own : 0);
            const uint32_t to = mapa_shared(smem_u32(sums + at), static_cast<uint32_t>(dst));
            const uint32_t acc = tmem + (static_cast<uint32_t>(warp * 32) << 16);
#pragma unroll 1
            for (int c = 0; c < TN && c < T; c += 16) {
                float v[16];
                tmem_ld16(acc + c, v);
                tmem_wait_ld();
#pragma unroll
                for (int i = 0; i < 16; ++i)
                    if (c + i < T) st_shared_cluster_f32(to + static_cast<uint32_t>((c + i) * pitch * 4), v[i]);
            }
        }
        tc_fence_before();
    }
    cluster_sync();
    if (warp == 5) {
        if (*abort_flag) {      // loads and MMAs already issued may still be under way: let them finish
            const uint64_t t0 = globaltimer_ns();
            while (globaltimer_ns() - t0 < 200ull * 1000ull) {
            }
        }
        tc_fence_after();
        tmem_dealloc(tmem, F::kTmemCols);
    }
    // ------------------------------------------------------------------------- epilogue
    const int pitch = KIND == kEpiGated ? 2 * own : own;
    const int base = n0 + rank * own;
    for (int i = threadIdx.x; i < T * own; i += kThreads) {
        const int t = i >> own_log, r = i & (own - 1), n = base + r;
        if (n >= p.epi.N) continue;
        float a0 = 0.0f, a1 = 0.0f;
        for (int s = 0; s < S; ++s) {
            const float* from = sums + (s * TN + t) * pitch + r;
            a0 += from[0];
            if constexpr (KIND == kEpiGated) a1 += from[own];
        }
        epilogue_element<__nv_bfloat16, KIND>(p.epi, t, n, a0, a1);
    }
    if (threadIdx.x == 0 && *abort_flag) atomicExch(p.status, static_cast<int>(DTP_ERR_NOT_CONVERGED));
    __syncthreads();
}

// ------------------------------------------------------------------------------------ host

static bool map_rows(CUtensorMap* m, const Mat& a, int64_t rows, int64_t K, int box_rows) {
    auto enc = tensor_map_encoder();
    if (!enc) return false;
    cuuint64_t dims[2] = {static_cast<cuuint64_t>(K), static_cast<cuuint64_t>(rows)};
    cuuint64_t strides[1] = {static_cast<cuuint64_t>(a.rs) * 2};
    cuuint32_t box[2] = {BK, static_cast<cuuint32_t>(box_rows)};
    cuuint32_t estr[2] = {1, 1};
    return enc(m, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, const_cast<void*>(a.p), dims, strides, box, estr,
               CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
               CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <int TN>
static int launch_form(const Product& p, int* status, int reset, int second, int sms, cudaStream_t stream) {
    using F = Form<TN>;
    const bool gated = p.epi.kind == kEpiGated;
    Args a;
    if (!map_rows(&a.w[0], p.B[0], p.N, p.K, BM / 2) || (gated && !map_rows(&a.w[1], p.B[1], p.N, p.K, BM / 2)) ||
        !map_rows(&a.x, p.A[0], p.M, p.K, TN))
        return DTP_ERR_CUDA;
    const int cols = gated ? BM / 2 : BM;
    const int tiles = (p.N + cols - 1) / cols;
    a.KB = static_cast<int>((p.K + BK - 1) / BK);
    // CTAs per tile: until the chip is covered, with at least two k blocks for each
    a.split = 1;
    while (a.split < kMaxSplit && static_cast<int64_t>(tiles) * a.split < sms && a.KB / (2 * a.split) >= 2) a.split *= 2;
    a.second = second;
    a.reset = reset;
    a.status = status;
    a.epi = p.epi;
    auto kernel = gated ? few_tokens_kernel<TN, kEpiGated> : few_tokens_kernel<TN, kEpiLinear>;
    DTP_CUDA_TRY(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                      static_cast<int>(F::kSmemBytes)));
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(static_cast<unsigned>(tiles * a.split));
    cfg.blockDim = dim3(kThreads);
    cfg.dynamicSmemBytes = F::kSmemBytes;
    cfg.stream = stream;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = static_cast<unsigned>(a.split);
    attr[0].val.clusterDim.y = 1;
    attr[0].val.clusterDim.z = 1;
    attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[1].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 2;
    DTP_CUDA_TRY(cudaLaunchKernelEx(&cfg, kernel, a));
    return DTP_OK;
}

// Whether this kernel takes the product: both operands with k contiguous, few tokens.  Up to 32 always (4096 x 4096, 32 tokens:
// 9.4 us here, 13.3 in the persistent tiles); from 33 to 64 where there are too few tiles to keep those busy (64 tokens: 4096 x
// 4096 11.8 and 13.5 us, 4096 x 14336 31.7 and 24.5).
bool takes(const Product& p) {
    const int cols = p.epi.kind == kEpiGated ? BM / 2 : BM;
    return p.M <= (p.N > 64 * cols ? 32 : 64) && p.segments == 1 && p.A[0].ks == 1 && p.B[0].ks == 1 &&
           p.epi.kind != kEpiGatedGrad;
}

// second: X was written by the launch before this one on the stream, which is this kernel too.
int launch(const Product& p, int* status, int reset, int second, cudaStream_t stream) {
    int dev = 0, sms = 0;
    DTP_CUDA_TRY(cudaGetDevice(&dev));
    DTP_CUDA_TRY(cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev));
    if (p.M <= 16) return launch_form<16>(p, status, reset, second, sms, stream);
    if (p.M <= 32) return launch_form<32>(p, status, reset, second, sms, stream);
    return launch_form<64>(p, status, reset, second, sms, stream);
}

}  // namespace few
}  // namespace dtp
