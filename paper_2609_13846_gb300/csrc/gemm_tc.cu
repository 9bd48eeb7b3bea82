// gemm_tc.cu -- the bf16 matrix products of the layer operators on the tcgen05 tensor cores, with their
// epilogues fused:
//
//     acc[m, n] = sum over segments s, k of A_s[m, k] B_s[n, k]     (fp32 in TMEM)
//
// then, by kind, act(acc + bias) + residual (and the pre-activation), act(gate) up (and both), or the gradients
// of gate and up from dH.  Each operand may be stored with k contiguous (weights and tokens in the forward
// products) or with its rows contiguous (the transposed operands of the gradients): both are loaded by TMA into
// 128-byte-swizzled tiles and described to the tensor core in their own order, so nothing is transposed in
// memory.
//
// Structure: persistent grid, one CTA per SM, twenty warps: warp 0 loads tiles by TMA, warp 1 issues the MMAs,
// sixteen warps in two sets drain the accumulator, which is double-buffered in TMEM: a set takes every second tile, so that
// it has two tiles' time for its epilogue (the block of 1024 x 3072 on 16384 tokens 173 us, with eight warps and one tile's
// time 193).  Two forms: CTA pairs share 256 x BN x 16 tcgen05.mma of cta_group::2 (each CTA stages 128 rows of A and half of
// B), single CTAs issue 128 x BN x 16 ones (up to 128 rows).  Shared memory bounds both: a 64-wide k
// block is written once and read once by the tensor core, 64 KB per CTA at 128 bytes a clock for 256 x 256 pairs, as long as
// its MMAs take (512 clocks), 384 clocks against 256 for 256 x 128 ones, 512 against 256 for single 128 x 128 tiles.
// Where tiles are fewer than the pairs that the chip holds, a cluster of two or four pairs shares a tile, each pair with its
// own range of k (kSplit): the partial sums meet in the shared memory that the stages leave free, are added in the order of
// the ranges, and each CTA finishes a slice of the columns.  Measured: 4096 x 14336 x 4096 1.83 PFLOP/s (254 us; 293 with whole
// left-over tiles), 8192^3 1.82, 1003 x 2048 x 1024 with a residual 9.6 us, 200 x 1024 x 1024 5.5 us.
#include <cuda.h>
#include <cudaTypedefs.h>
#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include <atomic>
#include <type_traits>

#include "dtp_common.cuh"
#include "layer_common.cuh"

namespace dtp {
namespace gtc {

using namespace layer;

constexpr int BM = 128;       // rows of A per CTA (TMEM lanes)
constexpr int BK = 64;
constexpr int UK = 16;
constexpr int kThreads = 640;
constexpr int kEpiWarps = 16;                     // two sets of 8, one per accumulator
constexpr int kEpiWarp0 = 4;
constexpr uint32_t kTileA = BM * BK * 2;          // 16 KB
constexpr uint32_t kStageOut = 32 * 64;           // a 32-row x 32-column bf16 box, 2 KB (64-byte swizzle)

// A stage holds two 64-wide k blocks of A and of B: the thread that issues the MMAs passes a barrier once for eight of them
// (one block per stage: 600 to 650 clocks a block, whatever the tile).
constexpr int kBoxes = 2;
template <bool kPair, int BN>
struct Form {
    static constexpr int kRowsB = kPair ? BN / 2 : BN;            // staged by this CTA
    static constexpr uint32_t kTileB = kRowsB * BK * 2;
    static constexpr uint32_t kBoxBytes = kTileA + kTileB;
    static constexpr uint32_t kStageBytes = kBoxes * kBoxBytes;
    static constexpr int STAGES = 192 * 1024 / kStageBytes;
    static constexpr uint32_t kTmemCols = 2 * BN;                 // two accumulators: a power of two
    static constexpr size_t kSmemBytes = 1024 + STAGES * kStageBytes + kEpiWarps * kStageOut + 512;
};

// A launch's products: one (of one or two segments, or with a second B or output), or up to three of the same K and
// operand orders whose tiles follow one another, so that the last round of one is filled by the next.
constexpr int kBatch = 3;
struct Args {
    CUtensorMap a[kBatch], b[kBatch], out[kBatch], z;     // by product; by segment, or gate and up, in a single one
    int segments;
    int KB;               // k blocks of 64 per segment
    int a_mn, b_mn;       // operand stored with its rows contiguous
    int tiles_m[kBatch], tiles_n[kBatch];     // per CTA or pair
    int last[kBatch];     // tiles of the products up to this one
    int64_t M[kBatch];
    int N[kBatch];
    int64_t ldo[kBatch];
    void* dst[kBatch];
    int direct[kBatch];   // out rows are not on 16-byte boundaries: plain stores
    int unit0, units;     // this launch's tiles: unit0 .. units - 1
    int split;            // pairs per tile (kSplit)
    int early;            // kSplit: begun while the launch before it, of the same product's other tiles, still runs
    uint32_t idesc;
    int direct_z;         // rows of Z are not on 16-byte boundaries
    int reset;            // this launch clears the status word
    int* status;
    Epilogue epi;
};

// `leave`: out of L2 first, for what only the backward pass reads again (Z); the operands stay.
template <bool kLeave>
__device__ __forceinline__ void tma_store_2d(const CUtensorMap* map, uint32_t src, int32_t x, int32_t y) {
    if constexpr (kLeave) {
        uint64_t policy;
        asm volatile("createpolicy.fractional.L2::evict_first.b64 %0, 1.0;" : "=l"(policy));
        asm volatile("cp.async.bulk.tensor.2d.global.shared::cta.bulk_group.L2::cache_hint [%0, {%2, %3}], [%1], %4;" ::"l"(
                         reinterpret_cast<uint64_t>(map)),
                     "r"(src), "r"(x), "r"(y), "l"(policy)
                     : "memory");
    } else {
        asm volatile("cp.async.bulk.tensor.2d.global.shared::cta.bulk_group [%0, {%2, %3}], [%1];" ::"l"(
                         reinterpret_cast<uint64_t>(map)),
                     "r"(src), "r"(x), "r"(y)
                     : "memory");
    }
}
__device__ __forceinline__ void bulk_commit() { asm volatile("cp.async.bulk.commit_group;" ::: "memory"); }
__device__ __forceinline__ void bulk_wait_read0() { asm volatile("cp.async.bulk.wait_group.read 0;" ::: "memory"); }
__device__ __forceinline__ void fence_async_smem() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }

__device__ __forceinline__ uint32_t pack_bf16(float a, float b) {
    const __nv_bfloat162 v = __floats2bfloat162_rn(a, b);
    return *reinterpret_cast<const uint32_t*>(&v);
}
__device__ __forceinline__ void unpack_bf16(uint32_t v, float& a, float& b) {
    a = __uint_as_float(v << 16);
    b = __uint_as_float(v & 0xFFFF0000u);
}

// Units of a persistent worker: row tiles in groups of 8, column tile by column tile within a group, so that the
// tiles in flight share their rows and columns in L2.
constexpr int kGroupM = 8;
template <int JOBS>
__device__ __forceinline__ void decode(const Args& p, int u, int& job, int& tm, int& tn) {
    job = 0;
    if constexpr (JOBS > 1) {
        job = (u >= p.last[0]) + (u >= p.last[1]);
        if (job) u -= p.last[job - 1];
    }
    const unsigned per = static_cast<unsigned>(kGroupM) * p.tiles_n[job];
    const unsigned g = static_cast<unsigned>(u) / per, rest = static_cast<unsigned>(u) - g * per;
    const int m0 = static_cast<int>(g) * kGroupM;
    const unsigned gm = p.tiles_m[job] - m0 < kGroupM ? p.tiles_m[job] - m0 : kGroupM;
    tn = static_cast<int>(rest / gm);
    tm = m0 + static_cast<int>(rest % gm);
}

__device__ __forceinline__ void st_shared_cluster_f32x4(uint32_t cluster_addr, float a, float b, float c, float d) {
    asm volatile("st.shared::cluster.v4.f32 [%0], {%1, %2, %3, %4};" ::"r"(cluster_addr), "f"(a), "f"(b), "f"(c), "f"(d)
                 : "memory");
}

// JOBS: products that the launch may hold.
template <bool kPair, int BN, int KIND, bool kSplit, int JOBS>
__global__ void __launch_bounds__(kThreads, 1) gemm_tc_kernel(const __grid_constant__ Args p) {
    using F = Form<kPair, BN>;
    constexpr int STAGES = F::STAGES;
    constexpr uint32_t kStageBytes = F::kStageBytes;
    // output columns per tile: the two accumulators of the gated kind share it
    constexpr int kCols = KIND == kEpiGated ? BN / 2 : BN;
    extern __shared__ uint8_t smem_raw[];
    uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
    uint8_t* tiles = smem;
    uint8_t* staging = smem + STAGES * kStageBytes;
    uint64_t* bars = reinterpret_cast<uint64_t*>(staging + kEpiWarps * kStageOut);
    // In the pair form full and acc_empty are used in the even CTA only; empty and acc_full receive its commits in both.
    uint64_t* full_bar = bars;
    uint64_t* empty_bar = bars + STAGES;
    uint64_t* acc_full = bars + 2 * STAGES;
    uint64_t* acc_empty = acc_full + 2;
    uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(acc_full + 4);
    volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);

    const int warp = __shfl_sync(0xFFFFFFFFu, static_cast<int>(threadIdx.x >> 5), 0);     // the same register in every lane
    const int lane = threadIdx.x & 31;
    const uint32_t cluster_rank = kPair ? cluster_ctarank() : 0u;
    const uint32_t rank = cluster_rank & 1u;                // 0: issues the MMAs; 1: its peer
    const uint32_t lead_rank = cluster_rank & ~1u;
    const uint16_t pair_mask = static_cast<uint16_t>(3u << lead_rank);
    const bool leader = rank == 0;
    // a worker (a CTA, a pair, or a cluster of pairs) takes tiles first, first + workers, ..
    const int ctas = kSplit ? 2 * p.split : kPair ? 2 : 1;
    const int first = p.unit0 + static_cast<int>(blockIdx.x) / ctas, workers = static_cast<int>(gridDim.x) / ctas;
    const int part = kSplit ? static_cast<int>(cluster_rank >> 1) : 0;
    const int all_blocks = p.segments * p.KB;
    const int kb0 = kSplit ? static_cast<int>(static_cast<int64_t>(all_blocks) * part / p.split) : 0;
    const int kb1 = kSplit ? static_cast<int>(static_cast<int64_t>(all_blocks) * (part + 1) / p.split) : all_blocks;

    if (threadIdx.x == 0) {
        for (int s = 0; s < STAGES; ++s) {
            mbar_init(smem_u32(&full_bar[s]), 1);
            mbar_init(smem_u32(&empty_bar[s]), 1);
        }
        for (int b = 0; b < 2; ++b) {
            mbar_init(smem_u32(&acc_full[b]), 1);
            mbar_init(smem_u32(&acc_empty[b]), (kPair ? 2 : 1) * kEpiWarps / 2);
        }
        *abort_flag = 0;
        fence_mbar_init();
        tma_prefetch_desc(&p.a[0]);
        tma_prefetch_desc(&p.b[0]);
        if (!p.direct[0]) tma_prefetch_desc(&p.out[0]);
    }
    if (warp == 1) {
        if constexpr (kPair) {
            tmem_alloc_pair(smem_u32(tmem_slot), F::kTmemCols);
            tmem_relinquish_pair();
        } else {
            tmem_alloc(smem_u32(tmem_slot), F::kTmemCols);
            tmem_relinquish();
        }
    }
    tc_fence_before();
    if constexpr (kPair)
        cluster_sync();   // both CTAs' barriers initialised and TMEM allocated before any remote access
    else
        __syncthreads();
    tc_fence_after();
    const uint32_t tmem = *tmem_slot;
    // An early launch works on other tiles than the one before it, which had itself waited: it waits at its end.
    if (!(kSplit && p.early)) grid_wait();
    grid_release();
    asm volatile("fence.proxy.async;" ::: "memory");     // what was stored plainly is loaded by TMA
    // Clears the status of earlier calls.  A wait of this launch gives up two seconds after it began, long after
    // block 0, which starts first, has passed here.
    if (p.reset && blockIdx.x == 0 && threadIdx.x == 0) *reinterpret_cast<volatile int*>(p.status) = DTP_OK;

    if (warp == 0) {
        // -------------------------------------------------------------------- producer: one lane issues
        const bool issuer = elect_one();
        const uint32_t full0 = smem_u32(full_bar), empty0 = smem_u32(empty_bar), tiles0 = smem_u32(tiles);
        const uint32_t full_lead = kPair ? mapa_shared(full0, lead_rank) : full0;
        int stage = 0;
        uint32_t phase = 0;
        bool ok = true;
        for (int u = first; ok && u < p.units; u += workers) {
            int job, tm, tn;
            decode<JOBS>(p, u, job, tm, tn);
            const int m0 = (kPair ? 2 * tm + static_cast<int>(rank) : tm) * BM;
            const int n0 = tn * kCols;
            for (int kb = kb0; kb < kb1; kb += kBoxes) {
                if (!warp_wait(empty0 + stage * 8u, phase ^ 1u, abort_flag)) { ok = false; break; }
                const int boxes = kb1 - kb < kBoxes ? kb1 - kb : kBoxes;      // the last stage may hold one block
                const uint32_t fb = full_lead + stage * 8u;
                if (issuer) {
                    if (leader) mbar_arrive_expect_tx(full0 + stage * 8u, (kPair ? 2u : 1u) * boxes * F::kBoxBytes);
#pragma unroll
                    for (int x = 0; x < kBoxes; ++x) {
                        if (x >= boxes) break;
                        const uint32_t sa = tiles0 + stage * kStageBytes + x * F::kBoxBytes, sb = sa + kTileA;
                        const int seg = kb + x >= p.KB, at = seg + job;
                        const int k0 = (kb + x - seg * p.KB) * BK;
                        auto load = [&](uint32_t dst, const CUtensorMap* map, int cx, int cy) {
                            if constexpr (kPair) tma_load_2d_pair(dst, map, fb, cx, cy);
                            else tma_load_2d(dst, map, fb, cx, cy);
                        };
                        if (p.a_mn) {
                            load(sa, &p.a[at], m0, k0);
                            load(sa + kTileA / 2, &p.a[at], m0 + 64, k0);
                        } else {
                            load(sa, &p.a[at], k0, m0);
                        }
                        // rows of B: halves of BN / 2, which are gate and up in the gated kind
#pragma unroll
                        for (int h = 0; h < F::kRowsB / (BN / 2); ++h) {
                            const int half = kPair ? static_cast<int>(rank) : h;
                            const CUtensorMap* map = KIND == kEpiGated ? &p.b[half] : &p.b[at];
                            const int r0 = KIND == kEpiGated ? n0 : n0 + half * (BN / 2);
                            const uint32_t dst = sb + h * (BN / 2) * BK * 2;
                            if (p.b_mn) {
#pragma unroll
                                for (int q = 0; q < BN / 128; ++q)       // BN >= 128 then
                                    load(dst + q * 64 * BK * 2, map, r0 + 64 * q, k0);
                            } else {
                                load(dst, map, k0, r0);
                            }
                        }
                    }
                }
                if (++stage == STAGES) { stage = 0; phase ^= 1u; }
            }
        }
    } else if (warp == 1 && leader) {
        // ------------------------------------- MMA issuer (one lane of the even CTA's warp of a pair)
        const bool issuer = elect_one();
        const uint32_t full0 = smem_u32(full_bar), empty0 = smem_u32(empty_bar);
        int stage = 0;
        uint32_t phase = 0, unit_count = 0;
        bool ok = true;
        // one step of 16 k: 32 bytes along a row of k, 16 rows of 128 bytes where the rows are contiguous
        const uint32_t step_a = p.a_mn ? (UK * 128) >> 4 : (UK * 2) >> 4;
        const uint32_t step_b = p.b_mn ? (UK * 128) >> 4 : (UK * 2) >> 4;
        const uint32_t low_a = desc_low(smem_u32(tiles), p.a_mn), low_b = desc_low(smem_u32(tiles) + kTileA, p.b_mn);
        const uint32_t idesc = p.idesc;
        auto wait = [&](uint32_t bar, uint32_t parity) {
            return kPair ? warp_wait_cluster(bar, parity, abort_flag) : warp_wait(bar, parity, abort_flag);
        };
        for (int u = first; ok && u < p.units; u += workers, ++unit_count) {
            const uint32_t buf = unit_count & 1u;
            const uint32_t use = (unit_count >> 1) & 1u;
            if (!wait(smem_u32(&acc_empty[buf]), use ^ 1u)) { ok = false; break; }
            tc_fence_after();
            const uint32_t d_acc = tmem + buf * BN;
            for (int kb = kb0; kb < kb1; kb += kBoxes) {
                if (!wait(full0 + stage * 8u, phase)) { ok = false; break; }
                tc_fence_after();
                const int boxes = kb1 - kb < kBoxes ? kb1 - kb : kBoxes;
                if (issuer) {
#pragma unroll
                    for (int x = 0; x < kBoxes; ++x) {
                        if (x >= boxes) break;
                        const uint32_t off = (stage * kStageBytes + x * F::kBoxBytes) >> 4;
#pragma unroll
                        for (int kk = 0; kk < BK / UK; ++kk) {
                            const uint32_t accumulate = (kb == kb0 && x == 0 && kk == 0) ? 0u : 1u;
                            const uint64_t da = desc(low_a + off + kk * step_a), db = desc(low_b + off + kk * step_b);
                            if constexpr (kPair) umma_bf16_pair(d_acc, da, db, idesc, accumulate);
                            else umma_bf16(d_acc, da, db, idesc, accumulate);
                        }
                    }
                    if constexpr (kPair) umma_commit_pair(empty0 + stage * 8u, pair_mask);
                    else umma_commit(empty0 + stage * 8u);
                }
                __syncwarp();
                if (++stage == STAGES) { stage = 0; phase ^= 1u; }
            }
            if (!ok) break;
            if (issuer) {
                if constexpr (kPair) umma_commit_pair(smem_u32(&acc_full[buf]), pair_mask);
                else umma_commit(smem_u32(&acc_full[buf]));
            }
            __syncwarp();
        }
    }
    if constexpr (kSplit) {
        // ------------------------------------------------- partial sums to the CTAs that finish them
        __syncwarp();
        const bool epi_warp = warp >= kEpiWarp0;
        bool ok = true;
        if (epi_warp) {
            ok = warp_wait(smem_u32(&acc_full[0]), 0, abort_flag);
            tc_fence_after();
        }
        cluster_sync();                  // every pair's MMAs are done: the stages may be written over
        constexpr int kAcc = BN / kCols;
        const int width = kCols / p.split;       // columns that a CTA finishes
        if (epi_warp && ok) {
            const int quad = warp & 3, quarter = (warp - kEpiWarp0) >> 2;
            const uint32_t lane_acc = tmem + (static_cast<uint32_t>(quad * 32) << 16);
#pragma unroll 1
            for (int c = quarter * (BN / 4); c < (quarter + 1) * (BN / 4); c += 16) {
                const int q = c / kCols, col = c % kCols, dst = col / width;
                float v[16];
                tmem_ld16(lane_acc + static_cast<uint32_t>(c), v);
                tmem_wait_ld();
                // at the destination: [pair][accumulator][group of 4 columns][row][4 columns]
                const int at = (((part * kAcc + q) * (width / 4) + col % width / 4) * BM + quad * 32 + lane) * 16;
                const uint32_t to = mapa_shared(smem_u32(tiles) + at, 2u * dst + rank);
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    st_shared_cluster_f32x4(to + i * BM * 16, v[4 * i], v[4 * i + 1], v[4 * i + 2], v[4 * i + 3]);
            }
            tc_fence_before();
        }
        cluster_sync();
    }
    if (warp >= kEpiWarp0) {
        // -------------------------------------------------------------------- epilogue
        const Epilogue& e = p.epi;
        const int quad = warp & 3;                       // TMEM lanes 32*quad ..: a row per thread
        const int half = ((warp - kEpiWarp0) >> 2) & 1;
        const int set = (warp - kEpiWarp0) >> 3;
        const uint32_t lane_base = tmem + (static_cast<uint32_t>(quad * 32) << 16);
        uint8_t* stg = staging + (warp - kEpiWarp0) * kStageOut;
        // of the tile's product
        int64_t M = p.M[0], ldo = p.ldo[0];
        int N = p.N[0], job = 0;
        const bool wide = (p.ldo[0] & 7) == 0;
        // 64 bytes of every lane's row into the staging buffer, once the store issued from it has read it
        auto stage_box = [&](const uint32_t* w) {
            if (lane == 0) bulk_wait_read0();
            __syncwarp();
            uint8_t* sb = stg + lane * 64;
#pragma unroll
            for (int c = 0; c < 4; ++c)
                *reinterpret_cast<uint4*>(sb + ((c ^ ((lane >> 1) & 3)) << 4)) =
                    make_uint4(w[4 * c], w[4 * c + 1], w[4 * c + 2], w[4 * c + 3]);
        };
        // a bulk store of the box of 32 rows, from column x
        auto store_box = [&](auto leave, const CUtensorMap* map, const uint32_t* w, int x, int row0) {
            stage_box(w);
            fence_async_smem();
            __syncwarp();
            if (lane == 0) {
                tma_store_2d<decltype(leave)::value>(map, smem_u32(stg), x, row0);
                bulk_commit();
            }
        };
        // the same where rows are not on 16-byte boundaries: element by element, the lanes along the rows
        auto store_elements = [&](auto* out, int64_t ld, const uint32_t* w, int x, int row0) {
            using V = std::remove_pointer_t<decltype(out)>;
            constexpr int kPer = 64 / sizeof(V);          // columns of a box
            stage_box(w);
            __syncwarp();
            const int c = lane % kPer;
#pragma unroll 4
            for (int r = lane / kPer; r < 32; r += 32 / kPer) {
                const int at = r * 64 + ((((c * sizeof(V)) >> 4) ^ ((r >> 1) & 3)) << 4) + ((c * sizeof(V)) & 15);
                if (row0 + r < M && x + c < N)
                    out[(static_cast<int64_t>(row0) + r) * ld + x + c] = *reinterpret_cast<const V*>(stg + at);
            }
            __syncwarp();
        };
        // 32 columns of the box's rows, from column n, into output i
        auto store32 = [&](int i, void* out, const uint32_t (&w)[16], int n, int row0) {
            if (p.direct[job]) store_elements(static_cast<__nv_bfloat16*>(out), ldo, w, n, row0);
            else store_box(std::false_type(), &p.out[i], w, n, row0);
        };
        uint32_t unit_count = static_cast<uint32_t>(set);
        for (int u = first + set * workers; u < p.units; u += 2 * workers, unit_count += 2) {
            int tm, tn;
            decode<JOBS>(p, u, job, tm, tn);
            if constexpr (JOBS > 1) M = p.M[job], N = p.N[job], ldo = p.ldo[job];
            const int row0 = (kPair ? 2 * tm + static_cast<int>(rank) : tm) * BM + quad * 32;
            const int64_t m = static_cast<int64_t>(row0) + lane;
            const uint32_t buf = unit_count & 1u;
            const int width = kSplit ? kCols / p.split : kCols;          // this CTA's columns of the tile, 32 at a time
            const int base = tn * kCols + (kSplit ? part * width : 0);
            // A box's residual (four lanes to a row's 64 bytes, eight rows at a time) and bias (a pair of columns in each
            // of 16 lanes) are loaded one box ahead, the first before the accumulator is waited for.
            uint4 rq[4];
            uint32_t bq = 0;
            auto fetch = [&](int c) {
                const int n = base + c;
                if (c >= width || n >= N || row0 >= M) return;
                if (e.bias) {
                    const __nv_bfloat16* b = reinterpret_cast<const __nv_bfloat16*>(e.bias) + n + 2 * (lane & 15);
                    const int left = N - n - 2 * (lane & 15);
                    bq = left >= 2 ? *reinterpret_cast<const uint32_t*>(b)
                                   : left == 1 ? *reinterpret_cast<const uint16_t*>(b) : 0u;
                }
                if (e.residual && wide) {
                    const int col = n + 8 * (lane & 3);
                    const __nv_bfloat16* r = reinterpret_cast<const __nv_bfloat16*>(e.residual) + col;
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const int64_t row = static_cast<int64_t>(row0) + (lane >> 2) + 8 * i;
                        rq[i] = row < M && col < N ? *reinterpret_cast<const uint4*>(r + row * ldo)
                                                       : make_uint4(0, 0, 0, 0);
                    }
                }
            };
            if constexpr (KIND == kEpiLinear) fetch(32 * half);
            if constexpr (!kSplit) {
                const uint32_t use = (unit_count >> 1) & 1u;
                if (!warp_wait(smem_u32(&acc_full[buf]), use, abort_flag)) break;
                tc_fence_after();
            }
            const uint32_t acc = lane_base + buf * BN;
            // 16 columns from column col of accumulator q
            auto get16 = [&](int q, int col, float* v) {
                if constexpr (kSplit) {
                    constexpr int kAcc = BN / kCols;
#pragma unroll
                    for (int i = 0; i < 16; ++i) v[i] = 0.0f;
                    for (int s = 0; s < p.split; ++s) {
                        const uint8_t* from =
                            tiles + (((s * kAcc + q) * (width / 4) + col / 4) * BM + quad * 32 + lane) * 16;
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            const float4 w = *reinterpret_cast<const float4*>(from + i * BM * 16);
                            v[4 * i] += w.x, v[4 * i + 1] += w.y, v[4 * i + 2] += w.z, v[4 * i + 3] += w.w;
                        }
                    }
                } else {
                    tmem_ld16(acc + static_cast<uint32_t>(q * (BN / 2) + col), v);
                }
            };
            auto got = [&] {
                if constexpr (!kSplit) tmem_wait_ld();
            };
#pragma unroll 1
            for (int c = 32 * half; c < width; c += 64) {
                const int n = base + c;
                if (n >= N || row0 >= M) continue;     // box entirely outside (warp-uniform)
                uint32_t w[16];
                if constexpr (KIND == kEpiLinear) {
                    float v[32];
                    get16(0, c, v);
                    get16(0, c + 16, v + 16);
                    got();
                    if (e.bias) {
#pragma unroll
                        for (int i = 0; i < 16; ++i) {
                            float lo, hi;
                            unpack_bf16(__shfl_sync(0xFFFFFFFFu, bq, i), lo, hi);
                            v[2 * i] += lo;
                            v[2 * i + 1] += hi;
                        }
                    }
                    if (e.Z) {
#pragma unroll
                        for (int q = 0; q < 2; ++q) {
                            if (n + 16 * q < N) {
#pragma unroll
                                for (int i = 0; i < 16; ++i) w[i] = __float_as_uint(v[16 * q + i]);
                                if (p.direct_z) store_elements(e.Z, static_cast<int64_t>(N), w, n + 16 * q, row0);
                                else store_box(std::true_type(), &p.z, w, n + 16 * q, row0);
                            }
                        }
                    }
                    act_values<true>(e.act, v);
                    if (e.residual && wide) {
                        // from the rows' quarters to the lane's row, through the staging buffer
                        if (lane == 0) bulk_wait_read0();
                        __syncwarp();
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            const int r = (lane >> 2) + 8 * i;
                            *reinterpret_cast<uint4*>(stg + r * 64 + (((lane & 3) ^ ((r >> 1) & 3)) << 4)) = rq[i];
                        }
                        __syncwarp();
#pragma unroll
                        for (int q = 0; q < 4; ++q) {
                            const uint4 x = *reinterpret_cast<const uint4*>(stg + lane * 64 + ((q ^ ((lane >> 1) & 3)) << 4));
                            const uint32_t words[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
                            for (int i = 0; i < 4; ++i) {
                                float lo, hi;
                                unpack_bf16(words[i], lo, hi);
                                v[8 * q + 2 * i] += lo;
                                v[8 * q + 2 * i + 1] += hi;
                            }
                        }
                        __syncwarp();
                    } else if (e.residual && m < M) {
                        const __nv_bfloat16* r = reinterpret_cast<const __nv_bfloat16*>(e.residual) + m * ldo;
#pragma unroll
                        for (int i = 0; i < 32; ++i)
                            if (n + i < N) v[i] += to_f32(r[n + i]);
                    }
                    fetch(c + 64);
#pragma unroll
                    for (int i = 0; i < 16; ++i) w[i] = pack_bf16(v[2 * i], v[2 * i + 1]);
                    store32(job, p.dst[job], w, n, row0);
                } else if constexpr (KIND == kEpiGated) {
                    float* pre = e.pre ? e.pre + pre_index(m, n, N) : nullptr;
#pragma unroll
                    for (int q = 0; q < 2; ++q) {
                        float g[16], v[16];
                        get16(0, c + 16 * q, g);
                        get16(1, c + 16 * q, v);
                        got();
                        if (pre) {       // whole tiles: rows and columns beyond the edges have their place
#pragma unroll
                            for (int i = 0; i < 4; ++i) {
                                float* to = pre + (4 * q + i) * kPreTile * 4;
                                __stcs(reinterpret_cast<float4*>(to),
                                       make_float4(g[4 * i], g[4 * i + 1], g[4 * i + 2], g[4 * i + 3]));
                                __stcs(reinterpret_cast<float4*>(to + kPreTile * kPreTile),
                                       make_float4(v[4 * i], v[4 * i + 1], v[4 * i + 2], v[4 * i + 3]));
                            }
                        }
                        act_values<true>(e.act, g);
#pragma unroll
                        for (int i = 0; i < 8; ++i)
                            w[8 * q + i] = pack_bf16(g[2 * i] * v[2 * i], g[2 * i + 1] * v[2 * i + 1]);
                    }
                    store32(job, p.dst[job], w, n, row0);
                } else {
                    // 16 columns at a time with all their saved values in flight: 144 us for 1024 x 3072 on 16384 tokens (four
                    // columns at a time 192 us, the loads' latency 32 times a tile).  dG goes to the staging buffer as it
                    // is computed, dU waits in registers.  Both have rows on 16-byte boundaries.
                    const float* pre = e.pre + pre_index(m, n, N);
                    uint32_t w2[16];
                    if (lane == 0) bulk_wait_read0();
                    __syncwarp();
#pragma unroll
                    for (int q = 0; q < 2; ++q) {
                        float4 g[4], v[4];
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            const float* from = pre + (4 * q + i) * kPreTile * 4;
                            g[i] = __ldcs(reinterpret_cast<const float4*>(from));
                            v[i] = __ldcs(reinterpret_cast<const float4*>(from + kPreTile * kPreTile));
                        }
                        float dh[16];
                        get16(0, c + 16 * q, dh);
                        got();
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            float value[4] = {g[i].x, g[i].y, g[i].z, g[i].w}, slope[4];
                            act_both4<true>(e.act, value, slope);
                            const float* d = dh + 4 * i;
                            w[2 * i] = pack_bf16(d[0] * v[i].x * slope[0], d[1] * v[i].y * slope[1]);
                            w[2 * i + 1] = pack_bf16(d[2] * v[i].z * slope[2], d[3] * v[i].w * slope[3]);
                            w2[8 * q + 2 * i] = pack_bf16(d[0] * value[0], d[1] * value[1]);
                            w2[8 * q + 2 * i + 1] = pack_bf16(d[2] * value[2], d[3] * value[3]);
                        }
#pragma unroll
                        for (int h = 0; h < 2; ++h)
                            *reinterpret_cast<uint4*>(stg + lane * 64 + (((2 * q + h) ^ ((lane >> 1) & 3)) << 4)) =
                                make_uint4(w[4 * h], w[4 * h + 1], w[4 * h + 2], w[4 * h + 3]);
                    }
                    fence_async_smem();
                    __syncwarp();
                    if (lane == 0) {
                        tma_store_2d<false>(&p.out[0], smem_u32(stg), n, row0);
                        bulk_commit();
                    }
                    store_box(std::false_type(), &p.out[1], w2, n, row0);
                }
            }
            if constexpr (!kSplit) {
                // its TMEM loads have completed (tcgen05.wait::ld): hand the buffer back without release ordering,
                // which would also wait for the warp's stores
                tc_fence_before();
                __syncwarp();
                if (lane == 0) {
                    if constexpr (kPair)
                        mbar_arrive_cluster_relaxed(mapa_shared(smem_u32(&acc_empty[buf]), lead_rank));
                    else
                        mbar_arrive_relaxed(smem_u32(&acc_empty[buf]));
                }
            }
        }
        if (lane == 0) bulk_wait_read0();      // the staging buffers may go; the writes end with the launch
        __syncwarp();
    }
    // a launch that began before the one ahead of it on the stream had ended does not end before it
    if (kSplit && p.early && threadIdx.x == 0) grid_wait();

    tc_fence_before();
    __syncthreads();
    // Every accumulator has been waited for, so every MMA and every load has completed.  After a wait gave up they may not
    // have: loads already issued may still be landing in this CTA's or the peer's shared memory; let them finish.
    if (threadIdx.x == 0 && *abort_flag) {
        const uint64_t t0 = globaltimer_ns();
        while (globaltimer_ns() - t0 < 200ull * 1000ull) {
        }
    }
    // the peer's arrivals on this CTA's barriers have landed before either leaves
    if constexpr (kPair) cluster_sync();
    else __syncthreads();
    if (warp == 1) {
        tc_fence_after();
        if constexpr (kPair)
            tmem_dealloc_pair(tmem, F::kTmemCols);
        else
            tmem_dealloc(tmem, F::kTmemCols);
    }
    if (threadIdx.x == 0 && *abort_flag) atomicExch(p.status, static_cast<int>(DTP_ERR_NOT_CONVERGED));
}

// ------------------------------------------------------------------------------------ host

static bool map_2d(CUtensorMap* m, const void* base, int64_t inner, int64_t outer, int64_t pitch, int box_x, int box_y,
                   CUtensorMapSwizzle swz, bool f32 = false) {
    auto enc = tensor_map_encoder();
    if (!enc) return false;
    cuuint64_t dims[2] = {static_cast<cuuint64_t>(inner), static_cast<cuuint64_t>(outer)};
    cuuint64_t strides[1] = {static_cast<cuuint64_t>(pitch) * (f32 ? 4 : 2)};
    cuuint32_t box[2] = {static_cast<cuuint32_t>(box_x), static_cast<cuuint32_t>(box_y)};
    cuuint32_t estr[2] = {1, 1};
    return enc(m, f32 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT32 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, const_cast<void*>(base),
               dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE, swz, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
               CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// rows x K operand: tiles of `box_rows` rows x 64 k, or where the rows are contiguous 64 rows x 64 k.
static bool map_operand(CUtensorMap* m, const Mat& a, int64_t rows, int64_t K, int box_rows) {
    if (a.ks == 1) return map_2d(m, a.p, K, rows, a.rs, BK, box_rows, CU_TENSOR_MAP_SWIZZLE_128B);
    return map_2d(m, a.p, rows, K, a.ks, 64, BK, CU_TENSOR_MAP_SWIZZLE_128B);
}

// Tiles unit0 .. unit0 + count - 1 of the product (count < 0: all the others), on at most `most` workers; `split`: pairs per
// tile; `early`: see Args.
template <bool kPair, int BN, bool kSplit>
static int launch_form(const Product& p, int* status, int reset, int split, int early, int64_t unit0, int64_t count,
                       int64_t most, cudaStream_t stream) {
    using F = Form<kPair, BN>;
    const bool gated = p.epi.kind == kEpiGated;
    const int rows = kPair ? 2 * BM : BM, cols = gated ? BN / 2 : BN;
    Args a;
    for (int s = 0; s < 2; ++s) {            // only the maps that the kernel reads: an encoding is host time
        if (s < p.segments && !map_operand(&a.a[s], p.A[s], p.M, p.K, BM)) return DTP_ERR_CUDA;
        if ((s < p.segments || gated) && !map_operand(&a.b[s], p.B[s], p.N, p.K, BN / 2)) return DTP_ERR_CUDA;
    }
    int64_t all = 0;
    for (int j = 0; j < kBatch; ++j) {
        a.last[j] = 0x7FFFFFFF;
        if (j >= p.batch) continue;
        const Also& x = p.also[j > 0 ? j - 1 : 0];
        if (j > 0 && (!map_operand(&a.a[j], x.A, x.M, p.K, BM) || !map_operand(&a.b[j], x.B, x.N, p.K, BN / 2)))
            return DTP_ERR_CUDA;
        a.M[j] = j > 0 ? x.M : p.M;
        a.N[j] = j > 0 ? x.N : p.N;
        a.ldo[j] = j > 0 ? x.ldo : p.epi.ldo;
        a.dst[j] = j > 0 ? x.out : p.epi.out;
        a.direct[j] = (a.ldo[j] & 7) != 0;
        if (!a.direct[j] && !map_2d(&a.out[j], a.dst[j], a.N[j], a.M[j], a.ldo[j], 32, 32, CU_TENSOR_MAP_SWIZZLE_64B))
            return DTP_ERR_CUDA;
        a.tiles_m[j] = static_cast<int>((a.M[j] + rows - 1) / rows);
        a.tiles_n[j] = (a.N[j] + cols - 1) / cols;
        all += static_cast<int64_t>(a.tiles_m[j]) * a.tiles_n[j];
        if (all > 0x3FFFFFFF) return DTP_ERR_UNSUPPORTED;
        if (j + 1 < p.batch) a.last[j] = static_cast<int>(all);
    }
    if (p.epi.out2 && !a.direct[0] &&
        !map_2d(&a.out[1], p.epi.out2, p.N, p.M, p.epi.ldo, 32, 32, CU_TENSOR_MAP_SWIZZLE_64B))
        return DTP_ERR_CUDA;
    a.direct_z = (p.N & 3) != 0;
    if (p.epi.Z && !a.direct_z && !map_2d(&a.z, p.epi.Z, p.N, p.M, p.N, 16, 32, CU_TENSOR_MAP_SWIZZLE_64B, true))
        return DTP_ERR_CUDA;
    a.segments = p.segments;
    a.KB = static_cast<int>((p.K + BK - 1) / BK);
    a.a_mn = p.A[0].ks != 1;
    a.b_mn = p.B[0].ks != 1;
    a.unit0 = static_cast<int>(unit0);
    a.units = static_cast<int>(count < 0 ? all : unit0 + count);
    a.split = split;
    a.early = early;
    // bits 15 and 16: A and B stored with their rows contiguous
    a.idesc = idesc_bf16_f32(kPair ? 2 * BM : BM, BN) | (a.a_mn ? 1u << 15 : 0u) | (a.b_mn ? 1u << 16 : 0u);
    a.reset = reset;
    a.status = status;
    a.epi = p.epi;
    auto kernel = gated ? gemm_tc_kernel<kPair, BN, kEpiGated, kSplit, 1> : gemm_tc_kernel<kPair, BN, kEpiLinear, kSplit, 1>;
    if constexpr (BN >= 128)
        if (p.epi.kind == kEpiGatedGrad) kernel = gemm_tc_kernel<kPair, BN, kEpiGatedGrad, kSplit, 1>;
    if constexpr (kPair && BN >= 128)
        if (p.batch > 1) kernel = gemm_tc_kernel<kPair, BN, kEpiLinear, kSplit, kBatch>;
    DTP_CUDA_TRY(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                      static_cast<int>(F::kSmemBytes)));
    const int64_t per = kSplit ? 2 * split : kPair ? 2 : 1;
    const int64_t units = a.units - unit0;
    cudaLaunchConfig_t cfg = {};
    // a split tile's cluster takes that tile alone
    cfg.gridDim = dim3(static_cast<unsigned>(per * (kSplit || units < most ? units : most)));
    cfg.blockDim = dim3(kThreads);
    cfg.dynamicSmemBytes = F::kSmemBytes;
    cfg.stream = stream;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = static_cast<unsigned>(per);
    attr[0].val.clusterDim.y = 1;
    attr[0].val.clusterDim.z = 1;
    attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[1].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 2;
    DTP_CUDA_TRY(cudaLaunchKernelEx(&cfg, kernel, a));
    return DTP_OK;
}

// Clusters of `split` pairs that the current device holds at once (they stay within a part of the chip).
static int cluster_room(int split, int sms) {
    static std::atomic<int> cached[2][16];
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || dev < 0) return 0;
    std::atomic<int>* slot = dev < 16 ? &cached[split == 4][dev] : nullptr;
    int n = slot ? slot->load(std::memory_order_relaxed) : 0;
    if (n) return n - 1;
    using F = Form<true, 256>;
    auto kernel = gemm_tc_kernel<true, 256, kEpiLinear, true, 1>;
    if (cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(F::kSmemBytes)) !=
        cudaSuccess)
        return 0;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(static_cast<unsigned>(sms / (2 * split) * 2 * split));
    cfg.blockDim = dim3(kThreads);
    cfg.dynamicSmemBytes = F::kSmemBytes;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = static_cast<unsigned>(2 * split);
    attr[0].val.clusterDim.y = 1;
    attr[0].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    if (cudaOccupancyMaxActiveClusters(&n, kernel, &cfg) != cudaSuccess) n = 0;
    if (slot) slot->store(n + 1, std::memory_order_relaxed);
    return n;
}

// bf16 operands whose rows are on 16-byte boundaries; M, N >= 1, K >= 1.
//
// The form is the one with the smallest estimate, in clocks, from what the forms measured on a GB300: a launch's start, pipeline
// fill and last epilogue (9000 for 256 x 256 pairs, 7000 for 256 x 128 and for single 128 x 128 tiles, which up to 128 rows may
// take, 5500 for 256 x 64, where B has k contiguous); per round of tiles and k block what the form's shared-memory traffic
// takes (515, 400, 500, 280), but no less than an epilogue; and for splitting a tile the exchange (8000 with 256 columns, 5000
// with 128).  Tiles left over after the full rounds of 256 x 256 pairs may be split in a launch of their own, which begins as
// the first one's SMs fall free (saving 4000).
int launch(const Product& p, int* status, int reset, cudaStream_t stream) {
    int dev = 0, sms = 0;
    DTP_CUDA_TRY(cudaGetDevice(&dev));
    DTP_CUDA_TRY(cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev));
    const int64_t pairs = sms / 2;
    const int64_t kb = (p.K + BK - 1) / BK * p.segments;
    const bool gated = p.epi.kind == kEpiGated;
    auto tiles = [&](int rows, int bn) {
        const int cols = gated ? bn / 2 : bn;
        int64_t n = (p.M + rows - 1) / rows * ((p.N + cols - 1) / cols);
        for (int j = 0; j + 1 < p.batch; ++j)
            n += (p.also[j].M + rows - 1) / rows * ((p.also[j].N + cols - 1) / cols);
        return n;
    };
    auto whole = [&](int64_t n, int64_t workers, int clocks, int fixed) {
        const int64_t round = kb * clocks > fixed / 3 ? kb * clocks : fixed / 3;
        return (n + workers - 1) / workers * round + fixed;
    };
    auto split_ok = [&](int64_t n, int bn, int split) {
        return kb >= 4 * split && (gated ? bn / 2 : bn) / split >= 32 && n <= cluster_room(split, sms);
    };
    auto split_clocks = [&](int bn, int split) {
        return (kb + split - 1) / split * (bn == 256 ? 515 : 400) + (bn == 256 ? 9000 + 8000 : 7000 + 5000);
    };
    const int64_t n256 = tiles(2 * BM, 256);
    int64_t best = whole(n256, pairs, 515, 9000), tail = 0;
    int best_bn = 256, best_split = 1;
    auto take = [&](int64_t estimate, int bn, int split, int64_t left) {
        if (estimate < best) best = estimate, best_bn = bn, best_split = split, tail = left;
    };
    take(whole(tiles(2 * BM, 128), pairs, 400, 7000), 128, 1, 0);
    if (p.B[0].ks == 1 && p.epi.kind != kEpiGatedGrad) take(whole(tiles(2 * BM, 64), pairs, 280, 5500), 64, 1, 0);
    if (p.M <= BM && p.batch == 1) take(whole(tiles(BM, 128), sms, 500, 7000), 0, 1, 0);
    const int64_t left = n256 % pairs;
    for (int split : {2, 4}) {
        for (int bn : {256, 128})
            if (split_ok(tiles(2 * BM, bn), bn, split)) take(split_clocks(bn, split), bn, split, 0);
        if (n256 > pairs && left > 0 && split_ok(left, 256, split))
            take(whole(n256 - left, pairs, 515, 9000) + split_clocks(256, split) - 4000, 256, split, left);
    }
    if (tail) {
        const int st = launch_form<true, 256, false>(p, status, reset, 1, 0, 0, n256 - tail, pairs, stream);
        if (st != DTP_OK) return st;
        return launch_form<true, 256, true>(p, status, 0, best_split, 1, n256 - tail, -1, pairs, stream);
    }
    if (best_bn == 0) return launch_form<false, 128, false>(p, status, reset, 1, 0, 0, -1, sms, stream);
    if (best_bn == 64) return launch_form<true, 64, false>(p, status, reset, 1, 0, 0, -1, pairs, stream);
    if (best_bn == 128)
        return best_split == 1 ? launch_form<true, 128, false>(p, status, reset, 1, 0, 0, -1, pairs, stream)
                               : launch_form<true, 128, true>(p, status, reset, best_split, 0, 0, -1, pairs, stream);
    return best_split == 1 ? launch_form<true, 256, false>(p, status, reset, 1, 0, 0, -1, pairs, stream)
                           : launch_form<true, 256, true>(p, status, reset, best_split, 0, 0, -1, pairs, stream);
}

}  // namespace gtc
}  // namespace dtp
