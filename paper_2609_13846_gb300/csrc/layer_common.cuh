// layer_common.cuh -- what the kernels of the layer operators (linear layer, gated feed-forward block)
// share: the activations with their derivatives, the epilogues of the matrix products, and the layout of the
// saved gate and up pre-activations.
#pragma once

#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include "dtp.h"
#include "dtp_common.cuh"

namespace dtp {
namespace layer {

// act(z).  kFast: the exponential of the special-function unit (relative error about 2^-21, far below a
// bf16 output's rounding of 2^-9); else the library's expf, for fp32 outputs.
template <bool kFast>
__device__ __forceinline__ float sigmoid(float z) {
    if constexpr (kFast) return __fdividef(1.0f, 1.0f + __expf(-z));
    else return 1.0f / (1.0f + expf(-z));
}

// Phi(z) and e^(-z^2/2).  kFast: erf by Abramowitz and Stegun 7.1.26 (absolute error 1.5e-7), whose exponential is the one
// of the density; the small side is computed and not subtracted from 1.
template <bool kFast>
__device__ __forceinline__ float normal_cdf(float z, float& bell) {
    if constexpr (kFast) {
        bell = __expf(-0.5f * z * z);
        const float t = __fdividef(1.0f, fmaf(0.3275911f * 0.70710678f, fabsf(z), 1.0f));
        float p = fmaf(1.061405429f, t, -1.453152027f);
        p = fmaf(p, t, 1.421413741f);
        p = fmaf(p, t, -0.284496736f);
        p = fmaf(p, t, 0.254829592f);
        const float q = 0.5f * p * t * bell;
        return z < 0.0f ? q : 1.0f - q;
    } else {
        bell = expf(-0.5f * z * z);
        return 0.5f * (1.0f + erff(z * 0.70710678118654752f));
    }
}

template <bool kFast>
__device__ __forceinline__ float act_value(int act, float z) {
    switch (act) {
        case DTP_ACT_SILU: return z * sigmoid<kFast>(z);
        case DTP_ACT_GELU: {
            float bell;
            return z * normal_cdf<kFast>(z, bell);
        }
        case DTP_ACT_RELU: return z <= 0.0f ? 0.0f : z;       // a NaN stays a NaN
        default: return z;
    }
}

// act(z) and act'(z).  silu' = s (1 + z (1 - s)); gelu' = Phi(z) + z phi(z); relu' = [z > 0].
template <bool kFast>
__device__ __forceinline__ void act_both(int act, float z, float& value, float& slope) {
    switch (act) {
        case DTP_ACT_SILU: {
            const float s = sigmoid<kFast>(z);
            slope = s * fmaf(z, 1.0f - s, 1.0f);
            value = z * s;
            return;
        }
        case DTP_ACT_GELU: {
            float bell;
            const float cdf = normal_cdf<kFast>(z, bell);
            slope = fmaf(z * 0.39894228040143268f, bell, cdf);
            value = z * cdf;
            return;
        }
        case DTP_ACT_RELU:
            value = z <= 0.0f ? 0.0f : z;
            slope = z > 0.0f ? 1.0f : 0.0f;
            return;
        default:
            value = z;
            slope = 1.0f;
    }
}

// act over an array in place: one switch for all of it.
template <bool kFast, int N>
__device__ __forceinline__ void act_values(int act, float (&v)[N]) {
    if (act == DTP_ACT_SILU) {
#pragma unroll
        for (int i = 0; i < N; ++i) v[i] = act_value<kFast>(DTP_ACT_SILU, v[i]);
    } else if (act == DTP_ACT_GELU) {
#pragma unroll
        for (int i = 0; i < N; ++i) v[i] = act_value<kFast>(DTP_ACT_GELU, v[i]);
    } else if (act == DTP_ACT_RELU) {
#pragma unroll
        for (int i = 0; i < N; ++i) v[i] = act_value<kFast>(DTP_ACT_RELU, v[i]);
    }
}
// act and act' of four values, the values in place.
template <bool kFast>
__device__ __forceinline__ void act_both4(int act, float (&v)[4], float (&slope)[4]) {
    if (act == DTP_ACT_SILU) {
#pragma unroll
        for (int i = 0; i < 4; ++i) act_both<kFast>(DTP_ACT_SILU, v[i], v[i], slope[i]);
    } else if (act == DTP_ACT_GELU) {
#pragma unroll
        for (int i = 0; i < 4; ++i) act_both<kFast>(DTP_ACT_GELU, v[i], v[i], slope[i]);
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) act_both<kFast>(act, v[i], v[i], slope[i]);
    }
}

// The layer kernels are launched so that a kernel's set-up overlaps the end of the one before it on the stream.  Each waits
// for that one (grid_wait) before it touches global memory, and only then lets the next one begin (grid_release): what
// begins early may rely on everything before its predecessor.  Memory may thus change while a kernel lives: these kernels
// take no __restrict__ pointers and read nothing through the read-only path (__ldg), whose loads need not stay behind the wait.
__device__ __forceinline__ void grid_wait() { asm volatile("griddepcontrol.wait;" ::: "memory"); }
__device__ __forceinline__ void grid_release() { asm volatile("griddepcontrol.launch_dependents;" ::: "memory"); }

// Shared-memory matrix descriptors (128-byte swizzle, version 1) as two words: the high word is the stride byte offset (1024
// >> 4) and the layout, the same for both orders.  With k contiguous a tile is rows of 64 k, 8-row groups 1024 bytes apart.
// With the rows contiguous it is 64-row blocks of [k][64 rows], 128 bytes per k: the stride byte offset leads from one group of
// 8 k to the next, the leading byte offset (64 k x 128 bytes) from one 64-row block to the next.
constexpr uint32_t kDescHigh = (1024u >> 4) | (1u << 14) | (2u << 29);
__device__ __forceinline__ uint32_t desc_low(uint32_t saddr, bool rows_contiguous) {
    return ((saddr & 0x3FFFFu) >> 4) | ((rows_contiguous ? (64u * 128u) >> 4 : 1u) << 16);
}
__device__ __forceinline__ uint64_t desc(uint32_t low) {
    uint64_t d;
    asm("mov.b64 %0, {%1, %2};" : "=l"(d) : "r"(low), "r"(kDescHigh));
    return d;
}

// A whole warp's bounded wait, with one outcome for all lanes: where some saw the phase complete and others the abort flag,
// all give up, so that none waits for the others at a warp barrier.
__device__ __forceinline__ bool warp_wait(uint32_t bar, uint32_t parity, volatile int* abort) {
    return __all_sync(0xFFFFFFFFu, mbar_wait(bar, parity, abort)) != 0;
}
__device__ __forceinline__ bool warp_wait_cluster(uint32_t bar, uint32_t parity, volatile int* abort) {
    return __all_sync(0xFFFFFFFFu, mbar_wait_cluster(bar, parity, abort)) != 0;
}

// One lane of the warp, the same every time.
__device__ __forceinline__ bool elect_one() {
    uint32_t p;
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "elect.sync _|p, 0xFFFFFFFF;\n\t"
        "selp.u32 %0, 1, 0, p;\n\t}\n"
        : "=r"(p));
    return p != 0;
}

// Element types of the operands.
template <typename E>
__device__ __forceinline__ float to_f32(E v) { return static_cast<float>(v); }
template <typename E>
__device__ __forceinline__ E from_f32(float v);
template <>
__device__ __forceinline__ float from_f32<float>(float v) { return v; }
template <>
__device__ __forceinline__ __nv_bfloat16 from_f32<__nv_bfloat16>(float v) { return __float2bfloat16_rn(v); }

template <typename E>
struct IsFast { static constexpr bool value = false; };
template <>
struct IsFast<__nv_bfloat16> { static constexpr bool value = true; };

// The saved gate and up pre-activations, fp32 (rounding them to bf16 would add 1.7e-3 of relative error to dG
// and dU, as much as the rounding that the tensor cores ask for), in tiles of 128 tokens x 128 neurons: per
// tile 128 x 128 gate values, then the up values, each as [group of 4 neurons][token][4 neurons], so that the
// 32 lanes of a warp, which hold 32 tokens, read and write 512 consecutive bytes.
constexpr int kPreTile = 128;
__host__ __device__ inline int64_t pre_tiles(int64_t n) { return (n + kPreTile - 1) / kPreTile; }
__host__ __device__ inline int64_t pre_floats(int64_t T, int64_t N) {
    return pre_tiles(T) * pre_tiles(N) * 2 * kPreTile * kPreTile;
}
// of the gate value of (t, n); its up value is kPreTile * kPreTile floats further on
__host__ __device__ inline int64_t pre_index(int64_t t, int64_t n, int64_t N) {
    const int64_t tile = (t / kPreTile) * pre_tiles(N) + n / kPreTile;
    const int64_t in = ((n % kPreTile) / 4 * kPreTile + t % kPreTile) * 4 + n % 4;
    return tile * 2 * kPreTile * kPreTile + in;
}

// What happens to a product's accumulators.
enum EpiKind {
    kEpiLinear = 0,     // out = act(acc + bias) + residual; Z = acc + bias
    kEpiGated = 1,      // out = act(acc0) acc1; pre = (acc0, acc1)
    kEpiGatedGrad = 2   // acc = dH: out = dG = dH U act'(G), out2 = dU = dH act(G)
};

struct Epilogue {
    int kind = kEpiLinear;
    int act = DTP_ACT_NONE;
    const void* bias = nullptr;       // [N]
    const void* residual = nullptr;   // [M, ldo]
    void* out = nullptr;              // [M, ldo]
    void* out2 = nullptr;
    int64_t ldo = 0;
    float* Z = nullptr;               // [M, N]
    float* pre = nullptr;
    int64_t M = 0;
    int N = 0;
};

// One element (m, n); a1 is the second accumulator of kEpiGated.
template <typename E, int KIND>
__device__ __forceinline__ void epilogue_element(const Epilogue& e, int64_t m, int n, float a0, float a1) {
    constexpr bool kFast = IsFast<E>::value;
    E* out = reinterpret_cast<E*>(e.out);
    const int64_t at = m * e.ldo + n;
    if constexpr (KIND == kEpiLinear) {
        float z = a0;
        if (e.bias) z += to_f32(reinterpret_cast<const E*>(e.bias)[n]);
        if (e.Z) e.Z[m * e.N + n] = z;
        float y = act_value<kFast>(e.act, z);
        if (e.residual) y += to_f32(reinterpret_cast<const E*>(e.residual)[at]);
        out[at] = from_f32<E>(y);
    } else if constexpr (KIND == kEpiGated) {
        if (e.pre) {
            const int64_t i = pre_index(m, n, e.N);
            e.pre[i] = a0;
            e.pre[i + kPreTile * kPreTile] = a1;
        }
        out[at] = from_f32<E>(act_value<kFast>(e.act, a0) * a1);
    } else {
        const int64_t i = pre_index(m, n, e.N);
        const float g = e.pre[i], u = e.pre[i + kPreTile * kPreTile];
        float v, s;
        act_both<kFast>(e.act, g, v, s);
        out[at] = from_f32<E>(a0 * u * s);
        reinterpret_cast<E*>(e.out2)[at] = from_f32<E>(a0 * v);
    }
}

// A matrix of a product: element (row, k) at p[row * rs + k * ks]; rs or ks is 1.
struct Mat {
    const void* p = nullptr;
    int64_t rs = 0, ks = 0;
};

// sum over the segments s of A_s [M, K] B_s [N, K]^T, then the epilogue.  kEpiGated: one segment, whose
// second accumulator takes B[1].
// `also`: up to two more products of the same K and operand orders, without an epilogue, for the same launch (bf16 only).
struct Also {
    Mat A, B;
    int64_t M = 0;
    int N = 0;
    void* out = nullptr;
    int64_t ldo = 0;
};
struct Product {
    int segments = 1;
    int batch = 1;
    Also also[2];
    Mat A[2], B[2];
    int64_t M = 0;
    int N = 0;
    int64_t K = 0;
    Epilogue epi;
};

}  // namespace layer
}  // namespace dtp
