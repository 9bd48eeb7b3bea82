// adamw.cu -- one AdamW step over many tensors:
//
//     g = c grad,  c = min(1, max_norm / norm)
//     m = b1 m + (1 - b1) g,   v = b2 v + (1 - b2) g^2
//     p = (1 - lr decay) p - lr / (1 - b1^t) m / (sqrt(v) / sqrt(1 - b2^t) + eps)
//
// Bound by memory: every value is read and written once.  A first launch of one thread takes the step's factors from the counter, the
// norm and the rate, which live on the device, and counts the step; the second, which begins while the first runs, updates the
// tensors.  These are cut into chunks of whole blocks of 256 elements, and each CTA takes a run of chunks, whatever the
// tensors' sizes; a warp takes a block at a time, 8 elements a lane.  The table of the tensors is a kernel argument; more of
// them than it holds take a launch per table.
//
// In 8 bits a block of 256 elements has a scale, and each moment is held as e4m3 times it, the second one as its root, so that
// both have the range of the gradients.  A moment changes by a small part of itself in a step (0.1% with b2 = 0.999, where
// e4m3 steps by 6 to 12%): rounded to the nearest value it would never move.  So it is rounded up with the probability of the
// fraction of the step that it has gone, by a hash of the element's index and the step's number, and is right on
// average.  Parameters in bf16, whose updates are as small, are rounded alike.  What the states will be is
// computed without contracted operations, so that the same inputs give the same codes wherever they are computed in fp32.
#include <cuda_bf16.h>
#include <cuda_fp8.h>
#include <cuda_runtime.h>
#include <math.h>
#include <stdint.h>

#include "dtp_common.cuh"
#include "layer_common.cuh"

namespace dtp {
namespace adamw {

using layer::grid_release;
using layer::grid_wait;

constexpr int kThreads = 256;
constexpr int kWarps = kThreads / 32;
constexpr int kBlock = 256;                       // elements of a scale, and of a warp's step
constexpr int64_t kMinChunk = kBlock * kWarps;    // elements
constexpr int64_t kManyChunks = 1 << 24;
constexpr int kBlocksPerSm = 3;
constexpr float kLeast = 7.888609e-31f;           // 2^-100: blocks below it are held as zeros

// What a step has in common, written by the first launch.
struct Factors {
    float clip, down;          // the gradients' factor is clip down down
    float b1, not_b1, b2, not_b2;
    float keep, size, root, eps;
    uint32_t key;
    int skip;
};

struct Flags { uint8_t p_f32, g_f32, aligned; };

template <int CAP>
struct Table {
    void* p[CAP];
    const void* g[CAP];
    void* m[CAP];
    void* v[CAP];
    float* ms[CAP];
    float* vs[CAP];
    __nv_bfloat16* copy[CAP];
    int64_t numel[CAP];
    int first[CAP + 1];                // first chunk of the tensor
    Flags flags[CAP];
    int count;
    int chunks;
    int64_t chunk;                     // elements
    const Factors* factors;
};
constexpr int kSmallTable = 64, kLargeTable = 440;
static_assert(sizeof(Table<kLargeTable>) <= 32000, "kernel arguments");

// ------------------------------------------------------------------------- the step's factors

struct Step {
    double lr, b1, log_b1, b2, log_b2, eps, decay, max_norm;
    const float* lr_at;
    const float* norm;
    int64_t* step;
    Factors* factors;
    int* status;
};

__global__ void factors_kernel(const Step s) {
    grid_wait();
    grid_release();
    *s.status = DTP_OK;                // nothing here can give up
    Factors f;
    const float n = s.norm ? *s.norm : 0.0f;
    f.skip = s.norm && !isfinite(n);
    f.clip = 1.0f, f.down = 1.0f;
    if (!f.skip && static_cast<double>(n) > s.max_norm) {
        const float c = __frcp_rn(n) * static_cast<float>(s.max_norm);
        if (n <= 1.0e37f && (c >= 1.0e-30f || s.max_norm == 0.0)) {
            f.clip = c;
        } else {                       // a factor among fp32's subnormal numbers would lose bits: in two parts
            const double r = s.max_norm / static_cast<double>(n);
            const int half = (-ilogb(r) - 1) / 2;
            f.clip = static_cast<float>(ldexp(r, 2 * half)), f.down = ldexpf(1.0f, -half);
        }
    }
    const int64_t t = *s.step + 1;
    const double lr = s.lr_at ? static_cast<double>(*s.lr_at) : s.lr;
    f.b1 = static_cast<float>(s.b1), f.not_b1 = static_cast<float>(1.0 - s.b1);
    f.b2 = static_cast<float>(s.b2), f.not_b2 = static_cast<float>(1.0 - s.b2);
    f.keep = static_cast<float>(1.0 - lr * s.decay);
    // 1 - b^t as -(e^(t log b) - 1) in fp32: exact to its rounding for small t too, and fp64's exponential would double the launch
    f.size = static_cast<float>(lr) / -expm1f(static_cast<float>(static_cast<double>(t) * s.log_b1));
    f.root = 1.0f / sqrtf(-expm1f(static_cast<float>(static_cast<double>(t) * s.log_b2)));
    f.eps = static_cast<float>(s.eps);
    f.key = static_cast<uint32_t>(t) * 0x9E3779B9u;
    *s.factors = f;
    if (!f.skip) *s.step = t;
}

// ------------------------------------------------------------------------------- elements

template <int CAP>
__device__ __forceinline__ int tensor_of(const Table<CAP>& t, int c) {
    int lo = 0, hi = t.count;
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (t.first[mid] <= c) lo = mid;
        else hi = mid;
    }
    return lo;
}

// Three numbers in [0, 2^32) of an element and a step.
__device__ __forceinline__ uint32_t mix(int64_t i, uint32_t key) {
    uint32_t x = static_cast<uint32_t>(i) + static_cast<uint32_t>(i >> 32) * 0x85EBCA6Bu + key;
    x = (x ^ (x >> 16)) * 0x7FEB352Du;
    x = (x ^ (x >> 15)) * 0x846CA68Bu;
    return x ^ (x >> 16);
}
// [0, 2^32) to [0, 1) in 23 bits
__device__ __forceinline__ float fraction(uint32_t x) { return __uint_as_float(0x3F800000u | (x >> 9)) - 1.0f; }

// The code of a in [0, 448] rounded up with probability u's share: a over its step (of at least the subnormal numbers'
// 2^-9) is in [8, 16) for normal numbers, and codes count steps across the binades.
__device__ __forceinline__ uint32_t encode(float a, float u) {
    const uint32_t least = 121u << 23, bits = __float_as_uint(a) & 0x7F800000u;
    const uint32_t e = bits > least ? bits : least;
    const float steps = __fadd_rn(__fmul_rn(a, __uint_as_float((257u << 23) - e)), u);
    const uint32_t k = __float_as_uint(__fadd_rd(steps, 8388608.0f)) & 0x1Fu;        // the whole steps: below 2^23 + 17
    const uint32_t code = ((e - least) >> 20) + k;
    return code < 0x7Eu ? code : 0x7Eu;
}
__device__ __forceinline__ void decode2(uint32_t codes, float& a, float& b) {        // the lower two
    const __half2_raw h = __nv_cvt_fp8x2_to_halfraw2(static_cast<__nv_fp8x2_storage_t>(codes), __NV_E4M3);
    const float2 v = __half22float2(__half2(h));
    a = v.x, b = v.y;
}

// A lane's eight elements of a block: four consecutive ones of either half, so that a warp's words are consecutive in every
// type (eight consecutive ones, two words of fp32 a lane: 16 bytes of every 32 at a time, 2030 us for 415M elements and 32 bits), or every
// 32nd of them where a tensor starts on another boundary or ends within the block.
template <bool kWide>
__device__ __forceinline__ int place(int j) {
    const int lane = threadIdx.x & 31;
    return kWide ? 4 * lane + (j & 3) + 128 * (j >> 2) : 32 * j + lane;
}
// What is read and written once a step does not stay in L2 for long: streaming loads and stores.
template <bool kWide>
__device__ __forceinline__ void load8(const float* p, int left, float (&v)[8]) {
    if constexpr (kWide) {
        const float4 a = __ldcs(reinterpret_cast<const float4*>(p + place<true>(0)));
        const float4 b = __ldcs(reinterpret_cast<const float4*>(p + place<true>(4)));
        v[0] = a.x, v[1] = a.y, v[2] = a.z, v[3] = a.w, v[4] = b.x, v[5] = b.y, v[6] = b.z, v[7] = b.w;
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = place<false>(j) < left ? p[place<false>(j)] : 0.0f;
    }
}
template <bool kWide>
__device__ __forceinline__ void load8(const __nv_bfloat16* p, int left, float (&v)[8]) {
    if constexpr (kWide) {
        const uint2 a = __ldcs(reinterpret_cast<const uint2*>(p + place<true>(0)));
        const uint2 b = __ldcs(reinterpret_cast<const uint2*>(p + place<true>(4)));
        const uint32_t w[4] = {a.x, a.y, b.x, b.y};
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = __uint_as_float(j & 1 ? w[j / 2] & 0xFFFF0000u : w[j / 2] << 16);
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = place<false>(j) < left ? layer::to_f32(p[place<false>(j)]) : 0.0f;
    }
}
template <bool kWide>
__device__ __forceinline__ void store8(float* p, int left, const float (&v)[8]) {
    if constexpr (kWide) {
        __stcs(reinterpret_cast<float4*>(p + place<true>(0)), make_float4(v[0], v[1], v[2], v[3]));
        __stcs(reinterpret_cast<float4*>(p + place<true>(4)), make_float4(v[4], v[5], v[6], v[7]));
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j)
            if (place<false>(j) < left) p[place<false>(j)] = v[j];
    }
}
template <bool kWide>
__device__ __forceinline__ void store8(__nv_bfloat16* p, int left, const float (&v)[8]) {
    if constexpr (kWide) {
        uint32_t w[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const __nv_bfloat162 b = __floats2bfloat162_rn(v[2 * j], v[2 * j + 1]);
            w[j] = *reinterpret_cast<const uint32_t*>(&b);
        }
        __stcs(reinterpret_cast<uint2*>(p + place<true>(0)), make_uint2(w[0], w[1]));
        __stcs(reinterpret_cast<uint2*>(p + place<true>(4)), make_uint2(w[2], w[3]));
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j)
            if (place<false>(j) < left) p[place<false>(j)] = __float2bfloat16_rn(v[j]);
    }
}
template <bool kWide>
__device__ __forceinline__ void load_codes(const uint8_t* p, int left, float (&v)[8]) {
    uint32_t w[4];
    if constexpr (kWide) {
        w[0] = __ldcs(reinterpret_cast<const uint32_t*>(p + place<true>(0))), w[1] = w[0] >> 16;
        w[2] = __ldcs(reinterpret_cast<const uint32_t*>(p + place<true>(4))), w[3] = w[2] >> 16;
    } else {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int a = place<false>(2 * j), b = place<false>(2 * j + 1);
            w[j] = (a < left ? p[a] : 0u) | (b < left ? static_cast<uint32_t>(p[b]) << 8 : 0u);
        }
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) decode2(w[j], v[2 * j], v[2 * j + 1]);
}
template <bool kWide>
__device__ __forceinline__ void store_codes(uint8_t* p, int left, const uint32_t (&v)[8]) {
    if constexpr (kWide) {
        __stcs(reinterpret_cast<uint32_t*>(p + place<true>(0)), v[0] | v[1] << 8 | v[2] << 16 | v[3] << 24);
        __stcs(reinterpret_cast<uint32_t*>(p + place<true>(4)), v[4] | v[5] << 8 | v[6] << 16 | v[7] << 24);
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j)
            if (place<false>(j) < left) p[place<false>(j)] = static_cast<uint8_t>(v[j]);
    }
}

// A block's values as codes over its scale.  kFine: they are all finite; else those that are not are held as NaN.
__device__ __forceinline__ uint32_t largest(const float (&x)[8]) {       // of the warp's sizes as bits: infinities and NaNs are above all
    uint32_t top = 0;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        const uint32_t b = __float_as_uint(x[j]) & 0x7FFFFFFFu;
        top = b > top ? b : top;
    }
    return __reduce_max_sync(0xFFFFFFFFu, top);
}
template <bool kRoot, typename F>
__device__ __forceinline__ void hold(const float (&x)[8], F u, float* scale, uint32_t (&code)[8]) {
    uint32_t top = largest(x);
    const bool fine = top < 0x7F800000u;
    if (!fine) {
        float y[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) y[j] = isfinite(x[j]) ? x[j] : 0.0f;
        top = largest(y);
    }
    const float size = __uint_as_float(top);
    const bool some = size >= kLeast;
    const float up = some ? __fmul_rn(__frcp_rn(size), 448.0f) : 0.0f;
    if ((threadIdx.x & 31) == 0) *scale = some ? __fmul_rn(size, 1.0f / 448.0f) : 0.0f;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        code[j] = encode(__fmul_rn(fabsf(x[j]), up), u(j));
        if constexpr (kRoot) code[j] = code[j] == 0 && x[j] > 0.0f ? 1u : code[j];       // a moment is never lost: its parameter would leap
        else code[j] |= x[j] < 0.0f ? 0x80u : 0u;
    }
    if (!fine) {
#pragma unroll
        for (int j = 0; j < 8; ++j)
            if (!isfinite(x[j])) code[j] = 0x7Fu;
    }
}

// One block of 256 elements by a warp, `left` of which the tensor has.
template <typename P, typename G, bool kEight, bool kWide, int CAP>
__device__ __forceinline__ void update(const Table<CAP>& t, int i, int64_t b, int left, const Factors& f) {
    const int64_t at = b * kBlock;
    P* p = static_cast<P*>(t.p[i]) + at;
    float x[8], g[8], m[8], v[8];
    load8<kWide>(p, left, x);
    load8<kWide>(static_cast<const G*>(t.g[i]) + at, left, g);
    if constexpr (kEight) {
        load_codes<kWide>(static_cast<const uint8_t*>(t.m[i]) + at, left, m);
        load_codes<kWide>(static_cast<const uint8_t*>(t.v[i]) + at, left, v);
        const float ms = t.ms[i][b], vs = t.vs[i][b];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            m[j] = __fmul_rn(m[j], ms);
            v[j] = __fmul_rn(v[j], vs);
            v[j] = __fmul_rn(v[j], v[j]);
        }
    } else {
        load8<kWide>(static_cast<const float*>(t.m[i]) + at, left, m);
        load8<kWide>(static_cast<const float*>(t.v[i]) + at, left, v);
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) g[j] = __fmul_rn(g[j], f.clip);
    if (f.down != 1.0f) {
#pragma unroll
        for (int j = 0; j < 8; ++j) g[j] = __fmul_rn(__fmul_rn(g[j], f.down), f.down);
    }
    float root[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        m[j] = __fadd_rn(__fmul_rn(m[j], f.b1), __fmul_rn(g[j], f.not_b1));
        v[j] = __fadd_rn(__fmul_rn(v[j], f.b2), __fmul_rn(__fmul_rn(g[j], g[j]), f.not_b2));
        root[j] = kEight ? __fsqrt_rn(v[j]) : sqrtf(v[j]);
        x[j] = x[j] * f.keep - f.size * __fdividef(m[j], fmaf(root[j], f.root, f.eps));
    }
    [[maybe_unused]] uint32_t h[8];
    if constexpr (kEight || sizeof(P) == 2) {
#pragma unroll
        for (int j = 0; j < 8; ++j) h[j] = mix(at + place<kWide>(j), f.key);
    }
    if constexpr (sizeof(P) == 2) {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const uint32_t up = (__float_as_uint(x[j]) + ((h[j] * 0x85EBCA77u) >> 16)) & 0xFFFF0000u;
            x[j] = isfinite(x[j]) ? __uint_as_float(up) : x[j];
        }
    }
    store8<kWide>(p, left, x);
    if constexpr (sizeof(P) == 4)
        if (t.copy[i]) store8<kWide>(t.copy[i] + at, left, x);
    if constexpr (kEight) {
        uint32_t code[8];
        hold<false>(m, [&](int j) { return fraction(h[j]); }, t.ms[i] + b, code);
        store_codes<kWide>(static_cast<uint8_t*>(t.m[i]) + at, left, code);
        hold<true>(root, [&](int j) { return fraction(h[j] * 0x9E3779B1u); }, t.vs[i] + b, code);
        store_codes<kWide>(static_cast<uint8_t*>(t.v[i]) + at, left, code);
    } else {
        store8<kWide>(static_cast<float*>(t.m[i]) + at, left, m);
        store8<kWide>(static_cast<float*>(t.v[i]) + at, left, v);
    }
}

__device__ __forceinline__ void prefetch(const void* p) { asm volatile("prefetch.global.L2 [%0];" ::"l"(p)); }

// The blocks of [a, e) of tensor i, whose values have types P and G.
template <typename P, typename G, bool kEight, int CAP>
__device__ __forceinline__ void update_run(const Table<CAP>& t, int i, int64_t a, int64_t e, const Factors& f) {
    const int64_t b1 = (e + kBlock - 1) / kBlock;
    for (int64_t b = a / kBlock + (threadIdx.x >> 5); b < b1; b += kWarps) {
        const int64_t left = t.numel[i] - b * kBlock;
        if (t.flags[i].aligned && left >= kBlock) update<P, G, kEight, true>(t, i, b, kBlock, f);
        else update<P, G, kEight, false>(t, i, b, left < kBlock ? static_cast<int>(left) : kBlock, f);
    }
}

template <int CAP, bool kEight>
__global__ void __launch_bounds__(kThreads, kBlocksPerSm) step_kernel(const __grid_constant__ Table<CAP> t) {
    const int c0 = static_cast<int>(static_cast<int64_t>(t.chunks) * blockIdx.x / gridDim.x);
    const int c1 = static_cast<int>(static_cast<int64_t>(t.chunks) * (blockIdx.x + 1) / gridDim.x);
    // elements [a, e) of tensor i in this block's chunks
    auto part = [&](int i, int64_t& a, int64_t& e) {
        a = c0 > t.first[i] ? (c0 - t.first[i]) * t.chunk : 0;
        e = c1 < t.first[i + 1] ? (c1 - t.first[i]) * t.chunk : t.numel[i];
    };
    const int i0 = tensor_of(t, c0);
    {   // the first block's values on their way while the factors are made
        int64_t a, e;
        part(i0, a, e);
        a += (threadIdx.x >> 5) * kBlock + place<true>(0);
        if (a < t.numel[i0]) {
            prefetch(static_cast<const uint8_t*>(t.p[i0]) + a * (t.flags[i0].p_f32 ? 4 : 2));
            prefetch(static_cast<const uint8_t*>(t.g[i0]) + a * (t.flags[i0].g_f32 ? 4 : 2));
            prefetch(static_cast<const uint8_t*>(t.m[i0]) + a * (kEight ? 1 : 4));
            prefetch(static_cast<const uint8_t*>(t.v[i0]) + a * (kEight ? 1 : 4));
        }
    }
    grid_wait();
    grid_release();
    const Factors f = *t.factors;
    if (f.skip || c0 >= c1) return;
    for (int i = i0; i < t.count && t.first[i] < c1; ++i) {
        int64_t a, e;
        part(i, a, e);
        if (t.flags[i].p_f32) {
            if (t.flags[i].g_f32) update_run<float, float, kEight>(t, i, a, e, f);
            else update_run<float, __nv_bfloat16, kEight>(t, i, a, e, f);
        } else {
            if (t.flags[i].g_f32) update_run<__nv_bfloat16, float, kEight>(t, i, a, e, f);
            else update_run<__nv_bfloat16, __nv_bfloat16, kEight>(t, i, a, e, f);
        }
    }
}

// ------------------------------------------------------------------------------------ host

bool sizes_ok(int count, const int64_t* numel) {
    int64_t total = 0;
    for (int i = 0; i < count; ++i) {
        if (numel[i] < 0 || numel[i] > (int64_t(1) << 46)) return false;
        total += numel[i];
        if (total > (int64_t(1) << 46)) return false;
    }
    return count < (1 << 24);
}

size_t workspace_bytes() { return kWorkspaceHeader + 256; }

template <typename K, typename A>
static int launch_overlapped(K kernel, int blocks, int threads, const A& arg, cudaStream_t stream) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(static_cast<unsigned>(blocks));
    cfg.blockDim = dim3(static_cast<unsigned>(threads));
    cfg.stream = stream;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    DTP_CUDA_TRY(cudaLaunchKernelEx(&cfg, kernel, arg));
    return DTP_OK;
}

template <int CAP>
static int launch_tables(void* const* params, const int* param_dtypes, const void* const* grads, const int* grad_dtypes,
                         void* const* m, void* const* v, float* const* m_scale, float* const* v_scale, void* const* copies,
                         const int64_t* numel, int count, bool eight, const Factors* factors, int sms, cudaStream_t stream) {
    Table<CAP> t;
    int64_t total = 0;
    for (int i = 0; i < count; ++i) total += numel[i];
    t.chunk = kMinChunk;
    while (total / t.chunk > kManyChunks) t.chunk *= 2;
    t.factors = factors;
    t.count = 0;
    int chunks = 0;
    auto flush = [&]() {
        t.chunks = chunks;
        t.first[t.count] = chunks;
        const int most = kBlocksPerSm * sms;
        const int st = launch_overlapped(eight ? step_kernel<CAP, true> : step_kernel<CAP, false>, chunks < most ? chunks : most,
                                         kThreads, t, stream);
        t.count = 0, chunks = 0;
        return st;
    };
    for (int i = 0; i < count; ++i) {
        if (numel[i] == 0) continue;
        if (t.count == CAP) {
            const int st = flush();
            if (st != DTP_OK) return st;
        }
        const int k = t.count++;
        t.p[k] = params[i], t.g[k] = grads[i], t.m[k] = m[i], t.v[k] = v[i];
        t.ms[k] = eight ? m_scale[i] : nullptr, t.vs[k] = eight ? v_scale[i] : nullptr;
        t.copy[k] = copies ? static_cast<__nv_bfloat16*>(copies[i]) : nullptr;
        t.numel[k] = numel[i];
        t.first[k] = chunks;
        t.flags[k].p_f32 = param_dtypes[i] == DTP_F32, t.flags[k].g_f32 = grad_dtypes[i] == DTP_F32;
        uintptr_t all = reinterpret_cast<uintptr_t>(params[i]) | reinterpret_cast<uintptr_t>(grads[i]) |
                        reinterpret_cast<uintptr_t>(t.copy[k]);
        // four codes are a word of 4 bytes
        const uintptr_t held = reinterpret_cast<uintptr_t>(m[i]) | reinterpret_cast<uintptr_t>(v[i]);
        all |= eight ? 4 * held : held;
        t.flags[k].aligned = (all & 15) == 0;
        chunks += static_cast<int>((numel[i] + t.chunk - 1) / t.chunk);
    }
    return t.count ? flush() : static_cast<int>(DTP_OK);
}

int launch(void* const* params, const int* param_dtypes, const void* const* grads, const int* grad_dtypes, void* const* m,
           void* const* v, float* const* m_scale, float* const* v_scale, void* const* copies, const int64_t* numel, int count,
           const dtp_adamw_opts* o, const float* lr, const float* norm, int64_t* step, void* workspace, cudaStream_t stream) {
    int dev = 0, sms = 0;
    DTP_CUDA_TRY(cudaGetDevice(&dev));
    DTP_CUDA_TRY(cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev));
    auto* factors = reinterpret_cast<Factors*>(static_cast<uint8_t*>(workspace) + kWorkspaceHeader);
    const Step s{o->lr, o->beta1, log(o->beta1), o->beta2, log(o->beta2), o->eps, o->weight_decay, o->max_norm, lr, norm, step,
                 factors, static_cast<int*>(workspace)};
    const int st = launch_overlapped(factors_kernel, 1, 1, s, stream);
    if (st != DTP_OK) return st;
    int filled = 0;
    for (int i = 0; i < count; ++i) filled += numel[i] != 0;
    const bool eight = o->state_bits == 8;
    auto go = filled <= kSmallTable ? launch_tables<kSmallTable> : launch_tables<kLargeTable>;
    return go(params, param_dtypes, grads, grad_dtypes, m, v, m_scale, v_scale, copies, numel, count, eight, factors, sms, stream);
}

}  // namespace adamw
}  // namespace dtp
