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
//
// fp32 parameters, bf16 gradients and copies, 415M elements: 32 bits 1.78 to 1.83 ms (6.4 TB/s of 28 bytes each); 8 bits 1.26 ms
// (5.3 TB/s of 16), bound by 89 instructions an element, issued in 70% of the cycles.  bf16 parameters in 301 tensors off their words,
// 60M: 0.24 ms.
#include <cuda_bf16.h>
#include <cuda_fp8.h>
#include <cuda_runtime.h>
#include <math.h>
#include <stdint.h>

#include <type_traits>

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
    float keep;
    float root, eps;           // the update is m / (root sqrt(v) + eps): the rate is in both
    uint32_t key;
    int skip;
};

struct Flags { uint8_t p_f32, g_f32; };

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
        // the reciprocal of a normal number up to 1e37, and a limit, that lose no bits; a limit of 0 is one
        const bool normal = n >= 1.2e-38f && n <= 1.0e37f && s.max_norm >= 1.2e-38;
        if (s.max_norm == 0.0 || (normal && c >= 1.0e-30f)) {
            f.clip = s.max_norm == 0.0 ? 0.0f : c;
        } else {                       // a factor among fp32's subnormal numbers would lose bits: in two parts
            const double r = s.max_norm / static_cast<double>(n);
            if (r < 1.0e-90) {         // no gradient times it is above half of fp32's least number
                f.clip = 0.0f;
            } else {
                const int half = (-ilogb(r) - 1) / 2;
                f.clip = static_cast<float>(ldexp(r, 2 * half)), f.down = ldexpf(1.0f, -half);
            }
        }
    }
    const int64_t t = *s.step + 1;
    const double lr = s.lr_at ? static_cast<double>(*s.lr_at) : s.lr;
    f.b1 = static_cast<float>(s.b1), f.not_b1 = static_cast<float>(1.0 - s.b1);
    f.b2 = static_cast<float>(s.b2), f.not_b2 = static_cast<float>(1.0 - s.b2);
    f.keep = static_cast<float>(1.0 - lr * s.decay);
    // 1 - b^t as -(e^(t log b) - 1) in fp32: exact to its rounding for small t too, and fp64's exponential would double the launch
    const float size = static_cast<float>(lr) / -expm1f(static_cast<float>(static_cast<double>(t) * s.log_b1));
    const float root = 1.0f / sqrtf(-expm1f(static_cast<float>(static_cast<double>(t) * s.log_b2)));
    // Rates below fp32's range of quotients (0 among them) have no update, a divisor of infinity; the least divisor is a normal number.
    f.root = root / size, f.eps = static_cast<float>(s.eps) / size;
    if (isinf(f.root) || isinf(f.eps)) f.root = 0.0f, f.eps = INFINITY;
    if (fabsf(f.eps) < 1.1754944e-38f) f.eps = copysignf(1.1754944e-38f, f.eps);
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

// A number in [0, 2^32) of an element and a step, by which the first moment is rounded; the second and the parameter go by its products
// with two odd numbers.
__device__ __forceinline__ uint32_t mix(int64_t i, uint32_t key) {
    uint32_t x = static_cast<uint32_t>(i) + static_cast<uint32_t>(i >> 32) * 0x85EBCA6Bu + key;
    x = (x ^ (x >> 16)) * 0x7FEB352Du;
    x = (x ^ (x >> 15)) * 0x846CA68Bu;
    return x ^ (x >> 16);
}

// The code of a in [0, 448], in the top byte: with a in steps t (of at least the subnormal numbers' 2^-9) and u, h's upper 23 bits as a
// part of one, the whole part of t + u rounded to fp32.  In normal numbers t is a multiple of 2^-20, the place of the rounded
// sum below its next whole number, so the sum is t's pattern with h added below the step and a half for the rounding.  a256
// is 256 a, whose exponent makes the upper bits the code itself.
constexpr float kLeastNormal = 4.0f;               // 256 x 2^-6
constexpr uint32_t kMost = 0x7EFFFFFFu;            // no code beyond 448's
__device__ __forceinline__ uint32_t encode_normal(float a256, uint32_t h) {
    const uint32_t w = (__float_as_uint(a256) << 4) + (h >> 8) + 8u;
    return w < kMost ? w : kMost;
}
__device__ __forceinline__ uint32_t encode(float a256, uint32_t h) {
    if (a256 >= kLeastNormal) return encode_normal(a256, h);
    const float u = __uint_as_float(0x3F800000u | (h >> 9)) - 1.0f;
    return static_cast<uint32_t>(__fadd_rn(a256 * 2.0f, u)) << 24;                  // a 2^9
}
__device__ __forceinline__ void decode2(uint32_t codes, float& a, float& b) {        // the lower two
    const __half2_raw h = __nv_cvt_fp8x2_to_halfraw2(static_cast<__nv_fp8x2_storage_t>(codes), __NV_E4M3);
    const float2 v = __half22float2(__half2(h));
    a = v.x, b = v.y;
}

// Pairs of fp32 products, each half rounded as the scalar one.  Sums of them stay scalar: a pair's sum of two pairs' products came out
// contracted (a rounding less in a fifth of the blocks' largest moments), explicit rounding or not.
__device__ __forceinline__ uint64_t pair(float a, float b) {
    uint64_t r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(a), "f"(b));
    return r;
}
__device__ __forceinline__ void split(uint64_t v, float& a, float& b) { asm("mov.b64 {%0, %1}, %2;" : "=f"(a), "=f"(b) : "l"(v)); }
__device__ __forceinline__ uint64_t mul2(uint64_t a, uint64_t b) {
    uint64_t r;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}
__device__ __forceinline__ float sqrt_fast(float x) {
    float y;
    asm("sqrt.approx.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
// of a normal number (its own unit's error, 2^-23; the quotient's way around subnormal divisors is a tenth of the 8-bit kernel's time)
__device__ __forceinline__ float rcp_fast(float x) {
    float y;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
// the larger, or NaN
__device__ __forceinline__ float max_nan(float a, float b) {
    float y;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(y) : "f"(a), "f"(b));
    return y;
}

// A lane's eight elements of a block: four consecutive ones of either half, so that a warp's words are consecutive in every
// type (eight consecutive ones, two words of fp32 a lane: 16 bytes of every 32 at a time, 2030 us for 415M elements and 32 bits), or every
// 32nd of them where a tensor ends within the block.
template <bool kWhole>
__device__ __forceinline__ int place(int j) {
    const int lane = threadIdx.x & 31;
    return kWhole ? 4 * lane + (j & 3) + 128 * (j >> 2) : 32 * j + lane;
}

// A lane's values as they were loaded, and what they are.  Loads come first for all tensors, so that they are in flight together;
// tensors that start within a word are then shifted into place, each lane taking the rest of its words from the next one (16 bytes
// and 2 bytes off a word: 60M elements of 2 + 2 + 1 + 1 bytes 253 us element by element).  What is read and written once a step does
// not stay in L2 for long: streaming loads and stores.
__device__ __forceinline__ uint32_t offset_in_word(const void* p) { return static_cast<uint32_t>(reinterpret_cast<uintptr_t>(p)) & 3u; }
template <typename T>
__device__ __forceinline__ const uint32_t* word_of(const T* p) {
    return reinterpret_cast<const uint32_t*>(reinterpret_cast<uintptr_t>(p) & ~uintptr_t(3));
}

template <typename T, bool kWhole>
struct Values;
template <typename T>
struct Values<T, false> {
    T e[8];
    __device__ __forceinline__ void load(const T* p, int left) {
#pragma unroll
        for (int j = 0; j < 8; ++j) e[j] = place<false>(j) < left ? p[place<false>(j)] : T(0);
    }
    __device__ __forceinline__ void get(const T*, float (&v)[8]) const {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            if constexpr (sizeof(T) == 1) {
                float none;
                decode2(e[j], v[j], none);
            } else {
                v[j] = layer::to_f32(e[j]);
            }
        }
    }
};
template <>
struct Values<float, true> {
    float e[8];
    __device__ __forceinline__ void load(const float* p, int) {
        if ((reinterpret_cast<uintptr_t>(p) & 15) == 0) {
            const float4 a = __ldcs(reinterpret_cast<const float4*>(p + place<true>(0)));
            const float4 b = __ldcs(reinterpret_cast<const float4*>(p + place<true>(4)));
            e[0] = a.x, e[1] = a.y, e[2] = a.z, e[3] = a.w, e[4] = b.x, e[5] = b.y, e[6] = b.z, e[7] = b.w;
        } else {
#pragma unroll
            for (int j = 0; j < 8; ++j) e[j] = p[place<true>(j)];
        }
    }
    __device__ __forceinline__ void get(const float*, float (&v)[8]) const {
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = e[j];
    }
};
template <>
struct Values<__nv_bfloat16, true> {
    uint32_t w[4], next;
    __device__ __forceinline__ void load(const __nv_bfloat16* p, int) {
        next = 0;
        if ((reinterpret_cast<uintptr_t>(p) & 7) == 0) {
            const uint2 a = __ldcs(reinterpret_cast<const uint2*>(p + place<true>(0)));
            const uint2 b = __ldcs(reinterpret_cast<const uint2*>(p + place<true>(4)));
            w[0] = a.x, w[1] = a.y, w[2] = b.x, w[3] = b.y;
        } else {
            const uint32_t* q = word_of(p) + 2 * (threadIdx.x & 31);
            w[0] = q[0], w[1] = q[1], w[2] = q[64], w[3] = q[65];
            if ((threadIdx.x & 31) == 31 && offset_in_word(p)) next = q[66];       // the block's last element is in it
        }
    }
    __device__ __forceinline__ void get(const __nv_bfloat16* p, float (&v)[8]) const {
        uint32_t x[4] = {w[0], w[1], w[2], w[3]};
        if (offset_in_word(p)) {
            const int lane = threadIdx.x & 31;
            const uint32_t a = __shfl_sync(0xFFFFFFFFu, lane == 0 ? w[2] : w[0], (lane + 1) & 31);
            const uint32_t c = __shfl_down_sync(0xFFFFFFFFu, w[2], 1);
            x[0] = __funnelshift_r(w[0], w[1], 16), x[1] = __funnelshift_r(w[1], a, 16);
            x[2] = __funnelshift_r(w[2], w[3], 16), x[3] = __funnelshift_r(w[3], lane == 31 ? next : c, 16);
        }
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = __uint_as_float(j & 1 ? x[j / 2] & 0xFFFF0000u : x[j / 2] << 16);
    }
};
template <>
struct Values<uint8_t, true> {
    uint32_t w[2], next;
    __device__ __forceinline__ void load(const uint8_t* p, int) {
        const uint32_t* q = word_of(p) + (threadIdx.x & 31);
        w[0] = __ldcs(q), w[1] = __ldcs(q + 32), next = 0;
        if ((threadIdx.x & 31) == 31 && offset_in_word(p)) next = q[33];
    }
    __device__ __forceinline__ void get(const uint8_t* p, float (&v)[8]) const {
        uint32_t x[2] = {w[0], w[1]};
        const uint32_t off = offset_in_word(p);
        if (off) {
            const int lane = threadIdx.x & 31;
            const uint32_t a = __shfl_sync(0xFFFFFFFFu, lane == 0 ? w[1] : w[0], (lane + 1) & 31);
            const uint32_t c = __shfl_down_sync(0xFFFFFFFFu, w[1], 1);
            x[0] = __funnelshift_r(w[0], a, 8 * off), x[1] = __funnelshift_r(w[1], lane == 31 ? next : c, 8 * off);
        }
        decode2(x[0], v[0], v[1]), decode2(x[0] >> 16, v[2], v[3]);
        decode2(x[1], v[4], v[5]), decode2(x[1] >> 16, v[6], v[7]);
    }
};

template <bool kWhole>
__device__ __forceinline__ void store8(float* p, int left, const float (&v)[8]) {
    if (kWhole && (reinterpret_cast<uintptr_t>(p) & 15) == 0) {
        __stcs(reinterpret_cast<float4*>(p + place<true>(0)), make_float4(v[0], v[1], v[2], v[3]));
        __stcs(reinterpret_cast<float4*>(p + place<true>(4)), make_float4(v[4], v[5], v[6], v[7]));
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j)
            if (kWhole || place<false>(j) < left) p[place<kWhole>(j)] = v[j];
    }
}
// Words that start within a word of memory: each lane completes the one before with its neighbour's end; the ends of the
// block, whose words are shared with others, go by elements.
template <bool kWhole>
__device__ __forceinline__ void store8(__nv_bfloat16* p, int left, const float (&v)[8]) {
    if constexpr (kWhole) {
        uint32_t w[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const __nv_bfloat162 b = __floats2bfloat162_rn(v[2 * j], v[2 * j + 1]);
            w[j] = *reinterpret_cast<const uint32_t*>(&b);
        }
        if ((reinterpret_cast<uintptr_t>(p) & 7) == 0) {
            __stcs(reinterpret_cast<uint2*>(p + place<true>(0)), make_uint2(w[0], w[1]));
            __stcs(reinterpret_cast<uint2*>(p + place<true>(4)), make_uint2(w[2], w[3]));
            return;
        }
        const int lane = threadIdx.x & 31;
        uint32_t* q = const_cast<uint32_t*>(word_of(p)) + 2 * lane;
        if (offset_in_word(p) == 0) {
            q[0] = w[0], q[1] = w[1], q[64] = w[2], q[65] = w[3];
            return;
        }
        const uint32_t a = __shfl_up_sync(0xFFFFFFFFu, w[1], 1);
        const uint32_t c = __shfl_sync(0xFFFFFFFFu, lane == 31 ? w[1] : w[3], (lane + 31) & 31);
        if (lane == 0) reinterpret_cast<uint16_t*>(p)[0] = static_cast<uint16_t>(w[0]);
        else q[0] = __funnelshift_l(a, w[0], 16);
        q[1] = __funnelshift_l(w[0], w[1], 16);
        q[64] = __funnelshift_l(c, w[2], 16), q[65] = __funnelshift_l(w[2], w[3], 16);
        if (lane == 31) reinterpret_cast<uint16_t*>(p)[255] = static_cast<uint16_t>(w[3] >> 16);
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j)
            if (place<false>(j) < left) p[place<false>(j)] = __float2bfloat16_rn(v[j]);
    }
}
// codes in the top bytes
template <bool kWhole>
__device__ __forceinline__ void store_codes(uint8_t* p, int left, const uint32_t (&v)[8]) {
    if constexpr (kWhole) {
        uint32_t w[2];
#pragma unroll
        for (int j = 0; j < 2; ++j)
            w[j] = __byte_perm(__byte_perm(v[4 * j], v[4 * j + 1], 0x0073), __byte_perm(v[4 * j + 2], v[4 * j + 3], 0x0073), 0x5410);
        const int lane = threadIdx.x & 31;
        uint32_t* q = const_cast<uint32_t*>(word_of(p)) + lane;
        const uint32_t off = offset_in_word(p);
        if (off == 0) {
            __stcs(q, w[0]);
            __stcs(q + 32, w[1]);
            return;
        }
        const uint32_t a = __shfl_up_sync(0xFFFFFFFFu, w[0], 1);
        const uint32_t c = __shfl_sync(0xFFFFFFFFu, lane == 31 ? w[0] : w[1], (lane + 31) & 31);
        if (lane == 0) {
            for (uint32_t k = 0; k < 4 - off; ++k) p[k] = static_cast<uint8_t>(w[0] >> 8 * k);
        } else {
            q[0] = __funnelshift_l(a, w[0], 8 * off);
        }
        q[32] = __funnelshift_l(c, w[1], 8 * off);
        if (lane == 31)
            for (uint32_t k = 4 - off; k < 4; ++k) p[252 + k] = static_cast<uint8_t>(w[1] >> 8 * k);
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j)
            if (place<false>(j) < left) p[place<false>(j)] = static_cast<uint8_t>(v[j] >> 24);
    }
}

// A block's values as codes over its scale, in the top bytes; those that are not finite are held as NaN.  kRoot: they are not negative, and
// none above zero is held as zero (its parameter would leap).  `h`: a random number for each.
template <bool kRoot, typename F>
__device__ __forceinline__ void hold(const float (&x)[8], F h, float* scale, uint32_t (&code)[8]) {
    auto largest = [](const float (&y)[8]) {              // of the warp's sizes, as bits: NaNs and infinities are above all
        float top = fabsf(y[0]);
#pragma unroll
        for (int j = 1; j < 8; ++j) top = max_nan(top, fabsf(y[j]));
        return __reduce_max_sync(0xFFFFFFFFu, __float_as_uint(top));
    };
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
    const float up = some ? __fmul_rn(__frcp_rn(size), 448.0f) * 256.0f : 0.0f;
    if ((threadIdx.x & 31) == 0) *scale = some ? __fmul_rn(size, 1.0f / 448.0f) : 0.0f;
    bool low = false;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        const float a = __fmul_rn(fabsf(x[j]), up);
        low |= !(a >= kLeastNormal);
        code[j] = encode_normal(a, h(j));
    }
    if (__any_sync(0xFFFFFFFFu, low || !fine)) {          // subnormal codes are few: blocks with one in 60 when the values are normal ones
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            code[j] = encode(__fmul_rn(fabsf(x[j]), up), h(j));
            if (kRoot && code[j] == 0 && x[j] > 0.0f) code[j] = 1u << 24;
            if (!isfinite(x[j])) code[j] = 0x7Fu << 24;
        }
    }
    if constexpr (!kRoot) {
#pragma unroll
        for (int j = 0; j < 8; ++j) code[j] |= __float_as_uint(x[j]) & 0x80000000u;
    }
}

// A tensor of the table.  Its pointers are read where they are used: held over the loop they cost registers that the block's values
// need (8 bits: 1440 us for 415M elements, and 1300).
template <typename P, typename G, bool kEight, int CAP>
struct Tensor {
    using S = std::conditional_t<kEight, uint8_t, float>;
    const Table<CAP>& t;
    int i;
    __device__ __forceinline__ P* p() const { return static_cast<P*>(t.p[i]); }
    __device__ __forceinline__ const G* g() const { return static_cast<const G*>(t.g[i]); }
    __device__ __forceinline__ S* m() const { return static_cast<S*>(t.m[i]); }
    __device__ __forceinline__ S* v() const { return static_cast<S*>(t.v[i]); }
    __device__ __forceinline__ float* ms() const { return t.ms[i]; }
    __device__ __forceinline__ float* vs() const { return t.vs[i]; }
    __device__ __forceinline__ __nv_bfloat16* copy() const { return t.copy[i]; }
};

// One block of 256 elements by a warp, `left` of which the tensor has.
template <bool kWhole, typename P, typename G, bool kEight, int CAP>
__device__ __forceinline__ void update(const Tensor<P, G, kEight, CAP>& t, int64_t b, int left, const Factors& f) {
    using S = typename Tensor<P, G, kEight, CAP>::S;
    const int64_t at = b * kBlock;
    P* p = t.p() + at;
    const G* g_at = t.g() + at;
    S *m_at = t.m() + at, *v_at = t.v() + at;
    float x[8], g[8], m[8], v[8], root[8];
    {
        Values<P, kWhole> px;
        Values<G, kWhole> gx;
        Values<S, kWhole> mx, vx;
        px.load(p, left);
        gx.load(g_at, left);
        mx.load(m_at, left);
        vx.load(v_at, left);
        uint64_t ms = 0, vs = 0;
        if constexpr (kEight) {
            const float a = t.ms()[b], c = t.vs()[b];
            ms = pair(a, a), vs = pair(c, c);
        }
        mx.get(m_at, m);
        vx.get(v_at, v);
        if constexpr (kEight) {
#pragma unroll
            for (int j = 0; j < 8; j += 2) {
                split(mul2(pair(m[j], m[j + 1]), ms), m[j], m[j + 1]);
                const uint64_t r = mul2(pair(v[j], v[j + 1]), vs);
                split(mul2(r, r), v[j], v[j + 1]);
            }
        }
        gx.get(g_at, g);
        px.get(p, x);
    }
    if (f.down != 1.0f) {
#pragma unroll
        for (int j = 0; j < 8; ++j) g[j] = __fmul_rn(__fmul_rn(g[j], f.down), f.down);
    }
    const uint64_t clip = pair(f.clip, f.clip), b1 = pair(f.b1, f.b1), c1 = pair(f.not_b1, f.not_b1), b2 = pair(f.b2, f.b2),
                   c2 = pair(f.not_b2, f.not_b2);
#pragma unroll
    for (int j = 0; j < 8; j += 2) {
        const uint64_t q = mul2(pair(g[j], g[j + 1]), clip);
        float a, b;
        split(mul2(pair(m[j], m[j + 1]), b1), m[j], m[j + 1]);
        split(mul2(q, c1), a, b);
        m[j] = __fadd_rn(m[j], a), m[j + 1] = __fadd_rn(m[j + 1], b);
        split(mul2(pair(v[j], v[j + 1]), b2), v[j], v[j + 1]);
        split(mul2(mul2(q, q), c2), a, b);
        v[j] = __fadd_rn(v[j], a), v[j + 1] = __fadd_rn(v[j + 1], b);
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        root[j] = kEight ? __fsqrt_rn(v[j]) : sqrt_fast(v[j]);
        x[j] = fmaf(x[j], f.keep, -m[j] * rcp_fast(fmaf(root[j], f.root, f.eps)));
    }
    if constexpr (!kEight) {
        store8<kWhole>(m_at, left, m);
        store8<kWhole>(v_at, left, v);
    }
    [[maybe_unused]] uint32_t h[8];
    if constexpr (kEight || sizeof(P) == 2) {
#pragma unroll
        for (int j = 0; j < 8; ++j) h[j] = mix(at + place<kWhole>(j), f.key);
    }
    if constexpr (sizeof(P) == 2) {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const uint32_t up = (__float_as_uint(x[j]) + ((h[j] * 0x85EBCA77u) >> 16)) & 0xFFFF0000u;
            x[j] = isfinite(x[j]) ? __uint_as_float(up) : x[j];
        }
    }
    store8<kWhole>(p, left, x);
    if constexpr (sizeof(P) == 4)
        if (t.copy()) store8<kWhole>(t.copy() + at, left, x);
    if constexpr (kEight) {
        uint32_t code[8];
        hold<false>(m, [&](int j) { return h[j]; }, t.ms() + b, code);
        store_codes<kWhole>(m_at, left, code);
        hold<true>(root, [&](int j) { return h[j] * 0x9E3779B1u; }, t.vs() + b, code);
        store_codes<kWhole>(v_at, left, code);
    }
}

__device__ __forceinline__ void prefetch(const void* p) { asm volatile("prefetch.global.L2 [%0];" ::"l"(p)); }

// A whole block's values on their way to L2 while the one before is computed on (8 bits: 357 us for 104M elements, without 374; 32 bits, whose
// loads are enough to keep memory busy, 473 and 461).
template <typename P, typename G, bool kEight, int CAP>
__device__ __forceinline__ void prefetch_block(const Tensor<P, G, kEight, CAP>& t, int64_t b) {
    const int lane = threadIdx.x & 31;
    // sectors of 32 bytes: 8 lanes for a byte an element, 16 for two, 32 for four
    auto bytes = [&](const auto* p, int sector) { prefetch(reinterpret_cast<const uint8_t*>(p + b * kBlock) + 32 * sector); };
    if constexpr (sizeof(P) == 4) bytes(t.p(), lane);
    else if (lane < 16) bytes(t.p(), lane);
    if constexpr (sizeof(G) == 4) bytes(t.g(), lane);
    else if (lane < 16) bytes(t.g(), lane);
    if (!kEight || lane < 8) bytes(t.m(), lane), bytes(t.v(), lane);
}

// The blocks of [a, e) of n elements, by all warps in turn.
template <typename P, typename G, bool kEight, int CAP>
__device__ __forceinline__ void update_run(const Tensor<P, G, kEight, CAP> t, int64_t n, int64_t a, int64_t e, const Factors& f) {
    const int64_t b1 = (e + kBlock - 1) / kBlock;
    for (int64_t b = a / kBlock + (threadIdx.x >> 5); b < b1; b += kWarps) {
        const int64_t left = n - b * kBlock;
        if (kEight && b + kWarps < b1 && left >= (kWarps + 1) * kBlock) prefetch_block(t, b + kWarps);
        if (left >= kBlock) update<true>(t, b, kBlock, f);
        else update<false>(t, b, static_cast<int>(left), f);
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
            if (t.flags[i].g_f32) update_run(Tensor<float, float, kEight, CAP>{t, i}, t.numel[i], a, e, f);
            else update_run(Tensor<float, __nv_bfloat16, kEight, CAP>{t, i}, t.numel[i], a, e, f);
        } else {
            if (t.flags[i].g_f32) update_run(Tensor<__nv_bfloat16, float, kEight, CAP>{t, i}, t.numel[i], a, e, f);
            else update_run(Tensor<__nv_bfloat16, __nv_bfloat16, kEight, CAP>{t, i}, t.numel[i], a, e, f);
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
