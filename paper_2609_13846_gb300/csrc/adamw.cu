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
    f.size = static_cast<float>(lr / -expm1(static_cast<double>(t) * s.log_b1));
    f.root = static_cast<float>(rsqrt(-expm1(static_cast<double>(t) * s.log_b2)));
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
__device__ __forceinline__ float fraction(uint32_t x) { return static_cast<float>(x >> 9) * 1.1920929e-7f; }   // [0, 1)

// The code of a in [0, 448] rounded up with probability u's share: a over its step (of at least the subnormal numbers'
// 2^-9) is in [8, 16) for normal numbers, and codes count steps across the binades.
__device__ __forceinline__ uint32_t encode(float a, float u) {
    const uint32_t least = 121u << 23, bits = __float_as_uint(a) & 0x7F800000u;
    const uint32_t e = bits > least ? bits : least;
    const uint32_t k = static_cast<uint32_t>(__fadd_rn(__fmul_rn(a, __uint_as_float((257u << 23) - e)), u));
    const uint32_t code = ((e - least) >> 20) + k;
    return code < 0x7Eu ? code : 0x7Eu;
}
__device__ __forceinline__ float decode(uint32_t code) {
    return __half2float(__half(__nv_cvt_fp8_to_halfraw(static_cast<__nv_fp8_storage_t>(code), __NV_E4M3)));
}

// Eight elements from element i (of the lane's in the aligned form), or every 32nd from i.
template <typename E, bool kAligned>
__device__ __forceinline__ void load8(const E* p, int64_t i, int left, float (&v)[8]) {
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        const int at = kAligned ? j : 32 * j;
        v[j] = at < left ? layer::to_f32(p[i + at]) : 0.0f;
    }
}

// One block of 256 elements by a warp.
template <typename P, typename G, bool kEight, int CAP>
__device__ __forceinline__ void update(const Table<CAP>& t, int i, int64_t b, const Factors& f) {
    const int lane = threadIdx.x & 31;
    const int64_t at = b * kBlock + lane;
    const int64_t rest = t.numel[i] - at;
    const int left = rest > kBlock ? kBlock : static_cast<int>(rest);       // elements from the lane's first
    P* p = static_cast<P*>(t.p[i]);
    float x[8], g[8], m[8], v[8];
    load8<P, false>(p, at, left, x);
    load8<G, false>(static_cast<const G*>(t.g[i]), at, left, g);
    if constexpr (kEight) {
        const float ms = t.ms[i][b], vs = t.vs[i][b];
        const uint8_t *mc = static_cast<const uint8_t*>(t.m[i]), *vc = static_cast<const uint8_t*>(t.v[i]);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            m[j] = 32 * j < left ? __fmul_rn(decode(mc[at + 32 * j]), ms) : 0.0f;
            const float r = 32 * j < left ? __fmul_rn(decode(vc[at + 32 * j]), vs) : 0.0f;
            v[j] = __fmul_rn(r, r);
        }
    } else {
        load8<float, false>(static_cast<const float*>(t.m[i]), at, left, m);
        load8<float, false>(static_cast<const float*>(t.v[i]), at, left, v);
    }
    float root[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        g[j] = __fmul_rn(__fmul_rn(__fmul_rn(g[j], f.clip), f.down), f.down);
        m[j] = __fadd_rn(__fmul_rn(m[j], f.b1), __fmul_rn(g[j], f.not_b1));
        v[j] = __fadd_rn(__fmul_rn(v[j], f.b2), __fmul_rn(__fmul_rn(g[j], g[j]), f.not_b2));
        root[j] = sqrtf(v[j]);
        x[j] = x[j] * f.keep - f.size * (m[j] / (root[j] * f.root + f.eps));
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        if (32 * j >= left) continue;
        if constexpr (sizeof(P) == 2) {
            const uint32_t bits = __float_as_uint(x[j]);
            const uint32_t up = (bits + ((mix(at + 32 * j, f.key) * 0x85EBCA77u) >> 16)) & 0xFFFF0000u;
            p[at + 32 * j] = isfinite(x[j]) ? __float2bfloat16_rn(__uint_as_float(up)) : __float2bfloat16_rn(x[j]);
        } else {
            p[at + 32 * j] = x[j];
            if (t.copy[i]) t.copy[i][at + 32 * j] = __float2bfloat16_rn(x[j]);
        }
        if constexpr (!kEight) {
            static_cast<float*>(t.m[i])[at + 32 * j] = m[j];
            static_cast<float*>(t.v[i])[at + 32 * j] = v[j];
        }
    }
    if constexpr (kEight) {
        float mt = 0.0f, vt = 0.0f;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            if (32 * j >= left) continue;
            if (isfinite(m[j])) mt = fmaxf(mt, fabsf(m[j]));
            if (isfinite(root[j])) vt = fmaxf(vt, root[j]);
        }
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) {
            mt = fmaxf(mt, __shfl_xor_sync(0xFFFFFFFFu, mt, o));
            vt = fmaxf(vt, __shfl_xor_sync(0xFFFFFFFFu, vt, o));
        }
        const float mu = mt >= kLeast ? __fmul_rn(__frcp_rn(mt), 448.0f) : 0.0f;
        const float vu = vt >= kLeast ? __fmul_rn(__frcp_rn(vt), 448.0f) : 0.0f;
        if (lane == 0) {
            t.ms[i][b] = mt >= kLeast ? __fmul_rn(mt, 1.0f / 448.0f) : 0.0f;
            t.vs[i][b] = vt >= kLeast ? __fmul_rn(vt, 1.0f / 448.0f) : 0.0f;
        }
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            if (32 * j >= left) continue;
            const uint32_t h = mix(at + 32 * j, f.key);
            uint32_t mc = 0x7Fu, vc = 0x7Fu;
            if (isfinite(m[j])) mc = encode(__fmul_rn(fabsf(m[j]), mu), fraction(h)) | (m[j] < 0.0f ? 0x80u : 0u);
            if (isfinite(root[j])) {
                vc = encode(__fmul_rn(root[j], vu), fraction(h * 0x9E3779B1u));
                if (vc == 0 && root[j] > 0.0f) vc = 1;      // a moment is never lost: its parameter would leap
            }
            static_cast<uint8_t*>(t.m[i])[at + 32 * j] = static_cast<uint8_t>(mc);
            static_cast<uint8_t*>(t.v[i])[at + 32 * j] = static_cast<uint8_t>(vc);
        }
    }
}

template <int CAP, bool kEight>
__global__ void __launch_bounds__(kThreads, kBlocksPerSm) step_kernel(const __grid_constant__ Table<CAP> t) {
    const int c0 = static_cast<int>(static_cast<int64_t>(t.chunks) * blockIdx.x / gridDim.x);
    const int c1 = static_cast<int>(static_cast<int64_t>(t.chunks) * (blockIdx.x + 1) / gridDim.x);
    grid_wait();
    grid_release();
    const Factors f = *t.factors;
    if (f.skip || c0 >= c1) return;
    for (int i = tensor_of(t, c0); i < t.count && t.first[i] < c1; ++i) {
        const int64_t a = c0 > t.first[i] ? (c0 - t.first[i]) * t.chunk : 0;
        const int64_t e = c1 < t.first[i + 1] ? (c1 - t.first[i]) * t.chunk : t.numel[i];
        const int64_t b1 = (e + kBlock - 1) / kBlock;
        for (int64_t b = a / kBlock + (threadIdx.x >> 5); b < b1; b += kWarps) {
            if (t.flags[i].p_f32) {
                if (t.flags[i].g_f32) update<float, float, kEight>(t, i, b, f);
                else update<float, __nv_bfloat16, kEight>(t, i, b, f);
            } else {
                if (t.flags[i].g_f32) update<__nv_bfloat16, float, kEight>(t, i, b, f);
                else update<__nv_bfloat16, __nv_bfloat16, kEight>(t, i, b, f);
            }
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
