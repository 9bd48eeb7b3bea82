// grad_clip.cu -- the global norm of many gradient tensors, and their clipping:
//
//     n = sqrt(sum over tensors and elements of g^2),  c = n > max_norm ? max_norm / n : 1,  out = c g
//
// Bound by memory: one read for the norm, then one read and one write, of which the second read finds in L2 what fits
// there.  The tensors are cut into chunks of 8 KB (more where that would be too many to count), and each block takes a
// run of them, so that all blocks have the same bytes to read whatever the tensors' sizes.  The first launch sums the squares
// of each block's run in fp32, each thread in rounds of four 16-byte words whose sums enter a compensated total, and writes
// one fp64 partial per block; the second, which is under way before the first ends and waits for it, adds all partials in the
// same order in every block and scales the runs, last words first.  (Both in one cooperative launch with a barrier over the
// grid: 9 us for the smallest call, most of it the launch.)  The table of the tensors is a kernel argument; more of them than
// it holds take a launch per table for the norm and one per table for the scaling.
// A block whose fp32 sum left the range in which it is exact to fp32's precision (overflow, or so small that
// squares were lost below 2^-126) sums again with its elements scaled by a power of two.
#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include "dtp_common.cuh"
#include "layer_common.cuh"

namespace dtp {
namespace clip {

using layer::from_f32;
using layer::to_f32;

constexpr int kThreads = 512;
constexpr int kWarps = kThreads / 32;
constexpr int64_t kMinChunk = 8192;    // bytes
constexpr int64_t kManyChunks = 1 << 24;
constexpr int R = 4;                   // 16-byte words in flight per thread
constexpr int kBlocksPerSm = 2;

template <int CAP>
struct Table {
    const void* src[CAP];
    void* dst[CAP];
    int64_t numel[CAP];
    int first[CAP + 1];                // first chunk of the tensor
    uint8_t f32[CAP];
    int count;
    int chunks;                        // of this table
    int partial0;                      // the table's first partial
    int partials;                      // of all tables
    int64_t chunk;                     // bytes
    float max_norm;
    double* partial;
    float* norm;
    int* status;
};
constexpr int kSmallTable = 64, kLargeTable = 1024;
static_assert(sizeof(Table<kLargeTable>) <= 32000, "kernel arguments");

// the tensor of chunk c: the last one whose first chunk is <= c (empty tensors are not in the table)
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

__device__ __forceinline__ float block_sum(float v, float* red) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xFFFFFFFFu, v, o);
    __syncthreads();
    if (lane == 0) red[warp] = v;
    __syncthreads();
    float s = 0.0f;
#pragma unroll
    for (int w = 0; w < kWarps; ++w) s += red[w];
    return s;
}

// The 16-byte words of n elements from p, and the elements before and after them.
template <typename E>
struct Span {
    static constexpr int kPer = 16 / sizeof(E);
    int head;
    int64_t words;
    __device__ __forceinline__ Span(const void* p, int64_t n) {
        const int64_t lead = ((16 - (reinterpret_cast<uintptr_t>(p) & 15)) & 15) / sizeof(E);
        head = static_cast<int>(lead < n ? lead : n);
        words = (n - head) / kPer;
    }
};

template <typename E>
__device__ __forceinline__ void unpack(const uint4& q, float (&v)[16 / sizeof(E)]) {
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

template <typename E>
__device__ __forceinline__ uint4 pack(const float (&v)[16 / sizeof(E)]) {
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if constexpr (sizeof(E) == 4) {
            w[i] = __float_as_uint(v[i]);
        } else {
            const __nv_bfloat162 b = __floats2bfloat162_rn(v[2 * i], v[2 * i + 1]);
            w[i] = *reinterpret_cast<const uint32_t*>(&b);
        }
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
}

// A sum of many fp32 terms with the rounding errors of the additions carried along.  An infinite sum stays infinite: the error of
// an addition to it would be inf - inf.
struct Total {
    float sum = 0.0f, lost = 0.0f;
    __device__ __forceinline__ void add(float x) {
        const float y = x - lost, t = sum + y;
        lost = isinf(t) ? 0.0f : (t - sum) - y;
        sum = t;
    }
};

// This thread's share of sum (scale p[i])^2.
template <typename E>
__device__ __forceinline__ void sum_squares(const E* p, int64_t n, float scale, Total& total) {
    const Span<E> s(p, n);
    const uint4* words = reinterpret_cast<const uint4*>(p + s.head);
    auto square = [&](float x, float& to) { x *= scale; to = fmaf(x, x, to); };
    auto word = [&](const uint4& q, float& to) {
        float v[Span<E>::kPer];
        unpack<E>(q, v);
#pragma unroll
        for (int i = 0; i < Span<E>::kPer; ++i) square(v[i], to);
    };
    int64_t i = threadIdx.x;
    for (; i + (R - 1) * kThreads < s.words; i += R * kThreads) {
        uint4 q[R];
        float r[R];
#pragma unroll
        for (int j = 0; j < R; ++j) q[j] = words[i + j * kThreads];
#pragma unroll
        for (int j = 0; j < R; ++j) r[j] = 0.0f, word(q[j], r[j]);
        total.add((r[0] + r[1]) + (r[2] + r[3]));
    }
    float rest = 0.0f;
    for (; i < s.words; i += kThreads) word(words[i], rest);
    if (static_cast<int>(threadIdx.x) < s.head) square(to_f32(p[threadIdx.x]), rest);
    const int64_t tail = s.head + s.words * Span<E>::kPer + threadIdx.x;
    if (tail < n) square(to_f32(p[tail]), rest);
    total.add(rest);
}

constexpr float kTiny = 8.271806e-25f;         // 2^-80
constexpr float kUp = 1.2676506e30f;           // 2^100
constexpr float kDown = 7.888609e-31f;         // 2^-100

// A factor c down down.  `down` is 1, or a power of two where the factor would leave few bits of c, or none, among fp32's subnormal
// numbers (large gradients, a small limit).
struct Factor {
    float c, down;
    __device__ __forceinline__ float operator()(float v) const { return v * c * down * down; }
};
// below 1, above 0
__device__ __forceinline__ Factor factor_of(double ratio) {
    const int half = ratio < 7.888609052210118e-31 ? (-ilogb(ratio) - 1) / 2 : 0;       // 2^-100; then c is in [1/4, 1)
    return Factor{static_cast<float>(ldexp(ratio, 2 * half)), ldexpf(1.0f, -half)};
}

// dst = f src, last words first.  Words where both are equally aligned; a factor of 1 copies bit for bit, NaNs too.
template <typename E>
__device__ __forceinline__ void scale_run(const E* src, E* dst, int64_t n, const Factor f) {
    const bool copy = f.c == 1.0f;
    if (copy && src == dst) return;
    auto one = [&](int64_t i) { dst[i] = copy ? src[i] : from_f32<E>(f(to_f32(src[i]))); };
    if ((reinterpret_cast<uintptr_t>(src) ^ reinterpret_cast<uintptr_t>(dst)) & 15) {
        for (int64_t i = threadIdx.x; i < n; i += kThreads) one(i);
        return;
    }
    const Span<E> s(src, n);
    const uint4* from = reinterpret_cast<const uint4*>(src + s.head);
    uint4* to = reinterpret_cast<uint4*>(dst + s.head);
    auto word = [&](const uint4& q) {
        if (copy) return q;
        float v[Span<E>::kPer];
        unpack<E>(q, v);
#pragma unroll
        for (int i = 0; i < Span<E>::kPer; ++i) v[i] = f(v[i]);
        return pack<E>(v);
    };
    const int64_t rounds = s.words / (R * kThreads) * (R * kThreads);
    for (int64_t i = rounds + threadIdx.x; i < s.words; i += kThreads) __stcs(to + i, word(from[i]));
    for (int64_t i = rounds - R * kThreads + threadIdx.x; i >= 0; i -= R * kThreads) {
        uint4 q[R];
#pragma unroll
        for (int j = 0; j < R; ++j) q[j] = from[i + j * kThreads];
#pragma unroll
        for (int j = 0; j < R; ++j) __stcs(to + i + j * kThreads, word(q[j]));
    }
    if (static_cast<int>(threadIdx.x) < s.head) one(threadIdx.x);
    const int64_t tail = s.head + s.words * Span<E>::kPer + threadIdx.x;
    if (tail < n) one(tail);
}

enum Mode { kNorm = 0, kScale = 1 };

template <int CAP, int MODE>
__global__ void __launch_bounds__(kThreads, kBlocksPerSm) clip_kernel(const __grid_constant__ Table<CAP> t) {
    __shared__ float red[kWarps];
    __shared__ Factor coef;
    // this block's chunks, and elements [a, b) of tensor i among them
    const int c0 = static_cast<int>(static_cast<int64_t>(t.chunks) * blockIdx.x / gridDim.x);
    const int c1 = static_cast<int>(static_cast<int64_t>(t.chunks) * (blockIdx.x + 1) / gridDim.x);
    auto part = [&](int i, int64_t& a, int64_t& b) {
        const int64_t per = t.chunk / (t.f32[i] ? 4 : 2);
        a = c0 > t.first[i] ? (c0 - t.first[i]) * per : 0;
        b = c1 < t.first[i + 1] ? (c1 - t.first[i]) * per : t.numel[i];
    };
    if (MODE == kNorm && blockIdx.x == 0 && threadIdx.x == 0) *t.status = DTP_OK;     // nothing here can give up
    if constexpr (MODE == kNorm) {
        asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
        auto squares = [&](float scale) {
            Total total;
            if (c0 < c1) {
                for (int i = tensor_of(t, c0); i < t.count && t.first[i] < c1; ++i) {
                    int64_t a, b;
                    part(i, a, b);
                    if (t.f32[i]) sum_squares(static_cast<const float*>(t.src[i]) + a, b - a, scale, total);
                    else sum_squares(static_cast<const __nv_bfloat16*>(t.src[i]) + a, b - a, scale, total);
                }
            }
            return block_sum(total.sum, red);          // the same value in every thread
        };
        float s = squares(1.0f), scale = 1.0f;
        if (!(s >= kTiny && s <= 3.0e38f)) {
            scale = s < kTiny ? kUp : kDown;           // (a NaN stays one either way)
            s = squares(scale);
        }
        if (threadIdx.x == 0)
            t.partial[t.partial0 + blockIdx.x] = static_cast<double>(s) / (static_cast<double>(scale) * scale);
    } else {
        asm volatile("griddepcontrol.wait;" ::: "memory");
        // one warp adds the partials: an SM has two fp64 additions a clock (all 512 threads taking part: 5 us)
        if (threadIdx.x < 32) {
            double s = 0.0;
            for (int c = threadIdx.x; c < t.partials; c += 32) s += __ldcg(t.partial + c);
#pragma unroll
            for (int o = 16; o > 0; o >>= 1) s += __shfl_xor_sync(0xFFFFFFFFu, s, o);
            if (threadIdx.x == 0) {
                const double r = sqrt(s);
                const float n = static_cast<float>(r);
                // a norm that is not finite, as the caller reads it, leaves the gradients as they are
                coef = !isfinite(n) || r <= static_cast<double>(t.max_norm) ? Factor{1.0f, 1.0f}
                       : t.max_norm > 0.0f                                  ? factor_of(t.max_norm / r)
                                                                            : Factor{0.0f, 1.0f};
                if (blockIdx.x == 0) *t.norm = n;
            }
        }
        __syncthreads();
        const Factor f = coef;
        if (c0 < c1) {
            for (int i = tensor_of(t, c1 - 1); i >= 0 && t.first[i + 1] > c0; --i) {
                int64_t a, b;
                part(i, a, b);
                if (t.f32[i])
                    scale_run(static_cast<const float*>(t.src[i]) + a, static_cast<float*>(t.dst[i]) + a, b - a, f);
                else
                    scale_run(static_cast<const __nv_bfloat16*>(t.src[i]) + a,
                              static_cast<__nv_bfloat16*>(t.dst[i]) + a, b - a, f);
            }
        }
    }
}

// ------------------------------------------------------------------------------------ host

static int64_t bytes_of(int64_t numel, int dtype) { return numel * (dtype == DTP_F32 ? 4 : 2); }

static int64_t chunk_bytes(int count, const int64_t* numel, const int* dtype) {
    int64_t total = 0, chunk = kMinChunk;
    for (int i = 0; i < count; ++i) total += bytes_of(numel[i], dtype[i]);
    while (total / chunk > kManyChunks) chunk *= 2;
    return chunk;
}

// Whether the sizes can be counted.
bool sizes_ok(int count, const int64_t* numel) {
    int64_t total = 0;
    for (int i = 0; i < count; ++i) {
        if (numel[i] < 0 || numel[i] > (int64_t(1) << 46)) return false;
        total += numel[i];
        if (total > (int64_t(1) << 46)) return false;
    }
    return count < (1 << 24);
}

// Blocks of a table's launch; a partial for each of them.
constexpr int kMostBlocks = 512;
size_t workspace_bytes(int count) {
    return kWorkspaceHeader + static_cast<size_t>(count / kLargeTable + 1) * kMostBlocks * sizeof(double);
}

static int blocks_of(int chunks, int sms) {
    const int most = kBlocksPerSm * sms < kMostBlocks ? kBlocksPerSm * sms : kMostBlocks;
    return chunks < 1 ? 1 : chunks < most ? chunks : most;
}

template <int CAP, int MODE>
static int launch_table(const Table<CAP>& t, bool early, int sms, cudaStream_t stream) {
    auto kernel = clip_kernel<CAP, MODE>;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(static_cast<unsigned>(blocks_of(t.chunks, sms)));
    cfg.blockDim = dim3(kThreads);
    cfg.stream = stream;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = early ? 1 : 0;
    DTP_CUDA_TRY(cudaLaunchKernelEx(&cfg, kernel, t));
    return DTP_OK;
}

// Tables of at most CAP non-empty tensors (one, perhaps empty, if there are none), each passed to fn.
template <int CAP, typename F>
static int each_table(const void* const* grads, void* const* out, const int64_t* numel, const int* dtype, int count,
                      int sms, Table<CAP>& t, F fn) {
    t.count = 0, t.partial0 = 0;
    int chunks = 0, launched = 0;
    auto flush = [&]() {
        t.chunks = chunks;
        t.first[t.count] = chunks;
        const int st = fn();
        t.partial0 += blocks_of(chunks, sms);
        t.count = 0, chunks = 0;
        ++launched;
        return st;
    };
    for (int i = 0; i < count; ++i) {
        if (numel[i] == 0) continue;
        if (t.count == CAP) {
            const int st = flush();
            if (st != DTP_OK) return st;
        }
        t.src[t.count] = grads[i];
        t.dst[t.count] = out ? out[i] : const_cast<void*>(grads[i]);
        t.numel[t.count] = numel[i];
        t.first[t.count] = chunks;
        t.f32[t.count] = dtype[i] == DTP_F32;
        ++t.count;
        chunks += static_cast<int>((bytes_of(numel[i], dtype[i]) + t.chunk - 1) / t.chunk);
    }
    return t.count || !launched ? flush() : static_cast<int>(DTP_OK);
}

template <int CAP>
static int launch_capacity(const void* const* grads, void* const* out, const int64_t* numel, const int* dtype,
                           int count, float max_norm, float* norm, void* workspace, int sms, cudaStream_t stream) {
    Table<CAP> t;
    t.chunk = chunk_bytes(count, numel, dtype);
    t.max_norm = max_norm;
    t.norm = norm;
    t.status = static_cast<int*>(workspace);
    t.partial = reinterpret_cast<double*>(static_cast<uint8_t*>(workspace) + kWorkspaceHeader);
    const int st = each_table(grads, out, numel, dtype, count, sms, t,
                              [&] { return launch_table<CAP, kNorm>(t, false, sms, stream); });
    if (st != DTP_OK) return st;
    t.partials = t.partial0;             // of all the tables
    bool early = true;                   // the launch before is the norm's
    return each_table(grads, out, numel, dtype, count, sms, t, [&] {
        const int r = launch_table<CAP, kScale>(t, early, sms, stream);
        early = false;
        return r;
    });
}

int launch(const void* const* grads, void* const* out, const int64_t* numel, const int* dtype, int count,
           float max_norm, float* norm, void* workspace, cudaStream_t stream) {
    int dev = 0, sms = 0;
    DTP_CUDA_TRY(cudaGetDevice(&dev));
    DTP_CUDA_TRY(cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev));
    int filled = 0;
    for (int i = 0; i < count; ++i) filled += numel[i] != 0;
    if (filled <= kSmallTable)
        return launch_capacity<kSmallTable>(grads, out, numel, dtype, count, max_norm, norm, workspace, sms, stream);
    return launch_capacity<kLargeTable>(grads, out, numel, dtype, count, max_norm, norm, workspace, sms, stream);
}

}  // namespace clip
}  // namespace dtp
