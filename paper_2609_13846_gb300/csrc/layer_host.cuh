// layer_host.cuh -- the host side that the operators on tokens share: launches that overlap their predecessors, the pieces of a
// workspace, and the matrix products of one call.
#pragma once

#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include "dtp_common.cuh"
#include "layer_common.cuh"

namespace dtp {
namespace simt {
int launch(const layer::Product& p, int dtype, int* status, cudaStream_t stream);
}  // namespace simt
namespace gtc {
int64_t most_chunks(int N);
int launch(const layer::Product& p, int* status, int reset, cudaStream_t stream, int64_t* chunks = nullptr);
// The time that launch_pair takes, in k blocks of a 256 x 256 tile, and the best number of parts for it.
int64_t pair_clocks(int64_t rows, int cols, int d, int* parts);
int launch_pair(const layer::GradPair& g, int* status, cudaStream_t stream);
}  // namespace gtc
namespace few {
bool takes(const layer::Product& p);
int launch(const layer::Product& p, int* status, int reset, int second, cudaStream_t stream);
}  // namespace few

namespace fews {
bool takes(const layer::Product& p, int dtype);
int launch(const layer::Product& p, int dtype, int* status, int second, cudaStream_t stream);
}  // namespace fews

// fp32, up to 32 tokens (few_loss_f32.cu)
namespace fewl {
int ranges_of(int64_t V, int d);
bool takes_logits(int64_t T, int d);
int launch_logits(const float* X, const float* W, int64_t T, int64_t V, int d, float* Z, cudaStream_t stream);
int launch_dx(const float* dZ, const float* W, int64_t T, int64_t V, int d, int ranges, float* parts, cudaStream_t stream);
int launch_dw(const float* dZ, const float* X, int64_t T, int64_t V, int d, float* dW, cudaStream_t stream);
}  // namespace fewl

namespace layer {

// A launch whose start may overlap the end of the one before it.
template <typename... P, typename... A>
int launch_blocks(void (*kernel)(P...), int64_t blocks, int threads, cudaStream_t stream, A... args) {
    if (blocks > 0x7FFFFFFF) return DTP_ERR_UNSUPPORTED;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(static_cast<unsigned>(blocks));
    cfg.blockDim = dim3(static_cast<unsigned>(threads));
    cfg.stream = stream;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    DTP_CUDA_TRY(cudaLaunchKernelEx(&cfg, kernel, args...));
    return DTP_OK;
}

template <typename... P, typename... A>
int launch_after(void (*kernel)(P...), int64_t blocks, cudaStream_t stream, A... args) {
    return launch_blocks(kernel, blocks, 256, stream, args...);
}

// Pieces of a workspace, in the order in which they are asked for.
struct Carver {
    uint8_t* base;
    size_t used = kWorkspaceHeader;
    explicit Carver(void* p) : base(static_cast<uint8_t*>(p)) {}
    void* take(size_t bytes) {
        void* r = base ? base + used : nullptr;
        used += align_up(bytes, 256);
        return r;
    }
};

inline size_t elem(int dtype) { return dtype == DTP_BF16 ? 2 : 4; }
inline int64_t padded(int64_t n) { return (n + 7) / 8 * 8; }
// bf16 [rows, cols] as the tensor cores can load it: itself, or a copy at an aligned pitch from the workspace.
struct Rows {
    const void* p;
    int64_t ld;
};
size_t repitch_bytes(int64_t rows, int cols, int dtype);
int aligned_rows(const void* p, int64_t rows, int cols, int dtype, Carver& c, cudaStream_t stream, Rows* out);

inline Mat by_row(const void* p, int64_t ld) { return Mat{p, ld, 1}; }      // [rows, K]
inline Mat by_col(const void* p, int64_t ld) { return Mat{p, 1, ld}; }      // [K, rows]

// One call's products, in order on its stream.  The first launch that may give up on a wait clears the status word.
struct Call {
    int dtype;
    void* workspace;
    cudaStream_t stream;
    bool fresh = true;          // the status word is still an earlier call's
    bool after_few = false;     // the last launch was a few-token kernel

    int run(const Product& p) {
        int* status = static_cast<int*>(workspace);
        const int reset = fresh;
        const bool second = after_few;
        after_few = false;
        if (p.K > 0 && p.M > 0 && fews::takes(p, dtype)) {
            fresh = false, after_few = true;
            return fews::launch(p, dtype, reset ? status : nullptr, second, stream);
        }
        if (dtype == DTP_BF16 && p.K > 0) {
            fresh = false;
            if (few::takes(p)) {
                after_few = true;
                return few::launch(p, status, reset, second, stream);
            }
            return gtc::launch(p, status, reset, stream);
        }
        if (p.K == 0) return simt::launch(p, dtype, nullptr, stream);
        fresh = false;
        return simt::launch(p, dtype, reset ? status : nullptr, stream);
    }
    // calls without such a launch
    int done() {
        if (!fresh) return DTP_OK;
        DTP_CUDA_TRY(cudaMemsetAsync(workspace, 0, sizeof(int), stream));
        return DTP_OK;
    }
};

// The weights' gradients are sums over the tokens, of which there may be 2^31, and an fp32 accumulator loses about 2^-26 of its sum for
// every 16 of them on the tensor cores (it cuts off: 10% of a sum of 2^26 terms of one sign) and what rounding leaves on the
// CUDA cores (0.1%).  So such a sum is made in runs of at most 2^18 tokens (2^-12), each a product of its own whose fp32 sums go
// to the workspace, and the runs are added in 64 bits.
constexpr int64_t kRun = 1 << 18;
size_t runs_bytes(int64_t T, int64_t rows, int64_t cols);
// out [rows, cols] = sum over T tokens of A's rows times B's columns, both stored token by token; `runs` of runs_bytes.  `unit` (device; of
// several runs only): what the sums are taken times.
int weight_gradient(Call& call, const Also& w, int64_t T, float* runs, const float* unit = nullptr);

}  // namespace layer
}  // namespace dtp
