// Host-side launchers of the training operators (internal to the library).
#pragma once

#include <cuda_runtime.h>
#include <stddef.h>
#include <stdint.h>

#include "../../include/pwlq.h"

namespace pwlq {

constexpr int kF32 = PWLQ_F32, kBf16 = PWLQ_BF16, kF16 = PWLQ_F16;

// An 8-bit checkpoint (format: include/pwlq.h).
struct Act8Tensor {
    uint8_t* codes;
    int64_t ldc;
    float* ranges;
    int64_t rows, cols;
    int group;
    float ratio;
    __host__ __device__ int64_t groups() const { return (cols + group - 1) / group; }
};

inline int group_shift(int group) { return group == 32 ? 5 : group == 64 ? 6 : group == 128 ? 7 : 8; }
inline size_t type_size(int dtype) { return dtype == kF32 ? 4 : 2; }

// Whether every row starts on a 16-byte boundary.
inline bool rows_aligned(const void* p, int64_t ld, size_t size) {
    return ((reinterpret_cast<uintptr_t>(p) | (uintptr_t)(ld * (int64_t)size)) & 15) == 0;
}

// Launches a kernel that may begin while the one before it in the stream still runs (it waits for that
// one's end itself, await_previous).
template <typename... P, typename... A>
cudaError_t launch_dependent(void (*kernel)(P...), dim3 blocks, dim3 threads, size_t smem, cudaStream_t stream,
                             const A&... args) {
    cudaLaunchAttribute attr;
    attr.id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr.val.programmaticStreamSerializationAllowed = 1;
    cudaLaunchConfig_t config = {};
    config.gridDim = blocks;
    config.blockDim = threads;
    config.dynamicSmemBytes = smem;
    config.stream = stream;
    config.attrs = &attr;
    config.numAttrs = 1;
    return cudaLaunchKernelEx(&config, kernel, args...);
}

cudaError_t launch_act8_encode(const void* x, int dtype, int64_t ldx, const Act8Tensor& a,
                               cudaStream_t stream);
// A copy of [rows, cols] 16-bit values to rows of `pitch` (a multiple of 8) values, zeros past cols, that
// a decode launch makes beside its own work (from null: none; first and rows_per_block are its own).
struct Realigned {
    const void* from = nullptr;
    int64_t ld = 0;
    void* to = nullptr;
    int64_t pitch = 8, cols = 0, rows = 0;
    unsigned first = 0, rows_per_block = 1;
};
cudaError_t launch_act8_decode(const Act8Tensor& a, void* y, int dtype, int64_t ldy, cudaStream_t stream,
                               const Realigned& beside = Realigned());

cudaError_t launch_block_norm(const pwlq_block_norm_args& a, cudaStream_t stream);
size_t block_norm_backward_workspace(int64_t rows, int64_t cols, int64_t gate_rows);
cudaError_t launch_block_norm_backward(const pwlq_block_norm_args& a, const pwlq_block_norm_grads& g,
                                       cudaStream_t stream);

struct WeightGrad {
    const void* dy;
    int dtype;
    int64_t rows, outputs, lddy;
    Act8Tensor x;
    void* dw;
    int dw_dtype;
    int64_t lddw;
    bool accumulate;
};
// aligned: dy's rows start on 16-byte boundaries (else the workspace holds a copy whose rows do).
size_t weight_grad_workspace(int64_t rows, int64_t outputs, int64_t cols, bool aligned);
cudaError_t launch_weight_grad(const WeightGrad& w, void* workspace, cudaStream_t stream);
// 1 if a bounded wait of these kernels has expired on the current device since the last call, -1 if
// the flag could not be read.
int take_weight_grad_timeout_flag();
int take_block_norm_timeout_flag();

}  // namespace pwlq
