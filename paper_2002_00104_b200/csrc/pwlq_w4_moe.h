// What the launches of the mixture-of-experts layer share.
#pragma once

#include <cooperative_groups.h>

#include "pwlq_w4.cuh"

namespace pwlq {

constexpr int kMaxExperts = PWLQ_W4_MOE_MAX_EXPERTS, kMaxTop = PWLQ_W4_MOE_MAX_TOP, kMaxTokens = PWLQ_W4_MOE_MAX_TOKENS;
constexpr unsigned kAll = 0xffffffffu;

// The choice of every token: its experts, largest score first, and their weights.
struct Routing {
    const int32_t* chosen;
    const float* weights;
    int tokens, experts, top;
};

// Binary32 values as the products take them, in three bf16 parts, and rows that do not lie in whole 16-byte blocks: the
// first launch leaves tokens like that in the workspace, each part in whole blocks of columns.
inline bool moe_copies(const pwlq_w4_moe_args& a) {
    return a.dtype == kF32 || a.up->cols % kBlockCols != 0 || !rows_aligned(a.x, a.ldx, 2);
}

cudaError_t launch_moe_route(const pwlq_w4_moe_args& a, const Routing& r, void* copy, cudaStream_t stream);
template <typename T>
cudaError_t launch_moe_products(const pwlq_w4_moe_args& a, const Routing& r, const void* copy, void* hidden,
                                cudaStream_t stream);

}  // namespace pwlq
