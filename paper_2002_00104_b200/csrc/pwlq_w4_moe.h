// What the launches of the mixture-of-experts layer share.
#pragma once

#include <cooperative_groups.h>

#include "pwlq_w4.cuh"

namespace pwlq {

constexpr int kMoeWarps = 8;
constexpr int kMaxExperts = PWLQ_W4_MOE_MAX_EXPERTS, kMaxTop = PWLQ_W4_MOE_MAX_TOP, kMaxTokens = PWLQ_W4_MOE_MAX_TOKENS;
constexpr unsigned kAll = 0xffffffffu;

// The choice of every token: its experts, largest score first, and their weights.
struct Routing {
    const int32_t* chosen;
    const float* weights;
    int tokens, experts, top;
};

inline int64_t w4_padded(int64_t cols) { return w4_blocks(cols) * kBlockCols; }

cudaError_t launch_moe_route(const pwlq_w4_moe_args& a, const Routing& r, cudaStream_t stream);
template <typename T>
cudaError_t launch_moe_products(const pwlq_w4_moe_args& a, const Routing& r, void* hidden, cudaStream_t stream);

}  // namespace pwlq
