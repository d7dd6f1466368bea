// A mixture-of-experts layer for a few tokens on experts in 4-bit weights: scores and choice, gate and up
// projections with the activation, down projections with the sum over a token's experts -- three launches, each
// a dependent of the one before.
#include "pwlq_w4_moe.h"

namespace pwlq {
namespace {

// The workspace: the choice and its weights (where the caller keeps neither), the tokens in parts, and what lies between
// the products in parts.
size_t whole(int64_t bytes) { return (size_t)(bytes + 255) / 256 * 256; }

}  // namespace

size_t w4_moe_workspace(int64_t tokens, int64_t top, int64_t features, int64_t hidden) {
    return 2 * whole(4 * tokens * top) + whole(6 * tokens * w4_padded(features)) + whole(6 * tokens * top * w4_padded(hidden));
}

cudaError_t launch_w4_moe(const pwlq_w4_moe_args& a, cudaStream_t stream) {
    uint8_t* memory = static_cast<uint8_t*>(a.workspace);
    auto take = [&](int64_t bytes) { uint8_t* const p = memory; memory += whole(bytes); return p; };
    uint8_t* const chosen = take(4 * a.tokens * a.top);
    uint8_t* const weights = take(4 * a.tokens * a.top);
    const Routing r = {a.chosen ? a.chosen : reinterpret_cast<int32_t*>(chosen),
                       a.weights ? a.weights : reinterpret_cast<float*>(weights), (int)a.tokens, (int)a.up->matrices,
                       (int)a.top};
    void* const copy = take(6 * a.tokens * w4_padded(a.up->cols));
    const cudaError_t err = launch_moe_route(a, r, copy, stream);
    if (err != cudaSuccess) return err;
    if (a.dtype == kF32) return launch_moe_products<float>(a, r, copy, memory, stream);
    if (a.dtype == kBf16) return launch_moe_products<__nv_bfloat16>(a, r, copy, memory, stream);
    return launch_moe_products<__half>(a, r, copy, memory, stream);
}

}  // namespace pwlq
