// A mixture-of-experts layer for a few tokens on experts in 4-bit weights: scores and choice, gate and up
// projections with the activation, down projections with the sum over a token's experts -- three launches, each
// a dependent of the one before.
#include "pwlq_w4_moe.h"

namespace pwlq {
namespace {

// The workspace: the choice and its weights (where the caller keeps neither), and what lies between the products.
int64_t part(int64_t pairs) { return (4 * pairs + 255) / 256 * 256; }

}  // namespace

size_t w4_moe_workspace(int64_t tokens, int64_t top, int64_t hidden) {
    const int64_t pairs = tokens * top;
    return (size_t)(2 * part(pairs) + pairs * w4_padded(hidden) * 4);
}

cudaError_t launch_w4_moe(const pwlq_w4_moe_args& a, cudaStream_t stream) {
    uint8_t* const memory = static_cast<uint8_t*>(a.workspace);
    const int64_t pairs = a.tokens * a.top;
    const Routing r = {a.chosen ? a.chosen : reinterpret_cast<int32_t*>(memory),
                       a.weights ? a.weights : reinterpret_cast<float*>(memory + part(pairs)), (int)a.tokens,
                       (int)a.up->matrices, (int)a.top};
    void* const hidden = memory + 2 * part(pairs);
    const cudaError_t err = launch_moe_route(a, r, stream);
    if (err != cudaSuccess) return err;
    if (a.dtype == kF32) return launch_moe_products<float>(a, r, hidden, stream);
    if (a.dtype == kBf16) return launch_moe_products<__nv_bfloat16>(a, r, hidden, stream);
    return launch_moe_products<__half>(a, r, hidden, stream);
}

}  // namespace pwlq
