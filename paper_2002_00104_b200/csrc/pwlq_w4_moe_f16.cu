#include "pwlq_w4_moe.cuh"

namespace pwlq {
template cudaError_t launch_moe_products<__half>(const pwlq_w4_moe_args&, const Routing&, const void*, void*, cudaStream_t);
}
