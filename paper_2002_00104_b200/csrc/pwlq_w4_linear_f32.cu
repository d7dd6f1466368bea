#include "pwlq_w4_linear.cuh"

namespace pwlq {
template cudaError_t w4_linear_of<float>(const pwlq_w4&, const void*, bool, int64_t, int64_t, void*, int64_t, cudaStream_t);
}
