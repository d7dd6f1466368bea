#include "pwlq_w4_wide.cuh"

namespace pwlq {
template cudaError_t w4_wide_of<float>(const pwlq_w4&, const void*, int64_t, int64_t, void*, int64_t, cudaStream_t);
}
