// Weight gradient of a projection from the 8-bit checkpoint of its input:
// dw[n, k] = sum over t of dy[t, n] * xhat[t, k], xhat rounded to dy's type.
#include "pwlq_act8.cuh"
#include "pwlq_train.h"

namespace pwlq {
namespace {

constexpr int kTile = 64, kStep = 16;

// One 64 x 64 tile of dw per CTA, 4 x 4 sums per thread, kStep rows staged at a time.
template <typename T, typename W>
__global__ void __launch_bounds__(256) weight_grad_kernel(WeightGrad w, int group_shift) {
    __shared__ float sy[kStep][kTile], sx[kStep][kTile];
    const T* dy = static_cast<const T*>(w.dy);
    const int64_t n0 = (int64_t)blockIdx.y * kTile, k0 = (int64_t)blockIdx.x * kTile;
    const int tn = threadIdx.x / 16, tk = threadIdx.x % 16;
    const int64_t groups = w.x.groups();
    float acc[4][4] = {};
    for (int64_t t0 = 0; t0 < w.rows; t0 += kStep) {
        for (int i = threadIdx.x; i < kStep * kTile; i += 256) {
            const int64_t t = t0 + i / kTile, n = n0 + i % kTile, k = k0 + i % kTile;
            sy[i / kTile][i % kTile] =
                t < w.rows && n < w.outputs ? to_f32(dy[t * w.lddy + n]) : 0.0f;
            float v = 0.0f;
            if (t < w.rows && k < w.x.cols)
                v = act8_value(w.x.codes[t * w.x.ldc + k],
                               act8_params(w.x.ranges[t * groups + (k >> group_shift)], w.x.ratio));
            sx[i / kTile][i % kTile] = to_f32(from_f32<T>(v));
        }
        __syncthreads();
#pragma unroll
        for (int t = 0; t < kStep; ++t)
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    acc[i][j] = fmaf(sy[t][tn * 4 + i], sx[t][tk + 16 * j], acc[i][j]);
        __syncthreads();
    }
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int64_t n = n0 + tn * 4 + i, k = k0 + tk + 16 * j;
            if (n >= w.outputs || k >= w.x.cols) continue;
            W* at = static_cast<W*>(w.dw) + n * w.lddw + k;
            *at = from_f32<W>(w.accumulate ? acc[i][j] + to_f32(*at) : acc[i][j]);
        }
}

template <typename T>
cudaError_t launch(const WeightGrad& w, cudaStream_t stream) {
    const dim3 grid((unsigned)((w.x.cols + kTile - 1) / kTile),
                    (unsigned)((w.outputs + kTile - 1) / kTile));
    auto* kernel = w.dw_dtype == kF32 ? weight_grad_kernel<T, float> : weight_grad_kernel<T, T>;
    kernel<<<grid, 256, 0, stream>>>(w, group_shift(w.x.group));
    return cudaGetLastError();
}

}  // namespace

size_t weight_grad_workspace(int64_t, int64_t, int64_t) { return 256; }

cudaError_t launch_weight_grad(const WeightGrad& w, void*, cudaStream_t stream) {
    return w.dtype == kBf16 ? launch<__nv_bfloat16>(w, stream) : launch<__half>(w, stream);
}

}  // namespace pwlq
