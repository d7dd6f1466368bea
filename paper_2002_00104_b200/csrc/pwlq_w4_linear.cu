// Product of a few tokens with 4-bit weights: y[t, n] = sum over k of x[t, k] w[n, k].
#include <cooperative_groups.h>

#include "pwlq_w4.cuh"

namespace pwlq {
namespace {

namespace cg = cooperative_groups;

constexpr int kWarps = 8;

template <typename T> struct LinearArgs {
    W4View w;
    const T* x;
    int64_t ldx, tokens;
    T* y;
    int64_t ldy;
};

// A CTA has kWarps / WK tiles of 16 rows, each of which WK warps share along the columns (with the other CTAs of its
// cluster, which is along z).  The warps' sums meet in shared memory and are added in a fixed order.
template <int NT, int WK, typename T, class S>
__global__ void __launch_bounds__(kWarps * 32) w4_linear_kernel(const LinearArgs<T> a) {
    constexpr int kTiles = kWarps / WK, kCols = 8 * NT;
    __shared__ float sums[kWarps][16][kCols + 1];
    cg::cluster_group cluster = cg::this_cluster();
    const int parts = (int)gridDim.z, part = (int)blockIdx.z;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int64_t first = (int64_t)blockIdx.x * kTiles, tile = first + warp / WK;
    const int64_t token = (int64_t)blockIdx.y * kCols;
    allow_dependents();
    const bool some = tile < a.w.tiles;
    const int64_t share = part * WK + warp % WK, shares = parts * WK;
    const int64_t begin = a.w.blocks * share / shares, end = a.w.blocks * (share + 1) / shares;
    await_previous();
    float acc[NT][4];
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int i = 0; i < 4; ++i) acc[n][i] = 0.0f;
    if (some && begin < end) {
        const T* row[NT];
        // columns past the last token repeat it; nobody reads their sums
#pragma unroll
        for (int n = 0; n < NT; ++n) row[n] = a.x + min(token + 8 * n + (lane >> 2), a.tokens - 1) * a.ldx;
        S source;
        source.cols = a.w.cols;
        w4_accumulate<NT>(acc, a.w.tile_codes(0, tile), a.w.tile_scales(0, tile), a.w, begin, end, source, row);
    }
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int i = 0; i < 4; ++i) sums[warp][(lane >> 2) + (i & 2) * 4][8 * n + 2 * (lane & 3) + (i & 1)] = acc[n][i];
    if (parts > 1) cluster.sync();
    else __syncthreads();
    if (part == 0) {
        const int64_t half = a.w.rows / 2;
        for (int i = threadIdx.x; i < kTiles * 8 * kCols; i += kWarps * 32) {
            const int c = i / 8 % kCols, r = i % 8, k = i / (8 * kCols);
            float lo = 0.0f, hi = 0.0f;
            for (int p = 0; p < parts; ++p) {
                const float* from = parts > 1 ? cluster.map_shared_rank(&sums[0][0][0], p) : &sums[0][0][0];
#pragma unroll
                for (int j = 0; j < WK; ++j) {
                    lo += from[((k * WK + j) * 16 + r) * (kCols + 1) + c];
                    hi += from[((k * WK + j) * 16 + r + 8) * (kCols + 1) + c];
                }
            }
            lo *= 256.0f;
            hi *= 256.0f;
            const int64_t t = token + c;
            if (t >= a.tokens) continue;
            T* const y = a.y + t * a.ldy;
            if (a.w.paired) {
                const int64_t n = (first + k) * 8 + r;
                if (n < half) y[n] = from_f32<T>(silu_of(lo) * hi);
            } else {
                const int64_t n = (first + k) * 16 + r;
                if (n < a.w.rows) y[n] = from_f32<T>(lo);
                if (n + 8 < a.w.rows) y[n + 8] = from_f32<T>(hi);
            }
        }
    }
    if (parts > 1) cluster.sync();                        // its shared memory is read by another CTA
}

template <int NT, int WK, typename T, class S>
cudaError_t launch(const LinearArgs<T>& a, int parts, cudaStream_t stream) {
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = 1;
    attr[1].val.clusterDim.y = 1;
    attr[1].val.clusterDim.z = (unsigned)parts;
    cudaLaunchConfig_t config = {};
    const int tiles = kWarps / WK;
    config.gridDim = dim3((unsigned)((a.w.tiles + tiles - 1) / tiles), (unsigned)((a.tokens + 8 * NT - 1) / (8 * NT)),
                          (unsigned)parts);
    config.blockDim = dim3(kWarps * 32);
    config.stream = stream;
    config.attrs = attr;
    config.numAttrs = parts > 1 ? 2 : 1;
    return cudaLaunchKernelEx(&config, w4_linear_kernel<NT, WK, T, S>, a);
}

template <typename T, class S>
cudaError_t linear(const LinearArgs<T>& a, cudaStream_t stream) {
    int parts = 1;
    while (parts < 8 && a.w.tiles * parts < 148 && a.w.blocks >= parts * 2 * kWarps) parts *= 2;
    if (a.tokens <= 8) return launch<1, 8, T, S>(a, parts, stream);
    if (a.tokens <= 16) return launch<2, 8, T, S>(a, parts, stream);
    return launch<4, 8, T, S>(a, parts, stream);
}

template <typename T>
cudaError_t linear_of(const pwlq_w4& w, const void* x, int64_t tokens, int64_t ldx, void* y, int64_t ldy, bool whole,
                      cudaStream_t stream) {
    const LinearArgs<T> a = {w4_view(w, !std::is_same<T, __half>::value), static_cast<const T*>(x), ldx, tokens,
                             static_cast<T*>(y), ldy};
    if constexpr (sizeof(T) == 2) {
        if (whole) return linear<T, RowsWhole<T>>(a, stream);
    }
    return linear<T, RowsAny<T>>(a, stream);
}

}  // namespace

cudaError_t launch_w4_linear(const pwlq_w4& w, const void* x, int dtype, int64_t tokens, int64_t ldx, void* y,
                             int64_t ldy, cudaStream_t stream) {
    const bool whole = w.cols % kBlockCols == 0 && rows_aligned(x, ldx, type_size(dtype));
    if (dtype == kF32) return linear_of<float>(w, x, tokens, ldx, y, ldy, whole, stream);
    if (dtype == kBf16) return linear_of<__nv_bfloat16>(w, x, tokens, ldx, y, ldy, whole, stream);
    return linear_of<__half>(w, x, tokens, ldx, y, ldy, whole, stream);
}

}  // namespace pwlq
