// Product of a few tokens with 4-bit weights: y[t, n] = sum over k of x[t, k] w[n, k].  The files that include this
// one instantiate it for a type each, so that they are compiled side by side.
#pragma once

#include "pwlq_w4.cuh"

namespace pwlq {
namespace {

constexpr int kWarps = 8;

// T: the type of y; S: how the activations lie.
template <typename T, class S> struct LinearArgs {
    W4View w;
    const typename S::Elem* x;
    int64_t ldx, tokens;
    int part;                              // columns of a row, or of one of its parts
    T* y;
    int64_t ldy;
    int team_shift;                        // log2 of the warps that share tiles
};

// A warp's part of MT tiles: one segment.
struct NoTag {};
template <int MT, typename T, class S> struct LinearSteps {
    const LinearArgs<T, S>* a;
    int64_t tile;
    int first, count;                                     // blocks
    int64_t token;                                        // of this lane's first column
    int bytes;                                            // of a block
    bool started = false;
    __device__ __forceinline__ bool next() { const bool yes = !started && count > 0; started = true; return yes; }
    __device__ __forceinline__ int blocks() const { return count; }
    // tiles past the last one repeat it; their sums go nowhere
    __device__ __forceinline__ const uint8_t* code(int m) const {
        return a->w.data + (min(tile + m, a->w.tiles - 1) * a->w.blocks + first) * bytes;
    }
    __device__ __forceinline__ NoTag tag() const { return {}; }
    __device__ __forceinline__ int column() const { return first * kBlockCols; }
    // columns past the last token repeat it; nobody reads their sums
    __device__ __forceinline__ const typename S::Elem* row(int n) const { return a->x + min(token + 8 * n, a->tokens - 1) * a->ldx; }
};

// A team of warps shares MT tiles along the columns.  The warps' sums meet in shared memory, where a warp's take its
// ring's place, and are added in a fixed order.
template <int MT, int NT, int ENDS, typename T, class S>
__global__ void __launch_bounds__(kWarps * 32, 2) w4_linear_kernel(const LinearArgs<T, S> a) {
    constexpr int kCols = 8 * NT, kRing = kRingBytes<MT, ENDS>, kPitch = kCols + 1;
    static_assert(kRing >= 16 * MT * kPitch * 4 && kRing % 16 == 0, "sums are larger than a ring");
    extern __shared__ __align__(16) uint8_t shared[];
    const int warp = warp_index(), lane = threadIdx.x & 31;
    const int team = 1 << a.team_shift, teams = kWarps >> a.team_shift;
    const int64_t first = (int64_t)blockIdx.x * teams, mine = first + (warp >> a.team_shift);
    const int64_t token = (int64_t)blockIdx.y * kCols;
    const int share = warp & (team - 1);
    const int begin = (a.w.blocks * share) >> a.team_shift, end = (a.w.blocks * (share + 1)) >> a.team_shift;
    float* const sums = reinterpret_cast<float*>(shared + warp * kRing);
    await_previous();
    bool none = true;
    if (mine * MT < a.w.tiles) {
        S source;
        source.cols = a.part;
        const LinearSteps<MT, T, S> steps = {&a, mine * MT, begin, end - begin, token + (lane >> 2), w4_block_bytes(ENDS)};
        w4_stream<MT, NT, ENDS>(steps, source, a.w.table, shared + warp * kRing,
                                [&](NoTag, const float (&acc)[MT][NT][4]) {
            none = false;
            __syncwarp();
#pragma unroll
            for (int m = 0; m < MT; ++m)
#pragma unroll
                for (int n = 0; n < NT; ++n)
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        sums[(16 * m + (lane >> 2) + (i & 2) * 4) * kPitch + 8 * n + 2 * (lane & 3) + (i & 1)] =
                            acc[m][n][i];
        });
    }
    if (none)
        for (int i = lane; i < 16 * MT * kPitch; i += 32) sums[i] = 0.0f;
    __syncthreads();
    const int columns = (int)min(a.tokens - token, (int64_t)kCols), each = 8 * MT * columns;
    const int64_t half = a.w.rows / 2;
    for (int i = threadIdx.x; i < teams * each; i += kWarps * 32) {
        const int k = i / each, r = i % 8, m = i / 8 % MT, c = i % each / (8 * MT);
        float lo = 0.0f, hi = 0.0f;
        for (int j = k * team; j < (k + 1) * team; ++j) {
            const float* const v = reinterpret_cast<const float*>(shared + j * kRing) + (16 * m + r) * kPitch + c;
            lo += v[0];
            hi += v[8 * kPitch];
        }
        lo *= kUnit<typename S::Mma>;
        hi *= kUnit<typename S::Mma>;
        const int64_t tile = (first + k) * MT + m;
        T* const y = a.y + (token + c) * a.ldy;
        if (a.w.paired) {
            if (tile * 8 + r < half) y[tile * 8 + r] = from_f32<T>(silu_of(lo) * hi);
        } else {
            if (tile * 16 + r < a.w.rows) y[tile * 16 + r] = from_f32<T>(lo);
            if (tile * 16 + r + 8 < a.w.rows) y[tile * 16 + r + 8] = from_f32<T>(hi);
        }
    }
}

template <int MT, int NT, int ENDS, typename T, class S>
cudaError_t launch(LinearArgs<T, S> a, cudaStream_t stream) {
    a.team_shift = 0;
    while (a.team_shift < 3 && a.w.blocks >> a.team_shift > 1) ++a.team_shift;
    const int teams = kWarps >> a.team_shift;
    const int64_t units = (a.w.tiles + MT - 1) / MT;
    constexpr size_t smem = kWarps * kRingBytes<MT, ENDS>;
    return launch_w4<smem>(w4_linear_kernel<MT, NT, ENDS, T, S>, a,
                           dim3((unsigned)((units + teams - 1) / teams), (unsigned)((a.tokens + 8 * NT - 1) / (8 * NT))),
                           kWarps * 32, smem, stream);
}

template <int ENDS, typename T, class S>
cudaError_t linear(const LinearArgs<T, S>& a, cudaStream_t stream) {
    // Two tiles at a time save a third of what is not a product, and leave half as many CTAs: 8192 x 8192 12.4
    // against 13.4 us, 22528 x 8192 27.3 against 30.1, but 14336 x 4096 13.2 against 12.2, 1024 x 4096 4.6 against 3.7.
    if (a.tokens <= 8)
        return a.w.blocks >= 64 && a.w.tiles >= 256 ? launch<2, 1, ENDS, T, S>(a, stream)
                                                    : launch<1, 1, ENDS, T, S>(a, stream);
    // sixteen at a time: the weights are taken apart again for every sixteen (64 x 8192 x 8192 bf16 45 us; decoding and a dense
    // product 60, which is less from 80 tokens on).  A kernel of larger tiles with the activations in shared memory was
    // 10 % faster at 64 x 16384 x 4096 and slower elsewhere.
    return launch<2, 2, ENDS, T, S>(a, stream);
}

template <typename T, class S>
cudaError_t linear(const LinearArgs<T, S>& a, cudaStream_t stream) {
    if (a.w.ends == 4) return linear<4, T, S>(a, stream);
    return a.w.ends == 2 ? linear<2, T, S>(a, stream) : linear<1, T, S>(a, stream);
}

}  // namespace

template <typename T>
cudaError_t w4_linear_of(const pwlq_w4& w, const void* x, bool copied, int64_t tokens, int64_t ldx, void* y, int64_t ldy,
                         cudaStream_t stream) {
    const W4View v = w4_view(w, !std::is_same<T, __half>::value);
    T* const out = static_cast<T*>(y);
    if constexpr (sizeof(T) == 2) {
        const T* const values = static_cast<const T*>(x);
        const bool aligned = copied || rows_aligned(x, ldx, sizeof(T));
        if (aligned && (copied || w.cols % kBlockCols == 0))
            return linear<T, RowsWhole<T>>({v, values, ldx, tokens, v.cols, out, ldy, 0}, stream);
        if (aligned && w.cols % 8 == 0) return linear<T, RowsEights<T>>({v, values, ldx, tokens, v.cols, out, ldy, 0}, stream);
    } else {
        if (copied)
            return linear<T, RowsParts<3>>({v, static_cast<const __nv_bfloat16*>(x), ldx, tokens, (int)w4_padded(w.cols), out,
                                            ldy, 0}, stream);
    }
    return linear<T, RowsAny<T>>({v, static_cast<const T*>(x), ldx, tokens, v.cols, out, ldy, 0}, stream);
}

}  // namespace pwlq
