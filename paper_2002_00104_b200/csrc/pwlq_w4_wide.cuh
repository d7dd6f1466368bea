// Product of some tens of tokens with 4-bit weights: what bounds it is no longer the weights but the matrix instructions
// and the activations, which every warp needs in full.
#pragma once

#include <algorithm>

#include "pwlq_w4.cuh"

namespace pwlq {
namespace {

constexpr int kWideWarps = 8;
constexpr int kWidePitch = 320;            // bytes of a token's block in shared memory: 256 and 64 against conflicts

template <typename T> struct WideArgs {
    W4View w;
    const T* x;
    int64_t ldx, tokens;
    T* y;
    int64_t ldy;
};

// Eight values of a token as its parts in 16 bits.
template <typename T> struct WidePieces {
    using Mma = T;
    static constexpr int kPieces = 1;
    static __device__ __forceinline__ void put(uint8_t* to, int, const Raw8<T>& r) { *reinterpret_cast<uint4*>(to) = r.w; }
};
template <> struct WidePieces<float> {
    using Mma = __nv_bfloat16;
    static constexpr int kPieces = 3;
    static __device__ __forceinline__ void put(uint8_t* to, int stride, const Raw8<float>& r) {
        RowsAny<float> rows;
        uint32_t b[3][4];
        rows.operand(r, b);
#pragma unroll
        for (int p = 0; p < 3; ++p) *reinterpret_cast<uint4*>(to + p * stride) = make_uint4(b[p][0], b[p][1], b[p][2], b[p][3]);
    }
};

template <int NT, typename T> constexpr int kWideStage = WidePieces<T>::kPieces * 8 * NT * kWidePitch;
template <int NT, int ENDS, typename T>
constexpr int kWideShared = std::max(2 * kWideStage<NT, T> + kWideWarps * kRingBytes<1, ENDS>,
                                     kWideWarps * 16 * (8 * NT + 1) * 4);

// A warp has a tile of 16 rows, a CTA those of its warps and 8 NT tokens; the CTAs of a cluster, along z, share the
// columns.  A block of all tokens (128 columns) lies in shared memory while the warps multiply it by their own; the
// next one is on its way in registers meanwhile.  Sums of a cluster are added in a fixed order.
template <int NT, int ENDS, bool VEC, typename T>
__global__ void __launch_bounds__(kWideWarps * 32, 1) w4_wide_kernel(const WideArgs<T> a) {
    using P = WidePieces<T>;
    constexpr int kTokens = 8 * NT, kStage = kWideStage<NT, T>, kBytes = w4_block_bytes(ENDS), kPitch = kTokens + 1;
    constexpr int kLoads = kTokens * 16 / (kWideWarps * 32), kRing = kRingBytes<1, ENDS>, kRows = kWideWarps * 16;
    extern __shared__ __align__(16) uint8_t shared[];     // two stages, rings
    const int warp = warp_index(), lane = threadIdx.x & 31, g = lane >> 2, q = lane & 3;
    const int parts = (int)gridDim.z, part = (int)blockIdx.z;
    const int begin = (int)((int64_t)a.w.blocks * part / parts), end = (int)((int64_t)a.w.blocks * (part + 1) / parts);
    const int64_t first = (int64_t)blockIdx.x * kWideWarps, token = (int64_t)blockIdx.y * kTokens;
    // tiles past the last one repeat it; their sums go nowhere
    const uint8_t* from = a.w.tile(0, min(first + warp, a.w.tiles - 1)) + (int64_t)begin * kBytes + lane * 16;
    uint8_t* const ring = shared + 2 * kStage + warp * kRing;
    const uint32_t to = (uint32_t)__cvta_generic_to_shared(ring) + lane * 16;
    const W4Table table = in_registers(a.w.table);
    Raw8<T> raw[kLoads];
    auto request = [&](int block) {
#pragma unroll
        for (int i = 0; i < kLoads; ++i) {
            const int u = (int)threadIdx.x + i * kWideWarps * 32, t = u >> 4, col = block * kBlockCols + (u & 15) * 8;
            const bool some = token + t < a.tokens;
            if (VEC && !(some && col < a.w.cols)) raw[i].clear();
            else load8<VEC>(raw[i], a.x + (some ? token + t : 0) * a.ldx + col, some ? a.w.cols - col : 0, col);
        }
    };
    auto put = [&](int stage) {
#pragma unroll
        for (int i = 0; i < kLoads; ++i) {
            const int u = (int)threadIdx.x + i * kWideWarps * 32;
            P::put(shared + stage * kStage + (u >> 4) * kWidePitch + (u & 15) * 16, kTokens * kWidePitch, raw[i]);
        }
    };
    int left = end - begin, stage = 0;
    auto fill = [&](int at) {
        copy16(to + at * kBytes, from, left > 0);
        copy16(to + at * kBytes + 512, from + 512, left > 0);
        copy16(to + at * kBytes + 1024, from + 1024, left > 0 && lane < 2 * ENDS);
        asm volatile("cp.async.commit_group;" ::: "memory");
        from += kBytes;
        --left;
    };
    await_previous();
    request(begin);
#pragma unroll
    for (int i = 0; i < kStages - 1; ++i) fill(i);
    put(0);
    __syncthreads();
    float acc[NT][4];
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int i = 0; i < 4; ++i) acc[n][i] = 0.0f;
    for (int b = begin; b < end; ++b) {
        if (b + 1 < end) request(b + 1);
        asm volatile("cp.async.wait_group %0;" ::"n"(kStages - 2) : "memory");
        __syncwarp();
        const uint8_t* const at = ring + stage * kBytes;
        const uint4 c0 = *reinterpret_cast<const uint4*>(at + lane * 16), c1 = *reinterpret_cast<const uint4*>(at + 512 + lane * 16);
        const uint32_t words[8] = {c0.x, c0.y, c0.z, c0.w, c1.x, c1.y, c1.z, c1.w};
        uint32_t scale[ENDS];
#pragma unroll
        for (int i = 0; i < ENDS; ++i) scale[i] = *reinterpret_cast<const uint32_t*>(at + 1024 + i * 32 + g * 4);
        fill((stage + kStages - 1) % kStages);
        stage = (stage + 1) % kStages;
        const uint8_t* const x = shared + ((b - begin) & 1) * kStage + g * kWidePitch + q * 16;
        float sum[NT][4];
#pragma unroll
        for (int h = 0; h < 4; ++h) {
            uint32_t operand[2][4];
#pragma unroll
            for (int j = 0; j < 2; ++j) w4_operand(words[2 * h + j], table, operand[j]);
#pragma unroll
            for (int p = 0; p < P::kPieces; ++p)
#pragma unroll
                for (int n = 0; n < NT; ++n) {
                    const uint4 v = *reinterpret_cast<const uint4*>(x + (p * kTokens + 8 * n) * kWidePitch + h * 64);
                    if (h * ENDS % 4 == 0 && p == 0) mma16816_first(sum[n], operand[0], v.x, v.y, typename P::Mma());
                    else mma16816(sum[n], operand[0], v.x, v.y, typename P::Mma());
                    mma16816(sum[n], operand[1], v.z, v.w, typename P::Mma());
                }
            if ((h + 1) * ENDS % 4 == 0) {
                const uint32_t v = scale[(h + 1) * ENDS / 4 - 1];
                const float lo = __uint_as_float(v << 16), hi = __uint_as_float(v & 0xffff0000u);
#pragma unroll
                for (int n = 0; n < NT; ++n) {
                    acc[n][0] = fmaf(lo, sum[n][0], acc[n][0]);
                    acc[n][1] = fmaf(lo, sum[n][1], acc[n][1]);
                    acc[n][2] = fmaf(hi, sum[n][2], acc[n][2]);
                    acc[n][3] = fmaf(hi, sum[n][3], acc[n][3]);
                }
            }
        }
        if (b + 1 < end) put((b + 1 - begin) & 1);
        __syncthreads();
    }
    asm volatile("cp.async.wait_all;" ::: "memory");
    __syncthreads();
    float* const sums = reinterpret_cast<float*>(shared);                // where stages and rings were
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int i = 0; i < 4; ++i) sums[(warp * 16 + g + (i & 2) * 4) * kPitch + 8 * n + 2 * q + (i & 1)] = acc[n][i];
    cooperative_groups::cluster_group cluster = cooperative_groups::this_cluster();
    if (parts > 1) cluster.sync();
    else __syncthreads();
    const int columns = (int)min(a.tokens - token, (int64_t)kTokens);
    const int64_t half = a.w.rows / 2;
    auto total = [&](int r, int c) {
        if (parts == 1) return sums[r * kPitch + c] * 256.0f;
        float s = 0.0f;
        for (int p = 0; p < parts; ++p) s += cluster.map_shared_rank(sums, p)[r * kPitch + c];
        return s * 256.0f;
    };
    // a CTA of a cluster delivers every parts-th token
    const int each = a.w.paired ? kRows / 2 : kRows;
    for (int i = threadIdx.x; i < each * ((columns - part + parts - 1) / parts); i += kWideWarps * 32) {
        const int r = i % each, c = part + i / each * parts;
        T* const y = a.y + (token + c) * a.ldy;
        if (a.w.paired) {
            const int64_t n = first * 8 + r;
            const int at = r / 8 * 16 + r % 8;
            if (n < half) y[n] = from_f32<T>(silu_of(total(at, c)) * total(at + 8, c));
        } else {
            const int64_t n = first * 16 + r;
            if (n < a.w.rows) y[n] = from_f32<T>(total(r, c));
        }
    }
    if (parts > 1) cluster.sync();                        // its shared memory is read by other CTAs
}

template <int NT, int ENDS, bool VEC, typename T>
cudaError_t launch_wide(const WideArgs<T>& a, cudaStream_t stream) {
    const int64_t ctas = (a.w.tiles + kWideWarps - 1) / kWideWarps, passes = (a.tokens + 8 * NT - 1) / (8 * NT);
    // 2, 4, 8 CTAs to a tile where there would be few: 64 x 4096 x 4096 in 24 us
    unsigned parts = 1;
    while (parts < 8 && ctas * passes * parts * 2 <= 148 && a.w.blocks >= 4 * (int)parts) parts *= 2;
    auto* const kernel = w4_wide_kernel<NT, ENDS, VEC, T>;
    const size_t smem = kWideShared<NT, ENDS, T>;
    const cudaError_t err = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
    if (err != cudaSuccess) return err;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = attr[1].val.clusterDim.y = 1;
    attr[1].val.clusterDim.z = parts;
    cudaLaunchConfig_t config = {};
    config.gridDim = dim3((unsigned)ctas, (unsigned)passes, parts);
    config.blockDim = dim3(kWideWarps * 32);
    config.dynamicSmemBytes = smem;
    config.stream = stream;
    config.attrs = attr;
    config.numAttrs = parts > 1 ? 2 : 1;
    return cudaLaunchKernelEx(&config, kernel, a);
}

template <int ENDS, bool VEC, typename T>
cudaError_t wide(const WideArgs<T>& a, cudaStream_t stream) {
    // 64 tokens at a time save taking the weights apart twice (64 x 16384 x 4096 in two passes of 32: as long, with twice
    // the CTAs); binary32 ones have three products to a value and not the registers
    if constexpr (sizeof(T) == 2) {
        if (a.tokens > 32) return launch_wide<8, ENDS, VEC, T>(a, stream);
    }
    return launch_wide<4, ENDS, VEC, T>(a, stream);
}
template <bool VEC, typename T>
cudaError_t wide(const WideArgs<T>& a, cudaStream_t stream) {
    if (a.w.ends == 4) return wide<4, VEC, T>(a, stream);
    return a.w.ends == 2 ? wide<2, VEC, T>(a, stream) : wide<1, VEC, T>(a, stream);
}

}  // namespace

// More tokens than w4_linear_of takes at a time.
template <typename T>
cudaError_t w4_wide_of(const pwlq_w4& w, const void* x, int64_t tokens, int64_t ldx, void* y, int64_t ldy,
                       cudaStream_t stream) {
    const WideArgs<T> a = {w4_view(w, !std::is_same<T, __half>::value), static_cast<const T*>(x), ldx, tokens,
                           static_cast<T*>(y), ldy};
    return w.cols % 8 == 0 && rows_aligned(x, ldx, sizeof(T)) ? wide<true, T>(a, stream) : wide<false, T>(a, stream);
}

}  // namespace pwlq
