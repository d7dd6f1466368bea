// A mixture-of-experts layer for a few tokens on experts in 4-bit weights: scores and choice, gate and up
// projections with the activation, down projections with the sum over a token's experts -- three launches, each
// a dependent of the one before.
#include <cooperative_groups.h>

#include "pwlq_w4.cuh"

namespace pwlq {
namespace {

namespace cg = cooperative_groups;

constexpr int kWarps = 8;
constexpr int kMaxExperts = PWLQ_W4_MOE_MAX_EXPERTS, kMaxTop = PWLQ_W4_MOE_MAX_TOP, kMaxTokens = PWLQ_W4_MOE_MAX_TOKENS;
constexpr unsigned kAll = 0xffffffffu;

// ---------------------------------------------------------------------------------- scores and choice
// A running sum in two binary32 parts, two sums at a time: every addition's rounding error is kept (two-sum) and,
// where the product itself is rounded, the product's too (a fused multiply-add).  The result is as good as a sum
// in twice the precision (Ogita, Rump, Oishi: Accurate sum and dot product): experts whose scores lie next to each
// other are chosen as the exact scores say, whatever the order of the sum.  Half the cost of binary64, whose
// conversions alone take longer.
template <bool ROUNDED> struct PairSum {
    u64 s = 0, c = 0;
    __device__ __forceinline__ void add(u64 x, u64 w) {
        const u64 minus = both(-1.0f);
        const u64 p = mul2(x, w);
        const u64 t = add2(s, p);
        const u64 z = fma2(s, minus, t);
        const u64 lost = add2(fma2(fma2(z, minus, t), minus, s), fma2(z, minus, p));
        c = add2(c, lost);
        if (ROUNDED) c = add2(c, fma2(x, w, mul2(p, minus)));
        s = t;
    }
    __device__ __forceinline__ double total() const {
        const double sum = (double)lo2(s) + (double)hi2(s), rest = (double)lo2(c) + (double)hi2(c);
        return isfinite(sum) ? sum + rest : sum;          // of an infinity there is no rounding error
    }
};

template <typename T, typename R> struct RouteArgs {
    const T* x;
    int64_t ldx, features;
    const R* router;
    int64_t ldr;
    int experts, top, normalize;
    int32_t* chosen;
    float* weights;
};

constexpr int kRouteCtas = 8;

// Order of the choice as whole numbers: larger scores first, NaN above all; 0 is below every score.
__device__ __forceinline__ u64 key_of(double v) {
    if (v != v) return ~0ull;
    const long long b = __double_as_longlong(v + 0.0);
    return b < 0 ? ~(u64)b : (u64)b | 1ull << 63;
}

// A cluster per token: its CTAs share the experts, one warp or several to a score; the first CTA's first warp
// chooses.
template <typename T, typename R>
__global__ void __launch_bounds__(kWarps * 32) __cluster_dims__(kRouteCtas, 1, 1)
    moe_route_kernel(const RouteArgs<T, R> a) {
    __shared__ double parts[kMaxExperts], scores[kMaxExperts];
    __shared__ u64 keys[kMaxExperts];
    cg::cluster_group cluster = cg::this_cluster();
    const int rank = (int)(blockIdx.x % kRouteCtas), warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int64_t token = blockIdx.y;
    allow_dependents();
    await_previous();
    cluster.sync();                                       // every CTA is there to be written to
    // several warps to an expert where a CTA has fewer than eight of them
    const int each = (a.experts + kRouteCtas - 1) / kRouteCtas;
    const int per = each >= 8 ? 1 : each > 3 ? 2 : each > 1 ? 4 : 8;
    const int sub = warp % per;
    double* const home = cluster.map_shared_rank(parts, 0);
    const T* const x = a.x + token * a.ldx;
    for (int i = warp / per; i < each; i += kWarps / per) {
        const int e = i * kRouteCtas + rank;
        if (e >= a.experts) break;
        const R* const r = a.router + e * a.ldr;
        PairSum<sizeof(T) == 4 || sizeof(R) == 4> sum[2];
        for (int64_t col = (sub * 32 + lane) * 8; col < a.features; col += per * 256) {
            Raw8<T> xr;
            Raw8<R> rr;
            const int valid = (int)min(a.features - col, (int64_t)64), before = (int)min(col, (int64_t)64);
            load8<false>(xr, x + col, valid, before);
            load8<false>(rr, r + col, valid, before);
            float u[8], v[8];
            xr.get(u);
            rr.get(v);
#pragma unroll
            for (int k = 0; k < 4; ++k) sum[k & 1].add(pack2(u[2 * k], u[2 * k + 1]), pack2(v[2 * k], v[2 * k + 1]));
        }
        double total = sum[0].total() + sum[1].total();
        for (int o = 16; o; o >>= 1) total += __shfl_xor_sync(kAll, total, o);
        if (lane == 0) home[e * per + sub] = total;
    }
    cluster.sync();
    if (rank != 0 || warp != 0) return;
    for (int e = lane; e < a.experts; e += 32) {
        double v = 0.0;
        for (int i = 0; i < per; ++i) v += parts[e * per + i];
        scores[e] = v;
        keys[e] = key_of(v);
    }
    __syncwarp();
    int best_of_lane = 0;
    for (int j = 0; j < a.top; ++j) {
        u64 best = 0;
        int at = kMaxExperts;
        for (int e = lane; e < a.experts; e += 32) {
            const u64 k = keys[e];
            if (k > best) { best = k; at = e; }           // the lowest of equal ones
        }
        const uint32_t high = __reduce_max_sync(kAll, (uint32_t)(best >> 32));
        if ((uint32_t)(best >> 32) != high) { best = 0; at = kMaxExperts; }
        const uint32_t low = __reduce_max_sync(kAll, (uint32_t)best);
        if ((uint32_t)best != low) at = kMaxExperts;
        at = (int)__reduce_min_sync(kAll, (unsigned)at);
        if (lane == at % 32) keys[at] = 0;
        if (lane == j) best_of_lane = at;
        __syncwarp();
    }
    const double top = scores[__shfl_sync(kAll, best_of_lane, 0)];
    // exp of a binary64 difference in binary32: exp(h + l) = exp(h) (1 + l), l below half a unit of h
    auto share = [&](double v) {
        const double d = v - top;
        const float h = (float)d;
        const float l = h > -1e30f ? (float)(d - (double)h) : 0.0f;
        const float e = expf(h);
        return fmaf(e, l, e);
    };
    const float own = lane < a.top ? share(scores[best_of_lane]) : 0.0f;
    float sum = own;
    if (!a.normalize) {
        sum = 0.0f;
        for (int e = lane; e < a.experts; e += 32) sum += share(scores[e]);
    }
    for (int o = 16; o; o >>= 1) sum += __shfl_xor_sync(kAll, sum, o);
    if (lane < a.top) {
        a.chosen[token * a.top + lane] = best_of_lane;
        a.weights[token * a.top + lane] = __fdiv_rn(own, sum);
    }
}

// ------------------------------------------------------------------------------------ the products
struct Routing {
    const int32_t* chosen;
    const float* weights;
    int tokens, experts, top;
};

// Who goes where, made by every CTA for itself: the experts that are chosen at all, and for each of them its
// (token, place) pairs, token * top + place, in ascending order.
struct Lists {
    u64 mask[kMaxExperts];                                // the tokens of an expert
    uint16_t index[kMaxExperts];
    uint16_t expert[kMaxExperts];
    uint16_t first[kMaxExperts + 1];
    uint16_t pair[kMaxTokens * kMaxTop];
    int active;
};

__device__ __forceinline__ void build_lists(Lists& l, const Routing& r) {
    const int pairs = r.tokens * r.top, threads = blockDim.x;
    for (int e = threadIdx.x; e < r.experts; e += threads) l.mask[e] = 0;
    __syncthreads();
    for (int i = threadIdx.x; i < pairs; i += threads) {
        const int t = i / r.top;
        atomicOr(reinterpret_cast<uint32_t*>(&l.mask[r.chosen[i]]) + (t >> 5), 1u << (t & 31));
    }
    __syncthreads();
    if (threadIdx.x < 32) {
        const int lane = threadIdx.x;
        int active = 0, before = 0;
        for (int base = 0; base < r.experts; base += 32) {
            const int e = base + lane;
            const int count = e < r.experts ? __popcll(l.mask[e]) : 0;
            const unsigned some = __ballot_sync(kAll, count > 0);
            int sum = count;
            for (int o = 1; o < 32; o <<= 1) {
                const int v = __shfl_up_sync(kAll, sum, o);
                if (lane >= o) sum += v;
            }
            if (count > 0) {
                const int at = active + __popc(some & ((1u << lane) - 1));
                l.index[e] = (uint16_t)at;
                l.expert[at] = (uint16_t)e;
                l.first[at] = (uint16_t)(before + sum - count);
            }
            active += __popc(some);
            before += __shfl_sync(kAll, sum, 31);
        }
        if (lane == 0) {
            l.first[active] = (uint16_t)before;
            l.active = active;
        }
    }
    __syncthreads();
    for (int i = threadIdx.x; i < pairs; i += threads) {
        const int t = i / r.top, e = r.chosen[i];
        l.pair[l.first[l.index[e]] + __popcll(l.mask[e] & ((1ull << t) - 1))] = (uint16_t)i;
    }
    __syncthreads();
}

// What lies between the two products, a row for each pair: binary32, or two bf16 parts (16 bits of each value:
// with them the result is rounded once, as if there were nothing between; one 16-bit value would add as much
// error again).  Rows are padded with zeros to whole blocks.
template <typename T> struct Hidden {
    using Source = RowsSplit;
    using Elem = __nv_bfloat16;
    static __host__ __device__ int64_t pitch(int64_t padded) { return 2 * padded; }
    static __device__ __forceinline__ void put(Elem* row, int64_t padded, int64_t i, float v) {
        const __nv_bfloat16 high = __float2bfloat16_rn(v);
        const float rest = v - __bfloat162float(high);
        row[i] = high;
        row[padded + i] = __float2bfloat16_rn(abs_bits(__bfloat162float(high)) < kInfBits ? rest : 0.0f);
    }
};
template <> struct Hidden<float> {
    using Source = RowsAny<float>;
    using Elem = float;
    static __host__ __device__ int64_t pitch(int64_t padded) { return padded; }
    static __device__ __forceinline__ void put(float* row, int64_t, int64_t i, float v) { row[i] = v; }
};

template <typename T> struct UpArgs {
    W4View w;                                             // [experts, 2 hidden, features], paired
    Routing r;
    const T* x;
    int64_t ldx;
    typename Hidden<T>::Elem* h;
    int64_t padded;                                       // hidden in whole blocks
};

template <typename T, class S>
__global__ void __launch_bounds__(kWarps * 32) moe_up_kernel(const UpArgs<T> a) {
    constexpr int kCols = 32;
    __shared__ Lists l;
    __shared__ float sums[kWarps][16][kCols + 1];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    allow_dependents();
    await_previous();
    build_lists(l, a.r);
    const int64_t items = (int64_t)l.active * a.w.tiles, hidden = a.w.rows / 2;
    const int64_t begin = a.w.blocks * warp / kWarps, end = a.w.blocks * (warp + 1) / kWarps;
    S source;
    source.cols = a.w.cols;
    for (int64_t item = blockIdx.x; item < items; item += gridDim.x) {
        const int at = (int)(item / a.w.tiles);
        const int64_t tile = item - at * a.w.tiles;
        const int e = l.expert[at], first = l.first[at], count = l.first[at + 1] - first;
        const uint4* const codes = a.w.tile_codes(e, tile);
        const uint32_t* const scales = a.w.tile_scales(e, tile);
        auto columns = [&](int c0, auto nt) {
            constexpr int NT = decltype(nt)::value;
            float acc[NT][4];
            const T* row[NT];
#pragma unroll
            for (int n = 0; n < NT; ++n) {
                const int c = min(c0 + 8 * n + (lane >> 2), count - 1);
                row[n] = a.x + (int64_t)(l.pair[first + c] / a.r.top) * a.ldx;
#pragma unroll
                for (int i = 0; i < 4; ++i) acc[n][i] = 0.0f;
            }
            w4_accumulate<NT>(acc, codes, scales, a.w, begin, end, source, row);
#pragma unroll
            for (int n = 0; n < NT; ++n)
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    sums[warp][(lane >> 2) + (i & 2) * 4][8 * n + 2 * (lane & 3) + (i & 1)] = acc[n][i];
        };
        for (int c0 = 0; c0 < count; c0 += kCols) {
            const int n = min(count - c0, kCols);
            if (n <= 8) columns(c0, std::integral_constant<int, 1>());
            else if (n <= 16) columns(c0, std::integral_constant<int, 2>());
            else columns(c0, std::integral_constant<int, 4>());
            __syncthreads();
            for (int i = threadIdx.x; i < 8 * n; i += kWarps * 32) {
                const int c = i >> 3, r = i & 7, pair = l.pair[first + c0 + c];
                float gate = 0.0f, up = 0.0f;
#pragma unroll
                for (int j = 0; j < kWarps; ++j) {
                    gate += sums[j][r][c];
                    up += sums[j][r + 8][c];
                }
                const int64_t f = tile * 8 + r;
                typename Hidden<T>::Elem* const row = a.h + pair * Hidden<T>::pitch(a.padded);
                if (f < a.padded)
                    Hidden<T>::put(row, a.padded, f,
                                   f < hidden ? silu_of(gate * 256.0f) * (up * 256.0f) * a.r.weights[pair] : 0.0f);
                if (tile == a.w.tiles - 1)
                    for (int64_t z = f + 8; z < a.padded; z += 8) Hidden<T>::put(row, a.padded, z, 0.0f);
            }
            __syncthreads();
        }
    }
}

template <typename T> struct DownArgs {
    W4View w;                                             // [experts, features, hidden]
    Routing r;
    const typename Hidden<T>::Elem* h;
    int64_t padded;
    T* y;
    int64_t ldy;
};

// A CTA (or a cluster along z) per 16 features: the blocks of all chosen experts' rows are one list that the
// warps share; a warp adds what an expert gives to its own sums, [16][tokens], and these are added in a fixed
// order at the end.
template <typename T>
__global__ void __launch_bounds__(kWarps * 32) moe_down_kernel(const DownArgs<T> a) {
    using H = Hidden<T>;
    __shared__ Lists l;
    extern __shared__ float sums[];                       // [kWarps][16][pitch]
    cg::cluster_group cluster = cg::this_cluster();
    const int parts = (int)gridDim.z, part = (int)blockIdx.z;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, q = lane & 3;
    const int pitch = a.r.tokens | 1;
    const int64_t tile = blockIdx.x;
    allow_dependents();
    float* const mine = sums + warp * 16 * pitch;
    for (int i = lane; i < 16 * pitch; i += 32) mine[i] = 0.0f;
    await_previous();
    build_lists(l, a.r);
    const int64_t blocks = a.w.blocks, total = l.active * blocks;
    const int64_t share = part * kWarps + warp, shares = parts * kWarps;
    int64_t begin = total * share / shares;
    const int64_t end = total * (share + 1) / shares;
    typename H::Source source;
    source.cols = a.padded;
    while (begin < end) {
        const int at = (int)(begin / blocks);
        const int64_t kb = begin - at * blocks, stop = min(blocks, kb + end - begin);
        const int e = l.expert[at], first = l.first[at], count = l.first[at + 1] - first;
        const uint4* const codes = a.w.tile_codes(e, tile);
        const uint32_t* const scales = a.w.tile_scales(e, tile);
        auto columns = [&](int c0, auto nt) {
            constexpr int NT = decltype(nt)::value;
            float acc[NT][4];
            const typename H::Elem* row[NT];
#pragma unroll
            for (int n = 0; n < NT; ++n) {
                row[n] = a.h + l.pair[first + min(c0 + 8 * n + g, count - 1)] * H::pitch(a.padded);
#pragma unroll
                for (int i = 0; i < 4; ++i) acc[n][i] = 0.0f;
            }
            w4_accumulate<NT>(acc, codes, scales, a.w, kb, stop, source, row);
#pragma unroll
            for (int n = 0; n < NT; ++n)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int c = c0 + 8 * n + 2 * q + (i & 1);
                    if (c < count) mine[(g + (i & 2) * 4) * pitch + l.pair[first + c] / a.r.top] += acc[n][i];
                }
            __syncwarp();
        };
        for (int c0 = 0; c0 < count; c0 += 32) {
            const int n = min(count - c0, 32);
            if (n <= 8) columns(c0, std::integral_constant<int, 1>());
            else if (n <= 16) columns(c0, std::integral_constant<int, 2>());
            else columns(c0, std::integral_constant<int, 4>());
        }
        begin += stop - kb;
    }
    if (parts > 1) cluster.sync();
    else __syncthreads();
    if (part == 0)
        for (int i = threadIdx.x; i < 16 * a.r.tokens; i += kWarps * 32) {
            const int r = i & 15, t = i >> 4;
            float sum = 0.0f;
            for (int p = 0; p < parts; ++p) {
                const float* from = parts > 1 ? cluster.map_shared_rank(sums, p) : sums;
#pragma unroll
                for (int j = 0; j < kWarps; ++j) sum += from[(j * 16 + r) * pitch + t];
            }
            const int64_t d = tile * 16 + r;
            if (d < a.w.rows) a.y[t * a.ldy + d] = from_f32<T>(sum * 256.0f);
        }
    if (parts > 1) cluster.sync();                        // its shared memory is read by another CTA
}

int64_t padded(int64_t hidden) { return w4_blocks(hidden) * kBlockCols; }

template <typename T, typename R>
cudaError_t route(const pwlq_w4_moe_args& a, const Routing& r, cudaStream_t stream) {
    const RouteArgs<T, R> q = {static_cast<const T*>(a.x), a.ldx, a.up->cols, static_cast<const R*>(a.router), a.ldrouter,
                               r.experts, r.top, a.normalize != 0, const_cast<int32_t*>(r.chosen),
                               const_cast<float*>(r.weights)};
    return launch_dependent(moe_route_kernel<T, R>, dim3(kRouteCtas, (unsigned)a.tokens), dim3(kWarps * 32), 0, stream, q);
}

template <typename T>
cudaError_t moe(const pwlq_w4_moe_args& a, cudaStream_t stream) {
    const int64_t pairs = a.tokens * a.top, pad = padded(a.down->cols);
    uint8_t* const memory = static_cast<uint8_t*>(a.workspace);
    Routing r = {};
    r.chosen = a.chosen ? a.chosen : reinterpret_cast<int32_t*>(memory);
    r.weights = a.weights ? a.weights : reinterpret_cast<float*>(memory + (4 * pairs + 255) / 256 * 256);
    r.tokens = (int)a.tokens;
    r.experts = (int)a.up->matrices;
    r.top = (int)a.top;
    auto* const h = reinterpret_cast<typename Hidden<T>::Elem*>(memory + 2 * ((4 * pairs + 255) / 256 * 256));
    const bool bf16 = !std::is_same<T, __half>::value;

    cudaError_t err = a.router_dtype == a.dtype ? route<T, T>(a, r, stream) : route<T, float>(a, r, stream);
    if (err != cudaSuccess) return err;

    const UpArgs<T> up = {w4_view(*a.up, bf16), r, static_cast<const T*>(a.x), a.ldx, h, pad};
    const int64_t most = std::min<int64_t>(r.experts, pairs) * up.w.tiles;
    const dim3 grid((unsigned)std::min<int64_t>(most, 148 * 4)), threads(kWarps * 32);
    const bool whole = a.up->cols % kBlockCols == 0 && rows_aligned(a.x, a.ldx, sizeof(T));
    if constexpr (sizeof(T) == 2) {
        err = whole ? launch_dependent(moe_up_kernel<T, RowsWhole<T>>, grid, threads, 0, stream, up)
                    : launch_dependent(moe_up_kernel<T, RowsAny<T>>, grid, threads, 0, stream, up);
    } else {
        err = launch_dependent(moe_up_kernel<T, RowsAny<T>>, grid, threads, 0, stream, up);
    }
    if (err != cudaSuccess) return err;

    const DownArgs<T> down = {w4_view(*a.down, true), r, h, pad, static_cast<T*>(a.y), a.ldy};
    int parts = 1;
    while (parts < 8 && down.w.tiles * parts < 2 * 148) parts *= 2;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = 1;
    attr[1].val.clusterDim.y = 1;
    attr[1].val.clusterDim.z = (unsigned)parts;
    cudaLaunchConfig_t config = {};
    config.gridDim = dim3((unsigned)down.w.tiles, 1, (unsigned)parts);
    config.blockDim = threads;
    config.dynamicSmemBytes = (size_t)kWarps * 16 * (r.tokens | 1) * 4;
    config.stream = stream;
    config.attrs = attr;
    config.numAttrs = parts > 1 ? 2 : 1;
    if (config.dynamicSmemBytes + sizeof(Lists) > 48 * 1024)
        err = cudaFuncSetAttribute(moe_down_kernel<T>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                   kWarps * 16 * (kMaxTokens | 1) * 4);
    return err == cudaSuccess ? cudaLaunchKernelEx(&config, moe_down_kernel<T>, down) : err;
}

}  // namespace

size_t w4_moe_workspace(int64_t tokens, int64_t top, int64_t hidden) {
    const int64_t pairs = tokens * top;
    return (size_t)(2 * ((4 * pairs + 255) / 256 * 256) + pairs * padded(hidden) * 4);
}

cudaError_t launch_w4_moe(const pwlq_w4_moe_args& a, cudaStream_t stream) {
    if (a.dtype == kF32) return moe<float>(a, stream);
    if (a.dtype == kBf16) return moe<__nv_bfloat16>(a, stream);
    return moe<__half>(a, stream);
}

}  // namespace pwlq
