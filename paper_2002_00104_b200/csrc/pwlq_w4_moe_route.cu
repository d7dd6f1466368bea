// Mixture of experts: the scores of a token and its choice of experts.
#include <utility>

#include "pwlq_w4_moe.h"

namespace pwlq {
namespace {

namespace cg = cooperative_groups;

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
    void* copy;                                           // of the tokens, or null
    int64_t padded;                                       // columns of a part
};

constexpr int kRouteCtas = 8;

// Order of the choice as whole numbers: larger scores first, NaN above all; 0 is below every score.
__device__ __forceinline__ u64 key_of(double v) {
    if (v != v) return ~0ull;
    const long long b = __double_as_longlong(v + 0.0);
    return b < 0 ? ~(u64)b : (u64)b | 1ull << 63;
}

constexpr int kMostWarps = 32;

// A token for the products: its values in 16 bits, or the three parts of binary32 ones, zeros behind the last column.
template <typename T, typename R>
__device__ __forceinline__ void copy_part(const RouteArgs<T, R>& a, const T* x, int64_t token, int first, int step) {
    for (int64_t i = first; i < a.padded; i += step) {
        const T v = i < a.features ? x[i] : from_f32<T>(0.0f);
        if constexpr (sizeof(T) == 4) {
            float p[3];
            split3(v, p[0], p[1], p[2]);
            __nv_bfloat16* const to = static_cast<__nv_bfloat16*>(a.copy) + token * 3 * a.padded + i;
#pragma unroll
            for (int k = 0; k < 3; ++k) to[k * a.padded] = __float2bfloat16_rn(p[k]);
        } else {
            static_cast<T*>(a.copy)[token * a.padded + i] = v;
        }
    }
}

// A cluster per token: its CTAs share the experts, all warps of a CTA are at work on them, several to a score where
// there are few; the first CTA's first warp chooses.  What it costs for one token is latency: a warp requests its
// first kBatch parts of a score at once (64 experts of 2048 7.9 us alone, 10.9 with eight warps to a CTA).  64 tokens, 128
// experts: 17 us, half of it issue.  VEC: rows on 16-byte boundaries, of whole eights.
template <bool VEC, typename T, typename R>
__global__ void __launch_bounds__(kMostWarps * 32) __cluster_dims__(kRouteCtas, 1, 1)
    moe_route_kernel(const RouteArgs<T, R> a) {
    constexpr int kBatch = 2;
    __shared__ double parts[kMaxExperts], scores[kMaxExperts];
    __shared__ u64 keys[kMaxExperts];
    cg::cluster_group cluster = cg::this_cluster();
    const int rank = (int)(blockIdx.x % kRouteCtas), warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int64_t token = blockIdx.y;
    allow_dependents();                                   // few CTAs: the next launch may take its places
    auto arrived = cluster.barrier_arrive();
    const int each = (a.experts + kRouteCtas - 1) / kRouteCtas;
    const int warps = blockDim.x >> 5;
    int per = 1;                                          // warps to a score
    while (each * per * 2 <= warps) per *= 2;
    const int sub = warp % per;
    double* const home = cluster.map_shared_rank(parts, 0);
    const T* const x = a.x + token * a.ldx;
    await_previous();
    if (a.copy) copy_part(a, x, token, rank * (int)blockDim.x + (int)threadIdx.x, kRouteCtas * (int)blockDim.x);
    bool met = false;
    for (int i = warp / per; i < each; i += warps / per) {
        const int e = i * kRouteCtas + rank;
        if (e >= a.experts) break;
        const R* const r = a.router + e * a.ldr;
        PairSum<sizeof(T) == 4 || sizeof(R) == 4> sum[2];
        for (int64_t at = (sub * 32 + lane) * 8; at < a.features; at += kBatch * per * 256) {
            Raw8<T> xr[kBatch];
            Raw8<R> rr[kBatch];
#pragma unroll
            for (int k = 0; k < kBatch; ++k) {
                const int64_t col = at + k * per * 256;
                const int valid = (int)max((int64_t)-8, min(a.features - col, (int64_t)64)), before = (int)min(col, (int64_t)64);
                if (VEC && valid <= 0) {
                    xr[k].clear();
                    rr[k].clear();
                } else {
                    load8<VEC>(xr[k], x + col, valid, before);
                    load8<VEC>(rr[k], r + col, valid, before);
                }
            }
#pragma unroll
            for (int k = 0; k < kBatch; ++k) {
                float u[8], v[8];
                xr[k].get(u);
                rr[k].get(v);
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    sum[j & 1].add(pack2(u[2 * j], u[2 * j + 1]), pack2(v[2 * j], v[2 * j + 1]));
            }
        }
        double total = sum[0].total() + sum[1].total();
        for (int o = 16; o; o >>= 1) total += __shfl_xor_sync(kAll, total, o);
        if (!met) {                                       // every CTA is there to be written to
            cluster.barrier_wait(std::move(arrived));
            met = true;
        }
        if (lane == 0) home[e * per + sub] = total;
    }
    if (!met) cluster.barrier_wait(std::move(arrived));
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

template <typename T, typename R>
cudaError_t route(const pwlq_w4_moe_args& a, const Routing& r, void* copy, cudaStream_t stream) {
    const RouteArgs<T, R> q = {static_cast<const T*>(a.x), a.ldx, a.up->cols, static_cast<const R*>(a.router), a.ldrouter,
                               r.experts, r.top, a.normalize != 0, const_cast<int32_t*>(r.chosen),
                               const_cast<float*>(r.weights), moe_copies(a) ? copy : nullptr, w4_padded(a.up->cols)};
    const bool vec = a.up->cols % 8 == 0 && rows_aligned(a.x, a.ldx, sizeof(T)) && rows_aligned(a.router, a.ldrouter, sizeof(R));
    // all warps that fit for a few tokens; for many the multiprocessors are full anyway
    const unsigned warps = a.tokens <= 8 ? kMostWarps : 8;
    return launch_dependent(vec ? moe_route_kernel<true, T, R> : moe_route_kernel<false, T, R>,
                            dim3(kRouteCtas, (unsigned)a.tokens), dim3(warps * 32), 0, stream, q);
}

}  // namespace

cudaError_t launch_moe_route(const pwlq_w4_moe_args& a, const Routing& r, void* copy, cudaStream_t stream) {
    if (a.dtype == kF32) return route<float, float>(a, r, copy, stream);
    if (a.dtype == kBf16)
        return a.router_dtype == kF32 ? route<__nv_bfloat16, float>(a, r, copy, stream)
                                      : route<__nv_bfloat16, __nv_bfloat16>(a, r, copy, stream);
    return a.router_dtype == kF32 ? route<__half, float>(a, r, copy, stream) : route<__half, __half>(a, r, copy, stream);
}

}  // namespace pwlq
