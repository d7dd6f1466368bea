// Mixture of experts: the products of the chosen experts.  The files that include this one instantiate it for a type
// each, so that they are compiled side by side.
#pragma once

#include <cmath>

#include "pwlq_w4_moe.h"

namespace pwlq {
namespace {

constexpr int kUpWarps = 8, kDownWarps = 16;

// Who goes where, made by every CTA for itself in shared memory: the experts that are chosen at all, and for each of
// them its (token, place) pairs, token * top + place, in ascending order.
struct Lists {
    u64* mask;                                            // the tokens of an expert
    uint16_t *index, *expert, *first, *pair;
    int* active;
    __device__ Lists(uint8_t* at, const Routing& r)
        : mask(reinterpret_cast<u64*>(at)), index(reinterpret_cast<uint16_t*>(mask + r.experts)), expert(index + r.experts),
          first(expert + r.experts), pair(first + r.experts + 1),
          active(reinterpret_cast<int*>(at + (bytes(r) - 16))) {}
    static constexpr __host__ __device__ int bytes(int experts, int pairs) {
        return (experts * 14 + 2 + pairs * 2 + 15) / 16 * 16 + 16;
    }
    static __host__ __device__ int bytes(const Routing& r) { return bytes(r.experts, r.tokens * r.top); }
};
constexpr int kMostLists = Lists::bytes(kMaxExperts, kMaxTokens * kMaxTop);

// Returns how many experts are active.
__device__ __forceinline__ int build_lists(const Lists& l, const Routing& r) {
    const int pairs = r.tokens * r.top, threads = blockDim.x;
    if (r.tokens == 1) {                                  // every expert once, in the order of its choice
        for (int i = threadIdx.x; i <= pairs; i += threads) {
            l.first[i] = (uint16_t)i;
            if (i < pairs) {
                l.expert[i] = (uint16_t)r.chosen[i];
                l.pair[i] = (uint16_t)i;
            }
        }
        __syncthreads();
        return pairs;
    }
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
            *l.active = active;
        }
    }
    __syncthreads();
    for (int i = threadIdx.x; i < pairs; i += threads) {
        const int t = i / r.top, e = r.chosen[i];
        l.pair[l.first[l.index[e]] + __popcll(l.mask[e] & ((1ull << t) - 1))] = (uint16_t)i;
    }
    __syncthreads();
    return *l.active;
}

// What lies between the two products, a row for each pair: three bf16 parts whose sum a value is (24 bits, and
// binary32's range), so that nothing is rounded there, whatever the tokens' type.  Two parts, 16 bits, would do for an
// error against the real numbers that a 16-bit result hides, but would move a few in a thousand results to the next
// 16-bit number, and lose what is left of large values that cancel.  Rows are padded with zeros to whole blocks.
struct Hidden {
    static constexpr int kParts = 3;
    using Source = RowsParts<kParts>;
    using Elem = __nv_bfloat16;
    static __device__ __forceinline__ void put(Elem* row, int64_t padded, int64_t i, float v) {
        float p[kParts];
        split3(v, p[0], p[1], p[2]);
#pragma unroll
        for (int k = 0; k < kParts; ++k) row[k * padded + i] = __float2bfloat16_rn(p[k]);
    }
};
// The tokens: as they are given, or the copy that the first launch has made.
template <typename T> struct Tokens { using Source = RowsWhole<T>; static constexpr int kParts = 1; };
template <> struct Tokens<float> { using Source = RowsParts<3>; static constexpr int kParts = 3; };

template <typename T> struct UpArgs {
    W4View w;                                             // [experts, 2 hidden, features], paired
    Routing r;
    const typename Tokens<T>::Source::Elem* x;
    int64_t ldx;
    int part;                                             // columns of a part of x
    Hidden::Elem* h;
    int64_t padded;                                       // hidden in whole blocks
    int team_shift;                                       // log2 of the warps of a team
};

// A warp's way through the items (MT tiles of an expert) of its team, 8 NT of the expert's tokens at a time.  A team's items
// are spread over all experts, some of which have more tokens than one pass takes.
struct UpTag { int tile, first, count; };                 // the expert's pairs of this pass
template <int MT, int NT, typename T> struct UpSteps {
    const Lists* l;
    const UpArgs<T>* a;
    int n_blocks, from, bytes;
    int at, tile, experts;                                // of the next item: the expert's number, the tile
    int step_at, step_tile, units;                        // from one item to the next, items of an expert
    int expert = 0, first = 0, count = 0;                 // count: of the expert's pairs from `first` on
    bool started = false;
    __device__ __forceinline__ bool next() {
        first += 8 * NT;
        count -= 8 * NT;
        if (count > 0) return true;
        if (started) {
            at += step_at;
            tile += step_tile;
            if (tile >= units) {
                tile -= units;
                ++at;
            }
        }
        started = true;
        if (at >= experts) return false;
        expert = l->expert[at];
        first = l->first[at];
        count = l->first[at + 1] - first;
        return true;
    }
    __device__ __forceinline__ int blocks() const { return n_blocks; }
    // a tile past the last one repeats it; its sums go nowhere
    __device__ __forceinline__ const uint8_t* code(int m) const {
        return a->w.data + ((expert * a->w.tiles + min((int64_t)tile * MT + m, a->w.tiles - 1)) * a->w.blocks + from) * bytes;
    }
    __device__ __forceinline__ UpTag tag() const { return {tile, first, count}; }
    __device__ __forceinline__ int column() const { return from * kBlockCols; }
    // columns past the last token repeat it; nobody reads their sums
    __device__ __forceinline__ const typename Tokens<T>::Source::Elem* row(int n) const {
        const int c = min(8 * n + ((int)(threadIdx.x & 31) >> 2), count - 1);
        return a->x + (int64_t)(l->pair[first + c] / a->r.top) * a->ldx;
    }
};

// A team of warps takes MT tiles, 8 gate rows and the 8 up rows that belong to them, of one expert, and shares the
// columns; teams go on from one such item to the next.
template <int MT, int NT, int ENDS, typename T>
__global__ void __launch_bounds__(kUpWarps * 32, 2) moe_up_kernel(const UpArgs<T> a) {
    constexpr int kPitch = 8 * NT + 1, kRing = kRingBytes<MT, ENDS>;
    constexpr float kScale = kUnit<typename Tokens<T>::Source::Mma>;
    extern __shared__ __align__(16) uint8_t shared[];     // rings, sums, lists
    float* const sums = reinterpret_cast<float*>(shared + kUpWarps * kRing);
    const Lists l(reinterpret_cast<uint8_t*>(sums + kUpWarps * MT * 16 * kPitch), a.r);
    const int warp = warp_index(), lane = threadIdx.x & 31;
    await_previous();
    allow_dependents();                                   // no CTA of this launch waits for a place
    const int active = build_lists(l, a.r);
    const int team = 1 << a.team_shift, teams = kUpWarps >> a.team_shift, mine = warp >> a.team_shift;
    const int part = warp & (team - 1), begin = (a.w.blocks * part) >> a.team_shift;
    const int count = ((a.w.blocks * (part + 1)) >> a.team_shift) - begin, hidden = (int)(a.w.rows / 2);
    auto meet = [&]() {                                   // the warps of a team
        if (team == 1) __syncwarp();
        else asm volatile("bar.sync %0, %1;" ::"r"(1 + mine), "r"(32 << a.team_shift) : "memory");
    };
    typename Tokens<T>::Source source;
    source.cols = a.part;
    const int item = (int)blockIdx.x * teams + mine, step = (int)gridDim.x * teams, units = (int)((a.w.tiles + MT - 1) / MT);
    const UpSteps<MT, NT, T> steps = {&l, &a, count, begin, w4_block_bytes(ENDS), item / units, item % units, active,
                                      step / units, step % units, units};
    w4_stream<MT, NT, ENDS>(steps, source, a.w.table, shared + warp * kRing,
                            [&](const UpTag& at, const float (&acc)[MT][NT][4]) {
#pragma unroll
        for (int m = 0; m < MT; ++m)
#pragma unroll
            for (int n = 0; n < NT; ++n)
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    sums[((warp * MT + m) * 16 + (lane >> 2) + (i & 2) * 4) * kPitch + 8 * n + 2 * (lane & 3) + (i & 1)] =
                        acc[m][n][i];
        meet();
        for (int i = threadIdx.x & (32 * team - 1); i < 8 * MT * min(at.count, 8 * NT); i += 32 * team) {
            const int r = i % 8, m = i / 8 % MT, c = i / (8 * MT), pair = l.pair[at.first + c];
            float gate = 0.0f, up = 0.0f;
            for (int j = mine * team; j < (mine + 1) * team; ++j) {
                gate += sums[((j * MT + m) * 16 + r) * kPitch + c];
                up += sums[((j * MT + m) * 16 + r + 8) * kPitch + c];
            }
            const int tile = at.tile * MT + m, f = tile * 8 + r;
            if (tile >= a.w.tiles) continue;
            Hidden::Elem* const to = a.h + pair * Hidden::kParts * a.padded;
            Hidden::put(to, a.padded, f,
                        f < hidden ? silu_of(gate * kScale) * (up * kScale) * a.r.weights[pair] : 0.0f);
            if (tile == a.w.tiles - 1)
                for (int z = f + 8; z < a.padded; z += 8) Hidden::put(to, a.padded, z, 0.0f);
        }
        meet();
    });
}

template <typename T> struct DownArgs {
    W4View w;                                             // [experts, features, hidden]
    Routing r;
    const Hidden::Elem* h;
    int64_t padded;
    T* y;
    int64_t ldy;
};

// A warp's way through its part of a tile's blocks, which are those of all chosen experts one after another.
struct DownTag { int first, count; };
template <int MT, typename T> struct DownSteps {
    const Lists* l;
    const DownArgs<T>* a;
    int64_t tile;                                         // the first of MT
    int now, end, bytes;                                  // the block after this segment, the last one
    int expert = 0, first = 0, count = 0, from = 0, n_blocks = 0;
    __device__ __forceinline__ bool next() {
        first += 8;
        count -= 8;
        if (count > 0) return true;
        if (now >= end) return false;
        const int at = now / a->w.blocks;
        from = now - at * a->w.blocks;
        n_blocks = min(a->w.blocks - from, end - now);
        now += n_blocks;
        expert = l->expert[at];
        first = l->first[at];
        count = l->first[at + 1] - first;
        return true;
    }
    __device__ __forceinline__ int blocks() const { return n_blocks; }
    // a tile past the last one repeats it; its sums go nowhere
    __device__ __forceinline__ const uint8_t* code(int m) const {
        return a->w.data + ((expert * a->w.tiles + min(tile + m, a->w.tiles - 1)) * a->w.blocks + from) * bytes;
    }
    __device__ __forceinline__ DownTag tag() const { return {first, count}; }
    __device__ __forceinline__ int column() const { return from * kBlockCols; }
    __device__ __forceinline__ const Hidden::Elem* row(int) const {
        const int c = min((int)(threadIdx.x & 31) >> 2, count - 1);
        return a->h + l->pair[first + c] * Hidden::kParts * a->padded;
    }
};

// A CTA per MT tiles of 16 features: the blocks of all chosen experts' rows are one list that the warps share; a warp
// adds what an expert gives to its own sums, [16 MT][tokens], and these are added in a fixed order at the end.  So no
// partial sum leaves the CTA; what is left is that 128 or 256 CTAs do not divide by 148.  An expert's tokens are taken eight
// at a time: sixteen leave too few registers for activations of three parts ahead (64 tokens, 8 of 32 experts of 3 x 768 x
// 2048 bf16, the whole layer: 109 us, 95 with eight; 2 of 8 of 3 x 2048 x 4096 131, 120).  4 tokens, 2 of 8 experts of 4096 x
// 8192: 50 us; with single tiles 55.
template <int MT, int ENDS, typename T>
__global__ void __launch_bounds__(kDownWarps * 32, 1) moe_down_kernel(const DownArgs<T> a) {
    constexpr int kRing = kRingBytes<MT, ENDS>, kRows = 16 * MT;
    extern __shared__ __align__(16) uint8_t shared[];     // rings, sums, lists
    const int warp = warp_index(), lane = threadIdx.x & 31, g = lane >> 2, q = lane & 3;
    const int pitch = a.r.tokens | 1;
    float* const sums = reinterpret_cast<float*>(shared + kDownWarps * kRing);
    float* const mine = sums + warp * kRows * pitch;
    const Lists l(reinterpret_cast<uint8_t*>(sums + kDownWarps * kRows * pitch), a.r);
    for (int i = lane; i < kRows * pitch; i += 32) mine[i] = 0.0f;
    await_previous();
    const int total = build_lists(l, a.r) * a.w.blocks;
    Hidden::Source source;
    source.cols = (int)a.padded;
    const DownSteps<MT, T> steps = {&l, &a, (int64_t)blockIdx.x * MT, (int)((int64_t)total * warp / kDownWarps),
                                        (int)((int64_t)total * (warp + 1) / kDownWarps), w4_block_bytes(ENDS)};
    w4_stream<MT, 1, ENDS>(steps, source, a.w.table, shared + warp * kRing,
                           [&](const DownTag& at, const float (&acc)[MT][1][4]) {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const int c = 2 * q + i;
            if (c >= at.count) continue;
            float* const to = mine + g * pitch + l.pair[at.first + c] / a.r.top;
#pragma unroll
            for (int m = 0; m < MT; ++m) {
                to[16 * m * pitch] += acc[m][0][i];
                to[(16 * m + 8) * pitch] += acc[m][0][i + 2];
            }
        }
        __syncwarp();
    });
    __syncthreads();
    for (int i = threadIdx.x; i < kRows * a.r.tokens; i += kDownWarps * 32) {
        const int r = i % kRows, t = i / kRows;
        float sum = 0.0f;
#pragma unroll
        for (int j = 0; j < kDownWarps; ++j) sum += sums[(j * kRows + r) * pitch + t];
        const int64_t d = (int64_t)blockIdx.x * kRows + r;
        if (d < a.w.rows) a.y[t * a.ldy + d] = from_f32<T>(sum * kUnit<Hidden::Source::Mma>);
    }
}

template <typename F>
cudaError_t with_ends(int ends, F f) {
    if (ends == 4) return f(std::integral_constant<int, 4>());
    return ends == 2 ? f(std::integral_constant<int, 2>()) : f(std::integral_constant<int, 1>());
}

template <int MT, int NT, typename T>
cudaError_t up_launch(UpArgs<T> a, cudaStream_t stream) {
    const int64_t units = (a.w.tiles + MT - 1) / MT, most = std::min<int64_t>(a.r.experts, (int64_t)a.r.tokens * a.r.top) * units;
    // Teams of two; larger ones where the items of as many experts as the tokens would choose at random leave
    // multiprocessors empty.  4 tokens, 8 experts of 2 x 8192 x 4096, single tiles: 72.5, 68.5, 73.4, 82.6 us with teams of
    // 1, 2, 4, 8 (the last ones meet more often than they multiply); 5 tokens, 17 experts of 2 x 515 x 1287: 21.1, 14.2, 11.2,
    // 12.4.
    const double spared = std::pow(1.0 - (double)a.r.top / a.r.experts, a.r.tokens);
    const double items = a.r.experts * (1.0 - spared) * (double)units;
    a.team_shift = a.w.blocks >= 2;
    while (a.team_shift < 3 && items * (1 << a.team_shift) < 12 * kMultiprocessors && a.w.blocks >> a.team_shift > 1) ++a.team_shift;
    const int64_t ctas = ((most << a.team_shift) + kUpWarps - 1) / kUpWarps;
    return with_ends(a.w.ends, [&](auto ends) {
        constexpr int kEnds = decltype(ends)::value;
        constexpr size_t kRings = kUpWarps * (kRingBytes<MT, kEnds> + MT * 16 * (8 * NT + 1) * 4);
        return launch_w4<kRings + kMostLists>(moe_up_kernel<MT, NT, kEnds, T>, a,
                                              dim3((unsigned)std::min<int64_t>(ctas, 2 * kMultiprocessors)), kUpWarps * 32,
                                              kRings + Lists::bytes(a.r), stream);
    });
}

constexpr int kPairedTokens = 8;         // of two tiles at a time: the warps' sums of many tokens leave no room for them

template <int MT, typename T>
cudaError_t down_launch(const DownArgs<T>& a, cudaStream_t stream) {
    return with_ends(a.w.ends, [&](auto ends) {
        constexpr int kEnds = decltype(ends)::value;
        const auto smem = [](int tokens) { return (size_t)kDownWarps * (kRingBytes<MT, kEnds> + MT * 16 * (tokens | 1) * 4); };
        return launch_w4<smem(MT == 2 ? kPairedTokens : kMaxTokens) + kMostLists>(
            moe_down_kernel<MT, kEnds, T>, a, dim3((unsigned)((a.w.tiles + MT - 1) / MT)), kDownWarps * 32,
            smem(a.r.tokens) + Lists::bytes(a.r), stream);
    });
}

// How much of a last round of single CTAs to a multiprocessor is used.
inline double filled(int64_t ctas) {
    return (double)ctas / (double)((ctas + kMultiprocessors - 1) / kMultiprocessors * kMultiprocessors);
}

template <int NT, typename T>
cudaError_t products(const pwlq_w4_moe_args& a, const Routing& r, const void* copy, void* hidden, cudaStream_t stream) {
    const int64_t padded = w4_padded(a.down->cols), part = w4_padded(a.up->cols);
    auto* const h = static_cast<Hidden::Elem*>(hidden);
    const bool copied = moe_copies(a);
    const UpArgs<T> up = {w4_view(*a.up, !std::is_same<T, __half>::value), r,
                          static_cast<const typename Tokens<T>::Source::Elem*>(copied ? copy : a.x),
                          copied ? part * Tokens<T>::kParts : a.ldx, (int)part, h, padded, 0};
    // two tiles at a time, eight tokens or fewer: as in the linear layer, where rows are long and many
    cudaError_t err;
    if constexpr (NT == 1) {
        err = up.w.blocks >= 32 && up.w.tiles >= 256 ? up_launch<2, NT, T>(up, stream) : up_launch<1, NT, T>(up, stream);
    } else {
        err = up_launch<1, NT, T>(up, stream);
    }
    if (err != cudaSuccess) return err;
    const DownArgs<T> down = {w4_view(*a.down, true), r, h, padded, static_cast<T*>(a.y), a.ldy};
    return a.tokens <= kPairedTokens && filled((down.w.tiles + 1) / 2) >= filled(down.w.tiles) ? down_launch<2, T>(down, stream)
                                                                                              : down_launch<1, T>(down, stream);
}

}  // namespace

template <typename T>
cudaError_t launch_moe_products(const pwlq_w4_moe_args& a, const Routing& r, const void* copy, void* hidden,
                                cudaStream_t stream) {
    // the up projections take an expert's tokens eight or sixteen at a time: they are, on average, few
    return a.tokens <= 8 || a.tokens * a.top <= 6 * r.experts ? products<1, T>(a, r, copy, hidden, stream)
                                                              : products<2, T>(a, r, copy, hidden, stream);
}

}  // namespace pwlq
