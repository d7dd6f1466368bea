// Norms around a gated residual block, forward and backward (formulas: include/pwlq.h).
//
// Both directions are bound by HBM: per value the forward pass reads x and f and writes r and h
// (and two bytes when it saves), the backward pass reads dh, dr and two bytes and writes dx and df.
// A row is owned by one CTA, eight consecutive values per thread and step, and stays on chip between
// the two reductions that depend on one another (of f, then of r; of the outer norm, then of the
// inner one), so every operand crosses HBM once.
//
// Times in this file are of whole calls (backward with its sums) in a CUDA graph of calls back to back, on
// operands larger than the L2 cache together, which still holds some of the last call's writes.
//
// Forms (the rules and both sides of each stand at the launches, at the end of this file):
//   narrow   rows of at most 1024 bytes: a few lanes per row, no barrier (400000 x 64 bf16: forward 36 us, a CTA
//            per row 236; backward 76 against 432)
//   ring     persistent CTAs walk the rows, and a ring of shared-memory stages holds the next ones, brought in by
//            bulk copies: a row's loads are in flight during the reductions of the rows before it, at no cost in
//            registers, and a thread works on 32 bytes of columns, which shares the cost of reductions and ranges
//            (16384 x 4096 bf16: with checkpoints 142 us = 4750 GB/s against 213, backward 152 us = 4440 GB/s against
//            243).  With checkpoints bound by instruction issue, 61 per value at 3.1 a cycle of 4.  Backward 52 per
//            value at 2.5 a cycle: 122 registers a thread leave 16 warps a multiprocessor, too few to cover the
//            latency of what they wait for, the barriers among it.
//            Backward, a pair of CTAs shares rows too wide for one CTA's registers (4096 x 12288: 218 against 314 us).
//            Binary32 weights beside 16-bit values take twice the registers and the loads (16384 x 4096 with a gate:
//            189 and 221 us against 147 and 163), and 12 bytes a thread spill, 124 backward on unaligned rows.
//   row      forward without checkpoints, one CTA per row, 32 bytes of columns per thread
//   direct   a thread loads its values itself, eight at a time: few rows, and rows off their alignment that the
//            ring does not take (see load8)
#include <algorithm>
#include <mutex>
#include <type_traits>

#include "pwlq_act8.cuh"
#include "pwlq_pipeline.cuh"
#include "pwlq_train.h"

namespace pwlq {

static __device__ int g_block_norm_timeout;     // a bounded wait expired

namespace {

// Stages of a ring.  Two hold the row at hand and the next one of every CTA, around 100 KB a multiprocessor in
// flight; what they leave is cache for the weights, which every row reads again (8 stages where they fit:
// 8192 x 8192 bf16 with gates backward 188 against 182 us, 10922 x 6144 200 against 194, 16384 x 4096 166 against
// 163; forward 0 to 2 % slower).
constexpr int kMaxStages = 2;

// Sum over the CTA (of up to 32 warps), the same value in every thread, in a fixed order.  Calls alternate between the
// two halves of `buf`, so one barrier per call is enough: a half is written again only after the
// barrier of the call in between.  After a call every thread of the CTA has arrived at it.
struct CtaSum {
    float (*buf)[32];
    int half = 0;
    // post() hands a thread's part in, total() waits for the others'; what does not need the sum goes
    // in between.
    __device__ __forceinline__ void post(float v) {
        for (int o = 16; o; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
        if ((threadIdx.x & 31) == 0) buf[half][threadIdx.x >> 5] = v;
    }
    __device__ __forceinline__ float total() {
        const int lane = threadIdx.x & 31, warps = blockDim.x >> 5;
        __syncthreads();
        float v = lane < warps ? buf[half][lane] : 0.0f;
        if (warps > 8) {
            v += __shfl_xor_sync(0xffffffffu, v, 16);
            v += __shfl_xor_sync(0xffffffffu, v, 8);
        }
        v += __shfl_xor_sync(0xffffffffu, v, 4);
        v += __shfl_xor_sync(0xffffffffu, v, 2);
        v += __shfl_xor_sync(0xffffffffu, v, 1);
        half ^= 1;
        return __shfl_sync(0xffffffffu, v, 0);
    }
    __device__ __forceinline__ float operator()(float v) {
        post(v);
        return total();
    }
};
// The same over a pair of CTAs of up to 16 warps each that share a row: every warp's part goes to both,
// and the barrier is the cluster's.
struct PairSum {
    float (*buf)[32];                     // zero at first
    uint32_t rank;
    int half = 0;
    __device__ __forceinline__ void post(float v) {
        for (int o = 16; o; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
        const int lane = threadIdx.x & 31;
        if (lane < 2) store_cluster(peer_addr(&buf[half][rank * 16 + (threadIdx.x >> 5)], (uint32_t)lane), v);
    }
    __device__ __forceinline__ float total() {
        __syncwarp();
        cluster_sync();
        float v = buf[half][threadIdx.x & 31];
        for (int o = 16; o; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
        half ^= 1;
        return v;
    }
    __device__ __forceinline__ float operator()(float v) {
        post(v);
        return total();
    }
};
__device__ __forceinline__ float sum8(u64 s) { return lo2(s) + hi2(s); }

template <typename T>
__device__ __forceinline__ void pairs8(const Raw8<T>& raw, u64* v) {
    float f[8];
    raw.get(f);
#pragma unroll
    for (int k = 0; k < 4; ++k) v[k] = pack2(f[2 * k], f[2 * k + 1]);
}
__device__ __forceinline__ void floats8(const u64* v, float* f) {
#pragma unroll
    for (int k = 0; k < 4; ++k) unpack2(v[k], f[2 * k], f[2 * k + 1]);
}
template <bool VEC, typename T>
__device__ __forceinline__ void store_pairs(const u64* v, T* p, int valid) {
    float f[8];
    floats8(v, f);
    store8<VEC>(f, p, valid);
}

// Eight values of one thread, not of a warp that works together.
template <bool VEC, typename T>
__device__ __forceinline__ void put8(const float* v, T* p, int valid) {
    if (VEC) store8<true>(v, p, valid);
    else store8_each(v, p, valid);
}

// Eight weights (or gates) from column c on, as binary32, plus `offset`.
template <bool VEC, typename T>
__device__ __forceinline__ void weights8(const void* p, bool f32, int64_t at, int c, int valid, float offset,
                                         u64* w) {
    if (f32) {
        Raw8<float> raw;
        load8<VEC>(raw, static_cast<const float*>(p) + at + c, valid, c);
        pairs8(raw, w);
    } else {
        Raw8<T> raw;
        load8<VEC>(raw, static_cast<const T*>(p) + at + c, valid, c);
        pairs8(raw, w);
    }
#pragma unroll
    for (int k = 0; k < 4; ++k) w[k] = add2(w[k], both(offset));
}

struct NormParams {
    pwlq_block_norm_args a;
    float scale, eps, offset, inv_cols, ratio;
    int64_t groups;
    int group_lanes, group_shift;
    bool wf32;
    int stages;
    unsigned row_bytes, code_bytes;       // of a row
    unsigned slot_bytes;                  // what a row of values takes in a stage
    int64_t gate_step, gate_rest;         // gridDim.x / gate_tokens and the remainder (forward)
};

// ---- the ring.  Stage s of CTA-local row number i is s = i % stages; full[s] completes when the
// row's copies have landed.
struct Ring {
    uint64_t* full;
    unsigned char* stage0;
    unsigned stage_bytes;
    int stages;
    int stage = 0;
    unsigned phase = 0;
    bool dead = false;                    // a wait expired: no more waiting, the results are void
    __device__ __forceinline__ unsigned char* wait() {
        if (!dead && !mbar_wait(&full[stage], phase)) {
            dead = true;
            g_block_norm_timeout = 1;
        }
        return stage0 + (size_t)stage * stage_bytes;
    }
    __device__ __forceinline__ void next() {
        if (++stage == stages) { stage = 0; phase ^= 1; }
    }
};

// Bytes of eight values of a row, and the range of their group (whose lanes call this together).
__device__ __forceinline__ void save8(const u64* pairs, const NormParams& q, int64_t row, int c,
                                      int valid, uint8_t* codes, float* ranges) {
    float v[8], top = 0.0f;
    floats8(pairs, v);
    if (valid < 8)                        // bytes of 0 past the row, where x * scale may be -0
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = i < valid ? v[i] : 0.0f;
#pragma unroll
    for (int i = 0; i < 8; ++i) top = max_abs(top, v[i]);
    top = group_max(top, q.group_lanes);
    const float m = act8_range(top);
    const PieceParams P = act8_params_paired(m, q.ratio);
    if (valid <= 0) return;
    uint8_t* at = codes + row * q.a.ldc + c;
    *reinterpret_cast<uint2*>(at) = act8_bytes8(v, m, P);
    // the row's last 16 bytes may need zeros that no value stands for
    if (valid <= 8 && (c & 8) == 0) *reinterpret_cast<uint2*>(at + 8) = make_uint2(0u, 0u);
    if ((c & ((1 << q.group_shift) - 1)) == 0) ranges[row * q.groups + (c >> q.group_shift)] = m;
}

// A row of values on its way to a stage.  ODD: rows of 16-bit values that start anywhere.  The copy then
// takes the aligned words that hold the row, so that the row begins as far past the slot's beginning
// as past the boundary; bytes outside the matrix are not touched: the ends of its first and last row
// that no aligned word inside the matrix holds are moved value by value.
template <typename T>
struct RowCopy {
    const unsigned char *from, *lo, *hi;   // the row; the words copied
    unsigned bytes, skip;                  // of the row; from the slot's beginning to it
    __device__ __forceinline__ RowCopy(const void* base, int64_t rows, int64_t ld, int64_t row, unsigned row_bytes) {
        const unsigned char* first = static_cast<const unsigned char*>(base);
        from = first + row * ld * (int64_t)sizeof(T);
        bytes = row_bytes;
        skip = (unsigned)((uintptr_t)from & 15);
        const uintptr_t in_lo = ((uintptr_t)first + 15) & ~(uintptr_t)15;
        const uintptr_t in_hi = ((uintptr_t)first + (rows - 1) * ld * (int64_t)sizeof(T) + bytes) & ~(uintptr_t)15;
        lo = reinterpret_cast<const unsigned char*>(max((uintptr_t)from - skip, in_lo));
        hi = reinterpret_cast<const unsigned char*>(min(((uintptr_t)from + bytes + 15) & ~(uintptr_t)15, in_hi));
        if (hi < lo) hi = lo;
    }
    __device__ __forceinline__ unsigned size() const { return (unsigned)(hi - lo); }
    // the ends, before the barrier is told of the copy; a later row's copy to the same bytes, which this thread
    // starts too, comes after them
    __device__ __forceinline__ void ends(unsigned char* slot) const {
        if (lo == from - skip && hi >= from + bytes) return;
        const unsigned char* origin = from - skip;
        for (const unsigned char* p = from; p < from + bytes; p += sizeof(T)) {
            if (p >= lo && p < hi) p = hi;                   // words end between values
            if (p >= from + bytes) break;
            *reinterpret_cast<T*>(slot + (p - origin)) = *reinterpret_cast<const T*>(p);
        }
        fence_proxy_async();
    }
    __device__ __forceinline__ void start(unsigned char* slot, uint64_t* bar) const {
        if (hi > lo) bulk_copy_g2s(slot + (lo - (from - skip)), lo, size(), bar);
    }
};

template <typename T, bool ODD>
__device__ __forceinline__ void request_forward(const NormParams& q, Ring& ring, int stage, int64_t row) {
    unsigned char* to = ring.stage0 + (size_t)stage * ring.stage_bytes;
    uint64_t* bar = &ring.full[stage];
    if (ODD) {
        const RowCopy<T> x(q.a.x, q.a.rows, q.a.ldx, row, q.row_bytes),
            f(q.a.f ? q.a.f : q.a.x, q.a.rows, q.a.f ? q.a.ldf : q.a.ldx, row, q.row_bytes);
        x.ends(to);
        if (q.a.f) f.ends(to + q.slot_bytes);
        mbar_expect_tx(bar, x.size() + (q.a.f ? f.size() : 0));
        x.start(to, bar);
        if (q.a.f) f.start(to + q.slot_bytes, bar);
        return;
    }
    mbar_expect_tx(bar, ring.stage_bytes);
    bulk_copy_g2s(to, static_cast<const T*>(q.a.x) + row * q.a.ldx, q.row_bytes, bar);
    if (q.a.f) bulk_copy_g2s(to + q.slot_bytes, static_cast<const T*>(q.a.f) + row * q.a.ldf, q.row_bytes, bar);
}

// How far past a 16-byte boundary a row starts.
template <typename T, bool ODD>
__device__ __forceinline__ unsigned row_skip(const void* base, int64_t ld, int64_t row) {
    return ODD ? (unsigned)(((uintptr_t)base + row * ld * (int64_t)sizeof(T)) & 15) : 0;
}
// The 32 bytes that begin `bytes` (the same in a whole warp, below 16) past the first of twelve words:
// a branch over the word, then one operation a word.
template <int K>
__device__ __forceinline__ void words_from(const uint32_t (&w)[12], uint32_t pick, Raw32& r) {
#pragma unroll
    for (int i = 0; i < 8; ++i) r.w[i] = __byte_perm(w[i + K], w[i + K + 1], pick);
}
__device__ __forceinline__ Raw32 window32(const uint4* q, unsigned bytes) {
    uint32_t w[12];
#pragma unroll
    for (int i = 0; i < 3; ++i) {
        const uint4 x = q[i];
        w[4 * i] = x.x; w[4 * i + 1] = x.y; w[4 * i + 2] = x.z; w[4 * i + 3] = x.w;
    }
    const uint32_t pick = bytes & 2 ? 0x5432 : 0x3210;
    Raw32 r;
    switch (bytes >> 2) {
        case 0: words_from<0>(w, pick, r); break;
        case 1: words_from<1>(w, pick, r); break;
        case 2: words_from<2>(w, pick, r); break;
        default: words_from<3>(w, pick, r);
    }
    return r;
}

// A thread's 32 bytes of a row in shared memory; the values from `valid` on read as 0.
template <typename T, bool ODD>
__device__ __forceinline__ Raw32 ring32(const unsigned char* at, int valid) {
    if (!ODD) return load32(at);
    const unsigned o = smem_addr(at) & 15;
    Raw32 r = window32(reinterpret_cast<const uint4*>(at - o), o);
    if (valid < 2 * kPairs32<T>)
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int n = valid - 2 * i;  // values of this word that exist
            r.w[i] = n <= 0 ? 0u : n == 1 ? r.w[i] & 0xffffu : r.w[i];
        }
    return r;
}
// A warp's 32 bytes per lane to a row.  ODD: the first lane's go to `row0`, where `rest` values of the row
// exist from there on; they are turned in shared memory, so that whole aligned 16-byte words are written
// and only the ends of the warp's stretch go value by value.  Every lane calls.
constexpr int kTurn = 65;                // words of a warp's turn: the last window ends one past them
template <typename T, bool ODD>
__device__ __forceinline__ void put32(T* to, const Raw32& v, bool live, uint4* turn, T* row0, int rest) {
    if (!ODD) {
        if (live) store32(to, v);
        return;
    }
    constexpr int kSize = sizeof(T);
    const int lane = threadIdx.x & 31;
    const int bytes = min(rest * kSize, 1024), head = min((int)(-(uintptr_t)row0 & 15), bytes);
    const int words = (bytes - head) >> 4;
    uint4* const mine = turn + (threadIdx.x >> 5) * kTurn;
    __syncwarp();
    mine[2 * lane] = make_uint4(v.w[0], v.w[1], v.w[2], v.w[3]);
    mine[2 * lane + 1] = make_uint4(v.w[4], v.w[5], v.w[6], v.w[7]);
    __syncwarp();
    const Raw32 x = window32(mine + 2 * lane, head);
    uint4* const out = reinterpret_cast<uint4*>(reinterpret_cast<unsigned char*>(row0) + head) + 2 * lane;
    if (2 * lane < words) out[0] = make_uint4(x.w[0], x.w[1], x.w[2], x.w[3]);
    if (2 * lane + 1 < words) out[1] = make_uint4(x.w[4], x.w[5], x.w[6], x.w[7]);
    const T* from = reinterpret_cast<const T*>(mine);
    const int tail = (head + 16 * words) / kSize + lane;
    if (lane * kSize < head) row0[lane] = from[lane];
    if (tail * kSize < bytes) row0[tail] = from[tail];
}
template <bool ODD>
__device__ __forceinline__ unsigned turn_bytes() { return ODD ? blockDim.x / 32 * kTurn * 16 : 0; }

// Forward, every thread loading its values itself, one row per CTA.  VC: chunks of eight columns per
// thread.
template <typename T, int VC, bool VEC, bool SAVE>
__global__ void __launch_bounds__(1024) block_norm_kernel(const __grid_constant__ NormParams q) {
    __shared__ float buf[2][32];
    CtaSum cta_sum{buf};
    const int cols = (int)q.a.cols;
    const int64_t row = blockIdx.x;
    const T* x = static_cast<const T*>(q.a.x) + row * q.a.ldx;
    const T* f = static_cast<const T*>(q.a.f) + row * q.a.ldf;
    Raw8<T> rx[VC], rf[VC];
#pragma unroll
    for (int i = 0; i < VC; ++i) {
        const int c = (threadIdx.x + i * blockDim.x) * 8;
        if (q.a.f) load8<VEC>(rf[i], f + c, cols - c, c);
        load8<VEC>(rx[i], x + c, cols - c, c);
    }
    u64 r[VC][4];
    float rstd_f = 1.0f;
    if (q.a.post_weight) {
        u64 s = 0ull;
#pragma unroll
        for (int i = 0; i < VC; ++i) {
            u64 v[4];
            pairs8(rf[i], v);
#pragma unroll
            for (int k = 0; k < 4; ++k) s = fma2(v[k], v[k], s);
        }
        rstd_f = rsqrtf(fmaf(cta_sum(sum8(s)), q.inv_cols, q.eps));
        if (SAVE && threadIdx.x == 0 && q.a.f_rstd) q.a.f_rstd[row] = rstd_f;
    }
    u64 s = 0ull;
    const int64_t gate_at = q.a.gate ? row / q.a.gate_tokens * q.a.ldgate : 0;
#pragma unroll
    for (int i = 0; i < VC; ++i) {
        const int c = (threadIdx.x + i * blockDim.x) * 8, valid = cols - c;
        pairs8(rx[i], r[i]);
#pragma unroll
        for (int k = 0; k < 4; ++k) r[i][k] = mul2(r[i][k], both(q.scale));
        if (q.a.f) {
            u64 v[4], w[4];
            pairs8(rf[i], v);
            if (SAVE && q.a.f_codes) save8(v, q, row, c, valid, q.a.f_codes, q.a.f_ranges);
            if (q.a.post_weight) {
                weights8<VEC, T>(q.a.post_weight, q.wf32, 0, c, valid, q.offset, w);
#pragma unroll
                for (int k = 0; k < 4; ++k) v[k] = mul2(mul2(v[k], both(rstd_f)), w[k]);
            }
            if (q.a.gate) {
                weights8<VEC, T>(q.a.gate, q.wf32, gate_at, c, valid, 0.0f, w);
#pragma unroll
                for (int k = 0; k < 4; ++k) v[k] = mul2(v[k], w[k]);
            }
#pragma unroll
            for (int k = 0; k < 4; ++k) r[i][k] = add2(r[i][k], v[k]);
        }
        if (q.a.r) store_pairs<VEC>(r[i], static_cast<T*>(q.a.r) + row * q.a.ldr + c, valid);
        if (SAVE && q.a.r_codes) save8(r[i], q, row, c, valid, q.a.r_codes, q.a.r_ranges);
        // columns past the row hold 0 here, or NaN where the whole row does
#pragma unroll
        for (int k = 0; k < 4; ++k) s = fma2(r[i][k], r[i][k], s);
    }
    if (!q.a.pre_weight) return;
    const float rstd_r = rsqrtf(fmaf(cta_sum(sum8(s)), q.inv_cols, q.eps));
    if (SAVE && threadIdx.x == 0 && q.a.r_rstd) q.a.r_rstd[row] = rstd_r;
#pragma unroll
    for (int i = 0; i < VC; ++i) {
        const int c = (threadIdx.x + i * blockDim.x) * 8, valid = cols - c;
        u64 w[4];
        weights8<VEC, T>(q.a.pre_weight, q.wf32, 0, c, valid, q.offset, w);
#pragma unroll
        for (int k = 0; k < 4; ++k) w[k] = mul2(mul2(r[i][k], both(rstd_r)), w[k]);
        store_pairs<VEC>(w, static_cast<T*>(q.a.h) + row * q.a.ldh + c, valid);
    }
}

// Weights (or gates) of a thread's 32 bytes of columns: requested early, unpacked where they are used.
// WF32: binary32 beside 16-bit values.
template <typename T, bool WF32>
struct Weights {
    static constexpr bool kWide = WF32 && sizeof(T) == 2;
    Raw32 raw[kWide ? 2 : 1];
    // rows of weights that need not be aligned, and of which `valid` values from there on exist
    __device__ __forceinline__ void load_odd(const void* p, int64_t row, int c, int valid) {
        if (kWide) {
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                Raw8<float> r;
                load8<false>(r, static_cast<const float*>(p) + row + c + 8 * i, valid - 8 * i, c + 8 * i);
                float v[8];
                r.get(v);
#pragma unroll
                for (int k = 0; k < 8; ++k) raw[kWide ? i : 0].w[k] = __float_as_uint(v[k]);
            }
        } else {
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                Raw8<T> r;
                load8<false>(r, static_cast<const T*>(p) + row + c + 8 * i, valid - 8 * i, c + 8 * i);
                const uint4 w = *reinterpret_cast<const uint4*>(&r);
                raw[0].w[4 * i] = w.x; raw[0].w[4 * i + 1] = w.y; raw[0].w[4 * i + 2] = w.z; raw[0].w[4 * i + 3] = w.w;
            }
        }
    }
    template <bool ODD> __device__ __forceinline__ void load(const void* p, int64_t row, int c, int valid) {
        if (ODD) load_odd(p, row, c, valid);
        else load(p, row + c);
    }
    __device__ __forceinline__ void load(const void* p, int64_t at) {
        if (kWide) {
            raw[0] = load32(static_cast<const float*>(p) + at);
            raw[kWide ? 1 : 0] = load32(static_cast<const float*>(p) + at + 8);
        } else {
            raw[0] = load32(static_cast<const T*>(p) + at);
        }
    }
    __device__ __forceinline__ void get(u64* w) const {
        if (kWide) {
            pairs32(raw[0], w, 0.0f);
            pairs32(raw[kWide ? 1 : 0], w + kPairs32<T> / 2, 0.0f);
        } else {
            pairs32(raw[0], w, T());
        }
    }
    __device__ __forceinline__ void get(u64* w, float offset) const {
        get(w);
#pragma unroll
        for (int k = 0; k < kPairs32<T>; ++k) w[k] = add2(w[k], both(offset));
    }
};

// Bytes of a thread's 32 bytes of values, and the range of their group.
template <typename T, bool ODD = false>
__device__ __forceinline__ void save32(const u64* v, const NormParams& q, bool live, int64_t row, int c,
                                       uint8_t* codes, float* ranges) {
    constexpr int kP = kPairs32<T>;
    float f[2 * kP], top = 0.0f;
#pragma unroll
    for (int k = 0; k < kP; ++k) unpack2(v[k], f[2 * k], f[2 * k + 1]);
    if (ODD && c + 2 * kP > (int)q.a.cols)
#pragma unroll
        for (int k = 0; k < 2 * kP; ++k) f[k] = c + k < (int)q.a.cols ? f[k] : 0.0f;     // bytes of 0 past the row
#pragma unroll
    for (int k = 0; k < 2 * kP; ++k) top = max_abs(top, f[k]);
    top = group_max(top, q.group_lanes);
    const float m = act8_range(top);
    const PieceParams P = act8_params_paired(m, q.ratio);
    if (!live) return;
    uint8_t* at = codes + row * q.a.ldc + c;
    const uint2 a = act8_bytes8(f, m, P);
    if (kP == 8) {
        const uint2 b = act8_bytes8(f + 2 * kP - 8, m, P);
        *reinterpret_cast<uint4*>(at) = make_uint4(a.x, a.y, b.x, b.y);
    } else {
        *reinterpret_cast<uint2*>(at) = a;
    }
    // the row's last 16 bytes may need zeros that no value stands for
    if ((c & 8) == 0 && c + 8 == (int)q.a.cols) *reinterpret_cast<uint2*>(at + 8) = make_uint2(0u, 0u);
    if ((c & ((1 << q.group_shift) - 1)) == 0) ranges[row * q.groups + (c >> q.group_shift)] = m;
}

// Forward with a ring: 32 bytes of columns per thread.
template <typename T, bool SAVE, bool WF32, bool ODD>
__global__ void __maxnreg__(ODD ? 80 : 64) block_norm_ring_kernel(const __grid_constant__ NormParams q) {
    constexpr int kP = kPairs32<T>;
    __shared__ float buf[2][32];
    __shared__ uint64_t full[kMaxStages];
    extern __shared__ __align__(16) unsigned char smem[];
    CtaSum cta_sum{buf};
    uint4* const turn = reinterpret_cast<uint4*>(smem);
    Ring ring{full, smem + turn_bytes<ODD>(), q.a.f ? 2 * q.slot_bytes : q.slot_bytes, q.stages};
    if (threadIdx.x == 0) {
        for (int s = 0; s < q.stages; ++s) mbar_init(&full[s], 1);
        fence_barrier_init();
        for (int s = 0; s < q.stages; ++s) {
            const int64_t row = blockIdx.x + (int64_t)s * gridDim.x;
            if (row < q.a.rows) request_forward<T, ODD>(q, ring, s, row);
        }
    }
    __syncthreads();
    // the row's gate, found by division once and by addition from then on
    int64_t gate = 0, in_gate = 0;
    if (q.a.gate) {
        gate = blockIdx.x / q.a.gate_tokens;
        in_gate = blockIdx.x - gate * q.a.gate_tokens;
    }
    // threads past the row repeat its last columns (so that a group's range stays its own) and
    // neither store nor count
    const bool live = (int)threadIdx.x * 2 * kP < (int)q.a.cols, post = q.a.post_weight, pre = q.a.pre_weight;
    const int cols = (int)q.a.cols, end = ODD ? (cols - 1) / (2 * kP) * (2 * kP) : cols - 2 * kP;
    const int c = live ? (int)threadIdx.x * 2 * kP : end;
    const int valid = ODD ? cols - c : 2 * kP;
    const int warp_c = (int)(threadIdx.x & ~31u) * 2 * kP;       // of the warp's first lane
    for (int64_t row = blockIdx.x; row < q.a.rows; row += gridDim.x) {
        u64 r[kP], w[kP], s = 0ull;
        Weights<T, WF32> wt;
        if (post) wt.template load<ODD>(q.a.post_weight, 0, c, valid);
        const unsigned char* at = ring.wait() + c * (int)sizeof(T);
        pairs32(ring32<T, ODD>(at + row_skip<T, ODD>(q.a.x, q.a.ldx, row), valid), r, T());
#pragma unroll
        for (int k = 0; k < kP; ++k) r[k] = mul2(r[k], both(q.scale));
        if (q.a.f) {
            u64 f[kP];
            pairs32(ring32<T, ODD>(at + q.slot_bytes + row_skip<T, ODD>(q.a.f, q.a.ldf, row), valid), f, T());
            if (post) {
#pragma unroll
                for (int k = 0; k < kP; ++k) s = fma2(f[k], f[k], s);
                cta_sum.post(live ? sum8(s) : 0.0f);
                if (SAVE && q.a.f_codes) save32<T, ODD>(f, q, live, row, c, q.a.f_codes, q.a.f_ranges);
                const float rstd_f = rsqrtf(fmaf(cta_sum.total(), q.inv_cols, q.eps));
                if (SAVE && threadIdx.x == 0 && q.a.f_rstd) q.a.f_rstd[row] = rstd_f;
                wt.get(w, q.offset);
                if (q.a.gate) wt.template load<ODD>(q.a.gate, gate * q.a.ldgate, c, valid);
#pragma unroll
                for (int k = 0; k < kP; ++k) f[k] = mul2(mul2(f[k], both(rstd_f)), w[k]);
            } else {
                if (q.a.gate) wt.template load<ODD>(q.a.gate, gate * q.a.ldgate, c, valid);
                if (SAVE && q.a.f_codes) save32<T, ODD>(f, q, live, row, c, q.a.f_codes, q.a.f_ranges);
            }
            if (q.a.gate) {
                wt.get(w);
#pragma unroll
                for (int k = 0; k < kP; ++k) r[k] = fma2(f[k], w[k], r[k]);
                gate += q.gate_step;
                in_gate += q.gate_rest;
                if (in_gate >= q.a.gate_tokens) { ++gate; in_gate -= q.a.gate_tokens; }
            } else {
#pragma unroll
                for (int k = 0; k < kP; ++k) r[k] = add2(r[k], f[k]);
            }
        }
        s = 0ull;
#pragma unroll
        for (int k = 0; k < kP; ++k) s = fma2(r[k], r[k], s);
        if (pre) {
            cta_sum.post(live ? sum8(s) : 0.0f);
            wt.template load<ODD>(q.a.pre_weight, 0, c, valid);
        }
        if (q.a.r && (ODD || live)) {
            T* const to = static_cast<T*>(q.a.r) + row * q.a.ldr;
            put32<T, ODD>(to + c, raw32(r, T()), live, turn, to + warp_c, cols - warp_c);
        }
        if (SAVE && q.a.r_codes) save32<T, ODD>(r, q, live, row, c, q.a.r_codes, q.a.r_ranges);
        float rstd_r = 0.0f;
        if (pre) rstd_r = rsqrtf(fmaf(cta_sum.total(), q.inv_cols, q.eps));
        else __syncthreads();
        // every thread has its values of this stage
        const int64_t ahead = row + (int64_t)q.stages * gridDim.x;
        if (threadIdx.x == 0 && ahead < q.a.rows && !ring.dead) request_forward<T, ODD>(q, ring, ring.stage, ahead);
        ring.next();
        if (!pre) continue;
        if (SAVE && threadIdx.x == 0 && q.a.r_rstd) q.a.r_rstd[row] = rstd_r;
        wt.get(w, q.offset);
#pragma unroll
        for (int k = 0; k < kP; ++k) w[k] = mul2(mul2(r[k], both(rstd_r)), w[k]);
        T* const to = static_cast<T*>(q.a.h) + row * q.a.ldh;
        put32<T, ODD>(to + c, raw32(w, T()), live, turn, to + warp_c, cols - warp_c);
    }
}

// Forward without checkpoints, weights of the values' type, a row per CTA and no ring: the arithmetic, and so
// the bits, of block_norm_ring_kernel.  A row is then so little work that many CTAs, each with its own loads in
// flight, keep the memory busier than a ring does (16384 x 4096 bf16, one norm: 80.5 us = 6670 GB/s, more than a
// copy of that size moves, since the cache still holds part of the results).
template <typename T>
__global__ void __maxnreg__(64) block_norm_row_kernel(const __grid_constant__ NormParams q) {
    constexpr bool WF32 = sizeof(T) == 4;
    constexpr int kP = kPairs32<T>;
    __shared__ float buf[2][32];
    CtaSum cta_sum{buf};
    const int64_t row = blockIdx.x;
    const bool live = (int)threadIdx.x * 2 * kP < (int)q.a.cols, post = q.a.post_weight, pre = q.a.pre_weight;
    const int c = live ? (int)threadIdx.x * 2 * kP : (int)q.a.cols - 2 * kP;
    const Raw32 x = load32_global(static_cast<const T*>(q.a.x) + row * q.a.ldx + c);
    u64 r[kP], w[kP], s = 0ull;
    Weights<T, WF32> wt;
    if (q.a.f) {
        const Raw32 raw = load32_global(static_cast<const T*>(q.a.f) + row * q.a.ldf + c);
        const int64_t gate = q.a.gate ? row / q.a.gate_tokens * q.a.ldgate + c : 0;
        u64 f[kP];
        if (post) {
            wt.load(q.a.post_weight, c);
            pairs32(raw, f, T());
#pragma unroll
            for (int k = 0; k < kP; ++k) s = fma2(f[k], f[k], s);
            const float rstd_f = rsqrtf(fmaf(cta_sum(live ? sum8(s) : 0.0f), q.inv_cols, q.eps));
            wt.get(w, q.offset);
            if (q.a.gate) wt.load(q.a.gate, gate);
#pragma unroll
            for (int k = 0; k < kP; ++k) f[k] = mul2(mul2(f[k], both(rstd_f)), w[k]);
        } else {
            if (q.a.gate) wt.load(q.a.gate, gate);
            pairs32(raw, f, T());
        }
        pairs32(x, r, T());
#pragma unroll
        for (int k = 0; k < kP; ++k) r[k] = mul2(r[k], both(q.scale));
        if (q.a.gate) wt.get(w);
#pragma unroll
        for (int k = 0; k < kP; ++k) r[k] = q.a.gate ? fma2(f[k], w[k], r[k]) : add2(r[k], f[k]);
    } else {
        pairs32(x, r, T());
#pragma unroll
        for (int k = 0; k < kP; ++k) r[k] = mul2(r[k], both(q.scale));
    }
    s = 0ull;
#pragma unroll
    for (int k = 0; k < kP; ++k) s = fma2(r[k], r[k], s);
    if (pre) {
        cta_sum.post(live ? sum8(s) : 0.0f);
        wt.load(q.a.pre_weight, c);
    }
    if (q.a.r && live) store32(static_cast<T*>(q.a.r) + row * q.a.ldr + c, raw32(r, T()));
    if (!pre) return;
    const float rstd_r = rsqrtf(fmaf(cta_sum.total(), q.inv_cols, q.eps));
    wt.get(w, q.offset);
#pragma unroll
    for (int k = 0; k < kP; ++k) w[k] = mul2(mul2(r[k], both(rstd_r)), w[k]);
    if (live) store32(static_cast<T*>(q.a.h) + row * q.a.ldh + c, raw32(w, T()));
}

// Sum over the aligned `lanes` (a power of two) lanes that share a row.
__device__ __forceinline__ float lanes_sum(float v, int lanes) {
#pragma unroll
    for (int o = 1; o < 32; o <<= 1)
        if (o < lanes) v += __shfl_xor_sync(0xffffffffu, v, o);
    return v;
}

// Forward, rows of up to 32 lanes' columns: `lanes` lanes own a row, a warp 32 / lanes rows at a time,
// and nothing waits for another warp (one CTA per row left most of a warp idle below 512 columns: at
// 64 columns it ran at a tenth of the copy rate).  The next rows' values are requested before the
// current ones are worked on.
constexpr int kNarrowThreads = 256;
template <typename T, bool SAVE, bool WF32>
__global__ void __launch_bounds__(kNarrowThreads, 2)
block_norm_narrow_kernel(const __grid_constant__ NormParams q, int lanes) {
    constexpr int kP = kPairs32<T>;
    const int lane = threadIdx.x & 31, in = lane & (lanes - 1);
    const bool inside = in * 2 * kP < (int)q.a.cols, post = q.a.post_weight, pre = q.a.pre_weight;
    const int c = inside ? in * 2 * kP : (int)q.a.cols - 2 * kP;       // idle lanes repeat the last columns
    const int64_t per_step = (int64_t)gridDim.x * kNarrowThreads / lanes;
    Weights<T, WF32> post_w, pre_w;
    if (post) post_w.load(q.a.post_weight, c);
    if (pre) pre_w.load(q.a.pre_weight, c);
    const unsigned every = (unsigned)min(q.a.gate_tokens, (int64_t)0x7fffffff);
    int64_t row = ((int64_t)blockIdx.x * kNarrowThreads + threadIdx.x) / lanes;
    Raw32 next_x, next_f;
    auto fetch = [&](int64_t r) {
        const int64_t at = min(r, q.a.rows - 1);
        next_x = load32_global(static_cast<const T*>(q.a.x) + at * q.a.ldx + c);
        if (q.a.f) next_f = load32_global(static_cast<const T*>(q.a.f) + at * q.a.ldf + c);
    };
    // a warp's lanes go round together, with rows past the end masked
    const int64_t warp_row = row - lane / lanes;
    fetch(row);
    for (int64_t at = warp_row; at < q.a.rows; at += per_step, row += per_step) {
        const Raw32 raw_x = next_x, raw_f = next_f;
        fetch(row + per_step);
        const bool live = inside && row < q.a.rows;
        u64 r[kP], w[kP], s;
        pairs32(raw_x, r, T());
#pragma unroll
        for (int k = 0; k < kP; ++k) r[k] = mul2(r[k], both(q.scale));
        if (q.a.f) {
            u64 f[kP];
            pairs32(raw_f, f, T());
            if (SAVE && q.a.f_codes) save32<T>(f, q, live, row, c, q.a.f_codes, q.a.f_ranges);
            if (post) {
                s = 0ull;
#pragma unroll
                for (int k = 0; k < kP; ++k) s = fma2(f[k], f[k], s);
                const float rstd_f =
                    rsqrtf(fmaf(lanes_sum(inside ? sum8(s) : 0.0f, lanes), q.inv_cols, q.eps));
                if (SAVE && in == 0 && live && q.a.f_rstd) q.a.f_rstd[row] = rstd_f;
                post_w.get(w, q.offset);
#pragma unroll
                for (int k = 0; k < kP; ++k) f[k] = mul2(mul2(f[k], both(rstd_f)), w[k]);
            }
            if (q.a.gate) {
                Weights<T, WF32> g;
                g.load(q.a.gate, (int64_t)((unsigned)min(row, q.a.rows - 1) / every) * q.a.ldgate + c);
                g.get(w);
#pragma unroll
                for (int k = 0; k < kP; ++k) r[k] = fma2(f[k], w[k], r[k]);
            } else {
#pragma unroll
                for (int k = 0; k < kP; ++k) r[k] = add2(r[k], f[k]);
            }
        }
        if (live && q.a.r) store32(static_cast<T*>(q.a.r) + row * q.a.ldr + c, raw32(r, T()));
        if (SAVE && q.a.r_codes) save32<T>(r, q, live, row, c, q.a.r_codes, q.a.r_ranges);
        if (!pre) continue;
        s = 0ull;
#pragma unroll
        for (int k = 0; k < kP; ++k) s = fma2(r[k], r[k], s);
        const float rstd_r = rsqrtf(fmaf(lanes_sum(inside ? sum8(s) : 0.0f, lanes), q.inv_cols, q.eps));
        if (SAVE && in == 0 && live && q.a.r_rstd) q.a.r_rstd[row] = rstd_r;
        pre_w.get(w, q.offset);
#pragma unroll
        for (int k = 0; k < kP; ++k) w[k] = mul2(mul2(r[k], both(rstd_r)), w[k]);
        if (live) store32(static_cast<T*>(q.a.h) + row * q.a.ldh + c, raw32(w, T()));
    }
}

// Backward.  CTA b owns the rows [b * rows_per_cta, ...) and its columns' sums over them; the sums
// go to the workspace and a second kernel adds them in a fixed order.  Within the rows of one gate g,
// the gate and the weight w are the same in every row, so one sum A = sum of e * n serves both
// gradients: dgate_g = w * A_g and dpost = sum over the gates of g * A_g.  Where the gate changes, and
// at the CTA's end, A is turned into them: dgate_g goes out at once if all its rows are this CTA's
// (a gate per token, say), dpost gathers in shared memory.  The running sums live in registers up to
// 8192 columns (16 per thread and chunk); wider rows keep them in shared memory too (WIDE), where
// every thread touches its own columns only.
// Workspace: [ctas][cols] of dpre, [ctas][cols] of dpost, [2 * ctas][cols] of dgate: CTA b's share of
// the gate of its first row, and of its last one if that is another.
// Factor on an f that enters without a norm, so that the lines of its values (act8_lines) stay in range up to
// the largest: A is a quarter of the sum then, and dgate is multiplied back (both exact).
constexpr float kAsItIs = 0.25f;
struct GradParams {
    NormParams q;
    pwlq_block_norm_grads g;
    int64_t rows_per_cta;
    float *dpre, *dpost, *dgate;          // workspace; nullptr: not wanted
    unsigned gathered;                    // where dpost gathers in shared memory (with gates)
    bool gates;                           // several gates; one gate for all rows is dealt with where A
                                          // has been added up, and `dpost` holds A then
};

// What a CTA does with A of eight columns from c on (the first `valid` of which exist) once it is past
// the rows of `gate`.
template <bool VEC, typename T>
__device__ __forceinline__ void finish_gate(const GradParams& p, int64_t cta, int64_t gate, int64_t first,
                                            int64_t last, int c, int valid, const u64* A, float* gathered) {
    const pwlq_block_norm_args& a = p.q.a;
    if (valid <= 0) return;
    u64 w[4], v[4];
    float f[8];
    if (p.dgate) {
#pragma unroll
        for (int k = 0; k < 4; ++k) v[k] = A[k];
        if (a.post_weight) {
            weights8<VEC, T>(a.post_weight, p.q.wf32, 0, c, valid, p.q.offset, w);
#pragma unroll
            for (int k = 0; k < 4; ++k) v[k] = mul2(v[k], w[k]);
        } else {
#pragma unroll
            for (int k = 0; k < 4; ++k) v[k] = mul2(v[k], both(1.0f / kAsItIs));
        }
        floats8(v, f);
        const int64_t from = gate * a.gate_tokens, to = min(from + a.gate_tokens, a.rows);
        if (from < first || to > last) {
            const int64_t slot = 2 * cta + (from > first);
            put8<VEC>(f, p.dgate + slot * a.cols + c, valid);
        } else if (p.q.wf32) {
            put8<VEC>(f, static_cast<float*>(p.g.dgate) + gate * a.cols + c, valid);
        } else {
            put8<VEC>(f, static_cast<T*>(p.g.dgate) + gate * a.cols + c, valid);
        }
    }
    if (p.dpost) {
        weights8<VEC, T>(a.gate, p.q.wf32, gate * a.ldgate, c, valid, 0.0f, w);
        ulonglong2* at = reinterpret_cast<ulonglong2*>(gathered + c);
        ulonglong2 x = at[0], y = at[1];
        x.x = fma2(A[0], w[0], x.x);
        x.y = fma2(A[1], w[1], x.y);
        y.x = fma2(A[2], w[2], y.x);
        y.y = fma2(A[3], w[3], y.y);
        at[0] = x;
        at[1] = y;
    }
}

enum { kDpre, kInner };

template <int VC, bool WIDE>
struct ColumnSums {
    u64 reg[2][WIDE ? 1 : VC][4] = {};
    ulonglong2* smem = nullptr;           // [2][VC][2][blockDim.x]
    __device__ __forceinline__ ulonglong2* at(int which, int i) const {
        return smem + ((which * VC + i) * 2) * blockDim.x + threadIdx.x;
    }
    __device__ __forceinline__ void clear(int which) {
        const u64 zero[4] = {};
#pragma unroll
        for (int i = 0; i < VC; ++i) set(which, i, zero);
    }
    __device__ __forceinline__ void set(int which, int i, const u64* v) {
        if (WIDE) {
            at(which, i)[0] = make_ulonglong2(v[0], v[1]);
            at(which, i)[blockDim.x] = make_ulonglong2(v[2], v[3]);
        } else {
#pragma unroll
            for (int k = 0; k < 4; ++k) reg[which][WIDE ? 0 : i][k] = v[k];
        }
    }
    __device__ __forceinline__ void get(int which, int i, u64* v) const {
        if (WIDE) {
            const ulonglong2 a = at(which, i)[0], b = at(which, i)[blockDim.x];
            v[0] = a.x; v[1] = a.y; v[2] = b.x; v[3] = b.y;
        } else {
#pragma unroll
            for (int k = 0; k < 4; ++k) v[k] = reg[which][WIDE ? 0 : i][k];
        }
    }
    template <bool VEC>
    __device__ __forceinline__ void put(int which, float* to, int cols) const {
#pragma unroll
        for (int i = 0; i < VC; ++i) {
            const int c = (threadIdx.x + i * blockDim.x) * 8;
            u64 v[4];
            get(which, i, v);
            float f[8];
            floats8(v, f);
            put8<VEC>(f, to + c, cols - c);
        }
    }
};

// The columns of `gathered` that a thread looks after.
template <int VC>
__device__ __forceinline__ void clear_gathered(float* gathered) {
#pragma unroll
    for (int i = 0; i < VC; ++i) {
        float4* at = reinterpret_cast<float4*>(gathered + (threadIdx.x + i * blockDim.x) * 8);
        at[0] = at[1] = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
    }
}

template <typename T, bool ODD>
__device__ __forceinline__ void request_backward(const GradParams& p, Ring& ring, int stage, int64_t row, int base) {
    const NormParams& q = p.q;
    unsigned char* to = ring.stage0 + (size_t)stage * ring.stage_bytes;
    uint64_t* bar = &ring.full[stage];
    unsigned char* const at_dr = to + (q.a.pre_weight ? q.slot_bytes + q.code_bytes : 0);
    if (ODD) {
        const bool pre = q.a.pre_weight, has_dr = p.g.dr;
        const RowCopy<T> dh(pre ? p.g.dh : p.g.dr, q.a.rows, pre ? p.g.lddh : p.g.lddr, row, q.row_bytes),
            dr(has_dr ? p.g.dr : p.g.dh, q.a.rows, has_dr ? p.g.lddr : p.g.lddh, row, q.row_bytes);
        if (pre) dh.ends(to);
        if (has_dr) dr.ends(at_dr);
        mbar_expect_tx(bar, (pre ? dh.size() + q.code_bytes : 0) + (has_dr ? dr.size() : 0) +
                                (q.a.f_codes ? q.code_bytes : 0));
        if (pre) dh.start(to, bar);
        if (has_dr) dr.start(at_dr, bar);
    } else {
        mbar_expect_tx(bar, ring.stage_bytes);
        if (q.a.pre_weight)
            bulk_copy_g2s(to, static_cast<const T*>(p.g.dh) + row * p.g.lddh + base, q.row_bytes, bar);
        if (p.g.dr) bulk_copy_g2s(at_dr, static_cast<const T*>(p.g.dr) + row * p.g.lddr + base, q.row_bytes, bar);
    }
    if (q.a.pre_weight)
        bulk_copy_g2s(to + q.slot_bytes, q.a.r_codes + row * q.a.ldc + base, q.code_bytes, bar);
    if (q.a.f_codes)
        bulk_copy_g2s(to + ring.stage_bytes - q.code_bytes, q.a.f_codes + row * q.a.ldc + base, q.code_bytes, bar);
}

// Eight bytes of a row from column c on; those past the row read as 0.
__device__ __forceinline__ uint2 bytes8(const uint8_t* row, int c, int valid) {
    uint2 b = make_uint2(0u, 0u);
    if (valid > 0) {
        b = *reinterpret_cast<const uint2*>(row + c);
        if (valid < 8) {
            b.x &= valid >= 4 ? 0xffffffffu : (1u << (8 * valid)) - 1;
            b.y &= valid > 4 ? (1u << (8 * (valid - 4))) - 1 : 0u;
        }
    }
    return b;
}

// Backward, every thread loading its values itself.
template <typename T, int VC, bool VEC, bool WIDE>
__global__ void __launch_bounds__(WIDE ? 512 : 1024)
block_norm_backward_kernel(const __grid_constant__ GradParams p) {
    __shared__ float buf[2][32];
    extern __shared__ __align__(16) unsigned char smem[];
    CtaSum cta_sum{buf};
    const NormParams& q = p.q;
    const int cols = (int)q.a.cols;
    const int64_t first = blockIdx.x * p.rows_per_cta, last = min(first + p.rows_per_cta, q.a.rows);
    const bool pre = q.a.pre_weight, post = q.a.post_weight, has_f = q.a.f_codes, has_dr = p.g.dr;
    ColumnSums<VC, WIDE> sums;
    if (WIDE) {
        sums.smem = reinterpret_cast<ulonglong2*>(smem);
        for (int which = 0; which < 2; ++which) sums.clear(which);
    }
    float* const gathered = reinterpret_cast<float*>(smem + p.gathered);
    const bool gates = p.gates && (p.dpost || p.dgate);
    if (gates && p.dpost) clear_gathered<VC>(gathered);
    auto finish = [&](int64_t gate) {
#pragma unroll
        for (int i = 0; i < VC; ++i) {
            const int c = (threadIdx.x + i * blockDim.x) * 8;
            u64 A[4];
            sums.get(kInner, i, A);
            finish_gate<VEC, T>(p, blockIdx.x, gate, first, last, c, cols - c, A, gathered);
        }
        sums.clear(kInner);
    };
    int64_t gate = q.a.gate ? first / q.a.gate_tokens : 0;
    int64_t gate_end = (gate + 1) * q.a.gate_tokens;

    // a row's ranges and factors, requested one row ahead
    float mr[VC], mf[VC], rstd_r = 0.0f, rstd_f = kAsItIs;
    auto fetch = [&](int64_t row) {
        if (pre) rstd_r = q.a.r_rstd[row];
        if (post) rstd_f = q.a.f_rstd[row];
#pragma unroll
        for (int i = 0; i < VC; ++i) {
            const int c = (threadIdx.x + i * blockDim.x) * 8;
            mr[i] = mf[i] = 0.0f;
            if (c < cols) {
                const int64_t at = row * q.groups + (c >> q.group_shift);
                if (pre) mr[i] = q.a.r_ranges[at];
                if (has_f) mf[i] = q.a.f_ranges[at];
            }
        }
    };
    if (first < last) fetch(first);

    for (int64_t row = first; row < last; ++row) {
        if (q.a.gate && row == gate_end) {
            if (gates) finish(gate);
            ++gate;
            gate_end += q.a.gate_tokens;
        }
        const float factor_r = rstd_r, factor_f = rstd_f;
        float now_r[VC], now_f[VC];
#pragma unroll
        for (int i = 0; i < VC; ++i) {
            now_r[i] = mr[i];
            now_f[i] = mf[i];
        }
        if (row + 1 < last) fetch(row + 1);
        const T* dh = static_cast<const T*>(p.g.dh) + row * p.g.lddh;
        const T* dr = static_cast<const T*>(p.g.dr) + row * p.g.lddr;
        const uint8_t* rb = q.a.r_codes + row * q.a.ldc;
        const uint8_t* fb = q.a.f_codes + row * q.a.ldc;
        u64 e[VC][4], n[VC][4], s = 0ull;
        // outer norm: e = dr + rstd * (u - n * mean(u n))
        if (pre) {
#pragma unroll
            for (int i = 0; i < VC; ++i) {
                const int c = (threadIdx.x + i * blockDim.x) * 8, valid = cols - c;
                Raw8<T> raw;
                load8<VEC>(raw, dh + c, valid, c);
                pairs8(raw, e[i]);
                act8_scaled8(bytes8(rb, c, valid), act8_lines(now_r[i], q.ratio, factor_r), n[i]);
                u64 w[4], d[4];
                weights8<VEC, T>(q.a.pre_weight, q.wf32, 0, c, valid, q.offset, w);
                sums.get(kDpre, i, d);
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    d[k] = fma2(e[i][k], n[i][k], d[k]);
                    e[i][k] = mul2(e[i][k], w[k]);
                    s = fma2(e[i][k], n[i][k], s);
                }
                sums.set(kDpre, i, d);
            }
            const float mean = cta_sum(sum8(s)) * q.inv_cols;
#pragma unroll
            for (int i = 0; i < VC; ++i)
#pragma unroll
                for (int k = 0; k < 4; ++k) e[i][k] = mul2(fma2(n[i][k], both(-mean), e[i][k]), both(factor_r));
        } else {
#pragma unroll
            for (int i = 0; i < VC; ++i)
#pragma unroll
                for (int k = 0; k < 4; ++k) e[i][k] = 0ull;
        }
        s = 0ull;
#pragma unroll
        for (int i = 0; i < VC; ++i) {
            const int c = (threadIdx.x + i * blockDim.x) * 8, valid = cols - c;
            u64 w[4];
            if (has_dr) {
                Raw8<T> raw;
                load8<VEC>(raw, dr + c, valid, c);
                pairs8(raw, w);
#pragma unroll
                for (int k = 0; k < 4; ++k) e[i][k] = add2(e[i][k], w[k]);
            }
            if (p.g.dx) {
#pragma unroll
                for (int k = 0; k < 4; ++k) w[k] = mul2(e[i][k], both(q.scale));
                store_pairs<VEC>(w, static_cast<T*>(p.g.dx) + row * p.g.lddx + c, valid);
            }
            if (!has_f) continue;
            // inner norm and gate; e becomes v = e * gate * w
            act8_scaled8(bytes8(fb, c, valid), act8_lines(now_f[i], q.ratio, factor_f), n[i]);
            u64 d[4];
            sums.get(kInner, i, d);
#pragma unroll
            for (int k = 0; k < 4; ++k) d[k] = fma2(e[i][k], n[i][k], d[k]);
            sums.set(kInner, i, d);
            if (q.a.gate) {
                weights8<VEC, T>(q.a.gate, q.wf32, gate * q.a.ldgate, c, valid, 0.0f, w);
#pragma unroll
                for (int k = 0; k < 4; ++k) e[i][k] = mul2(e[i][k], w[k]);
            }
            if (post) {
                weights8<VEC, T>(q.a.post_weight, q.wf32, 0, c, valid, q.offset, w);
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    e[i][k] = mul2(e[i][k], w[k]);
                    s = fma2(e[i][k], n[i][k], s);
                }
            }
        }
        float mean = 0.0f;
        if (post) mean = cta_sum(sum8(s)) * q.inv_cols;
        if (!p.g.df) continue;
#pragma unroll
        for (int i = 0; i < VC; ++i) {
            const int c = (threadIdx.x + i * blockDim.x) * 8;
            u64 w[4];
#pragma unroll
            for (int k = 0; k < 4; ++k)
                w[k] = post ? mul2(fma2(n[i][k], both(-mean), e[i][k]), both(factor_f)) : e[i][k];
            store_pairs<VEC>(w, static_cast<T*>(p.g.df) + row * p.g.lddf + c, cols - c);
        }
    }
    if (p.dpre) sums.template put<VEC>(kDpre, p.dpre + (int64_t)blockIdx.x * cols, cols);
    if (gates) finish(gate);
    if (!p.dpost) return;
    float* const to = p.dpost + (int64_t)blockIdx.x * cols;
    if (!gates) {
        sums.template put<VEC>(kInner, to, cols);
        return;
    }
#pragma unroll
    for (int i = 0; i < VC; ++i) {
        const int c = (threadIdx.x + i * blockDim.x) * 8;
        put8<VEC>(gathered + c, to + c, cols - c);
    }
}

// A thread's 32 bytes of columns times `factor`, from its bytes.
// The bytes from `valid` on read as 0.
template <typename T>
__device__ __forceinline__ void held32(const unsigned char* bytes, int valid, float m, float ratio, float factor,
                                       u64* n) {
    const Act8Lines L = act8_lines(m, ratio, factor);
    constexpr int kWords = kPairs32<T> / 2;
    uint32_t b[4];
    if (kWords == 4) {
        const uint4 x = *reinterpret_cast<const uint4*>(bytes);
        b[0] = x.x; b[1] = x.y; b[2] = x.z; b[3] = x.w;
    } else {
        const uint2 x = *reinterpret_cast<const uint2*>(bytes);
        b[0] = x.x; b[1] = x.y; b[2] = b[3] = 0u;
    }
    if (valid < 4 * kWords)
#pragma unroll
        for (int i = 0; i < kWords; ++i) {
            const int k = valid - 4 * i;  // bytes of this word that exist
            b[i] = k >= 4 ? b[i] : k <= 0 ? 0u : b[i] & (0xffffffffu >> (32 - 8 * k));
        }
    act8_scaled8(make_uint2(b[0], b[1]), L, n);
    if (kWords == 4) act8_scaled8(make_uint2(b[2], b[3]), L, n + kPairs32<T> - 4);
}

__device__ __forceinline__ void set_rank(CtaSum&, uint32_t) {}
__device__ __forceinline__ void set_rank(PairSum& s, uint32_t rank) { s.rank = rank; }

// Backward with a ring: 32 bytes of columns per thread, sums in registers.  PAIR: a cluster of two CTAs
// shares the rows, half the columns each (rows too wide for one CTA's registers).
template <typename T, bool WF32, bool PAIR, bool ODD>
__global__ void __launch_bounds__(512)
block_norm_backward_ring_kernel(const __grid_constant__ GradParams p) {
    constexpr int kP = kPairs32<T>;
    __shared__ float buf[2][32];
    __shared__ uint64_t full[kMaxStages];
    extern __shared__ __align__(16) unsigned char smem[];
    const uint32_t rank = PAIR ? cluster_rank() : 0;
    typename std::conditional<PAIR, PairSum, CtaSum>::type cta_sum{buf};
    const NormParams& q = p.q;
    const int64_t cta = PAIR ? blockIdx.x >> 1 : blockIdx.x;
    const int cols = PAIR ? (int)q.a.cols / 2 : (int)q.a.cols, base = (int)rank * cols;
    const int64_t first = cta * p.rows_per_cta, last = min(first + p.rows_per_cta, q.a.rows);
    const bool pre = q.a.pre_weight, post = q.a.post_weight, has_f = q.a.f_codes, has_dr = p.g.dr;
    uint4* const turn = reinterpret_cast<uint4*>(smem);
    Ring ring{full, smem + turn_bytes<ODD>(),
              (pre ? q.slot_bytes + q.code_bytes : 0) + (has_dr ? q.slot_bytes : 0) + (has_f ? q.code_bytes : 0),
              q.stages};
    if (PAIR && threadIdx.x < 64) buf[threadIdx.x >> 5][threadIdx.x & 31] = 0.0f;
    if (threadIdx.x == 0) {
        for (int s = 0; s < q.stages; ++s) mbar_init(&full[s], 1);
        fence_barrier_init();
        for (int s = 0; s < q.stages; ++s)
            if (first + s < last) request_backward<T, ODD>(p, ring, s, first + s, base);
    }
    __syncthreads();
    if (PAIR) {
        set_rank(cta_sum, rank);
        cluster_sync();                   // the other CTA writes to this one's sums
    }
    // threads past the row repeat its last columns and neither store nor count
    const bool live = (int)threadIdx.x * 2 * kP < cols;
    const int local = live ? (int)threadIdx.x * 2 * kP : (cols - 1) / (2 * kP) * (2 * kP), c = base + local;
    const int valid = ODD ? cols - local : 2 * kP;
    const int warp_c = (int)(threadIdx.x & ~31u) * 2 * kP;       // of the warp's first lane
    // where this thread's part of each operand lies in a stage
    const unsigned at_dh = local * (int)sizeof(T), at_rb = q.slot_bytes + local,
                   at_dr = (pre ? q.slot_bytes + q.code_bytes : 0) + local * (int)sizeof(T),
                   at_fb = ring.stage_bytes - q.code_bytes + local;
    int64_t gate = q.a.gate ? first / q.a.gate_tokens : 0;
    int64_t gate_end = (gate + 1) * q.a.gate_tokens;
    u64 dpre[kP] = {}, inner[kP] = {};
    allow_dependents();
    float* const gathered = reinterpret_cast<float*>(smem + p.gathered) - base;
    const bool gates = p.gates && (p.dpost || p.dgate);
    if (gates && p.dpost && live)
#pragma unroll
        for (int k = 0; k < 2 * kP; ++k) gathered[c + k] = 0.0f;
    auto finish = [&](int64_t gate) {
        if (live)
#pragma unroll
            for (int k = 0; k < kP; k += 4)
                finish_gate<!ODD, T>(p, cta, gate, first, last, c + 2 * k, valid - 2 * k, inner + k, gathered);
#pragma unroll
        for (int k = 0; k < kP; ++k) inner[k] = 0ull;
    };
    auto put = [&](const u64* v, float* to) {
        if (!live) return;
#pragma unroll
        for (int k = 0; k < kP; k += 4) {
            if (!ODD) {
                store32(to + c + 2 * k, raw32(v + k, 0.0f));
                continue;
            }
            float f[8];
            floats8(v + k, f);
            put8<false>(f, to + c + 2 * k, valid - 2 * k);
        }
    };

    // a row's ranges and factors, requested one row ahead
    float next_mr = 0.0f, next_mf = 0.0f, next_rr = 0.0f, next_rf = kAsItIs;
    auto fetch = [&](int64_t row) {
        if (pre) next_rr = q.a.r_rstd[row];
        if (post) next_rf = q.a.f_rstd[row];
        const int64_t at = row * q.groups + (c >> q.group_shift);
        if (pre) next_mr = q.a.r_ranges[at];
        if (has_f) next_mf = q.a.f_ranges[at];
    };
    if (first < last) fetch(first);

    for (int64_t row = first; row < last; ++row) {
        if (q.a.gate && row == gate_end) {
            if (gates) finish(gate);
            ++gate;
            gate_end += q.a.gate_tokens;
        }
        const float mr = next_mr, mf = next_mf, rr = next_rr, rf = next_rf;
        if (row + 1 < last) fetch(row + 1);
        u64 e[kP], n[kP], w[kP];
        Weights<T, WF32> wt, gt;
        if (pre) wt.template load<ODD>(q.a.pre_weight, 0, c, valid);
        const unsigned char* at = ring.wait();
        // outer norm: e = dr + rstd * (u - n * mean(u n))
        if (pre) {
            pairs32(ring32<T, ODD>(at + at_dh + row_skip<T, ODD>(p.g.dh, p.g.lddh, row), valid), e, T());
            held32<T>(at + at_rb, valid, mr, q.ratio, rr, n);
            wt.get(w, q.offset);
            if (post) wt.template load<ODD>(q.a.post_weight, 0, c, valid);
            if (q.a.gate) gt.template load<ODD>(q.a.gate, gate * q.a.ldgate, c, valid);
            u64 s = 0ull;
#pragma unroll
            for (int k = 0; k < kP; ++k) {
                dpre[k] = fma2(e[k], n[k], dpre[k]);
                e[k] = mul2(e[k], w[k]);
                s = fma2(e[k], n[k], s);
            }
            cta_sum.post(live ? sum8(s) : 0.0f);
            Raw32 raw_dr;
            if (has_dr) raw_dr = ring32<T, ODD>(at + at_dr + row_skip<T, ODD>(p.g.dr, p.g.lddr, row), valid);
            const float mean = cta_sum.total() * q.inv_cols;
#pragma unroll
            for (int k = 0; k < kP; ++k) e[k] = mul2(fma2(n[k], both(-mean), e[k]), both(rr));
            if (has_dr) {
                pairs32(raw_dr, w, T());
#pragma unroll
                for (int k = 0; k < kP; ++k) e[k] = add2(e[k], w[k]);
            }
        } else {                          // without the outer norm dr is all there is
            if (post) wt.template load<ODD>(q.a.post_weight, 0, c, valid);
            if (q.a.gate) gt.template load<ODD>(q.a.gate, gate * q.a.ldgate, c, valid);
            pairs32(ring32<T, ODD>(at + at_dr + row_skip<T, ODD>(p.g.dr, p.g.lddr, row), valid), e, T());
        }
        if (p.g.dx && (ODD || live)) {
#pragma unroll
            for (int k = 0; k < kP; ++k) w[k] = mul2(e[k], both(q.scale));
            T* const to = static_cast<T*>(p.g.dx) + row * p.g.lddx;
            put32<T, ODD>(to + c, raw32(w, T()), live, turn, to + warp_c, cols - warp_c);
        }
        // inner norm and gate; e becomes v = e * gate * w
        float mean = 0.0f;
        if (has_f) {
            held32<T>(at + at_fb, valid, mf, q.ratio, rf, n);
#pragma unroll
            for (int k = 0; k < kP; ++k) inner[k] = fma2(e[k], n[k], inner[k]);
            if (q.a.gate) {
                gt.get(w);
#pragma unroll
                for (int k = 0; k < kP; ++k) e[k] = mul2(e[k], w[k]);
            }
            u64 s = 0ull;
            if (post) {
                wt.get(w, q.offset);
#pragma unroll
                for (int k = 0; k < kP; ++k) {
                    e[k] = mul2(e[k], w[k]);
                    s = fma2(e[k], n[k], s);
                }
            }
            if (post) mean = cta_sum(live ? sum8(s) : 0.0f) * q.inv_cols;
        }
        if (!post) __syncthreads();
        // every thread has its values of this stage
        const int64_t ahead = row + q.stages;
        if (threadIdx.x == 0 && ahead < last && !ring.dead) request_backward<T, ODD>(p, ring, ring.stage, ahead, base);
        ring.next();
        if (!p.g.df || (!ODD && !live)) continue;
        if (post)
#pragma unroll
            for (int k = 0; k < kP; ++k) e[k] = mul2(fma2(n[k], both(-mean), e[k]), both(rf));
        T* const to = static_cast<T*>(p.g.df) + row * p.g.lddf;
        put32<T, ODD>(to + c, raw32(e, T()), live, turn, to + warp_c, cols - warp_c);
    }
    if (p.dpre) put(dpre, p.dpre + cta * q.a.cols);
    if (gates) finish(gate);
    if (!p.dpost) return;
    if (gates && live)
#pragma unroll
        for (int k = 0; k < kP; ++k) inner[k] = pack2(gathered[c + 2 * k], gathered[c + 2 * k + 1]);
    put(inner, p.dpost + cta * q.a.cols);
}

// Backward of narrow rows (see block_norm_narrow_kernel), for one gate at most.  The CTA's rows are not
// neighbours here, but its sums are those of one CTA all the same.  16-bit values: at the 128 registers that
// two CTAs a multiprocessor leave, 200 bytes a thread spill (weights and sums of 16 columns live over the loop).
template <typename T, bool WF32>
__global__ void __launch_bounds__(kNarrowThreads, 2)
block_norm_backward_narrow_kernel(const __grid_constant__ GradParams p, int lanes) {
    constexpr int kP = kPairs32<T>, kWarps = kNarrowThreads / 32;
    __shared__ __align__(16) float part[kWarps][32 * 2 * kP];
    const NormParams& q = p.q;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, in = lane & (lanes - 1);
    const bool pre = q.a.pre_weight, post = q.a.post_weight, has_f = q.a.f_codes, has_dr = p.g.dr;
    const bool inside = in * 2 * kP < (int)q.a.cols;
    const int c = inside ? in * 2 * kP : (int)q.a.cols - 2 * kP;
    const int64_t per_step = (int64_t)gridDim.x * kNarrowThreads / lanes;
    Weights<T, WF32> post_w, pre_w, gate_w;
    if (post) post_w.load(q.a.post_weight, c);
    if (pre) pre_w.load(q.a.pre_weight, c);
    if (q.a.gate) gate_w.load(q.a.gate, c);
    allow_dependents();
    u64 dpre[kP] = {}, inner[kP] = {};
    int64_t row = ((int64_t)blockIdx.x * kNarrowThreads + threadIdx.x) / lanes;
    for (int64_t at = row - lane / lanes; at < q.a.rows; at += per_step, row += per_step) {
        const bool live = inside && row < q.a.rows;
        const int64_t t = min(row, q.a.rows - 1), range = t * q.groups + (c >> q.group_shift);
        Raw32 raw_dh, raw_dr;
        float mr = 0.0f, mf = 0.0f, rr = 0.0f, rf = kAsItIs;
        uint4 rb, fb;
        auto bytes = [&](const uint8_t* codes) {
            const uint8_t* from = codes + t * q.a.ldc + c;
            if (kP == 8) return *reinterpret_cast<const uint4*>(from);
            const uint2 b = *reinterpret_cast<const uint2*>(from);
            return make_uint4(b.x, b.y, 0u, 0u);
        };
        if (pre) {
            raw_dh = load32_global(static_cast<const T*>(p.g.dh) + t * p.g.lddh + c);
            rb = bytes(q.a.r_codes);
            mr = q.a.r_ranges[range];
            rr = q.a.r_rstd[t];
        }
        if (has_dr) raw_dr = load32_global(static_cast<const T*>(p.g.dr) + t * p.g.lddr + c);
        if (has_f) {
            fb = bytes(q.a.f_codes);
            mf = q.a.f_ranges[range];
            if (post) rf = q.a.f_rstd[t];
        }
        u64 e[kP], n[kP], w[kP], s = 0ull;
        if (pre) {
            pairs32(raw_dh, e, T());
            held32<T>(reinterpret_cast<const unsigned char*>(&rb), 2 * kP, mr, q.ratio, rr, n);
            pre_w.get(w, q.offset);
            if (live)
#pragma unroll
                for (int k = 0; k < kP; ++k) dpre[k] = fma2(e[k], n[k], dpre[k]);
#pragma unroll
            for (int k = 0; k < kP; ++k) {
                e[k] = mul2(e[k], w[k]);
                s = fma2(e[k], n[k], s);
            }
            const float mean = lanes_sum(inside ? sum8(s) : 0.0f, lanes) * q.inv_cols;
#pragma unroll
            for (int k = 0; k < kP; ++k) e[k] = mul2(fma2(n[k], both(-mean), e[k]), both(rr));
            if (has_dr) {
                pairs32(raw_dr, w, T());
#pragma unroll
                for (int k = 0; k < kP; ++k) e[k] = add2(e[k], w[k]);
            }
        } else {
            pairs32(raw_dr, e, T());
        }
        if (p.g.dx && live) {
#pragma unroll
            for (int k = 0; k < kP; ++k) w[k] = mul2(e[k], both(q.scale));
            store32(static_cast<T*>(p.g.dx) + row * p.g.lddx + c, raw32(w, T()));
        }
        float mean = 0.0f;
        if (has_f) {
            held32<T>(reinterpret_cast<const unsigned char*>(&fb), 2 * kP, mf, q.ratio, rf, n);
            if (live)
#pragma unroll
                for (int k = 0; k < kP; ++k) inner[k] = fma2(e[k], n[k], inner[k]);
            if (q.a.gate) {
                gate_w.get(w);
#pragma unroll
                for (int k = 0; k < kP; ++k) e[k] = mul2(e[k], w[k]);
            }
            if (post) {
                post_w.get(w, q.offset);
                s = 0ull;
#pragma unroll
                for (int k = 0; k < kP; ++k) {
                    e[k] = mul2(e[k], w[k]);
                    s = fma2(e[k], n[k], s);
                }
                mean = lanes_sum(inside ? sum8(s) : 0.0f, lanes) * q.inv_cols;
            }
        }
        if (!p.g.df || !live) continue;
        if (post)
#pragma unroll
            for (int k = 0; k < kP; ++k) e[k] = mul2(fma2(n[k], both(-mean), e[k]), both(rf));
        store32(static_cast<T*>(p.g.df) + row * p.g.lddf + c, raw32(e, T()));
    }
    // a warp's rows, then the warps, in a fixed order
    auto reduce = [&](u64* v) {
        for (int o = lanes; o < 32; o <<= 1)
#pragma unroll
            for (int k = 0; k < kP; ++k) v[k] = add2(v[k], __shfl_xor_sync(0xffffffffu, v[k], o));
        __syncthreads();
        if (lane < lanes)
#pragma unroll
            for (int k = 0; k < kP; k += 2)
                *reinterpret_cast<ulonglong2*>(&part[warp][in * 2 * kP + 2 * k]) = make_ulonglong2(v[k], v[k + 1]);
        __syncthreads();
        if (warp == 0 && lane < lanes)
            for (int j = 1; j < kWarps; ++j)
#pragma unroll
                for (int k = 0; k < kP; k += 2) {
                    const ulonglong2 x = *reinterpret_cast<const ulonglong2*>(&part[j][in * 2 * kP + 2 * k]);
                    v[k] = add2(v[k], x.x);
                    v[k + 1] = add2(v[k + 1], x.y);
                }
    };
    const bool mine = warp == 0 && lane < lanes && inside;
    if (p.dpre) {
        reduce(dpre);
        if (mine)
#pragma unroll
            for (int k = 0; k < kP; k += 4)
                store32(p.dpre + (int64_t)blockIdx.x * q.a.cols + c + 2 * k, raw32(dpre + k, 0.0f));
    }
    if (!p.dpost) return;
    reduce(inner);
    if (mine)
#pragma unroll
        for (int k = 0; k < kP; k += 4)
            store32(p.dpost + (int64_t)blockIdx.x * q.a.cols + c + 2 * k, raw32(inner + k, 0.0f));
}

// Adds the CTAs' sums of V columns per thread (4 where the columns allow it): 64 parts of the CTAs side
// by side, eight loads of a part in flight, then the parts.  blockIdx.y 0: dpre, 1: dpost, 2: zeros for
// the gates without rows and, where few CTAs share a gate (`few`), the gates that do not end in the CTA
// they begin in, one per threadIdx.y; else 3 + g: gate g.
constexpr int kSumLanes = 8, kSumParts = 64, kFewShares = 16;
template <int V> struct alignas(4 * V) Columns {
    float v[V];
    __device__ __forceinline__ void add(const float* p) {
        const Columns x = *reinterpret_cast<const Columns*>(p);
#pragma unroll
        for (int k = 0; k < V; ++k) v[k] += x.v[k];
    }
    template <typename W> __device__ __forceinline__ void times(const W* w, int c, float offset) {
#pragma unroll
        for (int k = 0; k < V; ++k) v[k] *= to_f32(w[c + k]) + offset;
    }
    __device__ __forceinline__ void times(float w) {
#pragma unroll
        for (int k = 0; k < V; ++k) v[k] *= w;
    }
    template <typename W> __device__ __forceinline__ void put(W* to) const {
#pragma unroll
        for (int k = 0; k < V; ++k) to[k] = from_f32<W>(v[k]);
    }
};
template <typename W, int V>
__global__ void __launch_bounds__(kSumLanes * kSumParts)
block_norm_sums_kernel(const __grid_constant__ GradParams p, int ctas, bool few, W* dpre, W* dpost, W* dgate) {
    __shared__ Columns<V> part[kSumParts][kSumLanes];
    const pwlq_block_norm_args& a = p.q.a;
    const int cols = (int)a.cols;
    const int c = (blockIdx.x * kSumLanes + threadIdx.x) * V;
    // rows and their quotients fit 32 bits
    const unsigned rows = (unsigned)a.rows, per_cta = (unsigned)p.rows_per_cta;
    const unsigned every = (unsigned)min(a.gate_tokens, (int64_t)0x7fffffff);
    await_previous();
    if (blockIdx.y == 2) {
        if (c >= cols) return;
        const int64_t used = (a.rows + a.gate_tokens - 1) / a.gate_tokens;
        for (int64_t g = used + threadIdx.y; g < a.gate_rows; g += kSumParts) Columns<V>{}.put(dgate + g * cols + c);
        if (!few) return;
        const float* src = p.dgate + c;
        if (every < per_cta) {             // a gate goes on into the next CTA, and ends there
            for (unsigned b = 1 + threadIdx.y; b < (unsigned)ctas; b += kSumParts) {
                if (b * per_cta % every == 0) continue;
                Columns<V> s = {};
                s.add(src + (int64_t)(2 * b - 1) * cols);
                s.add(src + (int64_t)(2 * b) * cols);
                s.put(dgate + (int64_t)(b * per_cta / every) * cols + c);
            }
            return;
        }
        for (unsigned g = threadIdx.y; g < (unsigned)used; g += kSumParts) {
            const unsigned from = g * every, lo = from / per_cta;
            const unsigned hi = (unsigned)((min((uint64_t)from + every, (uint64_t)rows) - 1) / per_cta);
            if (lo == hi) continue;
            Columns<V> s = {};
            s.add(src + (int64_t)(2 * lo + (from > lo * per_cta)) * cols);
            for (unsigned b = lo + 1; b <= hi; ++b) s.add(src + (int64_t)(2 * b) * cols);
            s.put(dgate + (int64_t)g * cols + c);
        }
        return;
    }
    W* out = blockIdx.y == 0 ? dpre : dpost;
    const float* src = (blockIdx.y == 0 ? p.dpre : p.dpost) + c;
    int lo = 0, hi = ctas;
    int64_t pitch = cols, first = 0;               // how far the first share lies beyond its CTA's others
    if (blockIdx.y > 2) {
        const unsigned g = blockIdx.y - 3, from = g * every;
        lo = (int)(from / per_cta);
        hi = (int)((min((uint64_t)from + every, (uint64_t)rows) - 1) / per_cta) + 1;
        if (hi == lo + 1) return;                  // written by that CTA
        out = dgate + (int64_t)g * cols;
        src = p.dgate + c;
        pitch = 2 * (int64_t)cols;
        first = from > lo * per_cta ? cols : 0;
    }
    if (blockIdx.y == 0 ? !out : !p.dpost && blockIdx.y == 1) return;
    Columns<V> s = {};
    if (c < cols) {
#pragma unroll 8
        for (int b = lo + threadIdx.y; b < hi; b += kSumParts) s.add(src + b * pitch + (b == lo ? first : 0));
    }
    part[threadIdx.y][threadIdx.x] = s;
    __syncthreads();
    // eight parts each, then the eight
#pragma unroll
    for (int step = 1; step < kSumParts; step *= 8) {
        if (threadIdx.y % (8 * step) == 0) {
#pragma unroll
            for (int j = 1; j < 8; ++j) s.add(part[threadIdx.y + j * step][threadIdx.x].v);
            part[threadIdx.y][threadIdx.x] = s;
        }
        __syncthreads();
    }
    if (threadIdx.y != 0 || c >= cols) return;
    if (blockIdx.y == 1 && a.gate && !p.gates) {   // s is A, of all rows
        Columns<V> x = s;
        if (a.post_weight) x.times(static_cast<const W*>(a.post_weight), c, p.q.offset);
        else x.times(1.0f / kAsItIs);
        if (dgate) x.put(dgate + c);
        s.times(static_cast<const W*>(a.gate), c, 0.0f);
    }
    if (out) s.put(out + c);
}

// ------------------------------------------------------------------------------ launching
// Multiprocessors of the current device (looked up once per device).
int sm_count() {
    static std::mutex mutex;
    static int known[64] = {};
    int dev = 0, sms = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) return 148;
    std::lock_guard<std::mutex> lock(mutex);
    if (!known[dev]) {
        if (cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess || sms < 1) return 148;
        known[dev] = sms;
    }
    return known[dev];
}

NormParams params(const pwlq_block_norm_args& a) {
    NormParams q;
    q.a = a;
    q.scale = (float)a.residual_scale;
    q.eps = (float)a.eps;
    q.offset = (float)a.weight_offset;
    q.inv_cols = 1.0f / (float)a.cols;
    q.ratio = (float)a.ratio;
    q.group_shift = group_shift((int)a.group);
    q.group_lanes = 1 << (q.group_shift - 3);
    q.groups = a.group > 0 ? (a.cols + a.group - 1) / a.group : 0;
    q.wf32 = a.wtype == kF32;
    q.stages = 0;
    q.gate_step = q.gate_rest = 0;
    q.row_bytes = (unsigned)(a.cols * type_size((int)a.dtype));
    q.code_bytes = (unsigned)((a.cols + 15) / 16 * 16);
    q.slot_bytes = q.row_bytes;
    return q;
}

// Rows that the kernels of 32 bytes per thread cannot take as they lie (ODD): a slot for the aligned
// words that hold one and for the 16 bytes after its last thread's part.
inline void odd_slots(NormParams& q) { q.slot_bytes = (q.row_bytes + 31) / 32 * 32 + 32; }
inline size_t turn_bytes(bool odd, int threads) { return odd ? (size_t)threads / 32 * kTurn * 16 : 0; }

inline bool weights_aligned(const pwlq_block_norm_args& a) {
    const size_t ws = type_size((int)a.wtype);
    return rows_aligned(a.post_weight, 0, ws) && rows_aligned(a.pre_weight, 0, ws) &&
           rows_aligned(a.gate, a.ldgate, ws);
}

inline int threads_for(int64_t cols, int per_thread) {
    const int64_t n = (cols + per_thread - 1) / per_thread;
    return (int)((n + 31) / 32 * 32);
}

// Shared memory above the default 48 KB has to be allowed to a kernel before its launch.  It is allowed
// the most that any call of its form asks for, never a call's own size: calls from several threads share
// the attribute, and a smaller one set between another's setting and launch made that launch fail.
constexpr size_t kSmemBudget = 160 * 1024;      // what a multiprocessor's rings may take for their stages
constexpr size_t kRingMost = kSmemBudget + 24 * kTurn * 16 + 8192 * sizeof(float);   // stages, turns, gathered
constexpr size_t kDirectMost = 512 * (2 * 4 * 8 + 32) * sizeof(float);               // sums, gathered
template <typename K>
cudaError_t allow_smem(K* kernel, size_t smem, size_t most) {
    if (smem <= 12 * 1024) return cudaSuccess;  // with the static part below 48 KB
    return cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)most);
}
template <typename K, typename P>
cudaError_t run(K* kernel, unsigned ctas, int threads, size_t smem, size_t most, cudaStream_t stream, const P& p) {
    if (const cudaError_t e = allow_smem(kernel, smem, most)) return e;
    kernel<<<ctas, threads, smem, stream>>>(p);
    return cudaGetLastError();
}

// A ring kernel's launch: threads of 32 bytes of columns each; CTAs that share a multiprocessor, as
// far as their registers allow (`threads_per_sm`); stages of `bytes` for each of them.
struct RingPlan { int threads, ctas, stages; };
// two stages of every width up to the ring's limits fit
RingPlan ring_plan(int64_t cols, size_t size, int threads_per_sm, size_t bytes) {
    RingPlan r;
    r.threads = threads_for(cols, (int)(32 / size));
    r.ctas = std::max(1, std::min(16, threads_per_sm / r.threads));
    r.stages = bytes ? (int)std::min<size_t>((kSmemBudget / r.ctas - 1024) / bytes, kMaxStages) : 0;
    return r;
}
// 32-byte accesses to values need rows, and columns per thread, on 32-byte boundaries.
inline bool rows_aligned32(const void* p, int64_t ld, size_t size) {
    return ((reinterpret_cast<uintptr_t>(p) | (uintptr_t)(ld * (int64_t)size)) & 31) == 0;
}

// Lanes per row of the narrow kernels; 0: the rows are too wide for them.
inline int narrow_lanes(int64_t cols, size_t size) {
    const int64_t n = (cols * (int64_t)size + 31) / 32;
    int lanes = 2;                        // a pair of lanes shares the reciprocals of a range
    while (lanes < n) lanes *= 2;
    return lanes <= 32 ? lanes : 0;
}
// CTAs of a narrow kernel: four per multiprocessor at most, whole rounds of rows where there are few.
inline int64_t narrow_ctas(int64_t rows, int lanes) {
    const int64_t per_cta = kNarrowThreads / lanes;
    return std::min<int64_t>((rows + per_cta - 1) / per_cta, 4 * (int64_t)sm_count());
}

template <typename T, bool SAVE>
cudaError_t forward(const pwlq_block_norm_args& a, cudaStream_t stream) {
    NormParams q = params(a);
    constexpr size_t kSize = sizeof(T);
    const bool rows32 = a.cols % (32 / kSize) == 0 && rows_aligned32(a.x, a.ldx, kSize) &&
                        rows_aligned32(a.f, a.ldf, kSize) && rows_aligned32(a.r, a.ldr, kSize) &&
                        rows_aligned32(a.h, a.ldh, kSize) && weights_aligned(a);
    const int lanes = narrow_lanes(a.cols, kSize);
    if (rows32 && lanes) {
        q.group_lanes = std::min((int)(a.group * kSize / 32), lanes);
        auto* kernel = q.wf32 ? block_norm_narrow_kernel<T, SAVE, true> : block_norm_narrow_kernel<T, SAVE, kSize == 4>;
        kernel<<<(unsigned)narrow_ctas(a.rows, lanes), kNarrowThreads, 0, stream>>>(q, lanes);
        return cudaGetLastError();
    }
    const bool vec = rows_aligned(a.x, a.ldx, kSize) && rows_aligned(a.f, a.ldf, kSize) &&
                     rows_aligned(a.r, a.ldr, kSize) && rows_aligned(a.h, a.ldh, kSize) && weights_aligned(a);
    // Rows that lie anywhere, 16-bit types: 16384 x 4095 234 -> 144 us (with checkpoints 305 -> 218) against
    // threads that load for themselves.  Not binary32 (16384 x 2047: 122 against 133 us), nor rows on
    // 16-byte boundaries that end inside a thread's part (16384 x 4104: 115 against 171 us).
    const bool odd = kSize == 2 && !vec;
    if (odd) odd_slots(q);
    const size_t stage = (a.f ? 2 : 1) * (size_t)q.slot_bytes;
    const RingPlan ring = ring_plan(a.cols, kSize, odd ? 768 : 1024, stage);
    const int64_t resident = (int64_t)ring.ctas * sm_count();
    // A ring pays once every CTA has a few rows to walk (with checkpoints, bf16 1776 x 4096 18.1 against 24.1 us,
    // 592 rows 7.7 against 9.2, but 148 rows 5.1 against 4.5; without them 592 rows 5.3 against 4.9).  The rule
    // does not ask for checkpoints, since saving them must not change r and h: it gives up the 592 rows with them.
    // (block_norm_row_kernel has the ring's bits, too, and could take these sizes without checkpoints; not measured.)
    if ((rows32 || odd) && ring.threads <= (odd ? 768 : 1024) && ring.stages >= 2 && a.rows >= 2 * resident) {
        // Without checkpoints, up to how many columns a CTA per row is faster than the ring: with one reduction
        // 8192 (bf16 83 against 96 us, binary32 169 against 184 us; 12288: 98 against 99), with two 4096 (88 against 96;
        // 8192: 99 against 91) or, binary32, 5120 (172 against 181; 6144: 247 against 179), with a gate between them
        // 2048 (88 against 91; 2560: 95 against 88) or 2560 (166 against 166; 4096: 192 against 171).
        constexpr bool kF = kSize == 4;
        const int64_t light = !a.f || !a.post_weight ? 8192 : a.gate ? (kF ? 2560 : 2048) : kF ? 5120 : 4096;
        if (!SAVE && !odd && q.wf32 == kF && a.cols <= light)
            return run(block_norm_row_kernel<T>, (unsigned)a.rows, ring.threads, 0, 0, stream, q);
        q.stages = ring.stages;
        q.group_lanes = (int)(a.group * kSize / 32);
        if (a.gate) {
            q.gate_step = resident / a.gate_tokens;
            q.gate_rest = resident % a.gate_tokens;
        }
        auto* kernel = q.wf32 ? block_norm_ring_kernel<T, SAVE, true, false>
                              : block_norm_ring_kernel<T, SAVE, kSize == 4, false>;
        if constexpr (kSize == 2) {
            if (odd) kernel = q.wf32 ? block_norm_ring_kernel<T, SAVE, true, true>
                                     : block_norm_ring_kernel<T, SAVE, false, true>;
        }
        return run(kernel, (unsigned)resident, ring.threads, turn_bytes(odd, ring.threads) + ring.stages * stage,
                   kRingMost, stream, q);
    }
    const unsigned rows = (unsigned)a.rows;
    if (a.cols <= 8192)
        return vec ? run(block_norm_kernel<T, 1, true, SAVE>, rows, threads_for(a.cols, 8), 0, 0, stream, q)
                   : run(block_norm_kernel<T, 1, false, SAVE>, rows, threads_for(a.cols, 8), 0, 0, stream, q);
    return vec ? run(block_norm_kernel<T, 2, true, SAVE>, rows, threads_for(a.cols, 16), 0, 0, stream, q)
               : run(block_norm_kernel<T, 2, false, SAVE>, rows, threads_for(a.cols, 16), 0, 0, stream, q);
}
template <typename T>
cudaError_t forward(const pwlq_block_norm_args& a, cudaStream_t stream) {
    return a.r_codes || a.f_codes || a.r_rstd || a.f_rstd ? forward<T, true>(a, stream) : forward<T, false>(a, stream);
}

// CTAs of the backward pass: the rows are shared out evenly over at most this many.  As many as fit at once
// where a thread has 16 columns (16-bit values); binary32 rings have 8, and so two rounds of CTAs.
inline int64_t backward_ctas(int64_t rows, int64_t cols) {
    const int64_t per_sm = cols > 8192 ? 1 : std::max(1, std::min(16, 512 / threads_for(cols, 16)));
    return std::min<int64_t>(rows, per_sm * sm_count());
}

// Whether the kernels that read 32 bytes of columns at a time do.
template <typename T>
bool rows32_backward(const pwlq_block_norm_args& a, const pwlq_block_norm_grads& g) {
    constexpr size_t kSize = sizeof(T);
    return a.cols % (32 / kSize) == 0 && (a.pre_weight || g.dr) && rows_aligned32(g.dh, g.lddh, kSize) &&
           rows_aligned32(g.dr, g.lddr, kSize) && rows_aligned32(g.dx, g.lddx, kSize) &&
           rows_aligned32(g.df, g.lddf, kSize) && rows_aligned(g.dgate, a.cols, type_size((int)a.wtype)) &&
           weights_aligned(a);
}

// The ring's stage of a row of `cols` columns.
inline size_t backward_stage(const GradParams& p) {
    const pwlq_block_norm_args& a = p.q.a;
    return (a.pre_weight ? p.q.slot_bytes + p.q.code_bytes : 0) + (p.g.dr ? p.q.slot_bytes : 0) +
           (a.f_codes ? p.q.code_bytes : 0);
}

// Rows that one CTA's registers cannot sum: a pair of CTAs, where the halves are whole threads'.
template <typename T>
bool pairs_backward(const GradParams& p) {
    const pwlq_block_norm_args& a = p.q.a;
    return threads_for(a.cols, 32 / sizeof(T)) > 512 && threads_for(a.cols, 64 / sizeof(T)) <= 512 &&
           a.cols % 32 == 0 && rows32_backward<T>(a, p.g);
}
template <typename T>
cudaError_t backward_pairs(GradParams& p, unsigned pairs, cudaStream_t stream) {
    const pwlq_block_norm_args& a = p.q.a;
    p.q.slot_bytes = p.q.row_bytes /= 2;
    p.q.code_bytes = (unsigned)(a.cols / 2);
    const size_t stage = backward_stage(p);
    const RingPlan ring = ring_plan(a.cols / 2, sizeof(T), 512, stage);
    p.q.stages = ring.stages;
    p.gathered = (unsigned)(ring.stages * stage);
    const size_t smem = p.gathered + (p.gates && p.g.dpost ? (size_t)a.cols / 2 * sizeof(float) : 0);
    auto* kernel = p.q.wf32 ? block_norm_backward_ring_kernel<T, true, true, false>
                            : block_norm_backward_ring_kernel<T, sizeof(T) == 4, true, false>;
    if (const cudaError_t e = allow_smem(kernel, smem, kRingMost)) return e;
    cudaLaunchAttribute attr;
    attr.id = cudaLaunchAttributeClusterDimension;
    attr.val.clusterDim.x = 2;
    attr.val.clusterDim.y = attr.val.clusterDim.z = 1;
    cudaLaunchConfig_t config = {};
    config.gridDim = dim3(2 * pairs);
    config.blockDim = dim3((unsigned)ring.threads);
    config.dynamicSmemBytes = smem;
    config.stream = stream;
    config.attrs = &attr;
    config.numAttrs = 1;
    return cudaLaunchKernelEx(&config, kernel, p);
}

template <typename T>
cudaError_t backward_rows(GradParams& p, unsigned ctas, cudaStream_t stream) {
    const pwlq_block_norm_grads& g = p.g;
    const pwlq_block_norm_args& a = p.q.a;
    constexpr size_t kSize = sizeof(T);
    const size_t wsize = type_size((int)a.wtype);
    const bool vec = rows_aligned(g.dh, g.lddh, kSize) && rows_aligned(g.dr, g.lddr, kSize) &&
                     rows_aligned(g.dx, g.lddx, kSize) && rows_aligned(g.df, g.lddf, kSize) &&
                     rows_aligned(g.dgate, a.cols, wsize) && a.cols % 4 == 0 && weights_aligned(a);
    const bool gathers = p.gates && g.dpost;
    if (a.cols > 8192) {
        const int threads = threads_for(a.cols, 32);
        p.gathered = (unsigned)((size_t)2 * 4 * 8 * sizeof(float) * threads);     // at most 128 KB of sums
        const size_t smem = p.gathered + (gathers ? (size_t)threads * 32 * sizeof(float) : 0);
        return vec ? run(block_norm_backward_kernel<T, 4, true, true>, ctas, threads, smem, kDirectMost, stream, p)
                   : run(block_norm_backward_kernel<T, 4, false, true>, ctas, threads, smem, kDirectMost, stream, p);
    }
    const bool rows32 = rows32_backward<T>(a, g);
    // Rows that lie anywhere, 16-bit types: 16384 x 4095 352 -> 254 us, 16384 x 4104 406 -> 382 us against
    // threads that load for themselves.  Not binary32 (16384 x 2047: 190 against 192 us), nor gates of a few
    // rows, whose gradients go value by value (8192 x 4095, a gate per row: 286 against 327 us).
    const bool odd = !rows32 && kSize == 2 && (!p.dgate || a.gate_tokens >= 8);
    if (odd) odd_slots(p.q);
    const size_t stage = backward_stage(p);
    const RingPlan ring = ring_plan(a.cols, kSize, 512, stage);
    if ((rows32 || odd) && ring.threads <= 512 && ring.stages >= 2 && (a.pre_weight || g.dr)) {
        p.q.stages = ring.stages;
        p.gathered = (unsigned)(turn_bytes(odd, ring.threads) + ring.stages * stage);
        const size_t smem = p.gathered + (gathers ? (size_t)(a.cols + 15) / 16 * 16 * sizeof(float) : 0);
        auto* kernel = p.q.wf32 ? block_norm_backward_ring_kernel<T, true, false, false>
                                : block_norm_backward_ring_kernel<T, kSize == 4, false, false>;
        if constexpr (kSize == 2) {
            if (odd) kernel = p.q.wf32 ? block_norm_backward_ring_kernel<T, true, false, true>
                                       : block_norm_backward_ring_kernel<T, false, false, true>;
        }
        return run(kernel, ctas, ring.threads, smem, kRingMost, stream, p);
    }
    const int threads = threads_for(a.cols, 8);
    const size_t smem = gathers ? (size_t)threads * 8 * sizeof(float) : 0;
    return vec ? run(block_norm_backward_kernel<T, 1, true, false>, ctas, threads, smem, kDirectMost, stream, p)
               : run(block_norm_backward_kernel<T, 1, false, false>, ctas, threads, smem, kDirectMost, stream, p);
}
template <typename W, int V>
cudaError_t sums(const GradParams& p, int64_t ctas, cudaStream_t stream) {
    const pwlq_block_norm_args& a = p.q.a;
    int64_t kinds = 2;
    bool few = true;
    if (p.g.dgate && p.gates) {
        few = a.gate_tokens / p.rows_per_cta + 2 <= kFewShares;
        kinds = few ? 3 : 3 + (a.rows + a.gate_tokens - 1) / a.gate_tokens;
    } else if (p.g.dgate && a.gate_rows > 1) {
        kinds = 3;                                 // zeros for the others
        few = false;
    }
    const dim3 grid((unsigned)((a.cols + kSumLanes * V - 1) / (kSumLanes * V)), (unsigned)kinds);
    return launch_dependent(block_norm_sums_kernel<W, V>, grid, dim3(kSumLanes, kSumParts), 0, stream, p, (int)ctas,
                            few, static_cast<W*>(p.g.dpre), static_cast<W*>(p.g.dpost), static_cast<W*>(p.g.dgate));
}
template <typename W>
cudaError_t sums(const GradParams& p, int64_t ctas, cudaStream_t stream) {
    return p.q.a.cols % 4 == 0 ? sums<W, 4>(p, ctas, stream) : sums<W, 1>(p, ctas, stream);
}
template <typename T>
cudaError_t backward(const pwlq_block_norm_args& a, const pwlq_block_norm_grads& g, cudaStream_t stream) {
    GradParams p;
    p.q = params(a);
    if (!a.gate && !a.post_weight) p.q.a.f_codes = nullptr;      // f enters as it is: nothing of it is needed
    p.g = g;
    int64_t ctas = backward_ctas(a.rows, a.cols);
    const int lanes = !a.gate || a.gate_tokens >= a.rows ? narrow_lanes(a.cols, sizeof(T)) : 0;
    const bool narrow = lanes && rows32_backward<T>(a, g), pairs = pairs_backward<T>(p);
    if (narrow) ctas = std::min(ctas, narrow_ctas(a.rows, lanes));
    if (pairs) ctas = std::min<int64_t>(ctas, std::max(1, sm_count() / 2));
    p.rows_per_cta = ctas ? (a.rows + ctas - 1) / ctas : 1;
    ctas = (a.rows + p.rows_per_cta - 1) / p.rows_per_cta;
    float* ws = static_cast<float*>(g.workspace);
    p.dpre = g.dpre ? ws : nullptr;
    p.gates = a.gate && a.gate_tokens < a.rows;
    p.dpost = g.dpost || (g.dgate && !p.gates) ? ws + ctas * a.cols : nullptr;
    p.dgate = g.dgate && p.gates ? ws + 2 * ctas * a.cols : nullptr;
    p.gathered = 0;
    if (ctas && narrow) {
        auto* kernel = p.q.wf32 ? block_norm_backward_narrow_kernel<T, true>
                                : block_norm_backward_narrow_kernel<T, sizeof(T) == 4>;
        kernel<<<(unsigned)ctas, kNarrowThreads, 0, stream>>>(p, lanes);
        if (const cudaError_t e = cudaGetLastError()) return e;
    } else if (ctas && pairs) {
        if (const cudaError_t e = backward_pairs<T>(p, (unsigned)ctas, stream)) return e;
    } else if (ctas) {
        if (const cudaError_t e = backward_rows<T>(p, (unsigned)ctas, stream)) return e;
    }
    if (!g.dpre && !g.dpost && !g.dgate) return cudaSuccess;
    return p.q.wf32 ? sums<float>(p, ctas, stream) : sums<T>(p, ctas, stream);
}

}  // namespace

cudaError_t launch_block_norm(const pwlq_block_norm_args& a, cudaStream_t stream) {
    if (a.dtype == kF32) return forward<float>(a, stream);
    if (a.dtype == kBf16) return forward<__nv_bfloat16>(a, stream);
    return forward<__half>(a, stream);
}

size_t block_norm_backward_workspace(int64_t rows, int64_t cols, int64_t gate_rows) {
    const int64_t ctas = backward_ctas(rows, cols);
    return (size_t)((gate_rows ? 4 : 2) * ctas) * (size_t)cols * sizeof(float);
}

cudaError_t launch_block_norm_backward(const pwlq_block_norm_args& a, const pwlq_block_norm_grads& g,
                                       cudaStream_t stream) {
    if (a.dtype == kF32) return backward<float>(a, g, stream);
    if (a.dtype == kBf16) return backward<__nv_bfloat16>(a, g, stream);
    return backward<__half>(a, g, stream);
}

int take_block_norm_timeout_flag() {
    int v = 0;
    const int zero = 0;
    if (cudaMemcpyFromSymbol(&v, g_block_norm_timeout, sizeof(v)) != cudaSuccess) return -1;
    if (v && cudaMemcpyToSymbol(g_block_norm_timeout, &zero, sizeof(zero)) != cudaSuccess) return -1;
    return v;
}

}  // namespace pwlq
