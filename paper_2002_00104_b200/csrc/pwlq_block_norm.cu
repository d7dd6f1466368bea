// Norms around a gated residual block, forward and backward (formulas: include/pwlq.h).
//
// Both directions are bound by HBM: per value the forward pass reads x and f and writes r and h
// (and two bytes when it saves), the backward pass reads dh, dr and two bytes and writes dx and df.
// A row is owned by one CTA, eight consecutive values per thread and step, and stays in registers
// between the two reductions that depend on one another (of f, then of r; of the outer norm, then
// of the inner one), so every operand crosses HBM once.
#include "pwlq_act8.cuh"
#include "pwlq_train.h"

namespace pwlq {
namespace {

// Sum over the CTA, the same value in every thread, in a fixed order.  Calls alternate between the
// two halves of `buf`, so one barrier per call is enough: a half is written again only after the
// barrier of the call in between.
template <int N>
struct CtaSum {
    float (*buf)[N][32];
    int half = 0;
    __device__ __forceinline__ void operator()(float (&v)[N]) {
        const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, warps = blockDim.x >> 5;
#pragma unroll
        for (int k = 0; k < N; ++k)
            for (int o = 16; o; o >>= 1) v[k] += __shfl_xor_sync(0xffffffffu, v[k], o);
        if (warps == 1) return;
        if (lane == 0)
#pragma unroll
            for (int k = 0; k < N; ++k) buf[half][k][warp] = v[k];
        __syncthreads();
#pragma unroll
        for (int k = 0; k < N; ++k) {
            v[k] = lane < warps ? buf[half][k][lane] : 0.0f;
            for (int o = 16; o; o >>= 1) v[k] += __shfl_xor_sync(0xffffffffu, v[k], o);
        }
        half ^= 1;
    }
};

// Eight weights (or gates) starting at column c, as binary32.
template <bool VEC, typename T>
__device__ __forceinline__ void weights8(const void* p, bool f32, int64_t c, int valid, float* w) {
    if (f32) {
        Raw8<float> raw;
        load8<VEC>(raw, static_cast<const float*>(p) + c, valid);
        raw.get(w);
    } else {
        Raw8<T> raw;
        load8<VEC>(raw, static_cast<const T*>(p) + c, valid);
        raw.get(w);
    }
}

struct NormParams {
    pwlq_block_norm_args a;
    float scale, eps, offset, inv_cols, ratio;
    int64_t groups;
    int group_lanes, group_shift;
    bool wf32;
};

// Bytes of eight values of a row, and the range of their group (whose lanes call this together).
__device__ __forceinline__ void save8(const float* v, const NormParams& q, int64_t row, int c,
                                      int valid, uint8_t* codes, float* ranges) {
    uint32_t top = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) top = max(top, abs_bits(v[i]));
    top = group_max(top, q.group_lanes);
    if (valid <= 0) return;
    const float m = act8_range(top);
    const PieceParams P = act8_params(m, q.ratio);
    const uint2 w = make_uint2(act8_word(v, m, P), act8_word(v + 4, m, P));
    uint8_t* at = codes + row * q.a.ldc + c;
    *reinterpret_cast<uint2*>(at) = w;
    // the row's last 16 bytes may need zeros that no value stands for
    if (valid <= 8 && (c & 8) == 0) *reinterpret_cast<uint2*>(at + 8) = make_uint2(0u, 0u);
    if ((c & ((1 << q.group_shift) - 1)) == 0) ranges[row * q.groups + (c >> q.group_shift)] = m;
}

// VC: chunks of eight columns per thread.
template <typename T, int VC, bool VEC, bool SAVE>
__global__ void __launch_bounds__(VC == 4 ? 512 : 256) block_norm_kernel(NormParams q) {
    __shared__ float buf[2][1][32];
    CtaSum<1> cta_sum{buf};
    const int64_t row = blockIdx.x;
    const int cols = (int)q.a.cols;
    const T* x = static_cast<const T*>(q.a.x) + row * q.a.ldx;
    const T* f = static_cast<const T*>(q.a.f) + row * q.a.ldf;
    Raw8<T> rx[VC], rf[VC];
#pragma unroll
    for (int i = 0; i < VC; ++i) {
        const int c = (threadIdx.x + i * blockDim.x) * 8;
        load8<VEC>(rx[i], x + c, cols - c);
        if (q.a.f) load8<VEC>(rf[i], f + c, cols - c);
    }
    float r[VC][8], sum[1];
    float rstd_f = 1.0f;
    if (q.a.post_weight) {
        sum[0] = 0.0f;
#pragma unroll
        for (int i = 0; i < VC; ++i) {
            float v[8];
            rf[i].get(v);
#pragma unroll
            for (int k = 0; k < 8; ++k) sum[0] = fmaf(v[k], v[k], sum[0]);
        }
        cta_sum(sum);
        rstd_f = rsqrtf(fmaf(sum[0], q.inv_cols, q.eps));
        if (SAVE && threadIdx.x == 0 && q.a.f_rstd) q.a.f_rstd[row] = rstd_f;
    }
    sum[0] = 0.0f;
#pragma unroll
    for (int i = 0; i < VC; ++i) {
        const int c = (threadIdx.x + i * blockDim.x) * 8, valid = cols - c;
        float v[8];
        rx[i].get(r[i]);
#pragma unroll
        for (int k = 0; k < 8; ++k) r[i][k] *= q.scale;
        if (q.a.f) {
            rf[i].get(v);
            if (SAVE && q.a.f_codes) save8(v, q, row, c, valid, q.a.f_codes, q.a.f_ranges);
            float w[8];
            if (q.a.post_weight) {
                weights8<VEC, T>(q.a.post_weight, q.wf32, c, valid, w);
#pragma unroll
                for (int k = 0; k < 8; ++k) v[k] = v[k] * rstd_f * (w[k] + q.offset);
            }
            if (q.a.gate) {
                weights8<VEC, T>(q.a.gate, q.wf32, row / q.a.gate_tokens * q.a.ldgate + c, valid, w);
#pragma unroll
                for (int k = 0; k < 8; ++k) v[k] *= w[k];
            }
#pragma unroll
            for (int k = 0; k < 8; ++k) r[i][k] += v[k];
        }
        if (q.a.r) store8<VEC>(r[i], static_cast<T*>(q.a.r) + row * q.a.ldr + c, valid);
        if (SAVE && q.a.r_codes) save8(r[i], q, row, c, valid, q.a.r_codes, q.a.r_ranges);
#pragma unroll
        for (int k = 0; k < 8; ++k)
            if (k < valid) sum[0] = fmaf(r[i][k], r[i][k], sum[0]);
    }
    if (!q.a.pre_weight) return;
    cta_sum(sum);
    const float rstd_r = rsqrtf(fmaf(sum[0], q.inv_cols, q.eps));
    if (SAVE && threadIdx.x == 0 && q.a.r_rstd) q.a.r_rstd[row] = rstd_r;
#pragma unroll
    for (int i = 0; i < VC; ++i) {
        const int c = (threadIdx.x + i * blockDim.x) * 8, valid = cols - c;
        float w[8];
        weights8<VEC, T>(q.a.pre_weight, q.wf32, c, valid, w);
#pragma unroll
        for (int k = 0; k < 8; ++k) w[k] = r[i][k] * rstd_r * (w[k] + q.offset);
        store8<VEC>(w, static_cast<T*>(q.a.h) + row * q.a.ldh + c, valid);
    }
}

// Backward.  CTA b owns the rows [b * rows_per_cta, ...) and its columns' sums over them; the sums
// go to the workspace once per CTA (those of the gate also where the gate changes) and a second
// kernel adds them in a fixed order.  The sums live in registers up to 8192 columns (24 per
// thread); wider rows, whose sums alone would take three quarters of the register file, keep them
// in shared memory (WIDE), where every thread touches its own columns only.
// Workspace: [ctas][cols] of dpre, [ctas][cols] of dpost, [ctas + gate_rows][cols] of dgate, whose
// slot b + g holds CTA b's share of gate g (every CTA and every gate moves on by at least one).
struct GradParams {
    NormParams q;
    pwlq_block_norm_grads g;
    int64_t rows_per_cta;
    float *dpre, *dpost, *dgate;          // workspace; nullptr: not wanted
};

enum { kDpre, kDpost, kDgate };

template <int VC, bool WIDE>
struct ColumnSums {
    float reg[3][WIDE ? 1 : VC][8] = {};
    float4* smem = nullptr;               // [3][VC][2][blockDim.x]
    __device__ __forceinline__ float4* at(int which, int i) const {
        return smem + ((which * VC + i) * 2) * blockDim.x + threadIdx.x;
    }
    __device__ __forceinline__ void clear(int which) {
#pragma unroll
        for (int i = 0; i < VC; ++i) {
            const float zero[8] = {};
            set(which, i, zero);
        }
    }
    __device__ __forceinline__ void set(int which, int i, const float* v) {
        if (WIDE) {
            at(which, i)[0] = make_float4(v[0], v[1], v[2], v[3]);
            at(which, i)[blockDim.x] = make_float4(v[4], v[5], v[6], v[7]);
        } else {
#pragma unroll
            for (int k = 0; k < 8; ++k) reg[which][WIDE ? 0 : i][k] = v[k];
        }
    }
    __device__ __forceinline__ void get(int which, int i, float* v) const {
        if (WIDE) {
            const float4 a = at(which, i)[0], b = at(which, i)[blockDim.x];
            v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w;
            v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
        } else {
#pragma unroll
            for (int k = 0; k < 8; ++k) v[k] = reg[which][WIDE ? 0 : i][k];
        }
    }
    template <bool VEC>
    __device__ __forceinline__ void put(int which, float* to, int cols) const {
#pragma unroll
        for (int i = 0; i < VC; ++i) {
            const int c = (threadIdx.x + i * blockDim.x) * 8;
            float v[8];
            get(which, i, v);
            store8<VEC>(v, to + c, cols - c);
        }
    }
};

template <typename T, int VC, bool VEC, bool WIDE>
__global__ void __launch_bounds__(WIDE ? 512 : 1024) block_norm_backward_kernel(GradParams p) {
    __shared__ float buf[2][1][32];
    extern __shared__ float4 wide[];
    CtaSum<1> cta_sum{buf};
    const NormParams& q = p.q;
    const int cols = (int)q.a.cols;
    const int64_t first = blockIdx.x * p.rows_per_cta, last = min(first + p.rows_per_cta, q.a.rows);
    const bool pre = q.a.pre_weight, post = q.a.post_weight, has_f = q.a.f_codes;
    ColumnSums<VC, WIDE> sums;
    if (WIDE) {
        sums.smem = wide;
        for (int which = 0; which < 3; ++which) sums.clear(which);
    }
    int64_t gate = q.a.gate ? first / q.a.gate_tokens : 0;
    int64_t gate_end = (gate + 1) * q.a.gate_tokens;

    for (int64_t row = first; row < last; ++row) {
        if (q.a.gate && row == gate_end) {
            if (p.dgate) sums.template put<VEC>(kDgate, p.dgate + (blockIdx.x + gate) * cols, cols);
            sums.clear(kDgate);
            ++gate;
            gate_end += q.a.gate_tokens;
        }
        const float rstd_r = pre ? q.a.r_rstd[row] : 0.0f;
        const float rstd_f = post ? q.a.f_rstd[row] : 1.0f;
        float e[VC][8], n[VC][8], sum[1] = {0.0f};
        // outer norm: e = dr + rstd * (u - n * mean(u n))
        if (pre) {
#pragma unroll
            for (int i = 0; i < VC; ++i) {
                const int c = (threadIdx.x + i * blockDim.x) * 8, valid = cols - c;
                Raw8<T> raw;
                float w[8];
                load8<VEC>(raw, static_cast<const T*>(p.g.dh) + row * p.g.lddh + c, valid);
                raw.get(e[i]);
                weights8<VEC, T>(q.a.pre_weight, q.wf32, c, valid, w);
                uint2 b = make_uint2(0u, 0u);
                PieceParams S = {};
                if (valid > 0) {
                    b = *reinterpret_cast<const uint2*>(q.a.r_codes + row * q.a.ldc + c);
                    S = act8_params(q.a.r_ranges[row * q.groups + (c >> q.group_shift)], q.ratio);
                }
                act8_values(b.x, S, n[i]);
                act8_values(b.y, S, n[i] + 4);
                float d[8];
                sums.get(kDpre, i, d);
#pragma unroll
                for (int k = 0; k < 8; ++k) {
                    n[i][k] *= rstd_r;
                    d[k] = fmaf(e[i][k], n[i][k], d[k]);
                    e[i][k] *= w[k] + q.offset;
                    if (k < valid) sum[0] = fmaf(e[i][k], n[i][k], sum[0]);
                }
                sums.set(kDpre, i, d);
            }
            cta_sum(sum);
            const float mean = sum[0] * q.inv_cols;
#pragma unroll
            for (int i = 0; i < VC; ++i)
#pragma unroll
                for (int k = 0; k < 8; ++k) e[i][k] = rstd_r * fmaf(-mean, n[i][k], e[i][k]);
        } else {
#pragma unroll
            for (int i = 0; i < VC; ++i)
#pragma unroll
                for (int k = 0; k < 8; ++k) e[i][k] = 0.0f;
        }
        sum[0] = 0.0f;
#pragma unroll
        for (int i = 0; i < VC; ++i) {
            const int c = (threadIdx.x + i * blockDim.x) * 8, valid = cols - c;
            float w[8];
            if (p.g.dr) {
                Raw8<T> raw;
                load8<VEC>(raw, static_cast<const T*>(p.g.dr) + row * p.g.lddr + c, valid);
                raw.get(w);
#pragma unroll
                for (int k = 0; k < 8; ++k) e[i][k] += w[k];
            }
            if (p.g.dx) {
#pragma unroll
                for (int k = 0; k < 8; ++k) w[k] = q.scale * e[i][k];
                store8<VEC>(w, static_cast<T*>(p.g.dx) + row * p.g.lddx + c, valid);
            }
            if (!has_f) continue;
            // inner norm and gate; e becomes v = e * gate * w
            uint2 b = make_uint2(0u, 0u);
            PieceParams S = {};
            if (valid > 0) {
                b = *reinterpret_cast<const uint2*>(q.a.f_codes + row * q.a.ldc + c);
                S = act8_params(q.a.f_ranges[row * q.groups + (c >> q.group_shift)], q.ratio);
            }
            act8_values(b.x, S, n[i]);
            act8_values(b.y, S, n[i] + 4);
            float gv[8], wv[8];
            if (q.a.gate) weights8<VEC, T>(q.a.gate, q.wf32, gate * q.a.ldgate + c, valid, gv);
            if (post) weights8<VEC, T>(q.a.post_weight, q.wf32, c, valid, wv);
            float d[8], dg[8];
            sums.get(kDpost, i, d);
            sums.get(kDgate, i, dg);
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                const float g = q.a.gate ? gv[k] : 1.0f, ww = post ? wv[k] + q.offset : 1.0f;
                n[i][k] *= rstd_f;
                dg[k] = fmaf(e[i][k] * ww, n[i][k], dg[k]);
                d[k] = fmaf(e[i][k] * g, n[i][k], d[k]);
                e[i][k] *= g * ww;
                if (k < valid) sum[0] = fmaf(e[i][k], n[i][k], sum[0]);
            }
            sums.set(kDpost, i, d);
            sums.set(kDgate, i, dg);
        }
        if (!p.g.df) continue;
        float mean = 0.0f;
        if (post) {
            cta_sum(sum);
            mean = sum[0] * q.inv_cols;
        }
#pragma unroll
        for (int i = 0; i < VC; ++i) {
            const int c = (threadIdx.x + i * blockDim.x) * 8;
            float w[8];
#pragma unroll
            for (int k = 0; k < 8; ++k)
                w[k] = post ? rstd_f * fmaf(-mean, n[i][k], e[i][k]) : e[i][k];
            store8<VEC>(w, static_cast<T*>(p.g.df) + row * p.g.lddf + c, cols - c);
        }
    }
    if (p.dpre) sums.template put<VEC>(kDpre, p.dpre + (int64_t)blockIdx.x * cols, cols);
    if (p.dpost) sums.template put<VEC>(kDpost, p.dpost + (int64_t)blockIdx.x * cols, cols);
    if (p.dgate) sums.template put<VEC>(kDgate, p.dgate + (blockIdx.x + gate) * cols, cols);
}

// Adds the CTAs' sums of one column per thread: eight parts of the CTAs side by side, then the
// parts.  blockIdx.y: 0 dpre, 1 dpost, 2 + g gate g.
constexpr int kSumCols = 32, kSumParts = 8;
template <typename W>
__global__ void __launch_bounds__(kSumCols * kSumParts)
block_norm_sums_kernel(GradParams p, int64_t ctas, W* dpre, W* dpost, W* dgate) {
    __shared__ float part[kSumParts][kSumCols];
    const int cols = (int)p.q.a.cols;
    const int c = blockIdx.x * kSumCols + threadIdx.x;
    for (int64_t which = blockIdx.y; which < 2 + (dgate ? p.q.a.gate_rows : 0); which += gridDim.y) {
        W* out = which == 0 ? dpre : which == 1 ? dpost : dgate + (which - 2) * cols;
        if (which < 2 && !out) continue;
        const float* src = which == 0 ? p.dpre : which == 1 ? p.dpost : p.dgate;
        int64_t lo = 0, hi = ctas;
        if (which >= 2) {
            const int64_t g = which - 2, r0 = g * p.q.a.gate_tokens;
            const int64_t r1 = min(r0 + p.q.a.gate_tokens, p.q.a.rows);
            lo = r0 / p.rows_per_cta;
            hi = r1 > r0 ? (r1 - 1) / p.rows_per_cta + 1 : lo;
            src += g * cols;                       // slot of CTA b: b + g
        }
        float s = 0.0f;
        if (c < cols)
            for (int64_t b = lo + threadIdx.y; b < hi; b += kSumParts) s += src[b * cols + c];
        part[threadIdx.y][threadIdx.x] = s;
        __syncthreads();
        if (threadIdx.y == 0 && c < cols) {
#pragma unroll
            for (int k = 1; k < kSumParts; ++k) s += part[k][threadIdx.x];
            out[c] = from_f32<W>(s);
        }
        __syncthreads();
    }
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
    return q;
}

inline bool pointers_aligned(const pwlq_block_norm_args& a) {
    const size_t ws = type_size((int)a.wtype);
    return rows_aligned(a.post_weight, 0, ws) && rows_aligned(a.pre_weight, 0, ws) &&
           rows_aligned(a.gate, a.ldgate, ws);
}

template <typename T, int VC>
cudaError_t forward(const NormParams& q, int threads, cudaStream_t stream) {
    const bool vec = rows_aligned(q.a.x, q.a.ldx, sizeof(T)) && rows_aligned(q.a.f, q.a.ldf, sizeof(T)) &&
                     rows_aligned(q.a.r, q.a.ldr, sizeof(T)) && rows_aligned(q.a.h, q.a.ldh, sizeof(T)) &&
                     pointers_aligned(q.a);
    const bool save = q.a.r_codes || q.a.f_codes || q.a.r_rstd || q.a.f_rstd;
    auto* kernel = vec ? (save ? block_norm_kernel<T, VC, true, true> : block_norm_kernel<T, VC, true, false>)
                       : (save ? block_norm_kernel<T, VC, false, true> : block_norm_kernel<T, VC, false, false>);
    kernel<<<(unsigned)q.a.rows, threads, 0, stream>>>(q);
    return cudaGetLastError();
}
template <typename T>
cudaError_t forward(const pwlq_block_norm_args& a, cudaStream_t stream) {
    const NormParams q = params(a);
    const int chunks = (int)((a.cols + 7) / 8);
    const int vc = chunks <= 256 ? 1 : chunks <= 512 ? 2 : 4;
    const int threads = ((chunks + vc - 1) / vc + 31) / 32 * 32;
    if (vc == 1) return forward<T, 1>(q, threads, stream);
    if (vc == 2) return forward<T, 2>(q, threads, stream);
    return forward<T, 4>(q, threads, stream);
}

// CTAs of the backward pass: the rows are shared out evenly over at most this many.
constexpr int64_t kBackwardCtas = 296;
inline int64_t backward_ctas(int64_t rows) { return rows < kBackwardCtas ? rows : kBackwardCtas; }

template <typename T, int VC, bool WIDE>
cudaError_t backward(const GradParams& p, unsigned ctas, int threads, cudaStream_t stream) {
    const pwlq_block_norm_grads& g = p.g;
    const bool vec = rows_aligned(g.dh, g.lddh, sizeof(T)) && rows_aligned(g.dr, g.lddr, sizeof(T)) &&
                     rows_aligned(g.dx, g.lddx, sizeof(T)) && rows_aligned(g.df, g.lddf, sizeof(T)) &&
                     p.q.a.cols % 4 == 0 && pointers_aligned(p.q.a);
    auto* kernel = vec ? block_norm_backward_kernel<T, VC, true, WIDE>
                       : block_norm_backward_kernel<T, VC, false, WIDE>;
    const size_t smem = WIDE ? (size_t)3 * VC * 8 * sizeof(float) * threads : 0;   // at most 192 KB
    if (WIDE) {
        const cudaError_t e = cudaFuncSetAttribute(
            kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
        if (e != cudaSuccess) return e;
    }
    kernel<<<ctas, threads, smem, stream>>>(p);
    return cudaGetLastError();
}
template <typename W>
cudaError_t sums(const GradParams& p, int64_t ctas, cudaStream_t stream) {
    const int64_t kinds = 2 + (p.dgate ? p.q.a.gate_rows : 0);
    const dim3 grid((unsigned)((p.q.a.cols + kSumCols - 1) / kSumCols),
                    (unsigned)(kinds < 65535 ? kinds : 65535));
    block_norm_sums_kernel<W><<<grid, dim3(kSumCols, kSumParts), 0, stream>>>(
        p, ctas, static_cast<W*>(p.g.dpre), static_cast<W*>(p.g.dpost), static_cast<W*>(p.g.dgate));
    return cudaGetLastError();
}
template <typename T>
cudaError_t backward(const pwlq_block_norm_args& a, const pwlq_block_norm_grads& g, cudaStream_t stream) {
    GradParams p;
    p.q = params(a);
    p.g = g;
    int64_t ctas = backward_ctas(a.rows);
    p.rows_per_cta = ctas ? (a.rows + ctas - 1) / ctas : 1;
    ctas = (a.rows + p.rows_per_cta - 1) / p.rows_per_cta;
    float* ws = static_cast<float*>(g.workspace);
    p.dpre = g.dpre ? ws : nullptr;
    p.dpost = g.dpost ? ws + ctas * a.cols : nullptr;
    p.dgate = g.dgate ? ws + 2 * ctas * a.cols : nullptr;
    const int chunks = (int)((a.cols + 7) / 8);
    const int vc = chunks <= 1024 ? 1 : 4;
    const int threads = ((chunks + vc - 1) / vc + 31) / 32 * 32;
    if (ctas) {
        const cudaError_t e = vc == 1 ? backward<T, 1, false>(p, (unsigned)ctas, threads, stream)
                                      : backward<T, 4, true>(p, (unsigned)ctas, threads, stream);
        if (e != cudaSuccess) return e;
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
    const int64_t ctas = backward_ctas(rows);
    return (size_t)(3 * ctas + gate_rows) * (size_t)cols * sizeof(float);
}

cudaError_t launch_block_norm_backward(const pwlq_block_norm_args& a, const pwlq_block_norm_grads& g,
                                       cudaStream_t stream) {
    if (a.dtype == kF32) return backward<float>(a, g, stream);
    if (a.dtype == kBf16) return backward<__nv_bfloat16>(a, g, stream);
    return backward<__half>(a, g, stream);
}

}  // namespace pwlq
