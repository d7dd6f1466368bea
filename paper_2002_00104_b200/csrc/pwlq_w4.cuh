// What the kernels on 4-bit weights share: the format's table, a tile of weights as the operand of a
// matrix instruction, activations as the other operand, and the sum over a range of columns.
#pragma once

#include "pwlq_act8.cuh"
#include "pwlq_w4.h"

namespace pwlq {

// The eight magnitudes that region and level can stand for, n / 256 in a 16-bit type (exact: n <= 192 has
// eight bits), as bytes: a byte permutation with four codes for selectors looks four values up at once.
struct W4Table {
    uint32_t high[2], low[2];
};

// A packed matrix (format: include/pwlq.h) as kernels see it.  A block of 16 rows x 64 columns is 32 lanes x
// 4 words; word j of lane 4 g + q holds rows g and g + 8, columns 32 (j / 2) + 8 q + 4 (j & 1) .. + 3, so that
// a word is the operand of one 16 x 8 x 16 matrix instruction and eight consecutive values of an activation
// row are a lane's part of the other operand of two of them (any order of the columns will do in a sum, as
// long as both operands have the same).
struct W4View {
    const uint4* codes;
    const uint32_t* scales;                // [tiles][groups][8]: rows g (low half) and g + 8 of a tile
    int64_t tiles, blocks, groups;
    int64_t rows, cols;
    int group_shift;                       // log2(group)
    int paired;
    W4Table table;
    __device__ __forceinline__ const uint4* tile_codes(int64_t matrix, int64_t tile) const {
        return codes + (matrix * tiles + tile) * blocks * 32;
    }
    __device__ __forceinline__ const uint32_t* tile_scales(int64_t matrix, int64_t tile) const {
        return scales + (matrix * tiles + tile) * groups * 8;
    }
};

W4View w4_view(const pwlq_w4& w, bool bf16);

// Four registers of the weight operand from a word: bits 0-2 of nibbles 0-3 are the magnitudes of row g, of
// nibbles 4-7 those of row g + 8; bit 3 of the odd nibbles holds row g's signs, of the even ones row g + 8's,
// so that a mask puts them on top of the high bytes.
__device__ __forceinline__ void w4_operand(uint32_t w, const W4Table& t, uint32_t (&a)[4]) {
    const uint32_t m = w & 0x77777777u, n = m >> 16;
    const uint32_t h0 = __byte_perm(t.high[0], t.high[1], m) ^ (w & 0x80808080u);
    const uint32_t h1 = __byte_perm(t.high[0], t.high[1], n) ^ ((w << 4) & 0x80808080u);
    const uint32_t l0 = __byte_perm(t.low[0], t.low[1], m);
    const uint32_t l1 = __byte_perm(t.low[0], t.low[1], n);
    a[0] = __byte_perm(l0, h0, 0x5140);
    a[2] = __byte_perm(l0, h0, 0x7362);
    a[1] = __byte_perm(l1, h1, 0x5140);
    a[3] = __byte_perm(l1, h1, 0x7362);
}

__device__ __forceinline__ void mma16816(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1,
                                         __nv_bfloat16) {
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, "
                 "{%0,%1,%2,%3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
                 : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ void mma16816(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1, __half) {
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, "
                 "{%0,%1,%2,%3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
                 : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}

// A binary32 value as three bf16 values whose sum it is (8 + 8 + 8 bits, cut off, not rounded, so that the
// largest values stay finite): three products with one operand give binary32 activations their full precision.
__device__ __forceinline__ void split3(float v, float& a, float& b, float& c) {
    a = __uint_as_float(__float_as_uint(v) & 0xffff0000u);
    b = c = 0.0f;
    if (abs_bits(v) < kInfBits) {
        const float r = v - a;
        b = __uint_as_float(__float_as_uint(r) & 0xffff0000u);
        c = r - b;
    } else if (v != v) {
        a = v;                                            // cutting a NaN's bits off could leave an infinity
    }
}
__device__ __forceinline__ uint32_t top16(float lo, float hi) {
    return __byte_perm(__float_as_uint(lo), __float_as_uint(hi), 0x7632);
}

// Activations as operands: eight consecutive values of a row are kPieces x 4 registers.
// 16-bit rows on 16-byte boundaries, whole blocks.
template <typename T> struct RowsWhole {
    using Elem = T;
    using Mma = T;
    static constexpr int kPieces = 1;
    struct Raw { uint4 w; };
    int64_t cols;
    __device__ __forceinline__ void load(Raw& r, const T* row, int64_t col) const {
        r.w = *reinterpret_cast<const uint4*>(row + col);
    }
    __device__ __forceinline__ void operand(const Raw& r, uint32_t (&b)[1][4]) const {
        b[0][0] = r.w.x; b[0][1] = r.w.y; b[0][2] = r.w.z; b[0][3] = r.w.w;
    }
};
// Rows that lie anywhere, of any length and type.
template <typename T> struct RowsAny {
    using Elem = T;
    using Mma = T;
    static constexpr int kPieces = 1;
    using Raw = Raw8<T>;
    int64_t cols;
    __device__ __forceinline__ void load(Raw& r, const T* row, int64_t col) const {
        load8<false>(r, row + col, (int)max((int64_t)-8, min(cols - col, (int64_t)64)), (int)min(col, (int64_t)64));
    }
    __device__ __forceinline__ void operand(const Raw& r, uint32_t (&b)[1][4]) const {
        b[0][0] = r.w.x; b[0][1] = r.w.y; b[0][2] = r.w.z; b[0][3] = r.w.w;
    }
};
template <> struct RowsAny<float> {
    using Elem = float;
    using Mma = __nv_bfloat16;
    static constexpr int kPieces = 3;
    using Raw = Raw8<float>;
    int64_t cols;
    __device__ __forceinline__ void load(Raw& r, const float* row, int64_t col) const {
        load8<false>(r, row + col, (int)max((int64_t)-8, min(cols - col, (int64_t)64)), (int)min(col, (int64_t)64));
    }
    __device__ __forceinline__ void operand(const Raw& r, uint32_t (&b)[3][4]) const {
        float v[8];
        r.get(v);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            float a0, b0, c0, a1, b1, c1;
            split3(v[2 * i], a0, b0, c0);
            split3(v[2 * i + 1], a1, b1, c1);
            b[0][i] = pack16(a0, a1, __nv_bfloat16());
            b[1][i] = top16(b0, b1);
            b[2][i] = pack16(c0, c1, __nv_bfloat16());
        }
    }
};
// Rows of two bf16 values each, high parts then low parts, whole blocks: 16 bits of a binary32 value.
struct RowsSplit {
    using Elem = __nv_bfloat16;
    using Mma = __nv_bfloat16;
    static constexpr int kPieces = 2;
    struct Raw { uint4 w[2]; };
    int64_t cols;                                         // of each part
    __device__ __forceinline__ void load(Raw& r, const __nv_bfloat16* row, int64_t col) const {
        r.w[0] = *reinterpret_cast<const uint4*>(row + col);
        r.w[1] = *reinterpret_cast<const uint4*>(row + cols + col);
    }
    __device__ __forceinline__ void operand(const Raw& r, uint32_t (&b)[2][4]) const {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            b[i][0] = r.w[i].x; b[i][1] = r.w[i].y; b[i][2] = r.w[i].z; b[i][3] = r.w[i].w;
        }
    }
};

// acc[n][..] += the tile's blocks [begin, end) times 8 NT activation rows (row[n]: the row of column 8 n + g for
// this lane).  acc holds sums of n / 256 * s * x: the caller multiplies by 256.  A block's products are summed by
// the matrix instructions in binary32 and enter acc times the scales of their rows.
template <int NT, class S>
__device__ __forceinline__ void w4_accumulate(float (&acc)[NT][4], const uint4* __restrict__ codes,
                                              const uint32_t* __restrict__ scales, const W4View& w, int64_t begin,
                                              int64_t end, const S& source, const typename S::Elem* const (&row)[NT]) {
    constexpr int U = 4;                                  // blocks requested at once
    const int lane = threadIdx.x & 31, g = lane >> 2, q = lane & 3;
    const bool narrow = w.group_shift == 5;               // two groups in a block
    codes += lane;
    scales += g;
    auto block = [&](int64_t kb, const uint4& c, uint32_t s0, uint32_t s1) {
        float part[NT][4];
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int i = 0; i < 4; ++i) part[n][i] = 0.0f;
        const uint32_t word[4] = {c.x, c.y, c.z, c.w};
#pragma unroll
        for (int half = 0; half < 2; ++half) {
            uint32_t b[NT][S::kPieces][4];
#pragma unroll
            for (int n = 0; n < NT; ++n) {
                typename S::Raw raw;
                source.load(raw, row[n], kb * kBlockCols + half * 32 + q * 8);
                source.operand(raw, b[n]);
            }
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                uint32_t a[4];
                w4_operand(word[2 * half + j], w.table, a);
#pragma unroll
                for (int n = 0; n < NT; ++n)
#pragma unroll
                    for (int p = 0; p < S::kPieces; ++p)
                        mma16816(part[n], a, b[n][p][2 * j], b[n][p][2 * j + 1], typename S::Mma());
            }
            if (half == 1 || narrow) {
                const uint32_t s = half == 0 ? s0 : s1;
                const float lo = __uint_as_float(s << 16), hi = __uint_as_float(s & 0xffff0000u);
#pragma unroll
                for (int n = 0; n < NT; ++n) {
                    acc[n][0] = fmaf(lo, part[n][0], acc[n][0]);
                    acc[n][1] = fmaf(lo, part[n][1], acc[n][1]);
                    acc[n][2] = fmaf(hi, part[n][2], acc[n][2]);
                    acc[n][3] = fmaf(hi, part[n][3], acc[n][3]);
#pragma unroll
                    for (int i = 0; i < 4; ++i) part[n][i] = 0.0f;
                }
            }
        }
    };
    // the second half of the last block may have no group of its own: its codes are 0
    auto scale = [&](int64_t kb, int half) {
        return __ldg(scales + 8 * min((kb * kBlockCols + 32 * half) >> w.group_shift, w.groups - 1));
    };
    int64_t kb = begin;
    for (; kb + U <= end; kb += U) {
        uint4 c[U];
        uint32_t s0[U], s1[U];
#pragma unroll
        for (int u = 0; u < U; ++u) c[u] = __ldg(codes + (kb + u) * 32);
#pragma unroll
        for (int u = 0; u < U; ++u) {
            s1[u] = scale(kb + u, 1);
            s0[u] = narrow ? scale(kb + u, 0) : s1[u];
        }
#pragma unroll
        for (int u = 0; u < U; ++u) block(kb + u, c[u], s0[u], s1[u]);
    }
    for (; kb < end; ++kb) {
        const uint4 c = __ldg(codes + kb * 32);
        const uint32_t s1 = scale(kb, 1);
        block(kb, c, narrow ? scale(kb, 0) : s1, s1);
    }
}

// x * sigmoid(x)
__device__ __forceinline__ float silu_of(float v) { return __fdiv_rn(v, 1.0f + expf(-v)); }

}  // namespace pwlq
