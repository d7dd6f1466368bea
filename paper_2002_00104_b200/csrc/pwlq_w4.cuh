// What the kernels on 4-bit weights share: the format's table, a tile of weights as the operand of a
// matrix instruction, activations as the other operand, and the sum over a range of columns.
#pragma once

#include <cooperative_groups.h>
#include <type_traits>

#include "pwlq_act8.cuh"
#include "pwlq_w4.h"

namespace pwlq {

// The eight magnitudes that region and level can stand for, n / kUnit in a 16-bit type (exact: n <= 192 has
// eight bits), as bytes: a byte permutation with four codes for selectors looks four values up at once.
struct W4Table {
    uint32_t high[2], low[2];
};
// The products of a group, 128 at a time, are summed before they meet their scale: 128 * 192 / 2^15 < 1, so that no sum
// of bf16 values (parts of binary32 ones among them) leaves the range that the values themselves are in, however small
// the scale makes the result.  fp16 values are below 2^16 and their table is above 2^-14: any unit between will do.
template <typename T> constexpr int kUnitBits = std::is_same<T, __half>::value ? 8 : 15;
template <typename T> constexpr float kUnit = (float)(1 << kUnitBits<T>);

// A packed matrix (format: include/pwlq.h) as kernels see it.  A block of 16 rows x 128 columns is 32 lanes x
// 8 words; word j of lane 4 g + q holds rows g and g + 8, columns 32 (j / 2) + 8 q + 4 (j & 1) .. + 3, so that
// a word is the operand of one 16 x 8 x 16 matrix instruction and eight consecutive values of an activation
// row are a lane's part of the other operand of two of them (any order of the columns will do in a sum, as
// long as both operands have the same).
// The scales follow: [groups of the block][8] words, rows g (low half) and g + 8.
struct W4View {
    const uint8_t* data;
    int64_t tiles, rows;
    int blocks, cols;                      // of a row
    int ends;                              // groups of a block
    int paired;
    W4Table table;
};

W4View w4_view(const pwlq_w4& w, bool bf16);

// __byte_perm clears the selectors' top bits, which are known to be 0 here, with an instruction of its own.
__device__ __forceinline__ uint32_t permute(uint32_t a, uint32_t b, uint32_t selectors) {
    uint32_t r;
    asm("prmt.b32 %0, %1, %2, %3;" : "=r"(r) : "r"(a), "r"(b), "r"(selectors));
    return r;
}

// Four registers of the weight operand from a word: bits 0-2 of nibbles 0-3 are the magnitudes of row g, of
// nibbles 4-7 those of row g + 8; bit 3 of the odd nibbles holds row g's signs, of the even ones row g + 8's,
// so that a mask puts them on top of the high bytes.
__device__ __forceinline__ void w4_operand(uint32_t w, const W4Table& t, uint32_t (&a)[4]) {
    const uint32_t m = w & 0x77777777u, n = m >> 16;
    const uint32_t h0 = permute(t.high[0], t.high[1], m) ^ (w & 0x80808080u);
    const uint32_t h1 = permute(t.high[0], t.high[1], n) ^ ((w << 4) & 0x80808080u);
    const uint32_t l0 = permute(t.low[0], t.low[1], m);
    const uint32_t l1 = permute(t.low[0], t.low[1], n);
    a[0] = permute(l0, h0, 0x5140);
    a[2] = permute(l0, h0, 0x7362);
    a[1] = permute(l1, h1, 0x5140);
    a[3] = permute(l1, h1, 0x7362);
}

__device__ __forceinline__ void mma16816(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1,
                                         __nv_bfloat16) {
    asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, "
                 "{%0,%1,%2,%3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
                 : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
// The same with sums that begin at zero.
__device__ __forceinline__ void mma16816_first(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1,
                                               __nv_bfloat16) {
    asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, "
        "{%10,%10,%10,%10};"
        : "=f"(c[0]), "=f"(c[1]), "=f"(c[2]), "=f"(c[3])
        : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1), "f"(0.0f));
}
__device__ __forceinline__ void mma16816_first(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1, __half) {
    asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, "
        "{%10,%10,%10,%10};"
        : "=f"(c[0]), "=f"(c[1]), "=f"(c[2]), "=f"(c[3])
        : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1), "f"(0.0f));
}
__device__ __forceinline__ void mma16816(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1, __half) {
    asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, "
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

// Activations as operands, columns behind the last one as 0: eight consecutive values of a row, from column + offset +
// within on (`row` points `within` values into the row), are kPieces x 4 registers.
// 16-bit rows on 16-byte boundaries, whole blocks.
template <typename T> struct RowsWhole {
    using Elem = T;
    using Mma = T;
    static constexpr int kPieces = 1;
    struct Raw { uint4 w; };
    int cols;
    __device__ __forceinline__ void load(Raw& r, const T* row, int column, int offset, int) const {
        r.w = *reinterpret_cast<const uint4*>(row + column + offset);
    }
    __device__ __forceinline__ void operand(const Raw& r, uint32_t (&b)[1][4]) const {
        b[0][0] = r.w.x; b[0][1] = r.w.y; b[0][2] = r.w.z; b[0][3] = r.w.w;
    }
};
// 16-bit rows on 16-byte boundaries, of whole eights.
template <typename T> struct RowsEights {
    using Elem = T;
    using Mma = T;
    static constexpr int kPieces = 1;
    struct Raw { uint4 w; };
    int cols;
    __device__ __forceinline__ void load(Raw& r, const T* row, int column, int offset, int within) const {
        r.w = make_uint4(0u, 0u, 0u, 0u);
        if (column + offset + within < cols) r.w = *reinterpret_cast<const uint4*>(row + column + offset);
    }
    __device__ __forceinline__ void operand(const Raw& r, uint32_t (&b)[1][4]) const {
        b[0][0] = r.w.x; b[0][1] = r.w.y; b[0][2] = r.w.z; b[0][3] = r.w.w;
    }
};
// Eight binary32 values in three parts.
__device__ __forceinline__ void parts3(const float (&v)[8], uint32_t (&b)[3][4]) {
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
// Rows that lie anywhere, of any length and type.
template <typename T> struct RowsAny {
    using Elem = T;
    using Mma = T;
    static constexpr int kPieces = 1;
    using Raw = Raw8<T>;
    int cols;
    __device__ __forceinline__ void load(Raw& r, const T* row, int column, int offset, int within) const {
        const int col = column + offset + within;
        load8<false>(r, row + column + offset, cols - col, col);
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
    int cols;
    __device__ __forceinline__ void load(Raw& r, const float* row, int column, int offset, int within) const {
        const int col = column + offset + within;
        load8<false>(r, row + column + offset, cols - col, col);
    }
    __device__ __forceinline__ void operand(const Raw& r, uint32_t (&b)[3][4]) const {
        float v[8];
        r.get(v);
        parts3(v, b);
    }
};
// Rows of P bf16 parts, one after another, whose sum a value is; whole blocks.
template <int P> struct RowsParts {
    using Elem = __nv_bfloat16;
    using Mma = __nv_bfloat16;
    static constexpr int kPieces = P;
    struct Raw { uint4 w[P]; };
    int cols;                                             // of a part
    __device__ __forceinline__ void load(Raw& r, const __nv_bfloat16* row, int column, int offset, int) const {
#pragma unroll
        for (int i = 0; i < P; ++i) r.w[i] = *reinterpret_cast<const uint4*>(row + i * cols + column + offset);
    }
    __device__ __forceinline__ void operand(const Raw& r, uint32_t (&b)[P][4]) const {
#pragma unroll
        for (int i = 0; i < P; ++i) {
            b[i][0] = r.w[i].x; b[i][1] = r.w[i].y; b[i][2] = r.w[i].z; b[i][3] = r.w[i].w;
        }
    }
};

// The warp's number as the same value in all lanes, so that branches on what follows from it need no convergence.
__device__ __forceinline__ int warp_index() { return __shfl_sync(0xffffffffu, (int)(threadIdx.x >> 5), 0); }

// Sixteen bytes to shared memory where `yes`; they are there when the group that they belong to has been waited
// for.
__device__ __forceinline__ void copy16(uint32_t to, const uint8_t* from, bool yes) {
    asm volatile("{\n.reg .pred p;\nsetp.ne.b32 p, %2, 0;\n@p cp.async.cg.shared.global [%0], [%1], 16;\n}" ::"r"(to),
                 "l"(from), "r"((int)yes)
                 : "memory");
}

// The table in registers: as kernel parameters its words would be moved there for every permutation.
__device__ __forceinline__ uint32_t keep(uint32_t v) {
    uint32_t r;
    asm volatile("mov.b32 %0, %1;" : "=r"(r) : "r"(v));
    return r;
}
__device__ __forceinline__ W4Table in_registers(const W4Table& t) {
    return {{keep(t.high[0]), keep(t.high[1])}, {keep(t.low[0]), keep(t.low[1])}};
}

// A warp's way through its blocks.  `Steps` is a list of segments, blocks of MT tiles with the same activation rows:
// next() goes on to one, of blocks() blocks, whose codes begin at code(tile), whose first column and rows (of column
// 8 n + g for this lane) are column() and row(n); tag() is what done(tag, acc) gets with the segment's sums,
// of n / kUnit * s * x.  The products of a group (of 128 columns, if it is longer) are summed by the matrix instructions
// in binary32 and enter acc times the scales of their rows.
//
// What bounds this for a few tokens is, next to the weights' bytes, the integer pipe, which takes an instruction in two
// cycles (address arithmetic, moves by multiplication and 16-bit arithmetic included): 13 to a word of eight weights, 28
// cycles with the matrix instruction.  At 1.9 GHz that is 5.1 TB/s of codes; so all else is kept small.  Two tiles
// share an activation operand; blocks come to shared memory by asynchronous copies, kStages - 1 steps ahead and across
// the ends of segments, and activations are requested a block ahead.  1 token 22528 x 8192: 27.4 us, 3.4 TB/s of codes,
// 43 cycles of 1.9 GHz a word; 38 of them while a multiprocessor has work, the integer pipe busy in 69 % of these, and the
// rest the beginning and 704 CTAs on 296 places.
constexpr int kStages = 4;
template <int MT, int ENDS> constexpr int kRingBytes = kStages * MT * w4_block_bytes(ENDS);       // of a warp

template <int MT, int NT, int ENDS, class S, class Steps, class Done>
__device__ __forceinline__ void w4_stream(Steps steps, const S& source, const W4Table& given, uint8_t* ring, Done done) {
    constexpr int kBytes = w4_block_bytes(ENDS), kCodes = MT * kCodeBytes, kMask = kStages * kCodes - 1;
    constexpr int kScales = MT * ENDS * 32;               // bytes of a stage, behind all stages' codes
    static_assert((kMask & (kMask + 1)) == 0, "the ring is a power of two");
    const int lane = threadIdx.x & 31, g = lane >> 2, q = lane & 3;
    const W4Table table = in_registers(given);
    // the copies
    const uint32_t to = (uint32_t)__cvta_generic_to_shared(ring) + lane * 16;
    const bool scaling = lane < 2 * ENDS;
    Steps ahead = steps;
    const uint8_t* from[MT];
    int left = 0;
    auto turn = [&]() {
        left = 0;
        if (ahead.next()) {
            left = ahead.blocks();
#pragma unroll
            for (int m = 0; m < MT; ++m) from[m] = ahead.code(m) + lane * 16;
        }
    };
    auto fill = [&](uint32_t stage) {                     // a stage's offset among the codes
        if (left > 0) {
#pragma unroll
            for (int m = 0; m < MT; ++m) {
                copy16(to + stage + m * kCodeBytes, from[m], true);
                copy16(to + stage + m * kCodeBytes + 512, from[m] + 512, true);
                copy16(to + kStages * kCodes + stage / kCodes * kScales + m * ENDS * 32, from[m] + 1024, scaling);
                from[m] += kBytes;
            }
            if (--left == 0) turn();
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
    };
    turn();
#pragma unroll
    for (int i = 0; i < kStages - 1; ++i) fill(i * kCodes);
    // the products
    // quarters of a block, of activations: as many as registers hold (three parts and one tile: 64 tokens, 8 of 128
    // experts of 3 x 768 x 2048 binary32 246 us with two quarters, 182 with four)
    constexpr int kAhead = NT == 1 && (S::kPieces < 3 || MT == 1) ? 4 : 2;
    typename S::Raw raw[kAhead][NT];
    const typename S::Elem* row[NT];
    int column = 0;
    bool more = steps.next();
    auto place = [&]() {
#pragma unroll
        for (int n = 0; n < NT; ++n) row[n] = steps.row(n) + q * 8;
        column = steps.column();
    };
    if (more) {
        place();
#pragma unroll
        for (int h = 0; h < kAhead; ++h)
#pragma unroll
            for (int n = 0; n < NT; ++n) source.load(raw[h][n], row[n], column, h * 32, q * 8);
    }
    uint32_t stage = 0;
    while (more) {
        const auto tag = steps.tag();
        float acc[MT][NT][4];
#pragma unroll
        for (int m = 0; m < MT; ++m)
#pragma unroll
            for (int n = 0; n < NT; ++n)
#pragma unroll
                for (int i = 0; i < 4; ++i) acc[m][n][i] = 0.0f;
#pragma unroll 1
        for (int b = steps.blocks(); b > 0;) {
            --b;
            asm volatile("cp.async.wait_group %0;" ::"n"(kStages - 2) : "memory");
            __syncwarp();
            uint32_t words[MT][8], scale[MT][ENDS];
#pragma unroll
            for (int m = 0; m < MT; ++m) {
                const uint8_t* const at = ring + stage + m * kCodeBytes + lane * 16;
                const uint4 c0 = *reinterpret_cast<const uint4*>(at), c1 = *reinterpret_cast<const uint4*>(at + 512);
                words[m][0] = c0.x; words[m][1] = c0.y; words[m][2] = c0.z; words[m][3] = c0.w;
                words[m][4] = c1.x; words[m][5] = c1.y; words[m][6] = c1.z; words[m][7] = c1.w;
#pragma unroll
                for (int i = 0; i < ENDS; ++i)
                    scale[m][i] = *reinterpret_cast<const uint32_t*>(ring + kStages * kCodes + stage / kCodes * kScales +
                                                                     (m * ENDS + i) * 32 + g * 4);
            }
            fill((stage + (kStages - 1) * kCodes) & kMask);              // in the place of the one before this one
            stage = (stage + kCodes) & kMask;
            float part[MT][NT][4];
#pragma unroll
            for (int h = 0; h < 4; ++h) {
                uint32_t x[NT][S::kPieces][4];
#pragma unroll
                for (int n = 0; n < NT; ++n) source.operand(raw[h % kAhead][n], x[n]);
#pragma unroll
                for (int j = 0; j < 2; ++j)
#pragma unroll
                    for (int m = 0; m < MT; ++m) {
                        uint32_t a[4];
                        w4_operand(words[m][2 * h + j], table, a);
#pragma unroll
                        for (int n = 0; n < NT; ++n)
#pragma unroll
                            for (int p = 0; p < S::kPieces; ++p) {
                                if (h * ENDS % 4 == 0 && j == 0 && p == 0)
                                    mma16816_first(part[m][n], a, x[n][p][2 * j], x[n][p][2 * j + 1], typename S::Mma());
                                else
                                    mma16816(part[m][n], a, x[n][p][2 * j], x[n][p][2 * j + 1], typename S::Mma());
                            }
                    }
                if (h + kAhead == 4) {                    // from here on the next block's
                    if (b > 0) {
                        column += kBlockCols;
                    } else {                              // after the last segment this block's again, unused
                        more = steps.next();
                        if (more) place();
                    }
                }
#pragma unroll
                for (int n = 0; n < NT; ++n)
                    source.load(raw[h % kAhead][n], row[n], column, (h + kAhead) % 4 * 32, q * 8);
                if ((h + 1) * ENDS % 4 == 0) {
#pragma unroll
                    for (int m = 0; m < MT; ++m) {
                        const uint32_t v = scale[m][(h + 1) * ENDS / 4 - 1];
                        const float lo = __uint_as_float(v << 16), hi = __uint_as_float(v & 0xffff0000u);
#pragma unroll
                        for (int n = 0; n < NT; ++n) {
                            acc[m][n][0] = fmaf(lo, part[m][n][0], acc[m][n][0]);
                            acc[m][n][1] = fmaf(lo, part[m][n][1], acc[m][n][1]);
                            acc[m][n][2] = fmaf(hi, part[m][n][2], acc[m][n][2]);
                            acc[m][n][3] = fmaf(hi, part[m][n][3], acc[m][n][3]);
                        }
                    }
                }
            }
        }
        done(tag, acc);
    }
    asm volatile("cp.async.wait_all;" ::: "memory");
}

// x * sigmoid(x)
__device__ __forceinline__ float silu_of(float v) { return __fdiv_rn(v, 1.0f + expf(-v)); }

// Launches a kernel as a dependent of the launch before it.  Its own dependents start when it ends: begun earlier,
// their CTAs take places on the multiprocessors from those of this one that still wait for theirs (4096 x 4096, one
// token, back to back: 5.0 us, 6.1 with the trigger at the beginning).
// kMost: the most shared memory that any call of this kernel asks for.  Calls from several threads share what a kernel is
// allowed, so that it is never a call's own size: a smaller one set between another's setting and launch made that fail.
constexpr size_t kMostShared = 227 * 1024;                // of a CTA
template <size_t kMost, typename A>
cudaError_t launch_w4(void (*kernel)(A), const A& args, dim3 grid, int threads, size_t smem, cudaStream_t stream) {
    static_assert(kMost <= kMostShared, "more shared memory than there is");
    if (smem > kMost) return cudaErrorInvalidValue;
    if (smem > 48 * 1024) {
        const cudaError_t err = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kMost);
        if (err != cudaSuccess) return err;
    }
    return launch_dependent(kernel, grid, dim3((unsigned)threads), smem, stream, args);
}

}  // namespace pwlq
