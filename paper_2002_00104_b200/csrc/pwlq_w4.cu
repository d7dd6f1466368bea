// 4-bit weights: encode and decode (format: include/pwlq.h).
#include "pwlq_w4.cuh"

namespace pwlq {

W4View w4_view(const pwlq_w4& w, bool bf16) {
    W4View v = {};
    v.data = static_cast<const uint8_t*>(w.data);
    v.rows = w.rows;
    v.cols = (int)w.cols;
    v.paired = w.paired != 0;
    v.tiles = w4_tiles(w.rows, v.paired);
    v.blocks = (int)w4_blocks(w.cols);
    v.ends = w4_ends(w.group);
    const int b = (int)w.breakpoint;
    for (int i = 0; i < 8; ++i) {
        const int n = i < 4 ? i * b : 3 * b + (i - 4) * (64 - b);
        uint32_t bits = 0;
        if (n > 0) {                                      // n / kUnit = 1.m * 2^(e - kUnitBits)
            int e = 0;
            while (n >> (e + 1)) ++e;
            bits = bf16 ? (uint32_t)(e - kUnitBits<__nv_bfloat16> + 127) << 7 | ((uint32_t)(n << 7) >> e & 127)
                        : (uint32_t)(e - kUnitBits<__half> + 15) << 10 | ((uint32_t)(n << 10) >> e & 1023);
        }
        v.table.high[i >> 2] |= (bits >> 8) << 8 * (i & 3);
        v.table.low[i >> 2] |= (bits & 255) << 8 * (i & 3);
    }
    return v;
}

namespace {

constexpr float kUnits = 192.0f;         // scales to a range

struct W4Write {
    uint8_t* data;
    int64_t tiles, blocks, rows, cols;
    int group_shift, ends, breakpoint, paired;
    __device__ __forceinline__ uint8_t* block(int64_t matrix, int64_t tile, int64_t b) const {
        return data + ((matrix * tiles + tile) * blocks + b) * w4_block_bytes(ends);
    }
    // row of the matrix that row r of a tile is, or -1
    __device__ __forceinline__ int64_t row_of(int64_t tile, int r) const {
        const int64_t half = rows / 2;
        const int64_t i = paired ? tile * 8 + (r & 7) : tile * 16 + r;
        if (i >= (paired ? half : rows)) return -1;
        return paired && r >= 8 ? half + i : i;
    }
};

// 1 where a > t, 0 elsewhere, for a and t in units of t's own size and 2^-40 times it or more: the sign of a - t is
// that of the fused product's exact sum, and its size at least an ulp.  One instruction of the multiply-add pipe; a
// comparison and a selection take four cycles of the integer pipe.
__device__ __forceinline__ float above(float a, float minus_t) {
    float r;
    asm("fma.rn.sat.f32 %0, %1, 0f53800000, %2;" : "=f"(r) : "f"(a), "f"(minus_t));      // 2^40
    return r;
}

// One CTA packs 16 rows x 256 columns, a multiple of every group length; a thread holds 16 values of a row, so
// that a range is a few shuffles between neighbours.  A code counts the bounds below |x|, four between levels of the
// center and the tail and the breakpoint itself.  A bound is (a half-integer of at most 9 bits) * (a scale of 8 bits),
// exact in binary32, so that the level is the nearest one, without a rounding on the way.
// It goes on to the tile below, so that what does not depend on the values is made once for several tiles.
// Bound by issue: 30 instructions to a value, 14 of them bounds and sums; 8192 x 8192 bf16 65 us, 168 MB at 2.6 TB/s.
template <bool VEC, typename T>
__global__ void __launch_bounds__(256) w4_encode_kernel(const T* __restrict__ x, int64_t ldx, int64_t ldm, W4Write w,
                                                        int tiles_each) {
    __shared__ uint16_t runs[2][16][66];                  // four codes each; two columns of padding against conflicts
    const int r = threadIdx.x >> 4, c = threadIdx.x & 15;
    const int64_t first = (int64_t)blockIdx.x * tiles_each, matrix = blockIdx.z;
    const int col = blockIdx.y * 256 + c * 16, cols = (int)w.cols;
    const int lanes = 1 << (w.group_shift - 4);           // threads of a group
    // the row of the first tile that this thread has, and how many it has in all
    const int64_t half = w.rows / 2, step = w.paired ? 8 : 16;
    const int64_t row = w.paired && r >= 8 ? half + first * 8 + r - 8 : first * step + r;
    const int64_t end = w.paired && r < 8 ? half : w.rows;
    const T* p = x + matrix * ldm + row * ldx + col;
    int rows = (int)min((int64_t)tiles_each, max((int64_t)0, (end - row + step - 1) / step));
    int tiles = (int)min((int64_t)tiles_each, w.tiles - first);
    uint8_t* to = w.block(matrix, first, (int64_t)blockIdx.y * 2);
    const int64_t tile_bytes = w.blocks * w4_block_bytes(w.ends);
    // a group's first thread writes its scale, of a group of 256 the first one of either block
    const bool scaling = (c & (min(lanes, 8) - 1)) == 0 && (c >> 3) + blockIdx.y * 2 < w.blocks;
    const int scale_at = (c >> 3) * w4_block_bytes(w.ends) + kCodeBytes + ((c & 7) / lanes) * 32 + (r & 7) * 4 + (r >> 3) * 2;
    // two words of a quarter of a block; a lane's words 0-3 are in the block's first 512 bytes, 4-7 in the next
    const int block = threadIdx.x >> 7, lane = (threadIdx.x & 127) >> 2, h = threadIdx.x & 3;
    const bool writing = blockIdx.y * 2 + block < w.blocks;
    const int words_at = block * w4_block_bytes(w.ends) + (h >> 1) * 512 + lane * 16 + (h & 1) * 8;
    const int runs_at = block * 32 + h * 8 + (lane & 3) * 2;
    const float b = (float)w.breakpoint, d = (float)(64 - w.breakpoint);
    const float center = -1099511627776.0f * b, tail = -1099511627776.0f * d;       // -2^40
    await_previous();
    for (int turn = 0; tiles > 0; --tiles, --rows, turn ^= 1, p += step * ldx, to += tile_bytes) {
        float v[16];
        {
            const int valid = rows > 0 ? cols - col : 0;
            Raw8<T> lo, hi;
            load8<VEC>(lo, p, valid, col);
            load8<VEC>(hi, p + 8, valid - 8, col + 8);
            lo.get(v);
            hi.get(v + 8);
        }
        uint32_t m = 0;                                   // as bits: a NaN is above infinity, infinity above the rest
#pragma unroll
        for (int i = 0; i < 16; ++i) m = max(m, abs_bits(v[i]));
        for (int o = 1; o < lanes; o <<= 1) m = max(m, __shfl_xor_sync(0xffffffffu, m, o));
        uint32_t bits = 0;
        if (m >= kInfBits) {
            bits = 0x7fc00000u;
        } else if (__uint_as_float(m) >= kAct8Tiny) {
            bits = (__float_as_uint(__fdiv_rn(__uint_as_float(m), kUnits)) + 0xffffu) & 0xffff0000u;
        }
        // s = unit * 2^e: bounds for values times 2^-e, so that no product leaves the range of binary32
        const bool some = m < kInfBits && bits != 0;
        const float unit = __uint_as_float((bits & 0x007fffffu) | 0x3f800000u);
        const float scale = __uint_as_float(some ? 0x7f000000u - (bits & 0x7f800000u) : 0u);
        const float bk = center * unit, dk = tail * unit;
        // halves go to the even level: at 1.5 steps up, so that the bound there is the number before it (a tail without
        // steps, at 64, has its bounds at the breakpoint)
        const float edge = 3.0f * bk;
        const float c1 = 0.5f * bk, c2 = __uint_as_float(__float_as_uint(1.5f * bk) - 1), c3 = 2.5f * bk;
        const float t1 = edge + 0.5f * dk, t2 = __uint_as_float(__float_as_uint(edge + 1.5f * dk) - (d > 0.0f)),
                    t3 = edge + 2.5f * dk;
        const float bounds[6] = {c2, c3, edge, t1, t2, t3};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            float run = 0.0f;
#pragma unroll
            for (int h2 = 2; h2 >= 0; h2 -= 2) {
                const float x0 = v[4 * i + h2] * scale, x1 = v[4 * i + h2 + 1] * scale;
                u64 count = pack2(above(fabsf(x0), c1), above(fabsf(x1), c1));
#pragma unroll
                for (int n = 0; n < 6; ++n) count = add2(count, pack2(above(fabsf(x0), bounds[n]), above(fabsf(x1), bounds[n])));
                // the sign of what is not held as 0
                run = fmaf(run, 16.0f, fmaf(above(-x1, c1), 8.0f, hi2(count)));
                run = fmaf(run, 16.0f, fmaf(above(-x0, c1), 8.0f, lo2(count)));
            }
            runs[turn][r][c * 4 + i] = (uint16_t)(some ? __float_as_uint(run + 8388608.0f) : 0u);
        }
        if (scaling) *reinterpret_cast<uint16_t*>(to + scale_at) = (uint16_t)(bits >> 16);
        __syncthreads();
        if (!writing) continue;
        uint32_t word[2];
        const uint32_t a2 = *reinterpret_cast<const uint32_t*>(&runs[turn][lane >> 2][runs_at]);
        const uint32_t e2 = *reinterpret_cast<const uint32_t*>(&runs[turn][(lane >> 2) + 8][runs_at]);
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            // magnitudes of row g below those of row g + 8; signs: bits 3, 7, 11, 15 go to 7, 15, 23, 31 for row g, to 3, 11,
            // 19, 27 for row g + 8
            const uint32_t both = permute(a2, e2, j ? 0x7632u : 0x5410u);
            const uint32_t s = permute(a2, 0u, j ? 0x4342u : 0x4140u), q = permute(e2, 0u, j ? 0x4342u : 0x4140u);
            word[j] = (both & 0x77777777u) | (s << 4 & 0x00800080u) | (s << 8 & 0x80008000u) | (q & 0x00080008u) |
                      (q << 4 & 0x08000800u);
        }
        *reinterpret_cast<uint2*>(to + words_at) = make_uint2(word[0], word[1]);
    }
}

// A warp per block; a lane has eight consecutive values of two rows in every quarter of the block.  Bound by DRAM for
// rows on 16-byte boundaries: 8192 x 8192 bf16 29.6 us, 5.7 TB/s.
template <bool VEC, typename T>
__global__ void __launch_bounds__(256) w4_decode_kernel(const W4View v, W4Write w, T* __restrict__ y, int64_t ldy,
                                                        int64_t ldm) {
    __shared__ T turn[VEC ? 1 : 8][16][33];
    const int lane = threadIdx.x & 31, g = lane >> 2, q = lane & 3;
    const int64_t tile = blockIdx.x, matrix = blockIdx.z;
    const int64_t block = (int64_t)blockIdx.y * 8 + (threadIdx.x >> 5);
    await_previous();
    if (block >= v.blocks) return;
    const uint8_t* const at = w.block(matrix, tile, block);
    const uint4 c0 = *reinterpret_cast<const uint4*>(at + lane * 16);
    const uint4 c1 = *reinterpret_cast<const uint4*>(at + 512 + lane * 16);
    const uint32_t words[8] = {c0.x, c0.y, c0.z, c0.w, c1.x, c1.y, c1.z, c1.w};
#pragma unroll
    for (int half = 0; half < 4; ++half) {
        const int64_t col = block * kBlockCols + half * 32 + q * 8;
        const uint32_t s = *reinterpret_cast<const uint32_t*>(at + kCodeBytes + (half * w.ends / 4) * 32 + g * 4);
        float out[2][8];
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            uint32_t a[4];
            w4_operand(words[2 * half + j], v.table, a);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                float lo, hi;
                unpack16(a[i], lo, hi, __nv_bfloat16());
                out[i & 1][4 * j + (i & 2)] = lo;
                out[i & 1][4 * j + (i & 2) + 1] = hi;
            }
        }
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const int64_t row = w.row_of(tile, g + 8 * i);
            const float scale = __uint_as_float(i ? s & 0xffff0000u : s << 16);
#pragma unroll
            for (int k = 0; k < 8; ++k) out[i][k] = (out[i][k] * kUnit<__nv_bfloat16>) * scale;
            if constexpr (VEC) {
                const int valid = row < 0 ? 0 : (int)max((int64_t)0, min(w.cols - col, (int64_t)8));
                T* const to = y + matrix * ldm + (row < 0 ? 0 : row) * ldy + col;
                if (valid == 8) {
                    Raw8<T> raw;
                    raw.set(out[i]);
                    raw.store(to);
                } else {
                    store8_each(out[i], to, valid);
                }
            } else {
#pragma unroll
                for (int k = 0; k < 8; ++k) turn[threadIdx.x >> 5][g + 8 * i][q * 8 + k] = from_f32<T>(out[i][k]);
            }
        }
        if constexpr (!VEC) {                             // rows off their alignment: a warp writes 32 neighbours at a time
            __syncwarp();
            const int64_t at_col = block * kBlockCols + half * 32 + lane;
            for (int r = 0; r < 16; ++r) {
                const int64_t row = w.row_of(tile, r);
                if (row >= 0 && at_col < w.cols) y[matrix * ldm + row * ldy + at_col] = turn[threadIdx.x >> 5][r][lane];
            }
            __syncwarp();
        }
    }
}

// Rows of activations for the products: whole blocks of columns, zeros behind the last one; binary32 values in three
// bf16 parts, one after another.  Made once, where every tile of the weights would make it for itself.
template <typename T>
__global__ void __launch_bounds__(128) w4_copy_kernel(const T* __restrict__ x, int64_t ldx, int64_t cols, void* __restrict__ copy,
                                                      int64_t padded) {
    const int64_t col = ((int64_t)blockIdx.y * 128 + threadIdx.x) * 8, token = blockIdx.x;
    allow_dependents();                                   // few CTAs: the next launch may take its places
    await_previous();
    if (col >= padded) return;
    Raw8<T> raw;
    load8<false>(raw, x + token * ldx + col, (int)max((int64_t)-8, min(cols - col, (int64_t)64)), (int)min(col, (int64_t)64));
    if constexpr (sizeof(T) == 4) {
        float v[8];
        uint32_t b[3][4];
        raw.get(v);
        parts3(v, b);
#pragma unroll
        for (int p = 0; p < 3; ++p)
            *reinterpret_cast<uint4*>(static_cast<__nv_bfloat16*>(copy) + (token * 3 + p) * padded + col) =
                make_uint4(b[p][0], b[p][1], b[p][2], b[p][3]);
    } else {
        raw.store(static_cast<T*>(copy) + token * padded + col);
    }
}

W4Write writer(const pwlq_w4& w) {
    const bool paired = w.paired != 0;
    return {static_cast<uint8_t*>(w.data), w4_tiles(w.rows, paired), w4_blocks(w.cols), w.rows, w.cols,
            group_shift((int)w.group), w4_ends(w.group), (int)w.breakpoint, paired};
}

template <typename T>
cudaError_t encode(const pwlq_w4& w, const T* x, int64_t ldx, int64_t ldm, cudaStream_t stream) {
    const W4Write to = writer(w);
    // several tiles to a CTA where that leaves enough of them: 8192 x 8192 bf16 82 -> 70 us with four
    const int64_t columns = (w.cols + 255) / 256;
    const int each = to.tiles * columns * w.matrices >= 4 * 8 * kMultiprocessors ? 4 : 1;
    const dim3 grid((unsigned)((to.tiles + each - 1) / each), (unsigned)columns, (unsigned)w.matrices);
    const bool aligned = rows_aligned(x, ldx, sizeof(T)) && (w.matrices == 1 || rows_aligned(x, ldm, sizeof(T)));
    return aligned ? launch_dependent(w4_encode_kernel<true, T>, grid, dim3(256), 0, stream, x, ldx, ldm, to, each)
                   : launch_dependent(w4_encode_kernel<false, T>, grid, dim3(256), 0, stream, x, ldx, ldm, to, each);
}

template <typename T>
cudaError_t decode(const pwlq_w4& w, T* y, int64_t ldy, int64_t ldm, cudaStream_t stream) {
    const W4Write at = writer(w);
    const dim3 grid((unsigned)at.tiles, (unsigned)((at.blocks + 7) / 8), (unsigned)w.matrices);
    const W4View v = w4_view(w, true);
    const bool aligned = rows_aligned(y, ldy, sizeof(T)) && (w.matrices == 1 || rows_aligned(y, ldm, sizeof(T)));
    return aligned ? launch_dependent(w4_decode_kernel<true, T>, grid, dim3(256), 0, stream, v, at, y, ldy, ldm)
                   : launch_dependent(w4_decode_kernel<false, T>, grid, dim3(256), 0, stream, v, at, y, ldy, ldm);
}

}  // namespace

cudaError_t launch_w4_encode(const pwlq_w4& w, const void* x, int dtype, int64_t ldx, int64_t ldm, cudaStream_t stream) {
    if (dtype == kF32) return encode(w, static_cast<const float*>(x), ldx, ldm, stream);
    if (dtype == kBf16) return encode(w, static_cast<const __nv_bfloat16*>(x), ldx, ldm, stream);
    return encode(w, static_cast<const __half*>(x), ldx, ldm, stream);
}

cudaError_t launch_w4_decode(const pwlq_w4& w, void* y, int dtype, int64_t ldy, int64_t ldm, cudaStream_t stream) {
    if (dtype == kF32) return decode(w, static_cast<float*>(y), ldy, ldm, stream);
    if (dtype == kBf16) return decode(w, static_cast<__nv_bfloat16*>(y), ldy, ldm, stream);
    return decode(w, static_cast<__half*>(y), ldy, ldm, stream);
}

cudaError_t launch_w4_copy(const void* x, int dtype, int64_t tokens, int64_t cols, int64_t ldx, void* copy, cudaStream_t stream) {
    const int64_t padded = w4_padded(cols);
    const dim3 grid((unsigned)tokens, (unsigned)((padded / 8 + 127) / 128)), threads(128);
    if (dtype == kF32)
        return launch_dependent(w4_copy_kernel<float>, grid, threads, 0, stream, static_cast<const float*>(x), ldx, cols, copy, padded);
    if (dtype == kBf16)
        return launch_dependent(w4_copy_kernel<__nv_bfloat16>, grid, threads, 0, stream, static_cast<const __nv_bfloat16*>(x),
                                ldx, cols, copy, padded);
    return launch_dependent(w4_copy_kernel<__half>, grid, threads, 0, stream, static_cast<const __half*>(x), ldx, cols, copy, padded);
}

cudaError_t launch_w4_linear(const pwlq_w4& w, const void* x, int dtype, int64_t tokens, int64_t ldx, void* y,
                             int64_t ldy, void* workspace, cudaStream_t stream) {
    const bool copied = w4_copies(w.rows, w.cols, dtype, rows_aligned(x, ldx, type_size(dtype)));
    if (copied) {
        const cudaError_t err = launch_w4_copy(x, dtype, tokens, w.cols, ldx, workspace, stream);
        if (err != cudaSuccess) return err;
        x = workspace;
        ldx = w4_padded(w.cols) * (dtype == kF32 ? 3 : 1);
    }
    if (dtype == kF32) return w4_linear_of<float>(w, x, copied, tokens, ldx, y, ldy, stream);
    if (dtype == kBf16) return w4_linear_of<__nv_bfloat16>(w, x, copied, tokens, ldx, y, ldy, stream);
    return w4_linear_of<__half>(w, x, copied, tokens, ldx, y, ldy, stream);
}

}  // namespace pwlq
