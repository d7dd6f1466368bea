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
        if (n > 0) {                                      // n / 256 = 1.m * 2^(e - 8)
            int e = 0;
            while (n >> (e + 1)) ++e;
            bits = bf16 ? (uint32_t)(e - 8 + 127) << 7 | ((uint32_t)(n << 7) >> e & 127)
                        : (uint32_t)(e - 8 + 15) << 10 | ((uint32_t)(n << 10) >> e & 1023);
        }
        v.table.high[i >> 2] |= (bits >> 8) << 8 * (i & 3);
        v.table.low[i >> 2] |= (bits & 255) << 8 * (i & 3);
    }
    return v;
}

namespace {

constexpr float kInv192 = 192.0f;

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

// One CTA packs 16 rows x 256 columns, a multiple of every group length; a thread holds 16 values of a row, so
// that a range is a few shuffles between neighbours.  Levels come from comparing |x| with halves of steps: a
// bound is (a half-integer of at most 9 bits) * (a scale of 8 bits), exact in binary32, so that the level is the
// nearest one, without a rounding on the way.
template <bool VEC, typename T>
__global__ void __launch_bounds__(256) w4_encode_kernel(const T* __restrict__ x, int64_t ldx, int64_t ldm, W4Write w) {
    __shared__ uint16_t runs[16][66];                     // four codes each; two columns of padding against conflicts
    const int r = threadIdx.x >> 4, c = threadIdx.x & 15;
    const int64_t tile = blockIdx.x, matrix = blockIdx.z;
    const int64_t col = (int64_t)blockIdx.y * 256 + c * 16;
    const int64_t row = w.row_of(tile, r);
    await_previous();
    float v[16];
    {
        const T* p = x + matrix * ldm + (row < 0 ? 0 : row) * ldx + col;
        const int64_t valid = row < 0 ? 0 : w.cols - col;
        Raw8<T> a, b;
        load8<VEC>(a, p, (int)max((int64_t)-8, min(valid, (int64_t)64)), (int)min(col, (int64_t)64));
        load8<VEC>(b, p + 8, (int)max((int64_t)-8, min(valid - 8, (int64_t)64)), (int)min(col, (int64_t)64) + 8);
        a.get(v);
        b.get(v + 8);
    }
    uint32_t m = 0;                                       // as bits: a NaN is above infinity, infinity above the rest
#pragma unroll
    for (int i = 0; i < 16; ++i) m = max(m, abs_bits(v[i]));
    const int lanes = 1 << (w.group_shift - 4);           // threads of a group
    for (int o = 1; o < lanes; o <<= 1) m = max(m, __shfl_xor_sync(0xffffffffu, m, o));
    uint32_t bits = 0;
    if (m >= kInfBits) {
        bits = 0x7fc00000u;
    } else if (__uint_as_float(m) >= kAct8Tiny) {
        bits = (__float_as_uint(__fdiv_rn(__uint_as_float(m), kInv192)) + 0xffffu) & 0xffff0000u;
    }
    const float s = m >= kInfBits ? 0.0f : __uint_as_float(bits);
    const float b = (float)w.breakpoint, d = (float)(64 - w.breakpoint);
    const float edge = 3.0f * b * s;
    const float c1 = 0.5f * b * s, c2 = 1.5f * b * s, c3 = 2.5f * b * s;
    const float t1 = (3.0f * b + 0.5f * d) * s, t2 = (3.0f * b + 1.5f * d) * s, t3 = (3.0f * b + 2.5f * d) * s;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        uint32_t run = 0;
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const float value = v[4 * i + k], a = fabsf(value);
            const bool tail = a > edge;
            // halves go to the even level
            uint32_t code = (a > (tail ? t1 : c1) ? 1u : 0u) + (a >= (tail ? t2 : c2) ? 1u : 0u) +
                            (a > (tail ? t3 : c3) ? 1u : 0u) + (tail ? 4u : 0u);
            if (value < 0.0f) code |= 8u;
            run |= code << 4 * k;
        }
        runs[r][c * 4 + i] = s > 0.0f ? (uint16_t)run : (uint16_t)0;
    }
    // a group's first thread writes its scale, of a group of 256 the first one of either block
    if ((c & (min(lanes, 8) - 1)) == 0 && col / kBlockCols < w.blocks)
        *reinterpret_cast<uint16_t*>(w.block(matrix, tile, col / kBlockCols) + kCodeBytes + ((c & 7) / lanes) * 32 +
                                     (r & 7) * 4 + (r >> 3) * 2) = (uint16_t)(bits >> 16);
    __syncthreads();
    const int64_t block = (int64_t)blockIdx.y * 2 + (threadIdx.x >> 7);
    if (block >= w.blocks) return;
    const int lane = (threadIdx.x & 127) >> 2, h = threadIdx.x & 3;     // two words each, of a quarter of the block
    uint32_t word[2];
#pragma unroll
    for (int j = 0; j < 2; ++j) {
        const int at = (threadIdx.x >> 7) * 32 + h * 8 + (lane & 3) * 2 + j;
        const uint32_t a = runs[lane >> 2][at], e = runs[(lane >> 2) + 8][at];
        word[j] = (a & 0x7777u) | (e & 0x7777u) << 16 |
                  (a & 0x8u) << 4 | (a & 0x80u) << 8 | (a & 0x800u) << 12 | (a & 0x8000u) << 16 |
                  (e & 0x8u) | (e & 0x80u) << 4 | (e & 0x800u) << 8 | (e & 0x8000u) << 12;
    }
    // a lane's words 0-3 in the block's first 512 bytes, 4-7 in the next
    *reinterpret_cast<uint2*>(w.block(matrix, tile, block) + (h >> 1) * 512 + lane * 16 + (h & 1) * 8) =
        make_uint2(word[0], word[1]);
}

// A warp per block; a lane has eight consecutive values of two rows in both halves of the block.
template <bool VEC, typename T>
__global__ void __launch_bounds__(256) w4_decode_kernel(const W4View v, W4Write w, T* __restrict__ y, int64_t ldy,
                                                        int64_t ldm) {
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
            for (int k = 0; k < 8; ++k) out[i][k] = (out[i][k] * 256.0f) * scale;
            const int valid = row < 0 ? 0 : (int)max((int64_t)0, min(w.cols - col, (int64_t)8));
            T* const to = y + matrix * ldm + (row < 0 ? 0 : row) * ldy + col;
            if (VEC && valid == 8) {
                Raw8<T> raw;
                raw.set(out[i]);
                raw.store(to);
            } else {
                store8_each(out[i], to, valid);
            }
        }
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
    const dim3 grid((unsigned)to.tiles, (unsigned)((w.cols + 255) / 256), (unsigned)w.matrices);
    const bool aligned = rows_aligned(x, ldx, sizeof(T)) && (w.matrices == 1 || rows_aligned(x, ldm, sizeof(T)));
    return aligned ? launch_dependent(w4_encode_kernel<true, T>, grid, dim3(256), 0, stream, x, ldx, ldm, to)
                   : launch_dependent(w4_encode_kernel<false, T>, grid, dim3(256), 0, stream, x, ldx, ldm, to);
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

cudaError_t launch_w4_linear(const pwlq_w4& w, const void* x, int dtype, int64_t tokens, int64_t ldx, void* y,
                             int64_t ldy, cudaStream_t stream) {
    if (dtype == kF32) return w4_linear_of<float>(w, x, tokens, ldx, y, ldy, stream);
    if (dtype == kBf16) return w4_linear_of<__nv_bfloat16>(w, x, tokens, ldx, y, ldy, stream);
    return w4_linear_of<__half>(w, x, tokens, ldx, y, ldy, stream);
}

}  // namespace pwlq
