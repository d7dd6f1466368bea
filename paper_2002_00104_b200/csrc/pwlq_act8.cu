// 8-bit activation checkpoints: encode (values -> bytes and group ranges) and decode.
//
// Both directions move each value once and keep nothing.  A thread owns 16 (or 8) consecutive values, the
// 2 ... 32 threads of a group are neighbours in a warp and find the group's range with shuffles, so the
// values are read once although the range must be known before the first byte.  The bound is HBM with the
// instructions close behind (15 and 11 per value): 16384 x 4096 bf16 in 35.8 and 33.2 us, 5670 and 6110 GB/s.
// Rows with gaps between them, or off their alignment, take the kernels that find a value's row first:
// 16384 x 4104 55 and 53 us, 16384 x 4095, whose values and results are shifted, 73 and 73 us.
#include <algorithm>

#include "pwlq_act8.cuh"
#include "pwlq_train.h"

namespace pwlq {
namespace {

constexpr int kThreads = 256;
// Values per thread: 16, so that every access to the bytes is 16 bytes wide; 8 where the rows of the
// values are off their alignment, since neighbouring threads then join their values (store8).
__host__ __device__ constexpr int chunk_of(bool vec) { return vec ? 16 : 8; }

// A matrix of 16-bit values whose rows do not start on 16-byte boundaries is copied to one whose rows
// do by extra blocks of a decode launch, from block `first` on: a launch of its own cost 3.7 us.
__device__ __forceinline__ void realign(const Realigned& r) {
    typedef __nv_bfloat16 T;                     // 16 bits, whatever they mean
    const unsigned per_row = (unsigned)(r.pitch / 8);
    const int64_t row0 = (int64_t)(blockIdx.x - r.first) * r.rows_per_block;
    const unsigned rows = (unsigned)min((int64_t)r.rows_per_block, r.rows - row0);
    for (unsigned i = threadIdx.x; i < rows * per_row; i += blockDim.x) {
        const unsigned row = i / per_row, c = (i - row * per_row) * 8;
        const T* from = reinterpret_cast<const T*>(r.from) + (row0 + row) * r.ld + c;
        Raw8<T> v;
        load8<false>(v, from, (int)r.cols - (int)c, (int)c);
        v.store(reinterpret_cast<T*>(r.to) + (row0 + row) * r.pitch + c);
    }
}

// Which chunk of which row a thread owns.  Rows of up to 256 chunks share a block (rows_per_block of
// them), longer ones take blocks_per_row equal blocks; a row's chunks are counted in whole groups, so
// that a group's threads are an aligned part of a warp.  A block has as many warps as that takes, so
// that a row of 172 chunks does not leave a third of 256 threads idle.
struct Act8Grid {
    int64_t rows, cols;
    int threads;
    int chunks_lo;                       // chunks per row inside one block
    int rows_per_block;
    unsigned blocks_per_row;
    unsigned magic;                      // tid / chunks_lo == (tid * magic) >> 16 for tid < 256
};

// valid: how many values the row has from the chunk's first on (<= 0: the thread has nothing to do).
__device__ __forceinline__ bool locate(const Act8Grid& g, int chunk, int64_t& row, int64_t& col, int& valid) {
    const unsigned rb = blockIdx.x / g.blocks_per_row, part = blockIdx.x - rb * g.blocks_per_row;
    const unsigned in = (threadIdx.x * g.magic) >> 16;
    row = (int64_t)rb * g.rows_per_block + in;
    col = ((int64_t)part * g.chunks_lo + (threadIdx.x - in * g.chunks_lo)) * chunk;
    valid = in < (unsigned)g.rows_per_block && row < g.rows ? (int)(g.cols - col) : 0;
    return valid > 0;
}

template <typename T, bool VEC>
__global__ void __launch_bounds__(kThreads)
act8_encode_kernel(const T* x, int64_t ldx, Act8Grid g, int group_shift, float ratio,
                   uint8_t* codes, int64_t ldc, float* ranges, int64_t groups) {
    constexpr int kChunk = chunk_of(VEC), kParts = kChunk / 8;
    int64_t row, col;
    int valid;
    const bool live = locate(g, kChunk, row, col, valid);
    Raw8<T> raw[kParts];
    const T* src = x + row * ldx + col;
#pragma unroll
    for (int i = 0; i < kParts; ++i)
        load8<VEC>(raw[i], src + 8 * i, valid - 8 * i, (int)min((int64_t)8, col) + 8 * i);
    float v[kChunk], top = 0.0f;
#pragma unroll
    for (int i = 0; i < kParts; ++i) raw[i].get(v + 8 * i);
#pragma unroll
    for (int i = 0; i < kChunk; ++i) top = max_abs(top, v[i]);
    top = group_max(top, (1 << group_shift) / kChunk);
    const float m = act8_range(top);
    const PieceParams P = act8_params_paired(m, ratio);
    if (!live) return;
    uint2 w[kParts];
#pragma unroll
    for (int i = 0; i < kParts; ++i) w[i] = act8_bytes8(v + 8 * i, m, P);
    uint8_t* to = codes + row * ldc + col;
    if (kParts == 2) {
        *reinterpret_cast<uint4*>(to) = make_uint4(w[0].x, w[0].y, w[kParts - 1].x, w[kParts - 1].y);
    } else {
        *reinterpret_cast<uint2*>(to) = w[0];
        // the row's last 16 bytes may need zeros that no value stands for
        if (valid <= 8 && (col & 8) == 0) *reinterpret_cast<uint2*>(to + 8) = make_uint2(0u, 0u);
    }
    if ((col & (((int64_t)1 << group_shift) - 1)) == 0) ranges[row * groups + (col >> group_shift)] = m;
}

template <typename T, bool VEC>
__global__ void __launch_bounds__(kThreads)
act8_decode_kernel(const uint8_t* codes, int64_t ldc, const float* ranges, int64_t groups,
                   Act8Grid g, int group_shift, float ratio, T* y, int64_t ldy, Realigned beside) {
    allow_dependents();
    if (blockIdx.x >= beside.first) return realign(beside);
    constexpr int kChunk = chunk_of(VEC), kParts = kChunk / 8;
    int64_t row, col;
    int valid;
    const bool live = locate(g, kChunk, row, col, valid);
    if (!__any_sync(0xffffffffu, live)) return;
    uint2 w[kParts] = {};
    float m = 0.0f;
    if (live) {
        const uint8_t* from = codes + row * ldc + col;
        if (kParts == 2) {
            const uint4 b = *reinterpret_cast<const uint4*>(from);
            w[0] = make_uint2(b.x, b.y);
            w[kParts - 1] = make_uint2(b.z, b.w);
        } else {
            w[0] = *reinterpret_cast<const uint2*>(from);
        }
        m = ranges[row * groups + (col >> group_shift)];
    }
    u64 v[4 * kParts];
    act8_decode<kParts>(w, m, ratio, v);
    T* dst = y + row * ldy + col;
#pragma unroll
    for (int i = 0; i < kParts; ++i) {
        float o[8];
#pragma unroll
        for (int k = 0; k < 4; ++k) unpack2(v[4 * i + k], o[2 * k], o[2 * k + 1]);
        store8<VEC>(o, dst + 8 * i, valid - 8 * i);
    }
}

// Without gaps between the rows, and with whole groups, there are no rows to find: chunk i is the 16
// values, and the 16 bytes, from 16 i on.  C of them per thread, a block's width apart, are requested
// together.  Both directions issue three instructions a cycle of four and move 80 to 95 % of what a copy
// moves (16384 x 4096 bf16: 35.8 and 33.2 us).  Two chunks per thread; of 16-bit values, once there are
// kManyValues, three to encode and four to decode (there 37.9 -> 35.8 and 35.5 -> 33.2 us; 4096 x 4096
// 10.4 against 10.8 and 7.6 against 7.9 us; binary32 16384 x 4096 50.0 against 50.4 and 52.3 against 53.2 us).
constexpr int64_t kManyValues = (int64_t)1 << 25;
template <typename T, int C>
__global__ void __launch_bounds__(kThreads)
act8_encode_flat_kernel(const T* x, int64_t chunks, int group_shift, float ratio, uint8_t* codes, float* ranges) {
    const int64_t first = (int64_t)blockIdx.x * (kThreads * C) + threadIdx.x;
    Raw8<T> raw[C][2];
#pragma unroll
    for (int j = 0; j < C; ++j) {
        const int64_t i = min(first + j * kThreads, chunks - 1);      // lanes past the end repeat it
        raw[j][0].load(x + 16 * i);
        raw[j][1].load(x + 16 * i + 8);
    }
#pragma unroll
    for (int j = 0; j < C; ++j) {
        const int64_t i = first + j * kThreads;
        float v[16], top = 0.0f;
        raw[j][0].get(v);
        raw[j][1].get(v + 8);
#pragma unroll
        for (int k = 0; k < 16; ++k) top = max_abs(top, v[k]);
        const float m = act8_range(group_max(top, 1 << (group_shift - 4)));
        const PieceParams P = act8_params_paired(m, ratio);
        if (i >= chunks) continue;           // the whole warp goes on: it shuffles
        const uint2 a = act8_bytes8(v, m, P), b = act8_bytes8(v + 8, m, P);
        *reinterpret_cast<uint4*>(codes + 16 * i) = make_uint4(a.x, a.y, b.x, b.y);
        if ((i & ((1 << (group_shift - 4)) - 1)) == 0) ranges[i >> (group_shift - 4)] = m;
    }
}
template <typename T, int C>
__global__ void __launch_bounds__(kThreads)
act8_decode_flat_kernel(const uint8_t* codes, const float* ranges, int64_t chunks, int group_shift, float ratio,
                        T* y, Realigned beside) {
    allow_dependents();
    if (blockIdx.x >= beside.first) return realign(beside);
    const int64_t first = (int64_t)blockIdx.x * (kThreads * C) + threadIdx.x;
    uint4 w[C];
    float m[C];
#pragma unroll
    for (int j = 0; j < C; ++j) {
        const int64_t i = min(first + j * kThreads, chunks - 1);
        w[j] = *reinterpret_cast<const uint4*>(codes + 16 * i);
        m[j] = ranges[i >> (group_shift - 4)];
    }
#pragma unroll
    for (int j = 0; j < C; ++j) {
        const int64_t i = first + j * kThreads;
        if (i >= chunks) return;
        const uint2 bytes[2] = {make_uint2(w[j].x, w[j].y), make_uint2(w[j].z, w[j].w)};
        u64 v[8];
        act8_decode<2>(bytes, m[j], ratio, v);
        T* to = y + 16 * i;
        store32(to, raw32(v, T()));
        if (sizeof(T) == 4) store32(to + 8, raw32(v + 4, T()));
    }
}
// Whether the flat kernels do: 32-byte boundaries, no gaps, whole groups.
inline bool is_flat(const void* values, int64_t ld, const Act8Tensor& a) {
    return (reinterpret_cast<uintptr_t>(values) & 31) == 0 && ld == a.cols && a.ldc == a.cols && a.cols % a.group == 0;
}
inline bool is_many(const Act8Tensor& a, size_t size) { return size == 2 && a.rows * a.cols >= kManyValues; }
inline unsigned flat_blocks(const Act8Tensor& a, int per_thread) {
    const int64_t per_block = kThreads * per_thread * 16;
    return (unsigned)((a.rows * a.cols + per_block - 1) / per_block);
}

void plan(int64_t rows, int64_t cols, int group, bool vec, Act8Grid& g, unsigned& blocks) {
    const int per_group = group / chunk_of(vec);
    const int64_t chunks = (cols + group - 1) / group * per_group;
    g.rows = rows;
    g.cols = cols;
    const int64_t per_row = (chunks + kThreads - 1) / kThreads;
    if (per_row == 1) {
        g.chunks_lo = (int)chunks;
        g.rows_per_block = kThreads / g.chunks_lo;
        g.threads = (g.chunks_lo * g.rows_per_block + 31) / 32 * 32;
    } else {
        g.rows_per_block = 1;
        g.threads = g.chunks_lo = (int)((chunks + per_row - 1) / per_row + 31) / 32 * 32;
    }
    g.magic = (unsigned)(65536 / g.chunks_lo + 1);
    const int64_t n = (rows + g.rows_per_block - 1) / g.rows_per_block * per_row;
    g.blocks_per_row = (unsigned)per_row;
    blocks = (unsigned)n;                // at most 2^31 - 1: the entry points check it
}

template <typename T>
cudaError_t encode(const void* x, const Act8Tensor& a, int64_t ldx, cudaStream_t stream) {
    Act8Grid g;
    unsigned blocks;
    if (is_flat(x, ldx, a)) {
        const bool many = is_many(a, sizeof(T));
        auto* kernel = act8_encode_flat_kernel<T, 2>;
        if constexpr (sizeof(T) == 2) {
            if (many) kernel = act8_encode_flat_kernel<T, 3>;
        }
        kernel<<<flat_blocks(a, many ? 3 : 2), kThreads, 0, stream>>>(
            static_cast<const T*>(x), a.rows * a.cols / 16, group_shift(a.group), a.ratio, a.codes, a.ranges);
        return cudaGetLastError();
    }
    const bool vec = rows_aligned(x, ldx, sizeof(T));
    plan(a.rows, a.cols, a.group, vec, g, blocks);
    const T* p = static_cast<const T*>(x);
    auto* kernel = vec ? act8_encode_kernel<T, true>
                                                   : act8_encode_kernel<T, false>;
    kernel<<<blocks, g.threads, 0, stream>>>(p, ldx, g, group_shift(a.group), a.ratio, a.codes,
                                            a.ldc, a.ranges, a.groups());
    return cudaGetLastError();
}
// Where the extra blocks begin, and how many they are.
unsigned place(Realigned& r, unsigned blocks) {
    r.first = blocks;
    if (!r.from) return 0;
    r.rows_per_block = (unsigned)std::max<int64_t>(1, 2048 / (r.pitch / 8));
    return (unsigned)((r.rows + r.rows_per_block - 1) / r.rows_per_block);
}

template <typename T>
cudaError_t decode(const Act8Tensor& a, void* y, int64_t ldy, Realigned beside, cudaStream_t stream) {
    Act8Grid g;
    unsigned blocks;
    if (is_flat(y, ldy, a)) {
        const bool many = is_many(a, sizeof(T));
        const unsigned extra = place(beside, flat_blocks(a, many ? 4 : 2));
        auto* kernel = act8_decode_flat_kernel<T, 2>;
        if constexpr (sizeof(T) == 2) {
            if (many) kernel = act8_decode_flat_kernel<T, 4>;
        }
        kernel<<<beside.first + extra, kThreads, 0, stream>>>(
            a.codes, a.ranges, a.rows * a.cols / 16, group_shift(a.group), a.ratio, static_cast<T*>(y), beside);
        return cudaGetLastError();
    }
    const bool vec = rows_aligned(y, ldy, sizeof(T));
    plan(a.rows, a.cols, a.group, vec, g, blocks);
    T* p = static_cast<T*>(y);
    auto* kernel = vec ? act8_decode_kernel<T, true>
                                                   : act8_decode_kernel<T, false>;
    const unsigned extra = place(beside, blocks);
    kernel<<<beside.first + extra, g.threads, 0, stream>>>(a.codes, a.ldc, a.ranges, a.groups(), g,
                                                           group_shift(a.group), a.ratio, p, ldy, beside);
    return cudaGetLastError();
}

}  // namespace

cudaError_t launch_act8_encode(const void* x, int dtype, int64_t ldx, const Act8Tensor& a,
                               cudaStream_t stream) {
    if (dtype == kF32) return encode<float>(x, a, ldx, stream);
    if (dtype == kBf16) return encode<__nv_bfloat16>(x, a, ldx, stream);
    return encode<__half>(x, a, ldx, stream);
}
cudaError_t launch_act8_decode(const Act8Tensor& a, void* y, int dtype, int64_t ldy, cudaStream_t stream,
                               const Realigned& beside) {
    if (dtype == kF32) return decode<float>(a, y, ldy, beside, stream);
    if (dtype == kBf16) return decode<__nv_bfloat16>(a, y, ldy, beside, stream);
    return decode<__half>(a, y, ldy, beside, stream);
}

}  // namespace pwlq
