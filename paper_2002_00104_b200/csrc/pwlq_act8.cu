// 8-bit activation checkpoints: encode (values -> bytes and group ranges) and decode.
//
// Both directions move each value once and keep nothing: they are bound by HBM.  A thread owns 16
// consecutive values (a 16-byte access to the bytes, two or four to the values), the 2 ... 16
// threads of a group are neighbours in a warp and find the group's range with shuffles, so the
// values are read once although the range must be known before the first byte.
#include "pwlq_act8.cuh"
#include "pwlq_train.h"

namespace pwlq {
namespace {

constexpr int kThreads = 256;
constexpr int kChunk = 16;               // values per thread

// Which chunk of which row a thread owns.  Rows of fewer than 256 chunks share a block
// (rows_per_block of them), longer ones take blocks_per_row blocks; `chunks` is the row's number of
// chunks rounded up to whole groups, so that a group's threads are an aligned part of a warp.
struct Act8Grid {
    int64_t rows, cols;
    int chunks_lo;                       // chunks per row inside one block
    int rows_per_block;
    unsigned blocks_per_row;
    unsigned magic;                      // tid / chunks_lo == (tid * magic) >> 16 for tid < 256
};

__device__ __forceinline__ bool locate(const Act8Grid& g, int64_t& row, int64_t& col) {
    const unsigned rb = blockIdx.x / g.blocks_per_row, part = blockIdx.x - rb * g.blocks_per_row;
    const unsigned in = (threadIdx.x * g.magic) >> 16;
    row = (int64_t)rb * g.rows_per_block + in;
    col = ((int64_t)part * kThreads + (threadIdx.x - in * g.chunks_lo)) * kChunk;
    return in < (unsigned)g.rows_per_block && row < g.rows && col < g.cols;
}

template <typename T, bool VEC>
__global__ void __launch_bounds__(kThreads)
act8_encode_kernel(const T* x, int64_t ldx, Act8Grid g, int group_shift, float ratio,
                   uint8_t* codes, int64_t ldc, float* ranges, int64_t groups) {
    int64_t row, col;
    const bool live = locate(g, row, col);
    const int valid = live ? (int)min((int64_t)kChunk, g.cols - col) : 0;
    Raw8<T> raw[2];
    const T* src = x + row * ldx + col;
    load8<VEC>(raw[0], src, valid);
    load8<VEC>(raw[1], src + 8, valid - 8);
    float v[kChunk];
    raw[0].get(v);
    raw[1].get(v + 8);
    uint32_t top = 0;
#pragma unroll
    for (int i = 0; i < kChunk; ++i) top = max(top, abs_bits(v[i]));
    top = group_max(top, 1 << (group_shift - 4));
    if (!live) return;
    const float m = act8_range(top);
    const PieceParams P = act8_params(m, ratio);
    uint4 w;
    w.x = act8_word(v, m, P);
    w.y = act8_word(v + 4, m, P);
    w.z = act8_word(v + 8, m, P);
    w.w = act8_word(v + 12, m, P);
    *reinterpret_cast<uint4*>(codes + row * ldc + col) = w;
    if ((col & (((int64_t)1 << group_shift) - 1)) == 0) ranges[row * groups + (col >> group_shift)] = m;
}

template <typename T, bool VEC>
__global__ void __launch_bounds__(kThreads)
act8_decode_kernel(const uint8_t* codes, int64_t ldc, const float* ranges, int64_t groups,
                   Act8Grid g, int group_shift, float ratio, T* y, int64_t ldy) {
    int64_t row, col;
    if (!locate(g, row, col)) return;
    const uint4 w = *reinterpret_cast<const uint4*>(codes + row * ldc + col);
    const PieceParams P = act8_params(ranges[row * groups + (col >> group_shift)], ratio);
    const int valid = (int)min((int64_t)kChunk, g.cols - col);
    T* dst = y + row * ldy + col;
    float v[8];
    act8_values(w.x, P, v);
    act8_values(w.y, P, v + 4);
    store8<VEC>(v, dst, valid);
    act8_values(w.z, P, v);
    act8_values(w.w, P, v + 4);
    store8<VEC>(v, dst + 8, valid - 8);
}

cudaError_t plan(int64_t rows, int64_t cols, int group, Act8Grid& g, unsigned& blocks) {
    const int per_group = group / kChunk;
    const int64_t chunks = (cols + group - 1) / group * per_group;
    g.rows = rows;
    g.cols = cols;
    g.chunks_lo = (int)(chunks < kThreads ? chunks : kThreads);
    g.rows_per_block = kThreads / g.chunks_lo;
    const int64_t per_row = (chunks + kThreads - 1) / kThreads;
    g.magic = (unsigned)(65536 / g.chunks_lo + 1);
    const int64_t n = (rows + g.rows_per_block - 1) / g.rows_per_block * per_row;
    if (n > ((int64_t)1 << 31) - 1) return cudaErrorInvalidConfiguration;
    g.blocks_per_row = (unsigned)per_row;
    blocks = (unsigned)n;
    return cudaSuccess;
}

template <typename T>
cudaError_t encode(const void* x, const Act8Tensor& a, int64_t ldx, cudaStream_t stream) {
    Act8Grid g;
    unsigned blocks;
    if (cudaError_t e = plan(a.rows, a.cols, a.group, g, blocks)) return e;
    const T* p = static_cast<const T*>(x);
    auto* kernel = rows_aligned(x, ldx, sizeof(T)) ? act8_encode_kernel<T, true>
                                                   : act8_encode_kernel<T, false>;
    kernel<<<blocks, kThreads, 0, stream>>>(p, ldx, g, group_shift(a.group), a.ratio, a.codes,
                                            a.ldc, a.ranges, a.groups());
    return cudaGetLastError();
}
template <typename T>
cudaError_t decode(const Act8Tensor& a, void* y, int64_t ldy, cudaStream_t stream) {
    Act8Grid g;
    unsigned blocks;
    if (cudaError_t e = plan(a.rows, a.cols, a.group, g, blocks)) return e;
    T* p = static_cast<T*>(y);
    auto* kernel = rows_aligned(y, ldy, sizeof(T)) ? act8_decode_kernel<T, true>
                                                   : act8_decode_kernel<T, false>;
    kernel<<<blocks, kThreads, 0, stream>>>(a.codes, a.ldc, a.ranges, a.groups(), g,
                                            group_shift(a.group), a.ratio, p, ldy);
    return cudaGetLastError();
}

}  // namespace

cudaError_t launch_act8_encode(const void* x, int dtype, int64_t ldx, const Act8Tensor& a,
                               cudaStream_t stream) {
    if (dtype == kF32) return encode<float>(x, a, ldx, stream);
    if (dtype == kBf16) return encode<__nv_bfloat16>(x, a, ldx, stream);
    return encode<__half>(x, a, ldx, stream);
}
cudaError_t launch_act8_decode(const Act8Tensor& a, void* y, int dtype, int64_t ldy,
                               cudaStream_t stream) {
    if (dtype == kF32) return decode<float>(a, y, ldy, stream);
    if (dtype == kBf16) return decode<__nv_bfloat16>(a, y, ldy, stream);
    return decode<__half>(a, y, ldy, stream);
}

}  // namespace pwlq
