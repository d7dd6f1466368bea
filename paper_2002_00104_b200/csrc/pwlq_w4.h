// Host-side launchers of the operators on 4-bit weights (internal to the library).
#pragma once

#include "pwlq_train.h"

namespace pwlq {

constexpr int kMultiprocessors = 148;    // of a B200
constexpr int kTileRows = 16;            // rows of a tile
constexpr int kBlockCols = 128;          // columns of a block: 16 x 128 values, and the scales of its groups
constexpr int kCodeBytes = kTileRows * kBlockCols / 2;

inline int64_t w4_blocks(int64_t cols) { return (cols + kBlockCols - 1) / kBlockCols; }
inline int64_t w4_tiles(int64_t rows, bool paired) { return paired ? (rows / 2 + 7) / 8 : (rows + 15) / 16; }
// Groups that end in a block (a group of 256 has its scales in both of its blocks), and a block's size.
__host__ __device__ constexpr int w4_ends(int64_t group) { return group == 32 ? 4 : group == 64 ? 2 : 1; }
__host__ __device__ constexpr int w4_block_bytes(int ends) { return kCodeBytes + ends * 2 * kTileRows; }

cudaError_t launch_w4_encode(const pwlq_w4& w, const void* x, int dtype, int64_t ldx, int64_t ldm, cudaStream_t stream);
cudaError_t launch_w4_decode(const pwlq_w4& w, void* y, int dtype, int64_t ldy, int64_t ldm, cudaStream_t stream);
// The product takes rows as they are, or in parts, a copy that a launch of its own makes (see include/pwlq.h), where they
// would otherwise be turned and taken apart for every tile of a large matrix, one of 4096 blocks and more.  us without and
// with the copy, of calls back to back in a graph; a call on its own pays 2.4 for the second launch (1 x 1000 x 2048
// binary32 5.0, 7.4):
//     blocks               binary32: 1, 8, 16 tokens             bf16, a column fewer
//      1024  1024 x 2048   4.6  4.0, 4.8  4.7,  9.5  7.6         2.7  3.4,  5.2  4.0,  8.5  4.8
//      4096  4096 x 2048   6.5  5.5, 6.8  6.7, 10.1 11.5         3.9  4.4,  6.3  5.0,  9.3  6.8
//      8192  4096 x 4096   10.8 7.3, 11.1 8.8, 16.9 18.0         5.6  5.9, 10.1  7.3, 16.6  9.7
//     32768  8192 x 8192   24.7 17.4, 25.6 18.1, 43.2 31.9       14.0 13.4, 21.5 14.0, 33.7 16.8
inline int64_t w4_padded(int64_t cols) { return w4_blocks(cols) * kBlockCols; }
inline bool w4_copies(int64_t rows, int64_t cols, int dtype, bool aligned) {
    return (dtype == kF32 || cols % 8 != 0 || !aligned) && (rows / 16) * w4_blocks(cols) >= 4096;
}
inline size_t w4_copy_bytes(int64_t tokens, int64_t cols, int dtype) {
    return (size_t)(tokens * w4_padded(cols) * (dtype == kF32 ? 6 : 2) + 255) / 256 * 256;
}
cudaError_t launch_w4_copy(const void* x, int dtype, int64_t tokens, int64_t cols, int64_t ldx, void* copy, cudaStream_t stream);
// copied: x is the copy.
template <typename T>
cudaError_t w4_linear_of(const pwlq_w4& w, const void* x, bool copied, int64_t tokens, int64_t ldx, void* y, int64_t ldy,
                         cudaStream_t stream);
cudaError_t launch_w4_linear(const pwlq_w4& w, const void* x, int dtype, int64_t tokens, int64_t ldx, void* y,
                             int64_t ldy, void* workspace, cudaStream_t stream);
size_t w4_moe_workspace(int64_t tokens, int64_t top, int64_t features, int64_t hidden);
cudaError_t launch_w4_moe(const pwlq_w4_moe_args& a, cudaStream_t stream);

}  // namespace pwlq
