// Host-side launchers of the operators on 4-bit weights (internal to the library).
#pragma once

#include "pwlq_train.h"

namespace pwlq {

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
// would otherwise be turned and taken apart for every tile of a large matrix: 1 token 8192 x 8192 binary32 24.8 -> 17.4 us,
// 8 tokens 8191 x 8191 bf16 21.4 -> 14.0, but 1 x 1000 x 2048 binary32, called one by one, 5.0 -> 7.4.
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
