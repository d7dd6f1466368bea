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
template <typename T>
cudaError_t w4_linear_of(const pwlq_w4& w, const void* x, int64_t tokens, int64_t ldx, void* y, int64_t ldy,
                         cudaStream_t stream);
template <typename T>
cudaError_t w4_wide_of(const pwlq_w4& w, const void* x, int64_t tokens, int64_t ldx, void* y, int64_t ldy,
                       cudaStream_t stream);
cudaError_t launch_w4_linear(const pwlq_w4& w, const void* x, int dtype, int64_t tokens, int64_t ldx, void* y,
                             int64_t ldy, cudaStream_t stream);
size_t w4_moe_workspace(int64_t tokens, int64_t top, int64_t features, int64_t hidden);
cudaError_t launch_w4_moe(const pwlq_w4_moe_args& a, cudaStream_t stream);

}  // namespace pwlq
