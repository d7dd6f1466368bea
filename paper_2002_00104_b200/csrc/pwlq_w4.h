// Host-side launchers of the operators on 4-bit weights (internal to the library).
#pragma once

#include "pwlq_train.h"

namespace pwlq {

constexpr int kTileRows = 16;            // rows of a tile
constexpr int kBlockCols = 64;           // columns of a block: 16 x 64 values in 512 bytes
constexpr int kBlockBytes = kTileRows * kBlockCols / 2;

inline int64_t w4_blocks(int64_t cols) { return (cols + kBlockCols - 1) / kBlockCols; }
inline int64_t w4_tiles(int64_t rows, bool paired) { return paired ? (rows / 2 + 7) / 8 : (rows + 15) / 16; }
inline int64_t w4_groups(int64_t cols, int64_t group) { return (cols + group - 1) / group; }

cudaError_t launch_w4_encode(const pwlq_w4& w, const void* x, int dtype, int64_t ldx, int64_t ldm, cudaStream_t stream);
cudaError_t launch_w4_decode(const pwlq_w4& w, void* y, int dtype, int64_t ldy, int64_t ldm, cudaStream_t stream);
cudaError_t launch_w4_linear(const pwlq_w4& w, const void* x, int dtype, int64_t tokens, int64_t ldx, void* y,
                             int64_t ldy, cudaStream_t stream);
size_t w4_moe_workspace(int64_t tokens, int64_t top, int64_t hidden);
cudaError_t launch_w4_moe(const pwlq_w4_moe_args& a, cudaStream_t stream);

}  // namespace pwlq
