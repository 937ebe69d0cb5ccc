// Layout of a matrix of 4-bit weights (docs/QUANT.md, section 2) and the launchers of its kernels.
#pragma once

#include "lc_quant.cuh"

namespace lc {

constexpr uint32_t kQ4TileRows = 16;    // rows of a tile: the m of one m16n8k16 product
constexpr uint32_t kQ4StepCols = 128;   // columns of a step; rows are filled up to whole steps
constexpr uint32_t kQ4StepBytes = kQ4TileRows * kQ4StepCols / 2;

// Codes: [tile][block of 64 columns][lane][4 words]. Lane 4 * r + t holds rows r and r + 8 of the tile and, of either half of the
// block (32 columns), the columns 8 t ... 8 t + 7: word 2 * half + j the four columns 8 t + 4 j + (0..3) of both rows, in the order
// in which an m16n8k16 product takes its first operand: bits 4 p and 16 + 4 p (p = 0..3) hold two neighbouring columns, p = 0 and 1
// the first two of row r and of row r + 8, p = 2 and 3 the last two.
// Scales (bf16), behind the codes at a multiple of 256: [tile][group][r][2]: rows r and r + 8 side by side.
// What is added to fill a matrix up has codes of 0 and scales of 0.
struct Q4Layout {
  uint32_t rows, cols, group;
  uint32_t tiles, steps, groups;  // groups: per row, with those of the columns added
  uint64_t scales_off, total;
};

inline Q4Layout q4_layout(uint64_t rows, uint64_t cols, int group) {
  Q4Layout L;
  L.rows = (uint32_t)rows;
  L.cols = (uint32_t)cols;
  L.group = (uint32_t)group;
  L.tiles = (uint32_t)((rows + kQ4TileRows - 1) / kQ4TileRows);
  L.steps = (uint32_t)((cols + kQ4StepCols - 1) / kQ4StepCols);
  L.groups = L.steps * (kQ4StepCols / (uint32_t)group);
  L.scales_off = (uint64_t)L.tiles * L.steps * kQ4StepBytes;  // a multiple of 1024
  L.total = align_up(L.scales_off + (uint64_t)L.tiles * L.groups * kQ4TileRows * 2, 256);
  return L;
}

// status: set to LC_ERR_NONFINITE where a weight is Inf or NaN
cudaError_t launch_q4_quantize(const Q4Layout& L, const void* w, int type, uint64_t row_stride, uint8_t* q4, int32_t* status, cudaStream_t cs);
cudaError_t launch_q4_read(const Q4Layout& L, const uint8_t* q4, void* out, int type, uint64_t row_stride, cudaStream_t cs);
cudaError_t launch_q4_matvec(const Q4Layout& L, const uint8_t* q4, const void* x, int type, uint32_t tokens, uint64_t x_stride, void* out,
                             int out_type, uint64_t out_stride, cudaStream_t cs);

}  // namespace lc
