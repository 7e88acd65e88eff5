// What the launches of the served layer share: its row tiles and the arguments of both sides.
#pragma once

#include "kq_common.hpp"

namespace kq {

// ---- row tiles ---------------------------------------------------------------------------------
// Rows are taken in units of 32 (row / 32); a tile is up to NT units of one expert, and the rows of
// a unit outside [lo, hi) belong to another tile. One layer without offsets has one expert.
struct LinearTile {
  int expert, unit, lo, hi;
};

// Column (of a chunk of 32) of element i of step jj of a lane's eight codes, in the order in which
// the codes of a packed chunk are spread to pairs of fp16.
__host__ __device__ inline int chunk_col(int bits, int jj, int i) {
  const int p = i >> 1, b = i & 1;
  if (bits == 2) return 16 * (jj >> 1) + 4 * (jj & 1) + p + 8 * b;
  if (bits == 8) return 8 * jj + 4 * (p >> 1) + (p & 1) + 2 * b;
  return 8 * jj + p + 4 * b;  // 3 and 4 bits
}

// A side's transform of d elements: columns of cols = min(m, 512) elements, d / cols of them.
struct LinearTurn {
  bool rotate, has28;
  int m, cols;
  float norm;
};
LinearTurn linear_turn(int64_t d, bool rotate);

// x' = T_in diag(mul_in) x as fp16 in fragment order, and what lies beside it
struct LinearIn {
  const void* x;
  int x_dtype;
  int64_t ldx, n_rows, d_in;
  const float *mul, *q28;
  LinearTurn turn;
  int bits, planes;
  uint16_t* xf;     // plane after plane
  int64_t plane;    // elements of a plane
  float* row_unit;  // [n_rows] what the rows were divided by
  // the weights' table (or null): per group and row a dword {s 2^24 / unit, -z s / unit} in fp16;
  // per row its unit
  uint32_t* table;
  float* w_unit;
  const float *scales, *zeros;
  int64_t ldsz;
  int gpq, ng;     // groups of 128 columns per quantisation group, and in a row
  int64_t w_rows;  // rows of W over all experts
  // the list of tiles of NT units (with offsets): max_tiles of them after a count in a slot of its own
  const int* offsets;
  int n_experts, nt;
  int64_t max_tiles;
  LinearTile* tiles;
};
int linear_in_launch(const LinearIn& a, hipStream_t s);

// y = act(diag(mul_out) T_out y' + bias) + residual with y' the sum of the splits
struct LinearOut {
  const float* part;      // [split][row][ld]
  int64_t ld, stride;     // of a row and a split
  int splits;
  const float* row_unit;  // or null (1)
  int64_t n_rows, d_out;
  const float *mul, *q28;
  LinearTurn turn;
  const float* bias;
  int act;
  const void* residual;
  int64_t ldr;
  void* y;
  int y_dtype;
  int64_t ldy;
  const int* offsets;
  int n_experts;
};
int linear_out_launch(const LinearOut& a, hipStream_t s);

}  // namespace kq
