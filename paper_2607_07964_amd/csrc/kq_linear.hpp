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

constexpr int LINEAR_BLOCK = 256;  // rows of W of an item

// The outputs are cut into items of a row tile and a block of rows of W, tile after tile, which
// `workers` workgroups share: whole items in full rounds, and the groups of columns of the items left
// over in equal parts, `per` groups a worker in item order. So the last round is as full as the others
// and few items keep the whole chip busy, however the rows fall to experts; a worker that begins inside
// an item keeps that part in a place of its own, for linear_out to add.
struct LinearDeal {
  int full, per;  // rounds of whole items; groups of the rest per worker
};
__host__ __device__ inline LinearDeal linear_deal(int items, int ng, int workers) {
  const int full = items / workers, rest = items - full * workers;
  int per = (rest * ng + workers - 1) / workers;
  // few groups a worker are mostly start and end, and a rest that nearly fills a round gains less
  // than its parts cost to write and read again
  if (per < 2) per = 2;
  if (per * 10 > ng * 9) per = ng;
  return LinearDeal{full, per};
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
  // the weights' table (or null): per group and row a dword {s / unit, -(1024 + z)} in fp16;
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
  int2* first;     // [n_experts] first tile and first unit of each expert
};
int linear_in_launch(const LinearIn& a, hipStream_t s);

// y = act(diag(mul_out) T_out y' + bias) + residual
struct LinearOut {
  // y' [row][ld] (with w_unit: to be multiplied by it); dealt (workers > 0), with the parts that workers
  // keep, [worker][32 nt][LINEAR_BLOCK]
  const float* part;
  int64_t ld;
  int workers, ng, nt, row_blocks, items;  // items without offsets
  const float* kept;
  const float* w_unit;
  const LinearTile* tiles;
  const int2* first;
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
  bool pairs;             // (set by the launch)
};
int linear_out_launch(const LinearOut& a, hipStream_t s);

}  // namespace kq
