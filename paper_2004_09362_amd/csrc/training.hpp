// training.hpp -- types shared by the C ABI of what a training step runs around
// its linear layers (training.cpp) and its kernels: layer norm, its gradient
// (norm.hip), and the orthogonalised update of a weight (orthogonal.hip).
#pragma once

#include <cstdint>

#include "layers.hpp"

namespace ar {

// How rows of `cols` columns are dealt out (norm.hip): groups of `V` columns,
// group t + q * lanes to lane t of a team, q < per.  wide: rows that no team
// holds in its registers.
struct RowTeams {
  int32_t V, lanes, per, wide;
};
constexpr int64_t kTeamColumns = 16384;  // the longest row that a team holds
RowTeams row_teams(int64_t cols);

struct NormCall {
  const void* x;
  const void* w;  // NULL: ones
  const void* b;  // NULL: zeros
  void* y;
  float* stats;   // [rows][lds]: mean, 1 / standard deviation; NULL: not kept
  int64_t ldx, ldy, lds, rows, cols;
  int32_t we, be;  // element types of w and b
  float eps;
};
int launch_norm(const NormCall& c, int32_t xe, int32_t ye, void* stream);

// dx = res + rstd (g - mean(g) - h mean(g h)); parts: the sums of dy * h and of dy
// over each workgroup's rows, [blocks][2][cols].
struct NormGradCall {
  const void* dy;
  const void* x;
  const void* w;    // NULL: ones
  const float* stats;
  const void* res;  // of x's type; NULL: none
  void* dx;         // of x's type; NULL: sums only
  float* parts;     // NULL: dx only
  int64_t lddy, ldx, lds, ldr, lddx, rows, cols;
  int32_t we, blocks;
};
// The workgroups of a gradient, each with parts of its own, and for rows that
// are wide the rows of each.
int32_t norm_grad_blocks(int64_t rows, int64_t cols);
int launch_norm_grad(const NormGradCall& c, int32_t xe, int32_t dye, void* stream);

// dw[n] = (accumulate ? dw[n] : 0) + sum over blocks of parts[block][0][n], and
// db of parts[block][1]; NULL: not wanted.
struct NormJoinCall {
  const float* parts;
  void* dw;
  void* db;
  int64_t cols;
  int32_t blocks, dwe, dbe, accumulate;
};
int launch_norm_join(const NormJoinCall& c, void* stream);

}  // namespace ar
