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

// The orthogonalised update (orthogonal.hip).  Its matrices lie in the workspace
// as halves, each value times a power of two: a value is the sum of two halves,
// "high" and "low" (22 bits), in two planes.  They have m rows and n columns, m
// the shorter side, padded with zeros to whole tiles (mp, np).
constexpr float kOrthoScaleX = 8192.0f, kOrthoScaleA = 8192.0f, kOrthoScaleQ = 4096.0f;

// x or y, in the user's layout: `rows` x `cols`; turned: m is its columns.
struct OrthoOuter {
  const void* data;
  int64_t ld, stride;  // elements from row to row, and from matrix to matrix
  int32_t elem;
};
struct OrthoShape {
  int64_t rows, cols, mp, np;
  int32_t batch, turned, blocks;  // blocks: of a matrix' sum of squares
};

// sums[matrix][block] of the squares of x, in 64 bits.
int launch_ortho_norm(const OrthoShape& s, const OrthoOuter& x, double* sums, void* stream);
// X = x / (|x| + eps), both planes.
int launch_ortho_load(const OrthoShape& s, const OrthoOuter& x, const double* sums, double eps, void* planes, void* stream);
// The three products of a step.
enum OrthoKind : int32_t {
  kOrthoGram = 0,    // A = X X^T
  kOrthoSquare = 1,  // Q = b A + c A A without its diagonal, which goes to diag in 32 bits
  kOrthoApply = 2    // X = a X + (Q + diag) X, or y of it
};

// Whether a product's tiles may be split: the first, which has the longest inner
// length and the fewest tiles, and the second on tiles of 128 with three products
// each.  Of the others plan_part's model finds none faster so, at any of 400 000 sizes.
constexpr bool ortho_splits(int32_t kind, int32_t planes, int32_t tile) {
  return tile != 64 && (kind == kOrthoGram || (kind == kOrthoSquare && planes == 2 && tile == 128));
}

// One product of each of `batch` matrices: out[m][n] of sums over k of
// left(m, k) right(n, k), or of left(m, k) right(k, n) for kOrthoApply.  Tiles are
// dealt out as steps (128 bytes of inner length of one tile and pair of planes):
// workgroup w takes steps [w share, (w + 1) share) of all.  A tile that lies in
// one share is finished there; of others (ortho_splits) the parts go to `parts` and
// are joined by a second launch.
struct OrthoProduct {
  const void* left;
  const void* right;
  const void* old;   // kOrthoSquare: A, kOrthoApply: X
  void* out;
  float* diag;       // [batch][M]
  float* parts;
  int64_t ld_left, ld_right, ld_out;              // elements
  int64_t plane_left, plane_right, plane_out;     // elements from the high plane to the low one
  int64_t batch_left, batch_right, batch_out;     // from matrix to matrix
  int32_t M, N, K;                                // multiples of the tile, K of 64
  int32_t tiles_m, tiles_n, tiles;                // of a matrix; symmetric results: those on and below the diagonal
  int32_t batch, steps, share, workgroups;        // steps of a tile
  float a, b, c;
  // The last product of all: y = residual + scale X (residual.data NULL: none);
  // rows and cols of y, which is turned where m is its columns.  y.data NULL: to out.
  OrthoOuter residual, y;
  int64_t rows, cols;
  int32_t turned;
  float scale;
};
// tile: 256, 128, or 64 (share = steps).
int launch_ortho_product(const OrthoProduct& g, int32_t kind, int32_t planes, int32_t tile, void* stream);

}  // namespace ar
