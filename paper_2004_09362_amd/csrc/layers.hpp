// layers.hpp -- types shared by the C ABI of the layer operators (layers.cpp)
// and their kernels: the linear layer with its epilogue, its gradient, and
// dropout from a counter-based generator.
#pragma once

#include <cstdint>

namespace ar {

// Element types as the kernels see them (ar_dtype without int32).
enum Elem : int32_t { kF32 = 0, kF16 = 1, kBF16 = 2 };
enum Act : int32_t { kActNone = 0, kActRelu = 1, kActGelu = 2, kActGeluTanh = 3, kActSilu = 4 };

// Dropout: element (i, j) is kept where its generator word is at most `last`.
// none = 1 keeps nothing (p = 1).  on = 0: no dropout.
struct DropArgs {
  int32_t on, none;
  uint32_t last, site, k0, k1;
  float scale;
  uint64_t row0;
};

// What follows a product: y = res + drop(act(v + bias)), z = v + bias.
struct Epilogue {
  void* y;           // [M, ldy], float where y_f32, else the operands' type
  const void* bias;  // [N], float where bias_f32, else the operands' type; or NULL
  const void* res;   // [M, ldr] of y's type, or NULL (y itself: accumulate)
  void* z;           // [M, ldz] of the operands' type, or NULL
  int64_t ldy, ldr, ldz;
  int32_t M, N;
  int32_t y_f32, bias_f32, act;
  DropArgs drop;
};

// One product: v[m][n] = sum over k of a(m, k) b(n, k).  An operand that is
// "k-major" holds k consecutively (row m, element k at m * lda + k);
// otherwise its rows are the inner index (row k, element m at k * lda + m).
struct GemmArgs {
  const void* a;
  const void* b;
  int64_t lda, ldb;
  int32_t K, open;  // open: tiles_open of both operands
  int32_t tiles_m, tiles_n;
  int32_t splits, k_split;  // inner length dealt out: split s takes [s * k_split, min(K, (s + 1) * k_split))
  float* part;              // splits > 1: partial sums [splits][M][ldp]
  int64_t ldp;
  Epilogue e;
};

enum GemmShape : int32_t { kTile256 = 0, kTile128 = 1 };

// Tile geometry that the host needs: rows and columns of a workgroup's tile,
// and the bytes of inner length it takes at a time.
constexpr int32_t kTileKBytes = 128;
constexpr int32_t tile_rows(int32_t shape) { return shape == kTile256 ? 256 : 128; }
// Tiles of a product are below this: 256 threads each, fewer than 2^32 in a launch.
constexpr int64_t kMaxTiles = int64_t(1) << 24;

// The largest distance of two rows in bytes at which a tile's offsets fit 32 bits.
constexpr int64_t kMaxTileLd = int64_t(1) << 23;

// Whether every tile but the last of an operand (rows along the output, inner
// indices, ld in elements) may be loaded through registers without a check:
// offsets within a tile fit 32 bits, and where the operand is not k-major, the
// last 16 bytes of the last row before the last tile end within that tile's rows.
// They do not where rows are much shorter than 16 bytes and few are left: 1
// column of halves whose inner length is 64 t + 1 to 6, 2 with 1 or 2, 3 with 1; of
// floats 1 column, 32 t + 1 or 2.  All tiles of such an operand are checked.
constexpr bool tiles_open(bool kmajor, int64_t rows, int64_t inner, int64_t ld, int64_t elem_bytes) {
  if (inner < 1 || rows < 1) return true;  // nothing is loaded
  const int64_t per = 16 / elem_bytes, tile = kTileKBytes / elem_bytes, last_rows = (inner - 1) % tile + 1;
  if (kmajor) return rows == 1 || ld * elem_bytes <= kMaxTileLd;
  if (inner <= tile) return true;  // the last tile is the only one
  return ld * elem_bytes <= kMaxTileLd && (rows - 1) / per * per + per <= last_rows * ld + rows;
}

// elem: Elem; a_kmajor / b_kmajor as above (a k-major b with a not is not
// provided); aligned: whether the asynchronous loads apply (see gemm.hpp).
int launch_gemm(const GemmArgs& g, int32_t elem, bool a_kmajor, bool b_kmajor, bool aligned, int32_t shape, void* stream);
int launch_gemm_f32(const GemmArgs& g, bool a_kmajor, bool b_kmajor, bool aligned, int32_t shape, void* stream);
int launch_gemm_f16(const GemmArgs& g, bool a_kmajor, bool b_kmajor, bool aligned, int32_t shape, void* stream);
int launch_gemm_bf16(const GemmArgs& g, bool a_kmajor, bool b_kmajor, bool aligned, int32_t shape, void* stream);

// The gradient's products with respect to x (a k-major, b not) and w (neither)
// in one launch, both on tiles of that shape.
int launch_gemm_pair(const GemmArgs& x, const GemmArgs& w, int32_t elem, bool aligned, int32_t shape, void* stream);
int launch_gemm_pair_f32(const GemmArgs& x, const GemmArgs& w, bool aligned, int32_t shape, void* stream);
int launch_gemm_pair_f16(const GemmArgs& x, const GemmArgs& w, bool aligned, int32_t shape, void* stream);
int launch_gemm_pair_bf16(const GemmArgs& x, const GemmArgs& w, bool aligned, int32_t shape, void* stream);

// Products of few rows (both operands k-major): gemm_few.hip.
constexpr int32_t kFewMaxRows = 64;
// The widest w of each (a launch has fewer than 2^32 threads: 1024 for 64 columns, and 256).
constexpr int64_t kFewMaxCols = (int64_t(1) << 28) - 64, kStreamMaxCols = (int64_t(1) << 30) - 64;
int launch_gemm_few(const GemmArgs& g, int32_t elem, void* stream);
// the same for operands that can be loaded asynchronously
int launch_gemm_stream(const GemmArgs& g, int32_t elem, void* stream);

// db[n] = (accumulate ? db[n] : 0) + sum over chunks of sums[chunk * ld + n]
struct SumsCall {
  const float* sums;  // NULL: none
  void* db;
  int64_t N, ld;
  int32_t chunks, elem, accumulate;
};

// What the launches before left in parts, in one launch: y of up to two
// products whose inner length was split (splits > 1; the others are passed
// over), the parts summed in order and then the epilogue; and column sums.
int launch_join(const GemmArgs& g, const GemmArgs& h, const SumsCall& s, int32_t elem, void* stream);

// y = res + drop(x), element types xe (x) and ye (y, res).
struct DropCall {
  const void* x;
  const void* res;
  void* y;
  int64_t ldx, ldr, ldy, rows, cols;
  DropArgs drop;
};
int launch_dropout(const DropCall& c, int32_t xe, int32_t ye, void* stream);

// dz = act'(z) * drop(dy) in dz's type, and the sums of its columns before
// that rounding: parts [chunks][N] of `rows_per` rows each.
struct SlopeCall {
  const void* dy;
  const void* z;  // NULL without an activation
  void* dz;       // NULL: sums only
  float* sums;    // NULL: dz only
  int64_t lddy, ldz, lddz, M, N;
  int32_t act;
  int32_t chunks;
  int64_t rows_per;
  DropArgs drop;
};
int launch_slope(const SlopeCall& c, int32_t dye, int32_t ze, void* stream);

}  // namespace ar
