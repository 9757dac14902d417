// layers.cpp -- the layer operators of the C ABI (include/ar.h): argument
// checks, the choice of kernels, and launches.  The kernels are in gemm.hpp,
// gemm_few.hip and rowwise.hip; nothing here computes on the host.
#include <hip/hip_runtime_api.h>

#include <algorithm>
#include <cmath>
#include <cstdint>
#include <exception>
#include <string>
#include <utility>

#include "../../include/ar.h"
#include "ar_internal.hpp"
#include "layers.hpp"

namespace ar {

int launch_gemm(const GemmArgs& g, int32_t elem, bool a_kmajor, bool b_kmajor, bool aligned, int32_t shape, void* stream) {
  switch (elem) {
    case kF32: return launch_gemm_f32(g, a_kmajor, b_kmajor, aligned, shape, stream);
    case kF16: return launch_gemm_f16(g, a_kmajor, b_kmajor, aligned, shape, stream);
    case kBF16: return launch_gemm_bf16(g, a_kmajor, b_kmajor, aligned, shape, stream);
  }
  return int(hipErrorInvalidValue);
}

int launch_gemm_pair(const GemmArgs& x, const GemmArgs& w, int32_t elem, bool aligned, int32_t shape, void* stream) {
  switch (elem) {
    case kF32: return launch_gemm_pair_f32(x, w, aligned, shape, stream);
    case kF16: return launch_gemm_pair_f16(x, w, aligned, shape, stream);
    case kBF16: return launch_gemm_pair_bf16(x, w, aligned, shape, stream);
  }
  return int(hipErrorInvalidValue);
}

}  // namespace ar

namespace {

constexpr int64_t kMaxLength = int64_t(1) << 30;
constexpr int64_t kMaxLd = int64_t(1) << 40;
constexpr int64_t kCus = 256;
constexpr int64_t kWorkspaceAlign = 256;

// A failed check: what to report.
struct Fault {
  ar_status status;
  std::string text;
};
[[noreturn]] void refuse(ar_status s, const std::string& text) { throw Fault{s, text}; }

// The body of an entry point: nothing that is thrown leaves it.
template <typename F>
ar_status guarded(F&& f) noexcept {
  try {
    f();
    return AR_OK;
  } catch (const Fault& x) {
    ar::set_failure_text(x.text.c_str());
    return x.status;
  } catch (const std::exception& x) {
    ar::set_failure_text(x.what());
    return AR_ERR_OUT_OF_MEMORY;
  } catch (...) {
    ar::set_failure_text("unknown failure");
    return AR_ERR_INTERNAL;
  }
}

void launched(int e, const char* what) {
  if (e != 0) refuse(AR_ERR_HIP, std::string(what) + ": " + hipGetErrorString(hipError_t(e)));
}

int32_t elem_of(ar_dtype t) { return t == AR_FLOAT32 ? ar::kF32 : t == AR_FLOAT16 ? ar::kF16 : ar::kBF16; }
int64_t size_of(ar_dtype t) { return t == AR_FLOAT32 ? 4 : 2; }
bool is_float(ar_dtype t) { return t == AR_FLOAT32 || t == AR_FLOAT16 || t == AR_BFLOAT16; }

int64_t round_up(int64_t v, int64_t m) { return (v + m - 1) / m * m; }
int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

void check_length(const char* name, int64_t v) {
  if (v < 0 || v > kMaxLength) refuse(AR_ERR_INVALID_ARG, std::string(name) + " must be in [0, 2^30]");
}

// m is a rows x cols matrix; type: what its dtype must be, or wide: that or float32.
void check_matrix(const char* name, const ar_matrix* m, int64_t rows, int64_t cols) {
  if (!m) refuse(AR_ERR_INVALID_ARG, std::string(name) + " is NULL");
  if (!is_float(m->dtype)) refuse(AR_ERR_UNSUPPORTED, std::string(name) + " must be float32, float16 or bfloat16");
  if (rows == 0 || cols == 0) return;
  if (!m->data) refuse(AR_ERR_INVALID_ARG, std::string(name) + "'s data is NULL");
  if (reinterpret_cast<uintptr_t>(m->data) % uintptr_t(size_of(m->dtype)) != 0)
    refuse(AR_ERR_INVALID_ARG, std::string(name) + "'s data is not on a multiple of its element's size");
  if (rows > 1 && (m->ld < cols || m->ld > kMaxLd))
    refuse(AR_ERR_INVALID_ARG, std::string(name) + "'s ld must be in [" + std::to_string(cols) + ", 2^40]");
}
void check_type(const char* name, const ar_matrix* m, ar_dtype type, bool or_float32) {
  if (m->dtype != type && !(or_float32 && m->dtype == AR_FLOAT32))
    refuse(AR_ERR_UNSUPPORTED, std::string(name) + (or_float32 ? " must have x's type or be float32" : " has the wrong type"));
}

void check_activation(ar_activation a) {
  if (int(a) < AR_ACT_NONE || int(a) > AR_ACT_SILU) refuse(AR_ERR_INVALID_ARG, "unknown activation");
}

ar::DropArgs drop_args(const ar_dropout* d) {
  ar::DropArgs r{};
  r.scale = 1.0f;
  if (!d) return r;
  if (!(d->p >= 0.0 && d->p <= 1.0)) refuse(AR_ERR_INVALID_ARG, "dropout's p must be in [0, 1]");
  if (d->p == 0.0) return r;
  const double limit = std::floor((1.0 - d->p) * 4294967296.0 + 0.5);  // words below it are kept
  r.on = 1;
  r.none = limit < 1.0;
  r.last = limit < 1.0 ? 0u : uint32_t(uint64_t(limit) - 1);
  r.scale = r.none ? 0.0f : float(1.0 / (1.0 - d->p));
  r.site = d->site;
  r.k0 = uint32_t(d->seed);
  r.k1 = uint32_t(d->seed >> 32);
  r.row0 = d->row0;
  return r;
}

// The bytes that a rows x cols matrix covers.
struct Extent {
  uintptr_t at = 0;
  int64_t pitch = 0, row = 0, rows = 0;  // bytes from row to row, of a row, and rows
  bool empty() const { return rows == 0 || row == 0; }
  uintptr_t end() const { return at + uintptr_t((rows - 1) * pitch + row); }
};
Extent extent(const ar_matrix* m, int64_t rows, int64_t cols) {
  Extent e;
  if (!m || rows == 0 || cols == 0) return e;
  e.at = reinterpret_cast<uintptr_t>(m->data);
  e.row = cols * size_of(m->dtype);
  e.pitch = rows > 1 ? m->ld * size_of(m->dtype) : e.row;
  e.rows = rows;
  return e;
}
// Whether two matrices share a byte.  Rows of one pitch are told apart exactly
// (columns of one wider matrix); otherwise ranges that meet count as shared.
bool overlap(const Extent& a, const Extent& b) {
  if (a.empty() || b.empty() || a.end() <= b.at || b.end() <= a.at) return false;
  const int64_t pitch = a.rows > 1 ? a.pitch : b.pitch;
  if ((a.rows > 1 && a.pitch != pitch) || (b.rows > 1 && b.pitch != pitch) || a.row > pitch || b.row > pitch) return true;
  const int64_t d = int64_t((a.at <= b.at ? b.at - a.at : uintptr_t(pitch) - (a.at - b.at) % uintptr_t(pitch)) % uintptr_t(pitch));
  return d < a.row || d + b.row > pitch;
}
void check_apart(const char* out, const Extent& o, const char* other, const Extent& x) {
  if (overlap(o, x)) refuse(AR_ERR_ALIAS, std::string(out) + " overlaps " + other);
}
bool same_place(const ar_matrix* a, const ar_matrix* b, int64_t rows) {
  return a->data == b->data && a->dtype == b->dtype && (rows <= 1 || a->ld == b->ld);
}

void check_device() {
  int device = -1;
  const hipError_t e = hipGetDevice(&device);
  if (e != hipSuccess) {
    (void)hipGetLastError();
    refuse(AR_ERR_NO_DEVICE, std::string("no usable GPU: ") + hipGetErrorString(e));
  }
}

// The part of the workspace that a call uses.
Extent check_workspace(void* w, int64_t have, int64_t need) {
  Extent e;
  if (need == 0) return e;
  if (!w || have < need) refuse(AR_ERR_INVALID_ARG, "the workspace must hold " + std::to_string(need) + " bytes");
  if (reinterpret_cast<uintptr_t>(w) % 16 != 0) refuse(AR_ERR_INVALID_ARG, "the workspace must lie on a 16-byte boundary");
  e.at = reinterpret_cast<uintptr_t>(w);
  e.row = e.pitch = need;
  e.rows = 1;
  return e;
}

// An operand of a product: `rows` of the output along it.
struct Operand {
  const void* data;
  int64_t ld;
  bool kmajor;
  int64_t rows;
};

// Whether an operand's chunks of 16 bytes can be loaded asynchronously: whole,
// on 16-byte boundaries, within 32-bit offsets of their tile's first one.  An
// operand that is not k-major also needs whole chunks of rows, so that none
// reaches past the end of the matrix.
bool can_load_async(const Operand& o, int64_t elem_bytes) {
  const int64_t per = 16 / elem_bytes;
  return reinterpret_cast<uintptr_t>(o.data) % 16 == 0 && o.ld % per == 0 && (o.kmajor || o.rows % per == 0) &&
         o.ld * elem_bytes <= ar::kMaxTileLd;
}

// How a product runs: on which kernel, in how many parts of the inner length.
enum Kind { kTiles, kFew, kStream };
struct Product {
  Kind kind = kTiles;
  bool aligned = false;
  int32_t shape = ar::kTile128, splits = 1, k_split = 0, tiles_m = 0, tiles_n = 0;
  int64_t ldp = 0, M = 0, N = 0, steps = 0, inner = 0;  // steps of `inner` make the inner length
  double micros = 0.0;                                   // on tiles: what the model says, without the join's launch
};

// Shape and parts of a product, whose sizes are there.
void set_parts(Product& p, int32_t shape, int64_t splits) {
  const int64_t tile = ar::tile_rows(shape), per = ceil_div(p.steps, splits);
  p.shape = shape;
  p.tiles_m = int32_t(ceil_div(p.M, tile));
  p.tiles_n = int32_t(ceil_div(p.N, tile));
  p.k_split = int32_t(std::min(per * p.inner, kMaxLength));
  p.splits = int32_t(ceil_div(p.steps, per));
}

// What a product on tiles takes, in microseconds, on this library's kernels at
// the rates that they measured on MI355X: a tile of 128 x 128 costs `fixed` and
// then `one` for every 128 bytes of inner length where it has a compute unit to
// itself, `two` where two share one (256 x 256: one always does).  Parts of a
// split inner length are written and read again by one more launch.
struct TileCost {
  double fixed, one, two;
};
constexpr TileCost kCost256 = {10.0, 1.42, 1.42};
constexpr TileCost kCost128[2][2] = {{{5.0, 0.90, 1.55}, {5.0, 0.68, 1.18}},   // halves: through registers, asynchronous
                                     {{5.0, 2.10, 4.00}, {5.0, 1.90, 3.60}}};  // floats
constexpr double kJoinMicros = 4.0, kJoinBytesPerMicro = 5e6;
const TileCost& tile_cost(const Product& p, int32_t shape, bool floats) {
  return shape == ar::kTile256 ? kCost256 : kCost128[floats][p.aligned];
}
// What the parts of a product add.
double parts_micros(const Product& p, int64_t splits) {
  return splits > 1 ? double(splits) * double(p.M) * double(p.ldp) * 8.0 / kJoinBytesPerMicro : 0.0;
}

double tile_micros(const TileCost& c, int64_t workgroups, int64_t steps, bool shared) {
  const int64_t at_once = shared ? 2 * kCus : kCus, rounds = workgroups / at_once, rest = workgroups % at_once;
  const double last = rest == 0 ? 0.0 : c.fixed + double(steps) * (rest > kCus ? c.two : c.one);
  return double(rounds) * (c.fixed + double(steps) * c.two) + last;
}

Product plan_product(int64_t M, int64_t N, int64_t K, ar_dtype type, const Operand& a, const Operand& b) {
  Product p;
  const int64_t eb = size_of(type);
  p.M = M;
  p.N = N;
  p.inner = ar::kTileKBytes / eb;
  p.steps = std::max<int64_t>(1, ceil_div(K, p.inner));
  p.ldp = round_up(N, 8);
  p.aligned = can_load_async(a, eb) && can_load_async(b, eb);
  const bool rows = a.kmajor && b.kmajor && M <= ar::kFewMaxRows;
  // Few rows.  Aligned, both kernels read w at the rate of memory; the one
  // through LDS keeps it up with more rows and longer inner lengths, the other
  // starts sooner.  M = 1 / 16 / 24 / 64, us in a graph, w beyond the caches:
  //   w               registers, bf16     LDS, bf16          registers, fp32  LDS, fp32
  //   4096 x 4096     8.4/10.5/13.1/23  12.4/12.7/13.0/14.3    17/21/25/46    24/23/23/31
  //   16384 x 4096     32/38/42/76        30/30/29/31          72/81/96/167   60/61/61/96
  //   4096 x 16384     30/37/44/79        29/29/30/33          57/70/91/170   63/63/64/100
  //   8192 x 2048     9.6/10.7/12.6/22  12.3/12.7/12.9/14.2    17/19/25/46    22/23/23/32
  //   16384 x 1024    8.4/10.4/12.6/21   9.1/9.2/9.5/11.2      17/19/24/45    18/19/19/28
  //   4096 x 1024     4.3/4.8/5.5/7.7    7.9/8.3/8.5/10.5     6.3/7.1/8.5/14  11/12/12/16
  //   1024 x 512      3.1/3.6/4.0/5.2    4.2/4.4/4.6/6.2      3.8/4.4/5.3/7.7  8/9/9/12
  // Where these bounds give time away: 3 to 5 us at 8192 x 2048 with up to 16 rows,
  // 6 at 4096 x 16384 fp32 with one, 3 to 10 at 16384 x 1024 bf16 and 4 at 4096 x
  // 1024 fp32 with more than 16.
  // Off the 16-byte boundaries, bf16, the registers' kernel takes 18.6 / 29 / 36 /
  // 64 for 4096 x 4095 and 7.6 / 10.5 / 11.7 / 18.7 for 2047 x 1023, tiles 33 / 36 /
  // 20 / 21 and 14 / 15 / 16 / 17; fp32 at 4096 x 4095 18 / 24 / 29 / 51 and 50 / 49 / 49 /
  // 48.  The bound sends all four of 4096 x 4095 to the tiles: right for 16 bits
  // from 17 rows on, 7 to 15 us late with fewer, and 20 to 32 in fp32 below 64.
  const int64_t row_tiles = M <= 16 ? 1 : M <= 32 ? 2 : 4;
  if (rows && p.aligned && N <= ar::kStreamMaxCols && (M <= 16 ? N >= 8192 || K * eb > 16384 : K * eb > 2048)) {
    p.kind = kStream;
    set_parts(p, ar::kTile128, std::max<int64_t>(1, std::min(kCus / ceil_div(N, 64), p.steps / 8)));
    return p;
  }
  if (rows && N <= ar::kFewMaxCols && (p.aligned || N * K * (1 + row_tiles) <= 20000000)) {
    p.kind = kFew;
    set_parts(p, ar::kTile128, std::max<int64_t>(1, std::min<int64_t>({kCus / ceil_div(N, 16), p.steps / 64, 64})));
    return p;
  }
  const int64_t small = ceil_div(M, 128) * ceil_div(N, 128), large = ceil_div(M, 256) * ceil_div(N, 256);
  if (small >= ar::kMaxTiles) refuse(AR_ERR_UNSUPPORTED, "the product would need 2^24 or more tiles of 128 x 128");
  const bool floats = type == AR_FLOAT32;
  int32_t shape = ar::kTile128;
  int64_t splits = 1;
  double best = 0.0;
  for (int64_t s = 1; s <= std::min<int64_t>(64, std::max<int64_t>(1, p.steps / 2)); ++s) {
    if (s > 1 && s * std::min(small, large) > 8 * kCus) break;  // more parts than the chip takes at once
    for (int32_t sh : {ar::kTile128, ar::kTile256}) {
      if (sh == ar::kTile256 && (!p.aligned || floats)) continue;
      const double t = tile_micros(tile_cost(p, sh, floats), s * (sh == ar::kTile256 ? large : small), ceil_div(p.steps, s),
                                   sh == ar::kTile128) + parts_micros(p, s) + (s > 1 ? kJoinMicros : 0.0);
      if (best > 0.0 && t >= best) continue;
      best = t;
      shape = sh;
      splits = s;
    }
  }
  set_parts(p, shape, splits);
  p.micros = best - (splits > 1 ? kJoinMicros : 0.0);
  return p;
}

// Two products in one launch: workgroups of both kinds take the places that the
// chip has, the longer ones first.
double pair_micros(const TileCost& c, int64_t n1, int64_t steps1, int64_t n2, int64_t steps2, bool shared) {
  const int64_t places = shared ? 2 * kCus : kCus;
  const double one = n1 + n2 > kCus ? c.two : c.one;
  double t1 = c.fixed + double(steps1) * one, t2 = c.fixed + double(steps2) * one;
  if (t2 > t1) {
    std::swap(t1, t2);
    std::swap(n1, n2);
  }
  const int64_t late = n1 % places, early = places - late;  // places that are free a round later, and the others
  double at0 = double(n1 / places) * t1, at1 = at0 + t1, end = late > 0 ? at1 : at0;
  for (int64_t left = n2; left > 0;) {
    const bool first = late == 0 || at0 <= at1;
    left -= first ? early : late;
    double& at = first ? at0 : at1;
    at += t2;
    end = std::max(end, at);
  }
  return end;
}

// Whether x and w, the gradient's two products, share a launch, and their parts
// then: where the model says that it takes less time than one after the other.
// One launch has one start and one end, and while some workgroups write their
// results others multiply.  bf16, each by itself, added / together, us: 16384 x
// 1024 x 1024 84 / 71, 8192 x 4096 x 1024 141 / 117, 8192 x 2048 x 2048 130 / 117;
// fp16 off the 16-byte boundaries 1000 x 2047 x 513 42 / 30.
bool plan_pair(Product& x, Product& w, ar_dtype type) {
  constexpr double kLaunchMicros = 4.0;  // a launch's start and end, seen from the next one
  constexpr int64_t kParts[] = {1, 2, 3, 4, 6, 8, 12, 16, 24, 32};
  if (x.aligned != w.aligned) return false;
  const bool floats = type == AR_FLOAT32;
  double best = x.micros + w.micros + kLaunchMicros + (x.splits > 1 || w.splits > 1 ? kJoinMicros : 0.0);
  int32_t shape = -1;
  int64_t sx = 1, sw = 1;
  for (int32_t sh : {ar::kTile128, ar::kTile256}) {
    if (sh == ar::kTile256 && (!x.aligned || floats)) continue;
    const int64_t tile = ar::tile_rows(sh), tx = ceil_div(x.M, tile) * ceil_div(x.N, tile), tw = ceil_div(w.M, tile) * ceil_div(w.N, tile);
    if (tx + tw > 8 * kCus) continue;  // the ends of long launches weigh little
    for (const int64_t i : kParts) {
      if (i > 1 && (i > x.steps / 2 || i * tx > 4 * kCus)) break;
      for (const int64_t j : kParts) {
        if (j > 1 && (j > w.steps / 2 || j * tw > 4 * kCus)) break;
        const double t = pair_micros(tile_cost(x, sh, floats), i * tx, ceil_div(x.steps, i), j * tw, ceil_div(w.steps, j), sh == ar::kTile128) +
                         parts_micros(x, i) + parts_micros(w, j) + (i > 1 || j > 1 ? kJoinMicros : 0.0);
        if (t >= best) continue;
        best = t;
        shape = sh;
        sx = i;
        sw = j;
      }
    }
  }
  if (shape < 0) return false;
  set_parts(x, shape, sx);
  set_parts(w, shape, sw);
  return true;
}
int64_t part_bytes(const Product& p, int64_t M) { return p.splits > 1 ? p.splits * M * p.ldp * 4 : 0; }

ar::GemmArgs gemm_args(const Product& p, int64_t K, ar_dtype type, const Operand& a, const Operand& b, const ar::Epilogue& e,
                       void* part) {
  ar::GemmArgs g{};
  g.a = a.data;
  g.b = b.data;
  g.lda = a.ld;
  g.ldb = b.ld;
  g.K = int32_t(K);
  g.open = ar::tiles_open(a.kmajor, a.rows, K, a.ld, size_of(type)) && ar::tiles_open(b.kmajor, b.rows, K, b.ld, size_of(type));
  g.tiles_m = p.tiles_m;
  g.tiles_n = p.tiles_n;
  g.splits = p.splits;
  g.k_split = p.k_split;
  g.part = static_cast<float*>(part);
  g.ldp = p.ldp;
  g.e = e;
  return g;
}

void run_product(const Product& p, const ar::GemmArgs& g, int32_t elem, bool a_kmajor, bool b_kmajor, hipStream_t stream,
                 const char* what) {
  launched(p.kind == kFew      ? ar::launch_gemm_few(g, elem, stream)
           : p.kind == kStream ? ar::launch_gemm_stream(g, elem, stream)
                               : ar::launch_gemm(g, elem, a_kmajor, b_kmajor, p.aligned, p.shape, stream),
           what);
}

Operand rows_of(const ar_matrix* m, int64_t rows) { return {m->data, m->ld, true, rows}; }

// What ar_linear_backward does with its workspace.
struct Backward {
  bool make_dz = false;     // dz differs from dy
  int64_t lddz = 0, dz_bytes = 0;
  int32_t chunks = 1;
  int64_t rows_per = 0, sums_bytes = 0;
  Product px, pw;
  bool pair = false;        // both products in one launch
  int64_t part_x = 0, part_w = 0;
  int64_t total() const { return dz_bytes + sums_bytes + part_x + part_w; }
};

Backward plan_backward(int64_t M, int64_t N, int64_t K, const ar_matrix* dy, const ar_matrix* x, const ar_matrix* w,
                       ar_activation act, const ar_dropout* drop, const ar_matrix* dx, const ar_matrix* dw,
                       const ar_matrix* db) {
  Backward p;
  const ar_dtype type = dw ? x->dtype : dx ? w->dtype : dy->dtype;
  p.make_dz = (dx || dw) && M > 0 && N > 0 && (act != AR_ACT_NONE || (drop && drop->p > 0.0) || dy->dtype != type);
  if (p.make_dz) {
    p.lddz = round_up(N, 128 / size_of(type));
    p.dz_bytes = round_up(M * p.lddz * size_of(type), kWorkspaceAlign);
  }
  // enough workgroups of 256 columns to fill the chip, of 32 rows at least
  p.chunks = int32_t(std::max<int64_t>(1, std::min(4 * kCus / std::max<int64_t>(1, ceil_div(N, 256)), ceil_div(M, 32))));
  p.rows_per = round_up(std::max<int64_t>(1, ceil_div(M, p.chunks)), 8);
  p.chunks = int32_t(std::max<int64_t>(1, ceil_div(M, p.rows_per)));
  if (db) p.sums_bytes = round_up(p.chunks * N * 4, kWorkspaceAlign);
  const Operand dz = {p.make_dz ? nullptr : dy->data, p.make_dz ? p.lddz : dy->ld, true, M};
  if (dx) p.px = plan_product(M, K, N, type, dz, {w->data, w->ld, false, K});
  if (dw) p.pw = plan_product(N, K, M, type, {dz.data, dz.ld, false, N}, {x->data, x->ld, false, K});
  p.pair = dx && dw && M > 0 && N > 0 && K > 0 && plan_pair(p.px, p.pw, type);
  if (dx) p.part_x = round_up(part_bytes(p.px, M), kWorkspaceAlign);
  if (dw) p.part_w = round_up(part_bytes(p.pw, N), kWorkspaceAlign);
  return p;
}

// The arguments of the gradient, in the order in which they make sense.
void check_backward(int64_t M, int64_t N, int64_t K, const ar_matrix* dy, const ar_matrix* x, const ar_matrix* w,
                    const ar_matrix* preact, ar_activation act, const ar_dropout* drop, const ar_matrix* dx,
                    const ar_matrix* dw, const ar_matrix* db) {
  check_length("M", M);
  check_length("N", N);
  check_length("K", K);
  check_activation(act);
  (void)drop_args(drop);
  check_matrix("dy", dy, M, N);
  ar_dtype type = dy->dtype;
  if (dw) {
    check_matrix("x", x, M, K);
    type = x->dtype;
  }
  if (dx) {
    check_matrix("w", w, N, K);
    if (dw) check_type("w", w, type, false);
    type = w->dtype;
  }
  if (act != AR_ACT_NONE) {
    check_matrix("preact", preact, M, N);
    if (dx || dw) check_type("preact", preact, type, false);
    else type = preact->dtype;
  }
  check_type("dy", dy, type, true);
  if (dx) {
    check_matrix("dx", dx, M, K);
    check_type("dx", dx, type, true);
  }
  if (dw) {
    check_matrix("dw", dw, N, K);
    check_type("dw", dw, type, true);
  }
  if (db) {
    check_matrix("db", db, 1, N);
    if (dx || dw || act != AR_ACT_NONE) check_type("db", db, type, true);
  }
}

}  // namespace

extern "C" {

ar_status ar_linear_forward_workspace(int64_t M, int64_t N, int64_t K, const ar_matrix* x, const ar_matrix* w,
                                      int64_t* bytes) {
  return guarded([&] {
    if (!bytes) refuse(AR_ERR_INVALID_ARG, "bytes is NULL");
    *bytes = 0;
    check_length("M", M);
    check_length("N", N);
    check_length("K", K);
    check_matrix("x", x, M, K);
    check_matrix("w", w, N, K);
    check_type("w", w, x->dtype, false);
    if (M > 0 && N > 0) *bytes = part_bytes(plan_product(M, N, K, x->dtype, rows_of(x, M), rows_of(w, N)), M);
  });
}

ar_status ar_linear_forward(int64_t M, int64_t N, int64_t K, const ar_matrix* x, const ar_matrix* w,
                            const ar_matrix* bias, const ar_matrix* residual, ar_activation act,
                            const ar_dropout* drop, const ar_matrix* y, const ar_matrix* preact, void* workspace,
                            int64_t workspace_bytes, hipStream_t stream) {
  return guarded([&] {
    check_length("M", M);
    check_length("N", N);
    check_length("K", K);
    check_activation(act);
    check_matrix("x", x, M, K);
    check_matrix("w", w, N, K);
    check_type("w", w, x->dtype, false);
    check_matrix("y", y, M, N);
    check_type("y", y, x->dtype, true);
    if (bias) {
      check_matrix("bias", bias, 1, N);
      check_type("bias", bias, x->dtype, true);
    }
    if (residual) {
      check_matrix("residual", residual, M, N);
      if (residual->dtype != y->dtype) refuse(AR_ERR_UNSUPPORTED, "residual must have y's type");
    }
    if (preact) {
      check_matrix("preact", preact, M, N);
      check_type("preact", preact, x->dtype, false);
    }
    ar::Epilogue e{};
    e.drop = drop_args(drop);
    if (M == 0 || N == 0) return;
    const Extent ey = extent(y, M, N), ex = extent(x, M, K), ew = extent(w, N, K), eb = extent(bias, 1, N);
    const Extent er = extent(residual, M, N), ez = extent(preact, M, N);
    check_apart("y", ey, "x", ex);
    check_apart("y", ey, "w", ew);
    check_apart("y", ey, "bias", eb);
    check_apart("y", ey, "preact", ez);
    check_apart("preact", ez, "x", ex);
    check_apart("preact", ez, "w", ew);
    check_apart("preact", ez, "bias", eb);
    check_apart("preact", ez, "residual", er);
    if (residual && !same_place(residual, y, M)) check_apart("y", ey, "residual", er);
    const Operand a = rows_of(x, M), b = rows_of(w, N);
    const Product p = plan_product(M, N, K, x->dtype, a, b);
    const Extent ews = check_workspace(workspace, workspace_bytes, part_bytes(p, M));
    const Extent* const all[] = {&ex, &ew, &eb, &er, &ey, &ez};
    const char* const names[] = {"x", "w", "bias", "residual", "y", "preact"};
    for (int i = 0; i < 6; ++i) check_apart("the workspace", ews, names[i], *all[i]);
    check_device();
    e.y = y->data;
    e.ldy = y->ld;
    e.M = int32_t(M);
    e.N = int32_t(N);
    e.y_f32 = y->dtype == AR_FLOAT32;
    e.act = int32_t(act);
    if (bias) {
      e.bias = bias->data;
      e.bias_f32 = bias->dtype == AR_FLOAT32;
    }
    if (residual) {
      e.res = residual->data;
      e.ldr = residual->ld;
    }
    if (preact) {
      e.z = preact->data;
      e.ldz = preact->ld;
    }
    const ar::GemmArgs g = gemm_args(p, K, x->dtype, a, b, e, workspace);
    run_product(p, g, elem_of(x->dtype), true, true, stream, "linear kernel launch");
    if (p.splits > 1) launched(ar::launch_join(g, ar::GemmArgs{}, ar::SumsCall{}, elem_of(x->dtype), stream), "join kernel launch");
  });
}

ar_status ar_linear_backward_workspace(int64_t M, int64_t N, int64_t K, const ar_matrix* dy, const ar_matrix* x,
                                       const ar_matrix* w, const ar_matrix* preact, ar_activation act,
                                       const ar_dropout* drop, const ar_matrix* dx, const ar_matrix* dw,
                                       const ar_matrix* db, int64_t* bytes) {
  return guarded([&] {
    if (!bytes) refuse(AR_ERR_INVALID_ARG, "bytes is NULL");
    *bytes = 0;
    check_backward(M, N, K, dy, x, w, preact, act, drop, dx, dw, db);
    *bytes = plan_backward(M, N, K, dy, x, w, act, drop, dx, dw, db).total();
  });
}

ar_status ar_linear_backward(int64_t M, int64_t N, int64_t K, const ar_matrix* dy, const ar_matrix* x,
                             const ar_matrix* w, const ar_matrix* preact, ar_activation act, const ar_dropout* drop,
                             const ar_matrix* dx, const ar_matrix* dw, const ar_matrix* db, int32_t accumulate,
                             void* workspace, int64_t workspace_bytes, hipStream_t stream) {
  return guarded([&] {
    check_backward(M, N, K, dy, x, w, preact, act, drop, dx, dw, db);
    const Extent ins[] = {extent(dy, M, N), extent(dw ? x : nullptr, M, K), extent(dx ? w : nullptr, N, K),
                          extent(act != AR_ACT_NONE ? preact : nullptr, M, N)};
    const char* const in_names[] = {"dy", "x", "w", "preact"};
    const Extent outs[] = {extent(dx, M, K), extent(dw, N, K), extent(db, 1, N)};
    const char* const out_names[] = {"dx", "dw", "db"};
    for (int o = 0; o < 3; ++o) {
      for (int i = 0; i < 4; ++i) check_apart(out_names[o], outs[o], in_names[i], ins[i]);
      for (int i = 0; i < o; ++i) check_apart(out_names[o], outs[o], out_names[i], outs[i]);
    }
    const Backward p = plan_backward(M, N, K, dy, x, w, act, drop, dx, dw, db);
    const Extent ews = check_workspace(workspace, workspace_bytes, p.total());
    for (int i = 0; i < 4; ++i) check_apart("the workspace", ews, in_names[i], ins[i]);
    for (int o = 0; o < 3; ++o) check_apart("the workspace", ews, out_names[o], outs[o]);
    const ar_dtype type = dw ? x->dtype : dx ? w->dtype : act != AR_ACT_NONE ? preact->dtype : dy->dtype;
    const bool any = (dx && M > 0 && K > 0) || (dw && N > 0 && K > 0) || (db && N > 0);
    if (!any) return;
    check_device();
    char* const base = static_cast<char*>(workspace);
    void* const dz = base;
    float* const sums = reinterpret_cast<float*>(base + p.dz_bytes);
    void* const part = base + p.dz_bytes + p.sums_bytes;
    if (p.make_dz || (db && N > 0)) {
      ar::SlopeCall c{};
      c.dy = dy->data;
      c.lddy = dy->ld;
      c.z = act != AR_ACT_NONE ? preact->data : nullptr;
      c.ldz = act != AR_ACT_NONE ? preact->ld : 0;
      c.dz = p.make_dz ? dz : nullptr;
      c.lddz = p.lddz;
      c.sums = db ? sums : nullptr;
      c.M = M;
      c.N = N;
      c.act = int32_t(act);
      c.chunks = p.chunks;
      c.rows_per = p.rows_per;
      c.drop = drop_args(drop);
      launched(ar::launch_slope(c, elem_of(dy->dtype), elem_of(type), stream), "linear gradient kernel launch");
    }
    ar::SumsCall s{};
    if (db && N > 0) {
      s.sums = sums;
      s.db = db->data;
      s.N = s.ld = N;
      s.chunks = p.chunks;
      s.elem = elem_of(db->dtype);
      s.accumulate = accumulate != 0;
    }
    const void* const gz = p.make_dz ? dz : dy->data;
    const int64_t ldg = p.make_dz ? p.lddz : dy->ld;
    ar::Epilogue e{};
    e.drop = drop_args(nullptr);
    ar::GemmArgs gx{}, gw{};
    const bool run_x = dx && M > 0 && K > 0, run_w = dw && N > 0 && K > 0;
    if (run_x) {
      e.y = dx->data;
      e.ldy = dx->ld;
      e.M = int32_t(M);
      e.N = int32_t(K);
      e.y_f32 = dx->dtype == AR_FLOAT32;
      gx = gemm_args(p.px, N, type, {gz, ldg, true, M}, {w->data, w->ld, false, K}, e, part);
    }
    if (run_w) {
      e.y = dw->data;
      e.ldy = dw->ld;
      e.M = int32_t(N);
      e.N = int32_t(K);
      e.y_f32 = dw->dtype == AR_FLOAT32;
      if (accumulate) {
        e.res = dw->data;
        e.ldr = dw->ld;
      }
      gw = gemm_args(p.pw, M, type, {gz, ldg, false, N}, {x->data, x->ld, false, K}, e, static_cast<char*>(part) + p.part_x);
    }
    if (run_x && run_w && p.pair) {
      launched(ar::launch_gemm_pair(gx, gw, elem_of(type), p.px.aligned, p.px.shape, stream), "gradient kernel launch");
    } else {
      if (run_x) run_product(p.px, gx, elem_of(type), true, false, stream, "input gradient kernel launch");
      if (run_w) run_product(p.pw, gw, elem_of(type), false, false, stream, "weight gradient kernel launch");
    }
    launched(ar::launch_join(gx, gw, s, elem_of(type), stream), "join kernel launch");
  });
}

ar_status ar_dropout_forward(int64_t rows, int64_t cols, const ar_matrix* x, const ar_matrix* residual,
                             const ar_dropout* drop, const ar_matrix* y, hipStream_t stream) {
  return guarded([&] {
    check_length("rows", rows);
    check_length("cols", cols);
    check_matrix("x", x, rows, cols);
    check_matrix("y", y, rows, cols);
    if (residual) {
      check_matrix("residual", residual, rows, cols);
      if (residual->dtype != y->dtype) refuse(AR_ERR_UNSUPPORTED, "residual must have y's type");
    }
    if (!drop) refuse(AR_ERR_INVALID_ARG, "drop is NULL");
    ar::DropCall c{};
    c.drop = drop_args(drop);
    if (rows == 0 || cols == 0) return;
    const Extent ey = extent(y, rows, cols);
    if (!same_place(x, y, rows)) check_apart("y", ey, "x", extent(x, rows, cols));
    if (residual && !same_place(residual, y, rows)) check_apart("y", ey, "residual", extent(residual, rows, cols));
    check_device();
    c.x = x->data;
    c.ldx = x->ld;
    c.y = y->data;
    c.ldy = y->ld;
    if (residual) {
      c.res = residual->data;
      c.ldr = residual->ld;
    }
    c.rows = rows;
    c.cols = cols;
    launched(ar::launch_dropout(c, elem_of(x->dtype), elem_of(y->dtype), stream), "dropout kernel launch");
  });
}

ar_status ar_dropout_backward(int64_t rows, int64_t cols, const ar_matrix* dy, const ar_dropout* drop,
                              const ar_matrix* dx, hipStream_t stream) {
  return ar_dropout_forward(rows, cols, dy, nullptr, drop, dx, stream);
}

}  // extern "C"
