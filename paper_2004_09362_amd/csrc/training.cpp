// training.cpp -- the C ABI of layer norm, its gradient and the orthogonalised
// update (include/ar.h, "Layer operators"): argument checks, the choice of
// kernels, and launches.  The kernels are in norm.hip and orthogonal.hip; nothing
// here computes on the host.
#include <hip/hip_runtime_api.h>

#include <algorithm>
#include <cfloat>
#include <cmath>
#include <cstdint>
#include <string>
#include <utility>

#include "../../include/ar.h"
#include "layer_checks.hpp"
#include "training.hpp"

namespace {

// A vector of parameters or of their gradient, NULL where there is none.
void check_vector(const char* name, const ar_matrix* m, int64_t cols) {
  if (m) check_matrix(name, m, 1, cols);
}

void check_stats(const ar_matrix* stats, int64_t rows) {
  check_matrix("stats", stats, rows, 2);
  if (stats->dtype != AR_FLOAT32) refuse(AR_ERR_UNSUPPORTED, "stats must be float32");
}

void check_norm_grad(int64_t rows, int64_t cols, const ar_matrix* dy, const ar_matrix* x, const ar_matrix* stats,
                     const ar_matrix* weight, const ar_matrix* residual, const ar_matrix* dx, const ar_matrix* dw,
                     const ar_matrix* db) {
  check_length("rows", rows);
  check_length("cols", cols);
  check_matrix("dy", dy, rows, cols);
  check_matrix("x", x, rows, cols);
  check_stats(stats, rows);
  check_vector("weight", weight, cols);
  if (dx) {
    check_matrix("dx", dx, rows, cols);
    if (dx->dtype != x->dtype) refuse(AR_ERR_UNSUPPORTED, "dx must have x's type");
  }
  if (residual) {
    check_matrix("residual", residual, rows, cols);
    if (residual->dtype != x->dtype) refuse(AR_ERR_UNSUPPORTED, "residual must have x's type");
  }
  check_vector("dw", dw, cols);
  check_vector("db", db, cols);
}

int64_t norm_grad_bytes(int64_t rows, int64_t cols, const ar_matrix* dw, const ar_matrix* db) {
  if ((!dw && !db) || rows == 0 || cols == 0) return 0;
  return int64_t(ar::norm_grad_blocks(rows, cols)) * 2 * cols * 4;
}

// ---- the orthogonalised update ----

constexpr int32_t kMaxSteps = 64;
constexpr int64_t kMaxShort = 32768, kMaxLong = int64_t(1) << 21, kMaxBatch = 65535, kMaxElements = int64_t(1) << 34;
constexpr int64_t kCus = 256;

// How one of a step's products runs.
struct OrthoPlanPart {
  int64_t tile = 0, tiles = 0, steps = 0, share = 0, workgroups = 0;
  double micros = 0.0;
  int64_t parts() const { return share % steps == 0 ? 0 : workgroups * 2 * tile * tile * 4; }
};

// The fastest way by a model of what the kernels measured.  rows, cols: of the
// result in units of 64, of which tiles divide them; steps of a tile.  Measured, us
// a launch of many, tile: workgroups x steps of a symmetric product, and of X's:
//   64:  1 x 1 3.4, 1 x 32 7.6, 1 x 128 17.9, 136 x 16 7.0, 136 x 64 15.2, 528 x 32 30;
//        256 x 16 8.0, 416 x 39 21, 1024 x 16 28, 1536 x 8 33
//   128: 10 x 8 7.5, 36 x 16 10.3, 36 x 64 31, 136 x 32 19.6, 240 x 8 9.3, 528 x 64 87;
//        64 x 16 13.4, 256 x 16 17, 256 x 32 25, 384 x 8 18.5, 1024 x 64 122, 4096 x 64 519
//   256: 36 x 32 42, 136 x 64 76, 136 x 256 264; 64 x 32 54, 256 x 64 101 to 116,
//        1024 x 64 464, four tiles to a workgroup 413
// Parts: 36 tiles of 128 x 64 steps over 128 workgroups 19.7, over 256 19.5; 136 tiles of
// 256 x 256 steps over 256 workgroups 340 (264 whole).
OrthoPlanPart plan_part(int64_t rows, int64_t cols, int32_t kind, int32_t planes, int64_t batch, int64_t steps) {
  const bool symmetric = kind != ar::kOrthoApply;
  OrthoPlanPart best;
  for (const int64_t tile : {64, 128, 256}) {
    const int64_t unit = tile / 64;
    if (rows % unit != 0 || cols % unit != 0) continue;
    const int64_t tm = rows / unit, tn = cols / unit, tiles = symmetric ? tm * (tm + 1) / 2 : tm * tn, all = tiles * batch * steps;
    auto offer = [&](int64_t share) {
      OrthoPlanPart p;
      p.tile = tile;
      p.tiles = tiles;
      p.steps = steps;
      p.share = share;
      p.workgroups = ceil_div(all, share);
      const bool split = share % steps != 0;
      const double busy = double(std::min(p.workgroups, kCus)) / double(kCus);
      const double pieces = split ? double(share) / double(steps) + 1.0 : double(share / steps);
      if (tile == 64) {
        const double rounds = double(ceil_div(p.workgroups, kCus));
        p.micros = 1.5 + rounds * (3.0 + double(steps) * (0.11 + 0.10 * busy));
      } else if (tile == 128) {
        const double rounds = std::max(1.0, double(p.workgroups) / double(2 * kCus));
        if (p.workgroups <= kCus) p.micros = 3.0 + pieces * (symmetric ? 1.7 : 3.0 + 3.0 * busy) + double(share) * (0.43 + 0.06 * busy);
        else p.micros = 3.0 + rounds * (pieces * (symmetric ? 2.5 : 7.0) + double(share) * (symmetric ? 1.35 : 0.88));
      } else {
        const double rounds = double(ceil_div(p.workgroups, kCus));
        // parts of one tile read other parts of the operands at a time than their neighbours: the memory bounds them
        const double step = split ? 0.9 + 1.3 * busy : symmetric ? 0.75 + 0.4 * busy : 0.9 + 0.4 * busy;
        p.micros = rounds * (2.0 + pieces * (symmetric ? 14.0 : 18.0) + double(share) * step);
      }
      if (split) p.micros += 4.5 + double(p.workgroups + tiles * batch) * double(tile * tile) * 8.0 / 5e6;
      if (best.share == 0 || p.micros < best.micros) best = p;
    };
    offer(steps);
    if (tile == 64) continue;
    if (tile == 256 && tiles * batch > kCus) offer(steps * ceil_div(tiles * batch, kCus));
    if (ar::ortho_splits(kind, planes, int32_t(tile)) && tiles * batch <= kCus) {
      for (const int64_t w : {kCus, kCus / 2, kCus / 4})
        if (ceil_div(all, w) >= 4 && ceil_div(all, w) < steps) offer(ceil_div(all, w));
    }
  }
  return best;
}

struct OrthoPlan {
  ar::OrthoShape s{};
  int32_t planes = 1;
  OrthoPlanPart part[3];
  int64_t sums = 0, x = 0, a = 0, diag = 0, parts = 0;  // bytes of each
  int64_t total() const { return sums + 2 * x + 2 * a + diag + parts; }
};

// Whether products towards y may take operands of 11 bits: below 65 rows or columns
// their roundings have few others to even out with (one element was off by 4e-3 of
// itself), and 22 bits cost 15 us of 69.
bool may_round(int64_t M, int64_t N, ar_dtype y) { return y == AR_BFLOAT16 && std::min(M, N) > 64; }

OrthoPlan plan_ortho(int64_t batch, int64_t M, int64_t N, int32_t planes) {
  OrthoPlan best;
  double least = 0.0;
  for (const int64_t whole : {64, 128, 256}) {  // the sides' multiple
    OrthoPlan p;
    p.planes = planes;
    p.s.rows = M;
    p.s.cols = N;
    p.s.batch = int32_t(batch);
    p.s.turned = M > N;
    const int64_t pairs = p.planes == 2 ? 3 : 1;
    p.s.mp = round_up(std::min(M, N), whole);
    p.s.np = round_up(std::max(M, N), whole);
    const int64_t m = p.s.mp / 64, n = p.s.np / 64;
    p.part[ar::kOrthoGram] = plan_part(m, m, ar::kOrthoGram, planes, batch, pairs * n);
    p.part[ar::kOrthoSquare] = plan_part(m, m, ar::kOrthoSquare, planes, batch, pairs * m);
    p.part[ar::kOrthoApply] = plan_part(m, n, ar::kOrthoApply, planes, batch, pairs * m);
    const double micros = p.part[0].micros + p.part[1].micros + p.part[2].micros;
    if (least > 0.0 && micros >= least) continue;
    least = micros;
    // four groups of 8 to a thread and more, and 8 workgroups to a compute unit
    p.s.blocks = int32_t(std::max<int64_t>(1, std::min(8 * kCus / batch, ceil_div(M * ceil_div(N, 8), 1024))));
    p.sums = round_up(batch * p.s.blocks * 8, kWorkspaceAlign);
    p.x = batch * 2 * p.s.mp * p.s.np * 2;
    p.a = batch * p.planes * p.s.mp * p.s.mp * 2;
    p.diag = round_up(batch * p.s.mp * 4, kWorkspaceAlign);
    p.parts = 0;
    for (const OrthoPlanPart& q : p.part) p.parts = std::max(p.parts, q.parts());
    best = p;
  }
  return best;
}

// The workspace of a call, whose coefficients say which of the two it is.
int64_t ortho_bytes(int64_t batch, int64_t M, int64_t N, ar_dtype y) {
  const int64_t two = plan_ortho(batch, M, N, 2).total();
  return may_round(M, N, y) ? std::max(two, plan_ortho(batch, M, N, 1).total()) : two;
}

void check_ortho_sizes(int64_t batch, int64_t M, int64_t N, const ar_matrix* y) {
  check_length("batch", batch);
  check_length("M", M);
  check_length("N", N);
  if (!y) refuse(AR_ERR_INVALID_ARG, "y is NULL");
  if (!is_float(y->dtype)) refuse(AR_ERR_UNSUPPORTED, "y must be float32, float16 or bfloat16");
  if (batch == 0 || M == 0 || N == 0) return;
  if (batch > kMaxBatch) refuse(AR_ERR_UNSUPPORTED, "batch must be below 65536");
  if (std::min(M, N) > kMaxShort || std::max(M, N) > kMaxLong)
    refuse(AR_ERR_UNSUPPORTED, "the shorter side of a matrix must be at most 32768, the longer one 2^21");
  if (round_up(M, 256) * round_up(N, 256) > kMaxElements / batch)
    refuse(AR_ERR_UNSUPPORTED, "the matrices have more than 2^34 elements in whole tiles");
}

// Whether matrices of M > 1 rows share an element: two that are d apart do where d
// strides are within N elements of fewer than M rows.
bool matrices_overlap(int64_t ld, int64_t stride, int64_t batch, int64_t M, int64_t N) {
  if (stride >= N && (batch - 1) * stride + N <= ld) return false;  // side by side
  for (int64_t d = 1; d < batch; ++d) {
    const int64_t row = d * stride / ld, past = d * stride % ld;
    if (row >= M) return false;
    if (past < N || (ld - past < N && row + 1 < M)) return true;
  }
  return false;
}

// `batch` matrices, `stride` elements from one to the next.
void check_stack(const char* name, const ar_matrix* m, int64_t stride, int64_t batch, int64_t M, int64_t N, bool written) {
  check_matrix(name, m, batch == 0 ? 0 : M, N);
  if (batch <= 1 || M == 0 || N == 0) return;
  const int64_t covers = (M > 1 ? (M - 1) * m->ld : 0) + N;
  if (stride < 0 || stride > (int64_t(1) << 44))
    refuse(AR_ERR_INVALID_ARG, std::string(name) + "'s stride must be in [0, 2^44]");
  if (written && stride < covers && (M == 1 || matrices_overlap(m->ld, stride, batch, M, N)))
    refuse(AR_ERR_INVALID_ARG, std::string(name) + "'s matrices overlap");
}
Extent stack_extent(const ar_matrix* m, int64_t stride, int64_t batch, int64_t M, int64_t N) {
  if (!m || batch == 0) return Extent();
  Extent e = extent(m, M, N);
  if (batch == 1 || e.empty()) return e;
  if (M > 1 && stride == M * m->ld) {  // rows of one pitch throughout
    e.rows = batch * M;
    return e;
  }
  if (stride >= N && (M == 1 || stride * batch == m->ld)) {  // the same, rows of the matrices in turn
    e.rows = batch * M;
    e.pitch = stride * size_of(m->dtype);
    return e;
  }
  const int64_t bytes = int64_t(e.end() - e.at) + (batch - 1) * stride * size_of(m->dtype);
  e.row = e.pitch = bytes;
  e.rows = 1;
  return e;
}

// Whether the coefficients of a step keep singular values that are at most `most`
// within the range that the halves hold; `most` becomes the bound after the step:
// the polynomial's, and what the roundings of X, A and Q to `rounding` of their size
// add where they all fall the same way, so that steps which magnify it are seen.
bool within_range(const double* step, double rounding, double& most) {
  // as the kernels take them
  const double a = float(step[0]), b = float(step[1]), c = float(step[2]);
  const double end = most * most;
  double value = 0.0, q = 0.0, slope = 0.0;
  auto look = [&](double s) {  // s: a square
    if (!(s >= 0.0 && s <= end)) return;
    value = std::max(value, std::sqrt(s) * std::fabs(a + s * (b + s * c)));
    q = std::max(q, std::fabs(s * (b + s * c)));
    slope = std::max(slope, std::fabs(s * (b + 2.0 * s * c)));
  };
  look(end);
  if (c != 0.0) {
    look(-b / (2.0 * c));
    look(-b / (4.0 * c));
  }
  // The ends of a + 3 b s + 5 c s^2, of which neither is a difference of numbers
  // of one size: for c next to 0 the second one is still -a / (3 b).
  const double root = 9.0 * b * b - 20.0 * a * c;
  if (root >= 0.0) {
    const double r = -0.5 * (3.0 * b + std::copysign(std::sqrt(root), b));
    if (c != 0.0) look(r / (5.0 * c));
    if (r != 0.0) look(a / r);
  }
  // X's rounding enters A twice, A's once, each with b s + 2 c s^2; Q's, and X's in
  // the product with Q, with b s + c s^2; the halves end at 2^-39 of an element
  most = value + rounding * (value + (3.0 * slope + 2.0 * q) * most) + 0x1p-22;
  return value <= 2.5 && q <= 15.0;
}
bool all_within_range(const double* coefficients, int32_t steps, double rounding) {
  double most = 1.0;
  for (int32_t k = 0; k < steps; ++k)
    if (!within_range(coefficients + 3 * k, rounding, most)) return false;
  return true;
}

}  // namespace

extern "C" {

ar_status ar_layer_norm_forward(int64_t rows, int64_t cols, const ar_matrix* x, const ar_matrix* weight,
                                const ar_matrix* bias, double eps, const ar_matrix* y, const ar_matrix* stats,
                                hipStream_t stream) {
  return guarded([&] {
    check_length("rows", rows);
    check_length("cols", cols);
    check_matrix("x", x, rows, cols);
    check_vector("weight", weight, cols);
    check_vector("bias", bias, cols);
    if (!(eps >= 0.0 && eps <= double(FLT_MAX)) || (eps > 0.0 && float(eps) == 0.0f))
      refuse(AR_ERR_INVALID_ARG, "eps must be finite in 32 bits and at least 0, and 0 there only if it is 0");
    check_matrix("y", y, rows, cols);
    if (stats) check_stats(stats, rows);
    if (rows == 0 || cols == 0) {
      if (stats && rows > 0) refuse(AR_ERR_INVALID_ARG, "rows without columns have no statistics");
      return;
    }
    const Extent ex = extent(x, rows, cols), ey = extent(y, rows, cols), es = extent(stats, rows, 2);
    const Extent ew = extent(weight, 1, cols), eb = extent(bias, 1, cols);
    if (!same_place(x, y, rows)) check_apart("y", ey, "x", ex);
    check_apart("y", ey, "weight", ew);
    check_apart("y", ey, "bias", eb);
    check_apart("y", ey, "stats", es);
    check_apart("stats", es, "x", ex);
    check_apart("stats", es, "weight", ew);
    check_apart("stats", es, "bias", eb);
    check_device();
    ar::NormCall c{};
    c.x = x->data;
    c.ldx = x->ld;
    c.y = y->data;
    c.ldy = y->ld;
    if (weight) {
      c.w = weight->data;
      c.we = elem_of(weight->dtype);
    }
    if (bias) {
      c.b = bias->data;
      c.be = elem_of(bias->dtype);
    }
    if (stats) {
      c.stats = static_cast<float*>(stats->data);
      c.lds = stats->ld;
    }
    c.rows = rows;
    c.cols = cols;
    c.eps = float(eps);
    launched(ar::launch_norm(c, elem_of(x->dtype), elem_of(y->dtype), stream), "layer norm kernel launch");
  });
}

ar_status ar_layer_norm_backward_workspace(int64_t rows, int64_t cols, const ar_matrix* dy, const ar_matrix* x,
                                           const ar_matrix* stats, const ar_matrix* weight, const ar_matrix* residual,
                                           const ar_matrix* dx, const ar_matrix* dw, const ar_matrix* db,
                                           int64_t* bytes) {
  return guarded([&] {
    if (!bytes) refuse(AR_ERR_INVALID_ARG, "bytes is NULL");
    *bytes = 0;
    check_norm_grad(rows, cols, dy, x, stats, weight, residual, dx, dw, db);
    *bytes = norm_grad_bytes(rows, cols, dw, db);
  });
}

ar_status ar_layer_norm_backward(int64_t rows, int64_t cols, const ar_matrix* dy, const ar_matrix* x,
                                 const ar_matrix* stats, const ar_matrix* weight, const ar_matrix* residual,
                                 const ar_matrix* dx, const ar_matrix* dw, const ar_matrix* db, int32_t accumulate,
                                 void* workspace, int64_t workspace_bytes, hipStream_t stream) {
  return guarded([&] {
    check_norm_grad(rows, cols, dy, x, stats, weight, residual, dx, dw, db);
    const Extent ins[] = {extent(dy, rows, cols), extent(x, rows, cols), extent(stats, rows, 2),
                          extent(weight, 1, cols), extent(dx ? residual : nullptr, rows, cols)};
    const char* const in_names[] = {"dy", "x", "stats", "weight", "residual"};
    const Extent outs[] = {extent(dx, rows, cols), extent(dw, 1, cols), extent(db, 1, cols)};
    const char* const out_names[] = {"dx", "dw", "db"};
    for (int o = 0; o < 3; ++o) {
      for (int i = 0; i < 5; ++i) {
        // a row is in registers before any of it is written
        if (o == 0 && dx && ((i == 0 && same_place(dy, dx, rows)) || (i == 4 && residual && same_place(residual, dx, rows)))) continue;
        check_apart(out_names[o], outs[o], in_names[i], ins[i]);
      }
      for (int i = 0; i < o; ++i) check_apart(out_names[o], outs[o], out_names[i], outs[i]);
    }
    const int64_t need = norm_grad_bytes(rows, cols, dw, db);
    const Extent ews = check_workspace(workspace, workspace_bytes, need);
    for (int i = 0; i < 5; ++i) check_apart("the workspace", ews, in_names[i], ins[i]);
    for (int o = 0; o < 3; ++o) check_apart("the workspace", ews, out_names[o], outs[o]);
    if (cols == 0 || (rows == 0 && !dw && !db) || (!dx && !dw && !db)) return;
    check_device();
    ar::NormJoinCall j{};
    j.cols = cols;
    j.accumulate = accumulate != 0;
    if (dw) {
      j.dw = dw->data;
      j.dwe = elem_of(dw->dtype);
    }
    if (db) {
      j.db = db->data;
      j.dbe = elem_of(db->dtype);
    }
    if (rows > 0) {
      ar::NormGradCall c{};
      c.dy = dy->data;
      c.lddy = dy->ld;
      c.x = x->data;
      c.ldx = x->ld;
      c.stats = static_cast<const float*>(stats->data);
      c.lds = stats->ld;
      if (weight) {
        c.w = weight->data;
        c.we = elem_of(weight->dtype);
      }
      if (dx) {
        c.dx = dx->data;
        c.lddx = dx->ld;
        if (residual) {
          c.res = residual->data;
          c.ldr = residual->ld;
        }
      }
      c.rows = rows;
      c.cols = cols;
      c.blocks = j.blocks = ar::norm_grad_blocks(rows, cols);
      j.parts = c.parts = need > 0 ? static_cast<float*>(workspace) : nullptr;
      launched(ar::launch_norm_grad(c, elem_of(x->dtype), elem_of(dy->dtype), stream), "layer norm gradient kernel launch");
    }
    if (dw || db) launched(ar::launch_norm_join(j, stream), "join kernel launch");
  });
}

ar_status ar_orthogonalize_workspace(int64_t batch, int64_t M, int64_t N, const ar_matrix* y, int64_t* bytes) {
  return guarded([&] {
    if (!bytes) refuse(AR_ERR_INVALID_ARG, "bytes is NULL");
    *bytes = 0;
    check_ortho_sizes(batch, M, N, y);
    if (batch > 0 && M > 0 && N > 0) *bytes = ortho_bytes(batch, M, N, y->dtype);
  });
}

ar_status ar_orthogonalize(int64_t batch, int64_t M, int64_t N, const ar_matrix* x, int64_t x_stride, int32_t steps,
                           const double* coefficients, double eps, double scale, const ar_matrix* residual,
                           int64_t residual_stride, const ar_matrix* y, int64_t y_stride, void* workspace,
                           int64_t workspace_bytes, hipStream_t stream) {
  return guarded([&] {
    check_ortho_sizes(batch, M, N, y);
    check_stack("x", x, x_stride, batch, M, N, false);
    check_stack("y", y, y_stride, batch, M, N, true);
    if (residual) {
      check_stack("residual", residual, residual_stride, batch, M, N, false);
      if (residual->dtype != y->dtype) refuse(AR_ERR_UNSUPPORTED, "residual must have y's type");
    }
    if (steps < 1 || steps > kMaxSteps) refuse(AR_ERR_INVALID_ARG, "steps must be in [1, 64]");
    if (!coefficients) refuse(AR_ERR_INVALID_ARG, "coefficients is NULL");
    for (int32_t i = 0; i < 3 * steps; ++i)
      if (!std::isfinite(float(coefficients[i]))) refuse(AR_ERR_INVALID_ARG, "the coefficients must be finite in 32 bits");
    if (!all_within_range(coefficients, steps, 0x1p-21))
      refuse(AR_ERR_INVALID_ARG, "the coefficients take a singular value past 2.5, or |b s + c s^2| of its square s past 15");
    if (!(eps >= 0.0) || !std::isfinite(eps)) refuse(AR_ERR_INVALID_ARG, "eps must be finite and at least 0");
    if (!(std::fabs(scale) <= double(FLT_MAX))) refuse(AR_ERR_INVALID_ARG, "scale must be finite in 32 bits");
    if (batch == 0 || M == 0 || N == 0) return;
    const Extent ex = stack_extent(x, x_stride, batch, M, N), ey = stack_extent(y, y_stride, batch, M, N);
    const Extent er = stack_extent(residual, residual_stride, batch, M, N);
    auto same = [&](const ar_matrix* m, int64_t stride) { return same_place(m, y, M) && (batch == 1 || stride == y_stride); };
    if (!same(x, x_stride)) check_apart("y", ey, "x", ex);
    if (residual && !same(residual, residual_stride)) check_apart("y", ey, "residual", er);
    // Steps that magnify 11 bits' rounding out of the range take 22 (eight published
    // steps that hold 1 at the edge gave infinities from equal entries).
    const OrthoPlan p = plan_ortho(batch, M, N, may_round(M, N, y->dtype) && all_within_range(coefficients, steps, 0x1p-11) ? 1 : 2);
    const Extent ews = check_workspace(workspace, workspace_bytes, ortho_bytes(batch, M, N, y->dtype));
    check_apart("the workspace", ews, "x", ex);
    check_apart("the workspace", ews, "y", ey);
    check_apart("the workspace", ews, "residual", er);
    check_device();
    char* at = static_cast<char*>(workspace);
    auto take = [&](int64_t bytes) {
      char* const here = at;
      at += bytes;
      return here;
    };
    double* const sums = reinterpret_cast<double*>(take(p.sums));
    void* X[2] = {take(p.x), nullptr};
    X[1] = take(p.x);
    void* const A = take(p.a);
    void* const Q = take(p.a);
    float* const diag = reinterpret_cast<float*>(take(p.diag));
    float* const parts = reinterpret_cast<float*>(take(p.parts));
    const ar::OrthoOuter ox{x->data, x->ld, x_stride, elem_of(x->dtype)}, oy{y->data, y->ld, y_stride, elem_of(y->dtype)};
    ar::OrthoOuter ores{};
    if (residual) ores = {residual->data, residual->ld, residual_stride, elem_of(residual->dtype)};
    launched(ar::launch_ortho_norm(p.s, ox, sums, stream), "norm kernel launch");
    launched(ar::launch_ortho_load(p.s, ox, sums, eps, X[0], stream), "load kernel launch");
    const int64_t plane_x = p.s.mp * p.s.np, plane_a = p.s.mp * p.s.mp;
    for (int32_t k = 0; k < steps; ++k) {
      for (const int32_t kind : {ar::kOrthoGram, ar::kOrthoSquare, ar::kOrthoApply}) {
        const OrthoPlanPart& q = p.part[kind];
        const bool gram = kind == ar::kOrthoGram, apply = kind == ar::kOrthoApply;
        ar::OrthoProduct g{};
        g.left = gram ? X[0] : apply ? Q : A;
        g.right = gram || apply ? X[0] : A;
        g.old = apply ? X[0] : A;
        g.out = gram ? A : apply ? X[1] : Q;
        g.diag = diag;
        g.parts = parts;
        g.ld_left = gram ? p.s.np : p.s.mp;
        g.ld_right = gram || apply ? p.s.np : p.s.mp;
        g.ld_out = apply ? p.s.np : p.s.mp;
        g.plane_left = gram ? plane_x : plane_a;
        g.plane_right = gram || apply ? plane_x : plane_a;
        g.plane_out = apply ? plane_x : plane_a;
        g.batch_left = gram ? 2 * plane_x : p.planes * plane_a;
        g.batch_right = gram || apply ? 2 * plane_x : p.planes * plane_a;
        g.batch_out = apply ? 2 * plane_x : p.planes * plane_a;
        g.M = int32_t(p.s.mp);
        g.N = int32_t(apply ? p.s.np : p.s.mp);
        g.K = int32_t(gram ? p.s.np : p.s.mp);
        g.tiles_m = int32_t(p.s.mp / q.tile);
        g.tiles_n = int32_t(g.N / q.tile);
        g.tiles = int32_t(q.tiles);
        g.batch = int32_t(batch);
        g.steps = int32_t(q.steps);
        g.share = int32_t(q.share);
        g.workgroups = int32_t(q.workgroups);
        g.a = float(coefficients[3 * k]);
        g.b = float(coefficients[3 * k + 1]);
        g.c = float(coefficients[3 * k + 2]);
        if (apply && k == steps - 1) {
          g.y = oy;
          g.residual = ores;
          g.rows = M;
          g.cols = N;
          g.turned = p.s.turned;
          g.scale = float(scale);
        }
        launched(ar::launch_ortho_product(g, kind, p.planes, int32_t(q.tile), stream), "Newton-Schulz product launch");
      }
      std::swap(X[0], X[1]);
    }
  });
}

}  // extern "C"
