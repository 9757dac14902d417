// training.cpp -- the C ABI of layer norm and its gradient (include/ar.h,
// "Layer operators"): argument checks, the choice of kernels, and launches.  The
// kernels are in norm.hip; nothing here computes on the host.
#include <hip/hip_runtime_api.h>

#include <algorithm>
#include <cmath>
#include <cstdint>
#include <string>

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
    if (!(eps >= 0.0) || !std::isfinite(eps)) refuse(AR_ERR_INVALID_ARG, "eps must be finite and at least 0");
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

}  // extern "C"
