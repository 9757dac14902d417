// layer_checks.hpp -- what the entry points of the layer operators share: how a
// refused call is reported, the checks of matrices, and which of them overlap.
#pragma once

#include <hip/hip_runtime_api.h>

#include <cstdint>
#include <exception>
#include <string>

#include "../../include/ar.h"
#include "ar_internal.hpp"
#include "layers.hpp"

namespace {

constexpr int64_t kMaxLength = int64_t(1) << 30;
constexpr int64_t kMaxLd = int64_t(1) << 40;
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

}  // namespace
