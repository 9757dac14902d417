"""Where the tiled products read, without a GPU.

The operands' loads of csrc/gemm.hpp are compiled for the host, with reads that
say where they are, and run for every thread and tile of a workgroup: whatever
they take lies between the first element of the operand's matrix and its last
one."""
import os
import subprocess

import pytest

from paper_2004_09362_amd import build as b

PROGRAM = r"""
#include <cstdio>
#include <initializer_list>

#include <hip/hip_runtime.h>

// The loads as the host sees them: they say where they read.
namespace ar {
typedef int32_t i32x4v __attribute__((ext_vector_type(4)));
void reads(const void* p, int64_t bytes);
template <typename T> __host__ i32x4v load_whole(const void* p) {
  reads(p, 16);
  return i32x4v{};
}
template <typename T> __host__ i32x4v load_end(const T* p, int64_t have);
template <typename T> __host__ i32x4v end_chunk(const i32x4v& raw, int64_t) { return raw; }
template <typename T> __host__ i32x4v short_chunk(const T* p, int64_t have) {
  const int64_t per = 16 / sizeof(T);
  if (have > 0) reads(p, (have < per ? have : per) * int64_t(sizeof(T)));
  return i32x4v{};
}
}  // namespace ar

#include "gemm.hpp"

namespace ar {
template <typename T> __host__ i32x4v load_end(const T* p, int64_t have) {
  reads(end_at(p, have), 16);
  return i32x4v{};
}
}  // namespace ar

using namespace ar;

// The matrix at hand, and what is read of it.
const char* first;
int64_t bytes;  // to the end of its last row
long checked = 0;
bool outside = false;
int64_t outside_from, outside_to;

void ar::reads(const void* p, int64_t n) {
  const int64_t from = static_cast<const char*>(p) - first;
  ++checked;
  if (from >= 0 && from + n <= bytes) return;
  outside = true;
  outside_from = from;
  outside_to = from + n;
}

template <typename T, bool KMAJOR, bool FIRST, int R>
struct Replay {
  using Op = Operand<T, KMAJOR, FIRST, R, 256>;
  int64_t rows, inner, ld;

  bool inside(const char* what, int64_t row0, int64_t k0, int t) {
    if (!outside) return true;
    std::printf("%s of %d-byte elements, kmajor %d, tile of %d rows: rows %ld, inner length %ld, ld %ld, from row %ld and inner index %ld, "
                "tile %d: bytes %ld to %ld of %ld\n", what, int(sizeof(T)), int(KMAJOR), R, long(rows), long(inner), long(ld), long(row0),
                long(k0), t, long(outside_from), long(outside_to), long(bytes));
    outside = false;
    return false;
  }

  // parts of the inner length of `part` tiles each
  bool run(int64_t rows_, int64_t inner_, int64_t pad, int64_t part) {
    rows = rows_;
    inner = inner_;
    const int64_t height = KMAJOR ? rows : inner, width = KMAJOR ? inner : rows;
    ld = width + pad;
    bytes = ((height - 1) * ld + width) * int64_t(sizeof(T));
    first = reinterpret_cast<const char*>(uintptr_t(1) << 40);
    // what the host asks of operands that are loaded asynchronously
    const bool open = tiles_open(KMAJOR, rows, inner, ld, sizeof(T));
    const bool async = ld % Op::kElems == 0 && (KMAJOR || rows % Op::kElems == 0);
    for (int64_t row0 = 0; row0 < rows; row0 += R) {
      for (int64_t k0 = 0; k0 < inner; k0 += part * Op::kInner) {
        const int64_t klen = inner - k0 < part * Op::kInner ? inner - k0 : part * Op::kInner;
        const int tiles = int((klen + Op::kInner - 1) / Op::kInner), whole = int(klen / Op::kInner);
        for (int tid = 0; tid < 256; ++tid) {
          Op op;
          op.init(reinterpret_cast<const T*>(first), ld, row0, k0, rows, inner, tid);
          for (int t = 0; t < tiles; ++t) {
            i32x4v reg[Op::kSlots];
            if (open && t + 1 < tiles) op.load(reg, t);
            if (!inside("unchecked tile", row0, k0, t)) return false;
            op.load_checked(reg, t, klen - int64_t(t) * Op::kInner, tid);
            if (!inside("checked tile", row0, k0, t)) return false;
            if (async && t < whole)
              for (int i = 0; i < Op::kSlots; ++i) reads(op.at(t) + op.voff[i], 16);
            if (!inside("asynchronous tile", row0, k0, t)) return false;
          }
        }
      }
    }
    return true;
  }

  bool all() {
    bool ok = true;
    for (int64_t rows_ : {1, 2, 3, 4, 5, 7, 8, 9, 12, 16, 127, 128, 130, 264})
      for (int64_t inner_ : {1, 2, 7, 8, 31, 32, 33, 34, 35, 63, 64, 65, 66, 67, 68, 69, 70, 71, 96, 97, 128, 129, 130, 200, 257, 321, 385, 449})
        for (int64_t pad : {0, 1, 8})
          for (int64_t part : {2, 5, 100}) ok = run(rows_, inner_, pad, part) && ok;
    return ok;
  }
};

template <typename T>
bool type() {
  bool ok = Replay<T, true, false, 128>().all();
  ok = Replay<T, true, true, 128>().all() && ok;
  ok = Replay<T, false, false, 128>().all() && ok;
  ok = Replay<T, false, true, 128>().all() && ok;
  ok = Replay<T, true, false, 256>().all() && ok;
  ok = Replay<T, false, false, 256>().all() && ok;
  ok = Replay<T, true, false, 32>().all() && ok;
  ok = Replay<T, true, false, 64>().all() && ok;
  return ok;
}

int main() {
  const bool halves = type<f16>(), floats = type<float>();
  std::printf("%ld reads\n", checked);
  return halves && floats ? 0 : 1;
}
"""


def test_tiles_read_within_their_matrix(tmp_path):
    if not os.path.exists(b.HIPCC):
        pytest.skip("hipcc is not installed")
    source, program = tmp_path / "reads.hip", str(tmp_path / "reads")
    source.write_text(PROGRAM)
    subprocess.run([b.HIPCC, "-O2", "-std=c++17", "--cuda-host-only", "-I" + b.CSRC, str(source), "-o", program], check=True,
                   capture_output=True, text=True)
    got = subprocess.run([program], capture_output=True, text=True, timeout=600)
    assert got.returncode == 0, "%d lines\n%s" % (got.stdout.count("\n"), got.stdout[:4000])
    assert int(got.stdout.split()[0]) > 10 ** 7
