"""Where the tiled products read, without a GPU.

The address arithmetic of csrc/gemm.hpp is compiled for the host and run for
every thread, slot and tile of a workgroup: whatever a tile's loads take lies
between the first element of the operand's matrix and its last one."""
import os
import subprocess

import pytest

from paper_2004_09362_amd import build as b

PROGRAM = r"""
#include <cstdio>
#include <initializer_list>

#include "gemm.hpp"

using namespace ar;

long checked = 0;

template <typename T, bool KMAJOR, bool FIRST, int R>
struct Replay {
  using Op = Operand<T, KMAJOR, FIRST, R, 256>;
  const char* first;
  int64_t bytes;  // of the matrix: to the end of its last row
  int64_t rows, inner, ld;

  bool inside(const void* p, int64_t n, const char* what, int64_t row0, int64_t k0, int t) {
    const int64_t from = static_cast<const char*>(p) - first;
    ++checked;
    if (from >= 0 && from + n <= bytes) return true;
    std::printf("%s of %d-byte elements, kmajor %d, tile of %d rows: rows %ld, inner length %ld, ld %ld, from row %ld and inner index %ld, "
                "tile %d: bytes %ld to %ld of %ld\n", what, int(sizeof(T)), int(KMAJOR), R, long(rows), long(inner), long(ld), long(row0),
                long(k0), t, long(from), long(from + n), long(bytes));
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
            const T* chunk[Op::kSlots];
            int64_t there[Op::kSlots];
            op.chunks(chunk, there, t, klen - int64_t(t) * Op::kInner, tid);
            for (int i = 0; i < Op::kSlots; ++i) {
              const char* const plain = op.at(t) + op.voff[i];
              if (open && t + 1 < tiles && !inside(plain, 16, "unchecked chunk", row0, k0, t)) return false;
              if (async && t < whole && !inside(plain, 16, "asynchronous chunk", row0, k0, t)) return false;
              const int64_t have = there[i];
              const T* const p = chunk[i];
              if (op.wide) {
                if (!inside(end_at(p, have), 16, "checked chunk", row0, k0, t)) return false;
              } else if (have > 0) {
                const int64_t n = have < Op::kElems ? have : Op::kElems;
                if (!inside(p, n * int64_t(sizeof(T)), "short chunk", row0, k0, t)) return false;
              }
            }
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
