"""Which tiles the orthogonalised update's products take, without a GPU: the planner of csrc/training.cpp, compiled for the host,
is asked about the sizes that tests/test_gpu_orthogonal_tiles.py runs, so that a change of its model cannot leave a kernel
without a test."""
import os
import shutil
import subprocess

import pytest

from paper_2004_09362_amd import ar
from paper_2004_09362_amd import build as b

PROGRAM = r"""
#include "training.cpp"
#include <cstdio>
int main() {
  long batch, M, N;
  int y;
  while (scanf("%ld %ld %ld %d", &batch, &M, &N, &y) == 4) {
    const OrthoPlan p = plan_ortho(batch, M, N, may_round(M, N, ar_dtype(y)) ? 1 : 2);
    printf("%d", p.planes);
    for (const OrthoPlanPart& q : p.part)
      printf(" %ld %s", long(q.tile), q.share % q.steps != 0 ? "split" : q.share > q.steps ? "several" : "whole");
    printf("\n");
  }
}
"""

# (batch, M, N): the ways of the three products of a step towards float32, and towards bfloat16.  whole: a tile to a
# workgroup; several: whole tiles, one after the other; split: tiles whose inner length several workgroups share.
TILES = {
    (1, 4096, 4096): ("256 whole, 256 whole, 256 whole", "256 whole, 256 whole, 256 whole"),
    (2, 4096, 4096): ("256 several, 256 several, 256 several", "256 several, 256 several, 256 several"),
    (1, 4096, 16384): ("256 whole, 256 whole, 256 several", "256 whole, 256 whole, 256 several"),
    (1, 2048, 8192): ("128 split, 128 split, 256 whole", "128 split, 128 whole, 256 whole"),
    (1, 16384, 2048): ("128 split, 128 split, 256 several", "128 split, 128 whole, 256 several"),
    (1, 2826, 16384): ("256 split, 256 whole, 256 several", "256 split, 256 whole, 256 several"),
    (1, 16384, 2900): ("256 split, 256 whole, 256 several", "256 split, 256 whole, 256 several"),
    (1, 2900, 8192): ("256 split, 256 whole, 256 several", "256 whole, 256 whole, 128 whole"),
    (3, 3300, 4096): ("256 several, 256 several, 256 several", "256 several, 256 several, 256 several"),
    (1, 8192, 128): ("128 split, 64 whole, 64 whole", "128 split, 64 whole, 64 whole"),
    (1, 132, 65536): ("128 split, 64 whole, 256 whole", "128 split, 64 whole, 128 whole"),
    (100, 128, 128): ("128 whole, 128 whole, 128 whole", "128 whole, 128 whole, 128 whole"),
    (24, 512, 512): ("128 whole, 128 whole, 128 whole", "128 whole, 128 whole, 128 whole"),
    (1, 1024, 1024): ("64 whole, 64 whole, 64 whole", "64 whole, 64 whole, 64 whole"),
}


@pytest.fixture(scope="module")
def planner(tmp_path_factory):
    rocm = os.environ.get("ROCM_PATH", "/opt/rocm")
    if shutil.which("g++") is None or not os.path.exists(os.path.join(rocm, "include/hip/hip_runtime_api.h")):
        pytest.skip("no host compiler or no HIP headers")
    at = tmp_path_factory.mktemp("plan")
    (at / "plan.cpp").write_text(PROGRAM)
    # the kernels' launchers are named by the calls, which the program does not make
    subprocess.run(["g++", "-O1", "-std=c++17", "-D__HIP_PLATFORM_AMD__", "-isystem", os.path.join(rocm, "include"), "-I" + b.CSRC,
                    "-I" + os.path.join(b.ROOT, "include"), str(at / "plan.cpp"), "-o", str(at / "plan"),
                    "-Wl,--unresolved-symbols=ignore-all"], check=True, capture_output=True, timeout=300)

    def ask(cases):
        text = "\n".join("%d %d %d %d" % c for c in cases)
        out = subprocess.run([str(at / "plan")], input=text, check=True, capture_output=True, text=True, timeout=300).stdout
        got = []
        for line in out.splitlines():
            f = line.split()
            got.append((int(f[0]), tuple("%s %s" % (f[i], f[i + 1]) for i in (1, 3, 5))))
        assert len(got) == len(cases)
        return got

    return ask


def asked(cases=None):
    return [(*size, dtype) for size in (TILES if cases is None else cases) for dtype in (ar.AR_FLOAT32, ar.AR_BFLOAT16)]


def test_the_tested_sizes_take_these_tiles(planner):
    got = planner(asked())
    for (batch, M, N, dtype), (planes, ways) in zip(asked(), got):
        assert planes == (2 if dtype == ar.AR_FLOAT32 else 1)
        assert ", ".join(ways) == TILES[batch, M, N][dtype == ar.AR_BFLOAT16], (batch, M, N, dtype)


def sweep():
    """Sizes over the whole range, a fine grid of them and many stacks."""
    sides = sorted({int(round(1.13 ** i)) for i in range(0, 86)} | {64 * i for i in range(1, 130)})
    long_sides = sorted({int(round(1.3 ** i)) for i in range(0, 56)})
    out = [(batch, m, n) for batch in (1, 2, 3, 5, 24, 40, 100) for m in sides for n in long_sides
           if m <= n and batch * m * n < 1 << 33]
    return out


def test_every_way_that_is_taken_is_tested(planner):
    """Of all (product, planes, tile, way) that any size of the sweep takes, each is among those of the tested sizes."""
    def ways(cases):
        return {(product, planes, way) for planes, three in planner(cases) for product, way in enumerate(three)}

    taken, tested = ways(asked(sweep())), ways(asked())
    assert taken <= tested, sorted(taken - tested)
