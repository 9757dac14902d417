"""What the compiler made of the Newton-Schulz products (csrc/orthogonal.hip), which run the loop of csrc/gemm.hpp and its
assembly, without a GPU: the wait states that tests/test_gemm_code.py looks for, and loops that keep everything in registers."""
import os
import subprocess

import pytest

from paper_2004_09362_amd import build as b
from test_gemm_code import faults, functions


@pytest.fixture(scope="module")
def listing(tmp_path_factory):
    if not os.path.exists(b.HIPCC):
        pytest.skip("hipcc is not installed")
    to = str(tmp_path_factory.mktemp("asm") / "orthogonal.s")
    flags = [f for f in b.FLAGS if f != "--offload-compress"]
    subprocess.run([b.HIPCC] + flags + ["-S", "--cuda-device-only", os.path.join(b.CSRC, "orthogonal.hip"), "-o", to], check=True,
                   capture_output=True)
    with open(to) as fh:
        return fh.read()


def test_wait_states_and_registers(listing):
    products = 0
    for name, body in functions(listing):
        assert not list(faults(name, body)), name
        if "ortho_product_kernel" not in name:
            continue
        products += 1
        loads = [i for i, (op, _) in enumerate(body) if op.startswith("global_load_lds")]
        loop = body[loads[-8 if "Li4ELi4E" in name else -16]:loads[-1]]
        assert sum(op.startswith("v_mfma") for op, _ in loop) > 10, name
        assert not any(op.startswith("scratch_") for op, _ in body), name
        assert "Li8ELi8E" not in name or not any(op.startswith("v_accvgpr") for op, _ in loop), name
    assert products == 20  # three products and four last ones, with one and with three pairs of planes, on two tiles
