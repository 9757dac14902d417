"""What the compiler made of the products' assembly, without a GPU.

The loads to LDS and the matrix instructions with pinned sums (csrc/gemm.hpp)
are written as assembly, for which the compiler inserts no wait states.  Here
the compiled instructions are read: between a vector instruction that writes a
scalar register and a load to LDS that takes its address there lie five; between
one that writes an operand and a pinned matrix instruction two; and none but a
matrix instruction touches sums of the last 18 instructions' pinned ones.  The
loops keep everything in registers."""
import concurrent.futures
import os
import re
import subprocess

import pytest

from paper_2004_09362_amd import build as b

UNITS = ["gemm_bf16.hip", "gemm_f16.hip", "gemm_f32.hip", "gemm_few.hip"]


@pytest.fixture(scope="module")
def listings(tmp_path_factory):
    if not os.path.exists(b.HIPCC):
        pytest.skip("hipcc is not installed")
    out = tmp_path_factory.mktemp("asm")

    def compile_(unit):
        to = str(out / (unit + ".s"))
        flags = [f for f in b.FLAGS if f != "--offload-compress"]
        subprocess.run([b.HIPCC] + flags + ["-S", "--cuda-device-only", os.path.join(b.CSRC, unit), "-o", to], check=True,
                       capture_output=True)
        with open(to) as fh:
            return fh.read()

    with concurrent.futures.ThreadPoolExecutor(4) as ex:
        return dict(zip(UNITS, ex.map(compile_, UNITS)))


def registers(text):
    m = re.fullmatch(r"([sva])\[(\d+):(\d+)\]", text)
    if m:
        return {m.group(1) + str(i) for i in range(int(m.group(2)), int(m.group(3)) + 1)}
    return {text} if re.fullmatch(r"[sva]\d+", text) else set()


def functions(listing):
    """(name, [(operation, operands)]) of each kernel."""
    name, body = None, []
    for line in listing.splitlines():
        line = line.split(";")[0].strip()
        m = re.fullmatch(r"(_Z\w+):", line)
        if m:
            name, body = m.group(1), []
        elif line.startswith("s_endpgm") and name:
            yield name, body
            name = None
        elif name and line and not line.startswith(".") and not line.endswith(":"):
            op, _, rest = line.partition(" ")
            body.append((op, [a.strip() for a in rest.split(",")] if rest else []))


def before(body, i, states):
    """The instructions up to `states` wait states before number i."""
    passed = 0
    for op, args in reversed(body[max(0, i - 40):i]):
        if passed >= states:
            return
        yield op, args
        passed += 1 + (int(args[0]) if op == "s_nop" else 0)


def faults(name, body):
    pinned = "Li8ELi8E" in name
    for i, (op, args) in enumerate(body):
        if op.startswith("global_load_lds"):
            need = registers(args[1])
            assert any(r.startswith("s") for r in need)
            if any(o.startswith("v_") and a and need & registers(a[0]) for o, a in before(body, i, 5)):
                yield "%s %s" % (op, args)
        elif pinned and op.startswith("v_mfma"):
            need = registers(args[1]) | registers(args[2])
            if any(o.startswith("v_") and not o.startswith("v_mfma") and need & registers(a[0])
                   for o, a in before(body, i, 2)):
                yield "%s %s" % (op, args)
        elif pinned and not op.startswith("s_"):
            sums = {r for a in args for r in registers(a) if r.startswith("a")}
            if sums and any(o.startswith("v_mfma") and sums & registers(a[0]) for o, a in before(body, i, 18)):
                yield "%s %s" % (op, args)


def test_the_check_finds_planted_faults():
    ok = [("v_readfirstlane_b32", ["s6", "v1"]), ("s_nop", ["4"]), ("global_load_lds_dwordx4", ["v2", "s[6:7]"])]
    assert not list(faults("k", ok))
    assert list(faults("k", ok[:1] + ok[2:]))
    mfma = ("v_mfma_f32_16x16x32_bf16", ["a[0:3]", "v[4:7]", "v[8:11]", "a[0:3]"])
    assert list(faults("Li8ELi8E", [("v_mov_b32", ["v5", "0"]), mfma])) and not list(faults("k", [("v_mov_b32", ["v5", "0"]), mfma]))
    assert list(faults("Li8ELi8E", [mfma, ("s_nop", ["15"]), ("v_accvgpr_read_b32", ["v1", "a2"])]))
    assert not list(faults("Li8ELi8E", [mfma, ("s_nop", ["15"]), ("s_nop", ["15"]), ("v_accvgpr_read_b32", ["v1", "a2"])]))


@pytest.mark.parametrize("unit", UNITS)
def test_wait_states(listings, unit):
    seen = 0
    for name, body in functions(listings[unit]):
        seen += sum(op.startswith("global_load_lds") for op, _ in body)
        assert not list(faults(name, body)), name
    assert seen > 0


@pytest.mark.parametrize("unit", ["gemm_bf16.hip", "gemm_f16.hip"])
def test_the_large_tiles_loop_stays_in_registers(listings, unit):
    """Nothing is spilled between a load to LDS and the next within the loop: 128 matrix instructions and 16 loads."""
    checked = 0
    for name, body in functions(listings[unit]):
        if "Li8ELi8E" not in name:
            continue
        loads = [i for i, (op, _) in enumerate(body) if op.startswith("global_load_lds")]
        loop = body[loads[-16]:loads[-1]]
        assert sum(op.startswith("v_mfma") for op, _ in loop) > 60
        assert not any(op.startswith(("scratch_", "v_accvgpr")) for op, _ in loop), name
        checked += 1
    assert checked == 5  # the forward product in two forms, the gradient's two, and these in one launch
