"""Which kernels of the orthogonalised update are compiled, and that those on tiles of 64 keep everything in registers, without a
GPU."""
from test_gemm_code import functions
from test_orthogonal_code import listing  # noqa: F401  (the fixture)


def test_no_join_is_compiled_that_no_call_reaches(listing):  # noqa: F811
    """The first product's on both large tiles with one and two planes, the second's on tiles of 128 with two."""
    joins = sorted(name for name, _ in functions(listing) if "ortho_join_kernel" in name)
    assert len(joins) == 5 and sum("Li0E" in n for n in joins) == 4, joins
    assert [n for n in joins if "ortho_join_kernelILi1ELi2ELi4ELi4E" in n], joins


def test_small_tiles_stay_in_registers(listing):  # noqa: F811
    """Three products and four last ones, with one and two planes.  The sums of a whole tile are a wave's: no scratch memory, and
    in the loop, between the first and the last loads to LDS, no moves to other registers and back."""
    seen = 0
    for name, body in functions(listing):
        if "ortho_small_kernel" not in name:
            continue
        seen += 1
        assert not any(op.startswith("scratch_") for op, _ in body), name
        loads = [i for i, (op, _) in enumerate(body) if op.startswith("global_load_lds")]
        loop = body[loads[-16]:loads[-1]]
        assert sum(op.startswith("v_mfma") for op, _ in loop) > 10, name
        assert not any(op.startswith("v_accvgpr") for op, _ in loop), name
    assert seen == 10
