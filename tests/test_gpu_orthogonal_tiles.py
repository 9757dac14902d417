"""The orthogonalised update on the GPU at sizes that take every tile its products have, from 64 to 256, one to a workgroup,
several, or shared by several workgroups, with one and with two planes of operands (tests/test_orthogonal_plan.py says which
size takes which)."""
import math

import pytest
import torch

import layer_reference as ref
from paper_2004_09362_amd import ar
from test_orthogonal_plan import TILES

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
SIZES = list(TILES)
REPEATS = 4


def hadamard_rows(ids, n):
    """Rows `ids` of the n x n Hadamard matrix of Sylvester's doubling: the parity of the bits that row and column share."""
    v = ids.to(DEV, torch.int32)[:, None] & torch.arange(n, device=DEV, dtype=torch.int32)
    for s in (16, 8, 4, 2, 1):
        v ^= v >> s
    return 1.0 - 2.0 * (v & 1).float()


def repeated(m, n, g):
    """(x, m'): m' rows and n' columns of the m x n matrix x, any of them, hold rows of a Hadamard matrix, each REPEATS times;
    the other rows and columns are 0.  m' n' is a power of four, so that the norm is a power of two."""
    rows, cols = 1 << (m.bit_length() - 1), 1 << (n.bit_length() - 1)
    if (rows * cols).bit_length() % 2 == 0:
        cols //= 2
    if rows > cols:
        rows //= 4
    which = torch.randperm(cols, generator=g)[:rows // REPEATS].repeat(REPEATS)[torch.randperm(rows, generator=g)]
    x = torch.zeros(m, n, device=DEV)
    at = torch.randperm(m, generator=g)[:rows].to(DEV), torch.randperm(n, generator=g)[:cols].to(DEV)
    x[at[0][:, None], at[1]] = hadamard_rows(which, cols)
    return x, rows, cols


@pytest.mark.parametrize("out", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("size", SIZES, ids=lambda s: "x".join(map(str, s)))
def test_exact_steps(size, out):
    """With m' rows that hold each direction four times, A is 1 / m' within the four and 0 elsewhere, Q is not diagonal, every
    product and sum is a number of few bits, and the result is x times a number in every bit: any wrong row, column, step or
    part breaks it."""
    batch, M, N = size
    m, n = min(M, N), max(M, N)
    g = torch.Generator().manual_seed(m + n)
    stack, rows, cols = [], 0, 0
    for k in range(batch):
        x, rows, cols = repeated(m, n, g)
        stack.append((x if M <= N else x.t().contiguous()) * 2.0 ** (k % 5 - 2))
    x = torch.stack(stack) if batch > 1 else stack[0]
    s2 = REPEATS / rows
    for a, b, c in ((1.5, -0.5, 0.0), (1.5, -1.0, 0.5), (0.0, 2.0, 0.0)):
        print("[gpu] exact tiles", size, out, (a, b, c), flush=True)
        y = ar.ar_orthogonalize(x, steps=1, coefficients=(a, b, c), eps=0.0, out_dtype=out)
        want = x.sign() * ((a + b * s2 + c * s2 * s2) / math.sqrt(rows * cols))
        assert torch.equal(y, want.to(out))


def steps_of(x, dtype):
    """Five steps of the default coefficients in `dtype` on the GPU, in the shorter side's products."""
    X = (x.t() if x.shape[0] > x.shape[1] else x).to(dtype).contiguous()
    X = X / (X.double().norm().to(dtype) + 1e-7)
    for _ in range(5):
        A = X @ X.t().contiguous()
        X = 3.4445 * X + (-4.7750 * A + 2.0315 * (A @ A)) @ X
    return X.t() if x.shape[0] > x.shape[1] else X


@pytest.mark.parametrize("size", [(1, 4096, 4096), (1, 2826, 16384), (1, 8192, 2900), (3, 3300, 4096), (1, 2048, 8192)],
                         ids=lambda s: "x".join(map(str, s)))
def test_against_64_bits(size):
    """Towards float32 and float16 at most twice as far off, in the Frobenius norm, as the same steps in float32, and 2^-22;
    towards bfloat16 2.5e-3; and one rounding."""
    batch, M, N = size
    g = torch.Generator(device=DEV).manual_seed(M + N)
    x = torch.empty(batch, M, N, device=DEV).normal_(0, 0.01, generator=g)
    r = torch.empty(batch, M, N, device=DEV).normal_(0, 0.02, generator=g)
    want = [steps_of(t, torch.float64) for t in x]
    in32 = [float((steps_of(t, torch.float32).double() - w).norm()) for t, w in zip(x, want)]
    for out in (torch.float32, torch.float16, torch.bfloat16):
        print("[gpu] tiles against 64 bits", size, out, flush=True)
        res = r.to(out)
        y = ar.ar_orthogonalize(x, residual=res, scale=-0.5, out_dtype=out)
        for t, rt, w, o in zip(y, res, want, in32):
            whole = rt.double() - 0.5 * w
            off = 0.5 * (2.5e-3 if out == torch.bfloat16 else 0) * float(w.norm())
            if out != torch.bfloat16:
                off = 0.5 * (2 * o + 2.0 ** -22 * float(w.norm())) + 2.0 ** -24 * float(whole.norm())  # the sum with the residual
            off += ref.U[out] * float(whole.norm()) + (2.0 ** -25 * math.sqrt(w.numel()) if out == torch.float16 else 0)
            assert float((t.double() - whole).norm()) <= off
