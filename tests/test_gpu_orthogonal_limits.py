"""The orthogonalised update on the GPU at the largest sizes that it takes: matrices in a call, and sides."""
import math

import pytest
import torch

from paper_2004_09362_amd import ar
from test_gpu_orthogonal_tiles import REPEATS, repeated

pytestmark = pytest.mark.gpu

DEV = "cuda:0"


@pytest.mark.parametrize("out", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
def test_65535_matrices(out):
    """Each has one element that is not 0, of singular value 1, which these steps keep."""
    i = torch.arange(65535, device=DEV)
    x = torch.zeros(65535, 1, 3, device=DEV)
    x[i, 0, i % 3] = torch.where(i % 5 < 2, 1.0, -1.0) * torch.exp2((i % 7 - 3).float())
    print("[gpu] 65535 matrices", out, flush=True)
    y = ar.ar_orthogonalize(x, steps=2, coefficients=(1.5, -0.5, 0.0), eps=0.0, out_dtype=out)
    assert torch.equal(y, x.sign().to(out))
    y = ar.ar_orthogonalize(x.transpose(1, 2).contiguous(), steps=2, coefficients=(1.5, -0.5, 0.0), eps=0.0, out_dtype=out)
    assert torch.equal(y[:, :, 0], x[:, 0].sign().to(out))


@pytest.mark.parametrize("size", [(70, 1 << 21), (1 << 21, 64), (32768, 32768)], ids=lambda s: "x".join(map(str, s)))
def test_longest_sides(size):
    """As test_exact_steps of the tiles: results that are exact in every bit."""
    if torch.cuda.mem_get_info()[0] < 60 << 30:
        pytest.skip("needs 50 GB")
    M, N = size
    x, rows, cols = repeated(min(size), max(size), torch.Generator().manual_seed(M))
    if M > N:
        x = x.t().contiguous()
    s2 = REPEATS / rows
    a, b = (1.5, -0.5) if rows < 32768 else (0.5, 2.0)  # the sum a + b s2 in 22 bits
    for out in (torch.float32, torch.bfloat16):
        print("[gpu] longest sides", size, out, flush=True)
        y = ar.ar_orthogonalize(x, steps=1, coefficients=(a, b, 0.0), eps=0.0, out_dtype=out)
        want = (x * ((a + b * s2) / math.sqrt(rows * cols))).to(out)
        assert torch.equal(y, want)
        del y, want
