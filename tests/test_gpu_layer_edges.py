"""The layer operators on the GPU where their ranges end: matrices narrower than
16 bytes, infinities and very large values, the longest dimensions."""
import math

import pytest
import torch

import layer_reference as ref
from paper_2004_09362_amd import ar

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
TYPES = [torch.bfloat16, torch.float16, torch.float32]
IDS = ["bf16", "f16", "f32"]


def matrix(g, rows, cols, dtype, std=1.0):
    return torch.empty(rows, cols, dtype=torch.float32).normal_(0, std, generator=g).to(dtype).to(DEV)


@pytest.mark.parametrize("dtype", TYPES, ids=IDS)
def test_gradients_of_narrow_layers(dtype):
    """1 to 3 outputs or inputs, with inner lengths that leave a few rows in the last tile, of few tiles and of many: dy, x
    and w as operands whose rows are shorter than the 16 bytes that a load takes."""
    for M in (33, 34, 65, 66, 67, 70, 129, 321, 385, 1000):
        for N, K in ((1, 40), (2, 9), (3, 64), (40, 1), (9, 2), (64, 3), (1, 1), (3, 2)):
            print("[gpu] narrow", dtype, M, N, K, flush=True)
            g = torch.Generator().manual_seed(M * 10007 + N * 101 + K)
            # of dx the inner length is N: here the long one
            for rows, cols, inner in ((M, N, K), (K, M, N), (K, M, 1)):
                dy, x, w = matrix(g, rows, cols, dtype, 0.1), matrix(g, rows, inner, dtype), matrix(g, cols, inner, dtype, 0.3)
                want = ref.backward(dy, x, w)
                for name, t in zip(("dx", "dw", "db"), ar.ar_linear_backward(dy, x, w, dw_dtype=torch.float32)):
                    ref.close(t, want[name][0], want[name][1], name)
