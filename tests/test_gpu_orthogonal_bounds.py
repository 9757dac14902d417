"""The orthogonalised update on the GPU where it is at its bounds: steps that magnify roundings."""
import pytest
import torch

import layer_reference as ref
import training_reference as tref
from paper_2004_09362_amd import ar
from test_orthogonal_bounds import EIGHT, SAFER

pytestmark = pytest.mark.gpu

DEV = "cuda:0"


def reach(s, steps, u):
    """How far from its exact value the singular value s may come, where X, A and Q are off by u of their sizes and all the same
    way: the ends of an interval that each step's polynomial moves and its roundings widen."""
    lo = hi = exact = s
    for a, b, c in steps:
        grid = torch.linspace(lo, hi, 2001, dtype=torch.float64)
        s2 = grid * grid
        p = grid * (a + s2 * (b + s2 * c))
        wide = u * hi * float((p.abs() / hi + 3 * (s2 * (b + 2 * c * s2)).abs() + 2 * (s2 * (b + c * s2)).abs()).max())
        lo, hi = float(p.min()) - wide, float(p.max()) + wide
        exact = exact * (a + exact ** 2 * (b + exact ** 2 * c))
    return max(hi - exact, exact - lo)


@pytest.mark.parametrize("steps", [EIGHT, SAFER], ids=["eight", "safer"])
@pytest.mark.parametrize("size", [(96, 200), (400, 100), (130, 260), (200, 300)], ids=lambda s: "x".join(map(str, s)))
def test_steps_that_magnify_roundings(size, steps):
    """Equal entries have one singular value, 1, which the first step takes to where the next ones magnify what it is off by
    ten times each; products of 11 bits reach infinity from some of these.  Of 22 bits, u = 2^-21 with the product of the low
    halves that is left out.  Of many values the distance from 64 bits is at most twice that of the same steps in float32, and
    2^-22.  y is rounded once."""
    ones = torch.ones(*size, device=DEV)
    many = torch.randn(*size, generator=torch.Generator().manual_seed(5)).to(DEV)
    for x in (ones, many):
        want = tref.orthogonal(x, steps=8, coefficients=steps)
        in32 = tref.orthogonal(x, steps=8, coefficients=steps, dtype=torch.float32)
        off = reach(1.0, steps, 2.0 ** -21) if x is ones else 2 * float((in32.double() - want).norm()) + 2.0 ** -22 * float(want.norm())
        for out in (torch.bfloat16, torch.float32):
            print("[gpu] magnified", size, out, flush=True)
            y = ar.ar_orthogonalize(x, steps=8, coefficients=steps, out_dtype=out).double().cpu()
            assert float((y - want).norm()) <= off + ref.U[out] * float(want.norm())
