"""The orthogonalised update on the GPU where it is at its bounds: steps that magnify roundings, and how far the interface says
that results may be off, for matrices whose roundings even out and for those whose roundings all fall the same way."""
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


STEPS = [(3.4445, -4.7750, 2.0315)] * 5


def shuffled(n, seed):
    return torch.eye(n)[torch.randperm(n, generator=torch.Generator().manual_seed(seed))]


# entries of one size, whose k singular values are k^(-1/2) each: name, matrix, k
EQUAL = [("identity 353", torch.eye(353), 353), ("permutation 320", shuffled(320, 1), 320), ("permutation 405", shuffled(405, 2), 405),
         ("ones 65 x 290", torch.ones(65, 290), 1), ("ones 2000 x 65", torch.ones(2000, 65), 1), ("ones 80 x 12245", torch.ones(80, 12245), 1),
         ("blocks of 318 x 544", torch.block_diag(*[torch.ones(318, 544)] * 4), 4)]


@pytest.mark.parametrize("name,x,k", EQUAL, ids=[e[0] for e in EQUAL])
def test_equal_entries(name, x, k):
    """All roundings fall the same way.  Towards float32 and float16 no further than 22 bits' roundings can take the singular
    value; towards bfloat16 than those of 11 bits, and what the interface says of them, 2.6e-2."""
    want = tref.orthogonal(x)
    size = float(want.norm())
    for out in (torch.bfloat16, torch.float16, torch.float32):
        print("[gpu] equal entries", name, out, flush=True)
        y = ar.ar_orthogonalize(x.to(DEV), out_dtype=out).double().cpu()
        off = reach(k ** -0.5, STEPS, 2.0 ** -11 if out == torch.bfloat16 else 2.0 ** -21) * k ** 0.5
        if out == torch.bfloat16:
            off = min(off, 2.6e-2 * size)
        assert float((y - want).norm()) <= off + ref.U[out] * size + (2.0 ** -25 * x.numel() ** 0.5 if out == torch.float16 else 0)


def differing():
    g = torch.Generator().manual_seed(11)
    n = lambda *s: torch.empty(*s).normal_(generator=g)
    q = torch.linalg.qr(n(300, 300).double())
    return [("random", n(300, 700), 2.5e-3), ("tall", n(900, 66), 2.5e-3), ("rank 1", n(150, 1) @ n(1, 400), 2.5e-3),
            ("rank 8", n(500, 8) @ n(8, 200), 2.5e-3), ("rank 16 and noise", n(256, 16) @ n(16, 512) * 0.25 + n(256, 512), 2.5e-3),
            ("signs", n(257, 384).sign(), 2.5e-3), ("diagonal", torch.diag(torch.rand(500, generator=g)), 2.5e-3),
            ("orthogonal", q[0].float().contiguous(), 4e-3), ("sparse", n(400, 600) * (torch.rand(400, 600, generator=g) < 0.003), 4e-3)]


@pytest.mark.parametrize("i", range(9))
def test_differing_entries_towards_bfloat16(i):
    """What the interface says of the products' 11 bits, and one rounding to bfloat16, off by half a step at most."""
    name, x, stated = differing()[i]
    print("[gpu] differing entries", name, flush=True)
    want = tref.orthogonal(x)
    y = ar.ar_orthogonalize(x.to(DEV), out_dtype=torch.bfloat16).double().cpu()
    assert float((y - want).norm()) <= (stated + ref.U[torch.bfloat16]) * float(want.norm())


@pytest.mark.parametrize("size", [(3, 1266), (64, 1586), (1586, 64), (35, 35)], ids=lambda s: "x".join(map(str, s)))
def test_sides_up_to_64_take_22_bits(size):
    """Of equal entries 11 bits would leave these off by 1e-2 (the last one, an identity, by 7e-3) towards bfloat16 too."""
    x, k = (torch.eye(35), 35) if size == (35, 35) else (torch.ones(*size), 1)
    want = tref.orthogonal(x)
    y = ar.ar_orthogonalize(x.to(DEV), out_dtype=torch.bfloat16).double().cpu()
    part = reach(k ** -0.5, STEPS, 2.0 ** -21) / (float(want.norm()) * k ** -0.5)  # of the singular value, and so of each entry
    assert bool(((y - want).abs() <= (part + ref.U[torch.bfloat16] * (1 + part)) * want.abs()).all())
