"""What ar_orthogonalize's check of coefficients admits, without a GPU: no admitted polynomial takes a singular value out of the
range in which X, A and Q are held, however its coefficients are chosen."""
import ctypes

import pytest
import torch

from paper_2004_09362_amd import ar

X, Y, WS = 0x10000000, 0x20000000, 0x30000000  # addresses that nothing is launched on


def status(*triples, dtype=ar.AR_FLOAT32, size=4):
    """What is said of these steps, on one matrix and without a workspace: that is asked for once the coefficients are admitted."""
    flat = (ctypes.c_double * (3 * len(triples)))(*[v for t in triples for v in t])
    m = lambda at: ctypes.byref(ar.Matrix(at, size, dtype))
    got = ar.lib.ar_orthogonalize(1, size, size, m(X), 0, len(triples), flat, 1e-7, 1.0, None, 0, m(Y), 0, None, 0, None)
    assert got == ar.AR_ERR_INVALID_ARG
    return ar.ar_last_error_message()


@pytest.mark.parametrize("steps", [
    # 10 s - 10 s^3 is 3.85 at s = 1 / sqrt(3), whether the third number is 0 or next to it
    [(10, -10, 0)], [(10, -10, 1e-17)], [(10, -10, 1e-20)], [(10, -10, -1e-17)], [(-10, 10, 1e-20)], [(14, -14, 1e-18)] * 3,
    [(8, -8, 1e-40)], [(8, -8, -1e-12)],
    # what is left of X after the first step is its rounding, which the second magnifies
    [(0, 0, 0), (1e30, 0, 0)], [(1e-12, 0, 0), (1e12, 0, 0)],
    # 1 stays 1, but what is above it by a rounding doubles its distance in each step
    [(0.5, 0.5, 0)] * 64,
], ids=lambda s: "%d steps from %s" % (len(s), s[0]))
def test_steps_that_leave_the_range_are_refused(steps):
    assert "past 2.5" in status(*steps)


@pytest.mark.parametrize("step", [(1e300, 0, 0), (0, 1e39, 0), (0, 0, -4e38)], ids=str)
def test_numbers_past_32_bits_are_refused(step):
    """Also where the bound of the step before is 0: the kernels would multiply zeros with an infinity."""
    for steps in ([step], [(0, 0, 0), step]):
        assert "finite in 32 bits" in status(*steps)


# published sequences: of a fixed triple, of five and of eight steps, the last as it is and made safer by 1 %
EIGHT = [(8.28721201814563, -23.595886519098837, 17.300387312530933), (4.107059111542203, -2.9478499167379106, 0.5448431082926601),
         (3.9486908534822946, -2.908902115962949, 0.5518191394370137), (3.3184196573706015, -2.488488024314874, 0.51004894012372),
         (2.300652019954817, -1.6689039845747493, 0.4188073119525673), (1.891301407787398, -1.2679958271945868, 0.37680408948524835),
         (1.8750014808534479, -1.2500016453999487, 0.3750001645474248), (1.875, -1.25, 0.375)]
SAFER = [(a / 1.01, b / 1.01 ** 3, c / 1.01 ** 5) for a, b, c in EIGHT[:-1]] + EIGHT[-1:]


@pytest.mark.parametrize("dtype", [ar.AR_FLOAT32, ar.AR_BFLOAT16], ids=["f32", "bf16"])
@pytest.mark.parametrize("steps", [
    [(3.4445, -4.7750, 2.0315)] * 64, [(1.5, -0.5, 0.0)] * 64, [(1.5, -0.5, 1e-20)] * 64, [(1.875, -1.25, 0.375)] * 64, [(1, 0, 0)] * 64,
    [(2.5, 0, 0)], [(0.5, 0.0, 2.0)], [(0, 0, 0)] * 3, [(0.5, 0.5, 0)] * 5,
    [(4.0848, -6.8946, 2.9270), (3.9505, -6.3029, 2.6377), (3.7418, -5.5913, 2.3037), (2.8769, -3.1427, 1.2046), (2.8366, -3.0525, 1.2012)],
    EIGHT, SAFER], ids=lambda s: "%d x %s" % (len(s), s[0]))
def test_usual_steps_are_admitted(steps, dtype):
    for size in (4, 400):
        assert "workspace must hold" in status(*steps, dtype=dtype, size=size)


def test_admitted_polynomials_stay_in_the_range():
    """Random coefficients, some of them tiny: the largest value over a fine grid of singular values says which may be admitted."""
    g = torch.Generator().manual_seed(3)
    grid = torch.linspace(0, 1, 20001, dtype=torch.float64)
    admitted = 0
    for _ in range(400):
        co = torch.empty(3, dtype=torch.float64).normal_(0, 6, generator=g)
        co *= 10.0 ** -(torch.randint(0, 3, (3,), generator=g) * torch.randint(0, 12, (3,), generator=g)).double()
        a, b, c = co.tolist()
        said = status((a, b, c))
        value = float((grid * (a + b * grid ** 2 + c * grid ** 4)).abs().max())
        q = float((b * grid ** 2 + c * grid ** 4).abs().max())
        # a grid of distance h = 1 / 20000 misses the largest value by h^2 / 8 of the second derivative, at most 6 |b| + 20 |c|
        # with |b| and |c| below 30: 3e-7; the numbers' rounding to 32 bits moves it by 90 * 2^-24 at most
        if "past 2.5" in said:
            assert value > 2.5 - 1e-5 or q > 15 - 1e-5, (a, b, c)
        else:
            assert "workspace must hold" in said and value <= 2.5 + 1e-5 and q <= 15 + 1e-5, (a, b, c)
            admitted += 1
    assert 20 < admitted < 380
