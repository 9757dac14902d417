"""Which eps layer norm takes, without a GPU."""
import ctypes

import pytest
import torch

from paper_2004_09362_amd import ar


def said(eps):
    x, y = (ctypes.byref(ar.Matrix(a, 6, ar.AR_BFLOAT16)) for a in (0x10000000, 0x20000000))
    # y overlaps the weight: asked once eps is admitted
    st = ar.lib.ar_layer_norm_forward(4, 6, x, y, None, eps, y, None, None)
    return st, ar.ar_last_error_message()


@pytest.mark.parametrize("eps", [1e-50, 5e-324, 2.0 ** -150])
def test_an_eps_that_would_become_0_is_refused(eps):
    """It would give NaN for a row of equal values, whose result is the bias."""
    st, text = said(eps)
    assert st == ar.AR_ERR_INVALID_ARG and "eps must be" in text


@pytest.mark.parametrize("eps", [0.0, 2.0 ** -149, 1e-40, 1e-12, 1e-5, 3e38])
def test_others_are_taken(eps):
    assert torch.tensor(eps, dtype=torch.float32) > 0 or eps == 0
    st, text = said(eps)
    assert st == ar.AR_ERR_ALIAS and "weight" in text


@pytest.mark.gpu
@pytest.mark.parametrize("cols", [5, 100, 20000])
def test_rows_of_equal_values_give_the_bias(cols):
    """With the smallest eps too; their rstd is 1 / sqrt(eps), to a root's and a quotient's rounding."""
    x, b = torch.full((3, cols), 2.0, device="cuda"), torch.arange(cols, device="cuda") / 8
    for eps in (1e-5, 1e-40, 2.0 ** -149):
        y, stats = ar.ar_layer_norm_forward(x, bias=b, eps=eps, stats=True)
        assert torch.equal(y, b.expand(3, cols)), eps
        want = float(torch.tensor(eps, dtype=torch.float32)) ** -0.5
        assert float((stats[:, 1].double() - want).abs().max()) <= 3 * 2.0 ** -24 * want
