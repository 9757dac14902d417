"""The host side of layer norm and its gradient, without a GPU: what the C entry
points refuse before anything is launched, what they say of their workspace, and
the Python binding's refusals."""
import ctypes
import math

import pytest
import torch

from paper_2004_09362_amd import ar

F32, F16, BF16 = ar.AR_FLOAT32, ar.AR_FLOAT16, ar.AR_BFLOAT16
INVALID, UNSUPPORTED, ALIAS = ar.AR_ERR_INVALID_ARG, ar.AR_ERR_UNSUPPORTED, ar.AR_ERR_ALIAS
A = 0x10000000  # addresses that nothing is launched on


def mat(address, ld, dtype=BF16):
    return ctypes.byref(ar.Matrix(address, ld, dtype))


X, W, B, Y, S = A, A + 0x100000, A + 0x200000, A + 0x300000, A + 0x400000


def norm(rows=4, cols=6, x=None, weight=None, bias=None, eps=1e-5, y=None, stats=None):
    return ar.lib.ar_layer_norm_forward(rows, cols, x or mat(X, 6), weight, bias, eps, y or mat(Y, 6), stats, None)


@pytest.mark.parametrize("status,kw,text", [
    (INVALID, dict(rows=-1), "rows must be"), (INVALID, dict(cols=(1 << 30) + 1), "cols must be"),
    (INVALID, dict(x=mat(None, 6)), "x's data is NULL"), (INVALID, dict(x=mat(X + 1, 6)), "multiple"),
    (INVALID, dict(x=mat(X, 5)), "x's ld"), (INVALID, dict(y=mat(Y, 1 << 50)), "y's ld"),
    (UNSUPPORTED, dict(x=mat(X, 6, 0)), "float32, float16"), (UNSUPPORTED, dict(weight=mat(W, 0, 0)), "weight must be"),
    (INVALID, dict(bias=mat(None, 0)), "bias's data"), (UNSUPPORTED, dict(stats=mat(S, 2, F16)), "stats must be float32"),
    (INVALID, dict(stats=mat(S, 1, F32)), "stats's ld"), (INVALID, dict(eps=-1e-9), "eps must be"),
    (INVALID, dict(eps=math.inf), "eps must be"), (INVALID, dict(eps=math.nan), "eps must be"),
    (INVALID, dict(eps=1e39), "eps must be"),
    (INVALID, dict(cols=0, stats=mat(S, 2, F32)), "no statistics"),
    (ALIAS, dict(y=mat(X + 2, 6)), "y overlaps x"), (ALIAS, dict(y=mat(X, 6, F16), x=mat(X, 6)), "y overlaps x"),
    (ALIAS, dict(y=mat(X, 8)), "y overlaps x"), (ALIAS, dict(weight=mat(Y, 0)), "y overlaps weight"),
    (ALIAS, dict(bias=mat(Y + 8, 0)), "y overlaps bias"), (ALIAS, dict(stats=mat(Y, 2, F32)), "y overlaps stats"),
    (ALIAS, dict(stats=mat(X, 2, F32)), "stats overlaps x"),
    (ALIAS, dict(weight=mat(S, 0), stats=mat(S, 2, F32)), "stats overlaps weight"),
    (ALIAS, dict(bias=mat(S, 0), stats=mat(S, 2, F32)), "stats overlaps bias"),
])
def test_norm_refusals(status, kw, text):
    assert norm(**kw) == status
    assert text in ar.ar_last_error_message()


def test_norm_with_nothing_to_do_or_no_gpu():
    assert norm(rows=0, x=mat(None, 0), y=mat(None, 0), stats=mat(None, 0, F32)) == ar.AR_OK
    assert norm(cols=0, x=mat(None, 0), y=mat(None, 0)) == ar.AR_OK
    if torch.cuda.is_available():
        pytest.skip("the calls below would be launched")
    for kw in (dict(), dict(y=mat(X, 6)), dict(x=mat(X, 20), y=mat(X + 12, 20)), dict(rows=1, x=mat(X, 0), y=mat(X, 0)),
               dict(weight=mat(W, 0, F32), bias=mat(B, 0, F16), stats=mat(S, 3, F32), eps=0.0)):
        assert norm(**kw) == ar.AR_ERR_NO_DEVICE, (kw, ar.ar_last_error_message())


DX, DW, DB, DY, R = A + 0x500000, A + 0x600000, A + 0x700000, A + 0x800000, A + 0x900000


def grad_args(rows=300, cols=70, dy=None, x=None, stats=None, weight=None, residual=None, dx=mat(DX, 70), dw=mat(DW, 0, F32),
              db=mat(DB, 0, F32)):
    return (rows, cols, dy or mat(DY, 70), x or mat(X, 70), stats or mat(S, 2, F32), weight, residual, dx, dw, db)


def need_of(**kw):
    need = ctypes.c_int64(-1)
    st = ar.lib.ar_layer_norm_backward_workspace(*grad_args(**kw), ctypes.byref(need))
    assert st == ar.AR_OK, ar.ar_last_error_message()
    return need.value


def grad(ws=A + 0xA00000, ws_bytes=1 << 20, accumulate=0, **kw):
    return ar.lib.ar_layer_norm_backward(*grad_args(**kw), accumulate, ws, ws_bytes, None)


@pytest.mark.parametrize("status,kw,text", [
    (INVALID, dict(rows=-1), "rows must be"), (INVALID, dict(cols=-1), "cols must be"),
    (INVALID, dict(dy=mat(None, 70)), "dy's data"), (INVALID, dict(x=mat(X, 69)), "x's ld"),
    (UNSUPPORTED, dict(stats=mat(S, 2)), "stats must be float32"), (INVALID, dict(stats=mat(None, 2, F32)), "stats's data"),
    (UNSUPPORTED, dict(dx=mat(DX, 70, F32)), "dx must have x's type"), (UNSUPPORTED, dict(residual=mat(R, 70, F16)), "residual must"),
    (UNSUPPORTED, dict(dw=mat(DW, 0, 0)), "dw must be"), (INVALID, dict(db=mat(DB + 2, 0, F32)), "multiple"),
    (ALIAS, dict(dx=mat(X, 70)), "dx overlaps x"), (ALIAS, dict(dx=mat(DY, 71)), "dx overlaps dy"),
    (ALIAS, dict(dx=mat(DY + 2, 70)), "dx overlaps dy"), (ALIAS, dict(dx=mat(R, 72), residual=mat(R, 70)), "dx overlaps residual"),
    (ALIAS, dict(dw=mat(DY, 0)), "dw overlaps dy"), (ALIAS, dict(db=mat(DW, 0)), "db overlaps dw"),
    (ALIAS, dict(dw=mat(DX, 0)), "dw overlaps dx"), (ALIAS, dict(db=mat(S, 0)), "db overlaps stats"),
    (ALIAS, dict(dw=mat(W, 0), weight=mat(W, 0)), "dw overlaps weight"),
    (INVALID, dict(ws=None), "workspace must hold"), (INVALID, dict(ws_bytes=100), "workspace must hold"),
    (INVALID, dict(ws=A + 0xA00008), "16-byte"),
    (ALIAS, dict(ws=X + 16), "the workspace overlaps x"), (ALIAS, dict(ws=DY + 16), "the workspace overlaps dy"),
    (ALIAS, dict(ws=S), "the workspace overlaps stats"), (ALIAS, dict(ws=DW), "the workspace overlaps dw"),
    (ALIAS, dict(ws=DX), "the workspace overlaps dx"), (ALIAS, dict(ws=DB), "the workspace overlaps db"),
    (ALIAS, dict(ws=W, weight=mat(W, 0)), "the workspace overlaps weight"),
    (ALIAS, dict(ws=R, residual=mat(R, 70)), "the workspace overlaps residual"),
])
def test_norm_gradient_refusals(status, kw, text):
    assert grad(**kw) == status
    assert text in ar.ar_last_error_message()


def test_norm_gradient_workspace_and_nothing_to_do():
    assert need_of() > 0 and need_of(rows=0) == 0 and need_of(cols=0) == 0
    assert need_of(dw=None, db=None) == 0 and need_of(dw=None) == need_of()
    assert need_of(cols=40000, dy=mat(DY, 40000), x=mat(X, 40000), dx=mat(DX, 40000)) > 0  # longer than a team of lanes holds
    ask = ar.lib.ar_layer_norm_backward_workspace
    assert ask(*grad_args(), None) == INVALID
    assert grad(dx=None, dw=None, db=None, ws=None, ws_bytes=0) == ar.AR_OK
    assert grad(cols=0, ws=None, ws_bytes=0) == ar.AR_OK
    assert grad(rows=0, dw=None, db=None, ws=None, ws_bytes=0) == ar.AR_OK
    if torch.cuda.is_available():
        pytest.skip("the calls below would be launched")
    for kw in (dict(), dict(dx=mat(DY, 70)), dict(residual=mat(R, 70), dx=mat(R, 70)), dict(rows=0, ws=None, ws_bytes=0),
               dict(dy=mat(DY, 70, F32), weight=mat(W, 0, F16), dw=None), dict(dw=None, db=None, ws=None, ws_bytes=0)):
        assert grad(**kw) == ar.AR_ERR_NO_DEVICE, (kw, ar.ar_last_error_message())


def test_binding_refusals_without_a_gpu():
    x = torch.zeros(4, 8)
    for call in (lambda: ar.ar_layer_norm_forward(x), lambda: ar.ar_layer_norm_backward(x, x, x[:, :2])):
        with pytest.raises(ar.ArError, match="not on a GPU"):
            call()
    with pytest.raises(ar.ArError, match="x must be a tensor"):
        ar.ar_layer_norm_forward([1.0])
    with pytest.raises(ar.ArError, match="float32, float16 or bfloat16"):
        ar.ar_layer_norm_forward(x, out_dtype=torch.int32)
    with pytest.raises(ar.ArError, match="x requires a gradient"):
        ar.ar_layer_norm_forward(torch.zeros(4, 8, requires_grad=True))
    with pytest.raises(ar.ArError, match="not on a GPU"):
        with torch.no_grad():
            ar.ar_layer_norm_forward(torch.zeros(4, 8, requires_grad=True))


CO = (ctypes.c_double * 15)(*(3.4445, -4.7750, 2.0315) * 5)


def coefficients(*triples):
    flat = [v for t in triples for v in t]
    return (ctypes.c_double * len(flat))(*flat), len(triples)


def ortho(batch=2, M=4, N=6, x=None, x_stride=24, steps=5, co=CO, eps=1e-7, scale=1.0, residual=None, residual_stride=24, y=None,
          y_stride=24, ws=A + 0xA00000, ws_bytes=1 << 40):
    return ar.lib.ar_orthogonalize(batch, M, N, x or mat(X, 6), x_stride, steps, co, eps, scale, residual, residual_stride,
                                   y or mat(Y, 6), y_stride, ws, ws_bytes, None)


def with_coefficients(*triples):
    co, n = coefficients(*triples)
    return dict(co=co, steps=n)


@pytest.mark.parametrize("status,kw,text", [
    (INVALID, dict(batch=-1), "batch must be"), (INVALID, dict(M=-1), "M must be"), (INVALID, dict(N=(1 << 30) + 1), "N must be"),
    (INVALID, dict(x=mat(None, 6)), "x's data"), (INVALID, dict(x=mat(X, 5)), "x's ld"), (INVALID, dict(y=mat(Y + 1, 6)), "multiple"),
    (UNSUPPORTED, dict(x=mat(X, 6, 0)), "float32, float16"), (UNSUPPORTED, dict(y=mat(Y, 6, 7)), "y must be"),
    (UNSUPPORTED, dict(residual=mat(R, 6, F32)), "residual must have y's type"),
    (INVALID, dict(x_stride=-1), "x's stride"), (INVALID, dict(y_stride=23), "y's matrices overlap"),
    (INVALID, dict(residual=mat(R, 6), residual_stride=-5), "residual's stride"),
    (INVALID, dict(steps=0), "steps must be"), (INVALID, dict(steps=65), "steps must be"), (INVALID, dict(co=None), "coefficients is NULL"),
    (INVALID, dict(eps=-1.0), "eps must be"), (INVALID, dict(eps=math.nan), "eps must be"), (INVALID, dict(scale=math.nan), "scale must be"),
    (INVALID, dict(scale=1e39), "scale must be"), (INVALID, dict(scale=-math.inf), "scale must be"),
    (INVALID, with_coefficients((math.inf, 0, 0)), "must be finite"), (INVALID, with_coefficients((2.6, 0, 0)), "past 2.5"),
    (INVALID, with_coefficients((3.0, 0, 0)), "past 2.5"), (INVALID, with_coefficients((0, 5.0, 0)), "past 2.5"),
    # 2.4 after the first step, past 2.5 after the second
    (INVALID, with_coefficients((2.4, 0, 0), (1.1, 0, 0)), "past 2.5"),
    # within 2.5, but Q reaches past 15 between
    (INVALID, with_coefficients((17.0, -33.0, 16.5)), "past 2.5, or"),
    (ALIAS, dict(y=mat(X, 6), y_stride=30), "y overlaps x"), (ALIAS, dict(y=mat(X + 2, 6)), "y overlaps x"),
    (ALIAS, dict(y=mat(X, 6, F16)), "y overlaps x"), (ALIAS, dict(residual=mat(Y + 12, 6)), "y overlaps residual"),
    (ALIAS, dict(residual=mat(Y, 6), residual_stride=0), "y overlaps residual"),
    (INVALID, dict(ws=None), "workspace must hold"), (INVALID, dict(ws_bytes=1000), "workspace must hold"),
    (INVALID, dict(ws=A + 0xA00004), "16-byte"),
    (ALIAS, dict(ws=X + 16), "the workspace overlaps x"), (ALIAS, dict(ws=Y - 0x1000), "the workspace overlaps y"),
    (ALIAS, dict(ws=R + 16, residual=mat(R, 6)), "the workspace overlaps residual"),
    (UNSUPPORTED, dict(batch=65536), "batch must be"), (UNSUPPORTED, dict(M=32769, N=40000), "shorter side"),
    (UNSUPPORTED, dict(N=(1 << 21) + 1), "shorter side"), (UNSUPPORTED, dict(batch=3, M=32768, N=1 << 18), "2\\^34"),
])
def test_orthogonalize_refusals(status, kw, text):
    import re

    assert ortho(**kw) == status
    assert re.search(text, ar.ar_last_error_message()), ar.ar_last_error_message()


def test_orthogonalize_workspace_and_nothing_to_do():
    def need_of(batch, M, N, dtype):
        need = ctypes.c_int64(-1)
        st = ar.lib.ar_orthogonalize_workspace(batch, M, N, mat(None, N, dtype), ctypes.byref(need))
        assert st == ar.AR_OK, ar.ar_last_error_message()
        return need.value

    for batch, M, N in ((0, 4, 4), (3, 0, 4), (3, 4, 0)):
        assert need_of(batch, M, N, F32) == 0
        assert ortho(batch=batch, M=M, N=N, x=mat(None, 6), y=mat(None, 6), ws=None, ws_bytes=0) == ar.AR_OK
    assert need_of(1, 1, 1, F32) > 0 and need_of(1, 4096, 1024, BF16) == need_of(1, 1024, 4096, BF16)
    # two buffers of X in two halves, A and Q, and little else: 10 bytes an element and 4 of the square
    assert need_of(1, 4096, 16384, BF16) >= 8 * 4096 * 16384 + 4 * 4096 * 4096
    assert ar.lib.ar_orthogonalize_workspace(1, 4, 4, mat(None, 4), None) == INVALID
    assert ar.lib.ar_orthogonalize_workspace(1, 4, 4, None, ctypes.byref(ctypes.c_int64())) == INVALID
    if torch.cuda.is_available():
        pytest.skip("the calls below would be launched")
    for kw in (dict(), dict(y=mat(X, 6)), dict(residual=mat(Y, 6)), dict(x_stride=0), dict(batch=1, x_stride=-7, y_stride=0),
               dict(x=mat(X, 12), y=mat(X + 12, 12), x_stride=48, y_stride=48),
               with_coefficients((2.0, -1.5, 0.5)), with_coefficients((8.28, -23.6, 17.3), (1.5, -0.24, 0.0)),
               with_coefficients(*[(1.5, -0.5, 0.0)] * 64)):
        assert ortho(**kw) == ar.AR_ERR_NO_DEVICE, (kw, ar.ar_last_error_message())


def test_the_bound_of_singular_values_holds_for_the_usual_coefficients():
    """Accepted step for step: the bound that the check carries along stays below 2.5 for 64 steps."""
    co, n = coefficients(*[(3.4445, -4.7750, 2.0315)] * 64)
    st = ortho(steps=n, co=co, ws=None)
    assert st == INVALID and "workspace" in ar.ar_last_error_message()


def test_orthogonalize_binding_refusals_without_a_gpu():
    x = torch.zeros(4, 8)
    with pytest.raises(ar.ArError, match="not on a GPU"):
        ar.ar_orthogonalize(x)
    for kw, text in ((dict(coefficients=(1.0, 2.0)), "one such triple for each"), (dict(coefficients=[(1, 0, 0)] * 4), "each of 5 steps"),
                     (dict(coefficients=None), "one such triple for each"),
                     (dict(steps=2.0), "steps must be"), (dict(steps=10 ** 12), "steps must be"), (dict(steps=0), "steps must be"),
                     (dict(out_dtype=torch.float64), "float32, float16 or bfloat16")):
        with pytest.raises(ar.ArError, match=text):
            ar.ar_orthogonalize(x, **kw)
    with pytest.raises(ar.ArError, match="x requires a gradient"):
        ar.ar_orthogonalize(torch.zeros(4, 8, requires_grad=True))
    with pytest.raises(ar.ArError, match="x must be a tensor"):
        ar.ar_orthogonalize("x")
    with pytest.raises(ar.ArError, match="dense"):
        ar.ar_orthogonalize(x.to_sparse())
