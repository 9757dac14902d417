"""The layer operators' host side, without a GPU: the generator's published
vectors in the reference that the GPU tests use, what the C entry points refuse
before anything is launched, what they say of their workspace, and the Python
binding's refusals."""
import ctypes
import math

import pytest
import torch

import layer_reference as ref
from paper_2004_09362_amd import ar

F32, F16, BF16 = ar.AR_FLOAT32, ar.AR_FLOAT16, ar.AR_BFLOAT16
A = 0x10000000  # addresses that nothing is launched on


def mat(address, ld, dtype=BF16):
    return ctypes.byref(ar.Matrix(address, ld, dtype))


def test_reference_generator_gives_the_published_words():
    """The vectors that the generator's authors publish for seven and ten rounds."""
    m = 0xFFFFFFFF
    for rounds, zeros, ones in ((7, "5f6fb709 0d893f64 4f121f81 4f730a48", "5207ddc2 45165e59 4d8ee751 8c52f662"),
                                (10, "6627e8d5 e169c58d bc57ac4c 9b00dbd8", "408f276d 41c83b0e a20bc7c6 6d5451fd")):
        assert ref.counter_words([0] * 4, [0] * 2, rounds) == [int(x, 16) for x in zeros.split()]
        assert ref.counter_words([m] * 4, [m] * 2, rounds) == [int(x, 16) for x in ones.split()]
    seed, site, row0, p = 0xABCDEF0123456789, 3, (1 << 32) - 1, 0.4
    mask = ref.keep_mask(3, 10, p, seed, site, row0)
    for i in range(3):
        for j in range(10):
            row = row0 + i
            w = ref.counter_words([j // 4, row & m, row >> 32, site], [seed & m, seed >> 32])[j % 4]
            assert bool(mask[i, j]) == (w < math.floor((1 - p) * 2 ** 32 + 0.5))


def forward(M=4, N=6, K=8, x=None, w=None, bias=None, residual=None, act=0, drop=None, y=None, preact=None, ws=None,
            ws_bytes=0):
    x = mat(A, 8) if x is None else x
    w = mat(A + 0x100000, 8) if w is None else w
    y = mat(A + 0x200000, 6) if y is None else y
    return ar.lib.ar_linear_forward(M, N, K, x, w, bias, residual, act, drop, y, preact, ws, ws_bytes, None)


def drop(p, seed=1, site=0, row0=0):
    return ctypes.byref(ar.DropoutArgs(p, seed, site, row0))


INVALID, UNSUPPORTED, ALIAS = ar.AR_ERR_INVALID_ARG, ar.AR_ERR_UNSUPPORTED, ar.AR_ERR_ALIAS


@pytest.mark.parametrize("status,kw,text", [
    (INVALID, dict(M=-1), "M must be"), (INVALID, dict(N=(1 << 30) + 1), "N must be"), (INVALID, dict(K=-5), "K must be"),
    (INVALID, dict(act=9), "activation"), (INVALID, dict(act=-1), "activation"),
    (INVALID, dict(x=mat(None, 8)), "x's data is NULL"), (INVALID, dict(x=mat(A + 1, 8)), "multiple"),
    (INVALID, dict(x=mat(A, 7)), "x's ld"), (INVALID, dict(y=mat(A + 0x200000, 5)), "y's ld"),
    (INVALID, dict(y=mat(A + 0x200000, 1 << 50)), "y's ld"),
    (UNSUPPORTED, dict(x=mat(A, 8, 0)), "float32, float16"), (UNSUPPORTED, dict(w=mat(A + 0x100000, 8, F16)), "wrong type"),
    (UNSUPPORTED, dict(y=mat(A + 0x200000, 6, F16)), "y must have x's type"),
    (UNSUPPORTED, dict(bias=mat(A + 0x300000, 0, F16)), "bias"),
    (UNSUPPORTED, dict(residual=mat(A + 0x300000, 6, F32)), "residual"),
    (UNSUPPORTED, dict(preact=mat(A + 0x300000, 6, F32)), "preact"),
    (INVALID, dict(drop=drop(-0.1)), "p must be"), (INVALID, dict(drop=drop(1.0001)), "p must be"),
    (INVALID, dict(drop=drop(math.nan)), "p must be"),
    (ALIAS, dict(y=mat(A + 16, 6)), "y overlaps x"), (ALIAS, dict(y=mat(A + 0x100000, 6)), "y overlaps w"),
    (ALIAS, dict(preact=mat(A + 0x200000, 6)), "y overlaps preact"),
    (ALIAS, dict(residual=mat(A + 0x200002, 6)), "y overlaps residual"),
    (ALIAS, dict(bias=mat(A + 0x200000, 0)), "y overlaps bias"),
    (ALIAS, dict(preact=mat(A, 6)), "preact overlaps x"),
    # columns of one matrix that overlap by one element; those that do not are found apart below
    (ALIAS, dict(x=mat(A, 20), y=mat(A + 14, 20)), "y overlaps x"),
    (ALIAS, dict(x=mat(A + 12, 13), y=mat(A + 0, 13)), "y overlaps x"),
    (INVALID, dict(M=100, N=64, K=8192, x=mat(A, 8192), w=mat(A + 0x1000000, 8192), y=mat(A + 0x2000000, 64)), "workspace must hold"),
    (INVALID, dict(M=100, N=64, K=8192, x=mat(A, 8192), w=mat(A + 0x1000000, 8192), y=mat(A + 0x2000000, 64),
                   ws=A + 0x3000004, ws_bytes=1 << 40), "16-byte"),
])
def test_forward_refusals(status, kw, text):
    assert forward(**kw) == status
    assert text in ar.ar_last_error_message()


def test_forward_with_nothing_to_do_or_no_gpu():
    assert forward(M=0, x=mat(None, 0), y=mat(None, 0)) == ar.AR_OK
    assert forward(N=0, w=mat(None, 0), y=mat(None, 0)) == ar.AR_OK
    if torch.cuda.is_available():
        pytest.skip("the calls below would be launched")
    for kw in (dict(), dict(K=0, x=mat(None, 0), w=mat(None, 0)), dict(x=mat(A, 20), y=mat(A + 16, 20)),
               dict(residual=mat(A + 0x200000, 6)), dict(M=1, x=mat(A, 0), y=mat(A + 16, 0))):
        assert forward(**kw) == ar.AR_ERR_NO_DEVICE, (kw, ar.ar_last_error_message())


def test_forward_workspace():
    need = ctypes.c_int64(-1)
    ask = ar.lib.ar_linear_forward_workspace
    assert ask(4096, 4096, 4096, mat(A, 4096), mat(A, 4096), ctypes.byref(need)) == ar.AR_OK and need.value == 0
    assert ask(100, 64, 8192, mat(A, 8192), mat(A, 8192), ctypes.byref(need)) == ar.AR_OK
    assert need.value > 0 and need.value % (100 * 64 * 4) == 0
    assert ask(0, 64, 8192, mat(None, 0), mat(A, 8192), ctypes.byref(need)) == ar.AR_OK and need.value == 0
    assert ask(4, 4, 4, mat(A, 4), mat(A, 3), ctypes.byref(need)) == INVALID
    assert ask(4, 4, 4, mat(A, 4), mat(A, 4), None) == INVALID
    assert ask(4, 4, 4, None, mat(A, 4), ctypes.byref(need)) == INVALID
    big = 1 << 30
    assert ask(big, big, 8, mat(A, 8), mat(A, 8), ctypes.byref(need)) == UNSUPPORTED and "tiles" in ar.ar_last_error_message()


def test_a_workspace_within_an_operand_is_refused():
    """The workspace is written while operands are read and results stored."""
    M, N, K, need = 100, 64, 8192, ctypes.c_int64()
    x, w, y = A, A + 0x1000000, A + 0x2000000
    kw = dict(M=M, N=N, K=K, x=mat(x, K), w=mat(w, K), y=mat(y, N), preact=mat(A + 0x3000000, N), residual=mat(A + 0x4000000, N),
              bias=mat(A + 0x5000000, 0))
    assert ar.lib.ar_linear_forward_workspace(M, N, K, kw["x"], kw["w"], ctypes.byref(need)) == ar.AR_OK and need.value > 0
    for at, name in ((x + 16, "x"), (w - need.value + 16, "w"), (y, "y"), (A + 0x3000000 + M * N * 2 - 16, "preact"),
                     (A + 0x4000000, "residual"), (A + 0x5000000 - need.value + 16, "bias")):
        assert forward(ws=at, ws_bytes=need.value, **kw) == ALIAS, name
        assert "the workspace overlaps " + name in ar.ar_last_error_message()
    if not torch.cuda.is_available():  # beside them it is taken: what is left to miss is the GPU
        assert forward(ws=A + 0x6000000, ws_bytes=1 << 40, **kw) == ar.AR_ERR_NO_DEVICE
    kw = dict(M=500, N=64, K=8, dy=mat(A, 64), x=mat(A + 0x100000, 8), w=mat(A + 0x200000, 8), z=mat(A + 0x300000, 64), act=2,
              dx=mat(A + 0x400000, 8), dw=mat(A + 0x500000, 8), db=mat(A + 0x600000, 0))
    for i, name in enumerate(("dy", "x", "w", "preact", "dx", "dw", "db")):
        assert backward(ws=A + i * 0x100000, n=1 << 40, **kw) == ALIAS, name
        assert "the workspace overlaps " + name in ar.ar_last_error_message()


def test_products_of_too_many_tiles_are_refused():
    """A launch of 256 threads for each tile of 128 x 128 holds fewer than 2^24 of them."""
    need = ctypes.c_int64()
    ask = lambda M, N: ar.lib.ar_linear_forward_workspace(M, N, 8, mat(A, 8), mat(A, 8), ctypes.byref(need))  # noqa: E731
    assert ask(1 << 19, 1 << 19) == UNSUPPORTED and "tiles" in ar.ar_last_error_message()
    assert ask((1 << 19) - 127, 1 << 19) == UNSUPPORTED
    assert ask((1 << 19) - 128, 1 << 19) == ar.AR_OK
    assert ask(1 << 30, 128) == ar.AR_OK and ask(1, 1 << 30) == ar.AR_OK and ask(64, 1 << 30) == ar.AR_OK


def backward(M=4, N=6, K=8, dy=None, x=None, w=None, z=None, act=0, d=None, dx=None, dw=None, db=None, acc=0, ws=None, n=0):
    dy, x, w = dy or mat(A, 6), x or mat(A + 0x100000, 8), w or mat(A + 0x200000, 8)
    return ar.lib.ar_linear_backward(M, N, K, dy, x, w, z, act, d, dx, dw, db, acc, ws, n, None)


@pytest.mark.parametrize("status,kw,text", [
    (INVALID, dict(M=-1), "M must be"), (INVALID, dict(act=5), "activation"), (INVALID, dict(d=drop(2.0)), "p must be"),
    (INVALID, dict(act=2, dw=mat(A + 0x400000, 8)), "preact is NULL"),
    (INVALID, dict(x=mat(A, 7), dw=mat(A + 0x400000, 8)), "x's ld"),
    (INVALID, dict(w=mat(None, 8), dx=mat(A + 0x400000, 8)), "w's data"),
    (UNSUPPORTED, dict(w=mat(A, 8, F16), dx=mat(A + 0x400000, 8), dw=mat(A + 0x500000, 8)), "w has the wrong type"),
    (UNSUPPORTED, dict(dy=mat(A, 6, F16), dx=mat(A + 0x400000, 8)), "dy must have"),
    (UNSUPPORTED, dict(dw=mat(A + 0x400000, 8, F16)), "dw must have"), (UNSUPPORTED, dict(dx=mat(A + 0x400000, 8, F16)), "dx must have"),
    (UNSUPPORTED, dict(dx=mat(A + 0x400000, 8), db=mat(A + 0x500000, 0, F16)), "db must have"),
    (UNSUPPORTED, dict(act=1, z=mat(A + 0x300000, 6, F32), dw=mat(A + 0x400000, 8)), "preact has"),
    (ALIAS, dict(dx=mat(A, 8)), "dx overlaps dy"), (ALIAS, dict(dw=mat(A + 0x100000, 8)), "dw overlaps x"),
    (ALIAS, dict(dx=mat(A + 0x400000, 8), dw=mat(A + 0x400010, 8)), "dw overlaps dx"),
    (ALIAS, dict(dw=mat(A + 0x400000, 8), db=mat(A + 0x400000, 0)), "db overlaps dw"),
    (INVALID, dict(db=mat(A + 0x400000, 0)), "workspace must hold"),
])
def test_backward_refusals(status, kw, text):
    assert backward(**kw) == status
    assert text in ar.ar_last_error_message()


def test_backward_reads_only_what_it_needs():
    """Operands of gradients that are not wanted may be anything."""
    if torch.cuda.is_available():
        pytest.skip("the calls below would be launched")
    none = mat(None, 0, 77)
    ws = dict(ws=A + 0x600000, n=1 << 30)
    for kw in (dict(x=none, dx=mat(A + 0x400000, 8)), dict(w=none, dw=mat(A + 0x400000, 8, F32)),
               dict(x=none, w=none, db=mat(A + 0x400000, 0, F32)),
               dict(x=none, w=none, act=2, z=mat(A + 0x300000, 6), db=mat(A + 0x400000, 0))):
        assert backward(**kw, **ws) == ar.AR_ERR_NO_DEVICE, ar.ar_last_error_message()
    assert backward(x=none, w=none) == ar.AR_OK  # nothing wanted


def test_dropout_refusals():
    call = lambda rows=4, cols=6, x=None, r=None, d=None, y=None: ar.lib.ar_dropout_forward(  # noqa: E731
        rows, cols, x or mat(A, 6), r, d, y or mat(A + 0x100000, 6, F32), None)
    for status, kw, text in ((INVALID, dict(d=None), "drop is NULL"), (INVALID, dict(d=drop(-1.0)), "p must be"),
                             (INVALID, dict(d=drop(0.5), rows=-1), "rows"), (INVALID, dict(d=drop(0.5), cols=1 << 31), "cols"),
                             (INVALID, dict(d=drop(0.5), x=mat(A, 5)), "x's ld"),
                             (UNSUPPORTED, dict(d=drop(0.5), x=mat(A, 6, 0)), "float32"),
                             (UNSUPPORTED, dict(d=drop(0.5), r=mat(A + 0x200000, 6, BF16)), "residual"),
                             (ALIAS, dict(d=drop(0.5), y=mat(A, 6, F32)), "y overlaps x"),
                             (ALIAS, dict(d=drop(0.5), r=mat(A + 0x100004, 6, F32)), "y overlaps residual")):
        assert call(**kw) == status and text in ar.ar_last_error_message(), (kw, ar.ar_last_error_message())
    assert call(rows=0, x=mat(None, 0), y=mat(None, 0), d=drop(0.5)) == ar.AR_OK
    assert ar.lib.ar_dropout_backward(4, 6, mat(A, 6), None, mat(A + 0x100000, 6), None) == INVALID
    if not torch.cuda.is_available():
        assert call(d=drop(0.5), x=mat(A, 6, F32), y=mat(A, 6, F32)) == ar.AR_ERR_NO_DEVICE
        assert ar.lib.ar_dropout_backward(4, 6, mat(A, 6), drop(0.5), mat(A, 6), None) == ar.AR_ERR_NO_DEVICE


def test_binding_refusals_without_a_gpu():
    x, w, d = torch.zeros(4, 8), torch.zeros(6, 8), ar.Dropout(0.5, 1)
    for call, text in ((lambda: ar.ar_linear_forward(x, w), "x is not on a GPU"),
                       (lambda: ar.ar_linear_forward([1.0], w), "x must be a tensor"),
                       (lambda: ar.ar_linear_forward(x, w, activation="tanh"), "one of none, relu"),
                       (lambda: ar.ar_linear_forward(x, w, out_dtype=torch.int32), "float32, float16 or bfloat16"),
                       (lambda: ar.ar_linear_backward(x, x, w), "dy is not on a GPU"),
                       (lambda: ar.ar_linear_backward(x, x, w, dw_dtype=torch.float64), "float32, float16 or bfloat16"),
                       (lambda: ar.ar_dropout_forward(x, d), "x is not on a GPU"),
                       (lambda: ar.ar_dropout_backward(x, d), "x is not on a GPU")):
        with pytest.raises(ar.ArError, match=text):
            call()


def test_tensors_that_require_a_gradient():
    """The forward calls refuse them while torch records, and go on to the next check where it does not; the gradients' calls
    take them."""
    x, w, b, r = (torch.zeros(s, requires_grad=True) for s in ((4, 8), (6, 8), (6,), (4, 6)))
    d = ar.Dropout(0.5, 1)
    plain = x.detach()
    for call, name in ((lambda: ar.ar_linear_forward(x, w), "x"), (lambda: ar.ar_linear_forward(plain, w), "w"),
                       (lambda: ar.ar_dropout_forward(x, d), "x")):
        with pytest.raises(ar.ArError, match=name + " requires a gradient"):
            call()
        with torch.no_grad(), pytest.raises(ar.ArError, match="not on a GPU"):
            call()
        with torch.inference_mode(), pytest.raises(ar.ArError, match="not on a GPU"):
            call()
    for call in (lambda: ar.ar_linear_backward(r, x, w), lambda: ar.ar_dropout_backward(x, d)):
        with pytest.raises(ar.ArError, match="not on a GPU"):
            call()


def test_negated_views_are_refused():
    """The imaginary part of a conjugate is a view of the number's memory, to be read with its sign turned."""
    t = torch.imag(torch.ones(4, 1, dtype=torch.complex64).conj())
    assert t.is_neg() and t.dtype == torch.float32
    for call in (lambda: ar.ar_linear_forward(t, torch.zeros(6, 1)), lambda: ar.ar_dropout_forward(t, ar.Dropout(0.5, 1)),
                 lambda: ar.ar_linear_backward(t, torch.zeros(4, 2), torch.zeros(1, 2))):
        with pytest.raises(ar.ArError, match="negated view"):
            call()


def test_plans_take_rank_buffer_types_only():
    h = ctypes.c_void_p()
    for code in (F16, BF16):
        assert ar.lib.ar_plan_create(4, 10, code, ar.AR_SUM, 4, ctypes.byref(h)) == UNSUPPORTED
