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


def extremes(dtype):
    big = [6e4, 65504.0] if dtype == torch.float16 else [1e4, 1.8e19, 2e19, 1e20, 1e30, 3e38]
    return torch.tensor([0.0, 1.0, -1.0, 30.0, -30.0, 300.0, -300.0] + big + [-v for v in big] + [math.inf, -math.inf, math.nan])


def act_far_out(z, act):
    """The activations in 64 bits, in forms that stay finite for finite z; at -inf they are -inf * 0."""
    if act == "relu":
        return torch.where(z > 0, z, 0.0 * z.nan_to_num(posinf=0, neginf=0, nan=math.nan))
    if act == "gelu":
        return z * torch.special.ndtr(z)
    u = z if act == "silu" else 2 * math.sqrt(2 / math.pi) * (z + 0.044715 * z ** 3)
    return z * torch.sigmoid(u)


def slope_far_out(z, act):
    """Their slopes: at infinities inf * 0, but for relu's, which is 0 at NaN too."""
    if act == "relu":
        return (z > 0).double()
    if act == "gelu":
        return torch.special.ndtr(z) + z * torch.exp(-z * z / 2) / math.sqrt(2 * math.pi)
    u, du = (z, torch.ones_like(z)) if act == "silu" else (2 * math.sqrt(2 / math.pi) * (z + 0.044715 * z ** 3),
                                                         2 * math.sqrt(2 / math.pi) * (1 + 0.134145 * z ** 2))
    s = torch.sigmoid(u)
    return s + z * s * (1 - s) * du


def agree(got, want, where):
    """NaN and infinities in the same places; elsewhere the size of the rounding, and of the activation's evaluation."""
    g, w = got.double().cpu(), want
    u = ref.U[got.dtype]
    w = torch.where(w.abs() > torch.finfo(got.dtype).max, w.sign() * math.inf, w)
    assert torch.equal(g.isnan(), w.isnan()), (where, g, w)
    assert torch.equal(g.isinf(), w.isinf()) and torch.equal(g.sign()[g.isinf()], w.sign()[w.isinf()]), (where, g, w)
    ok = w.isfinite()
    assert bool(((g - w).abs()[ok] <= (u + 2.0 ** -22) * w.abs()[ok] + 2.0 ** -20).all()), (where, g, w)


@pytest.mark.parametrize("act", ["relu", "gelu", "gelu_tanh", "silu"])
@pytest.mark.parametrize("dtype", TYPES, ids=IDS)
def test_activations_at_infinities_and_far_out(dtype, act):
    """Every kernel that applies an activation: of few rows, of tiles (at a matrix' edge, whole ones, through 16-byte
    boundaries and not), and the join of a split product."""
    v = extremes(dtype)
    z1 = v.to(dtype)
    for M, N, K, pad in ((len(v), 1, 1, 0), (1, len(v), 1, 0), (len(v), 70, 1, 3), (200, 130, 1, 0), (200, 136, 8, 0), (len(v), 24, 9000, 0),
                         (256 * 15 + 40, 256 * 13 - 24, 200, 0)):
        print("[gpu] far out", dtype, act, M, N, K, flush=True)
        x = torch.zeros(M, K + pad, dtype=dtype)[:, :K]
        w = torch.zeros(N, K + pad, dtype=dtype)[:, :K]
        if M == 1:  # a row of values
            x[:, 0] = 1
            w[:, 0] = z1
        else:
            x[:, 0] = z1[torch.arange(M) % len(v)]
            w[:, 0] = 1
        x, w = x.to(DEV), w.to(DEV)
        y, z = ar.ar_linear_forward(x, w, activation=act, preact=True)
        want = z1.double() if M == 1 else z1.double()[torch.arange(M) % len(v)][:, None].expand(M, N)
        if K > 1:  # the zeros of w make an infinity's row NaN only where they meet it, which is nowhere
            assert torch.equal(z.cpu().isnan(), want.reshape(M, N).isnan())
        agree(y, act_far_out(want.reshape(M, N), act), (M, N, K))


@pytest.mark.parametrize("act", ["relu", "gelu", "gelu_tanh", "silu"])
@pytest.mark.parametrize("dtype", TYPES, ids=IDS)
def test_slopes_at_infinities_and_far_out(dtype, act):
    """db of one row is the slope in 32 bits; dx of one column is it in the operands' type; rows of 8 columns and shorter ones."""
    v = extremes(dtype)
    z1 = v.to(dtype)
    want = slope_far_out(z1.double(), act)
    row = z1[None].to(DEV)
    _, _, db = ar.ar_linear_backward(torch.ones_like(row), torch.ones(1, 1, dtype=dtype, device=DEV),
                                     torch.ones(len(v), 1, dtype=dtype, device=DEV), preact=row, activation=act, dx=False, dw=False,
                                     dw_dtype=torch.float32)
    agree(db, want, "db")
    for i in range(0, len(v), 5):  # rows shorter than 8
        _, _, db = ar.ar_linear_backward(torch.ones(1, 5, dtype=dtype, device=DEV)[:, :len(v) - i], torch.ones(1, 1, dtype=dtype, device=DEV),
                                         torch.ones(min(5, len(v) - i), 1, dtype=dtype, device=DEV), preact=row[:, i:i + 5], activation=act,
                                         dx=False, dw=False, dw_dtype=torch.float32)
        agree(db, want[i:i + 5], "db of short rows")
    column = z1[:, None].to(DEV)
    dx, _, _ = ar.ar_linear_backward(torch.ones_like(column), column, torch.ones(1, 1, dtype=dtype, device=DEV), preact=column,
                                     activation=act, dw=False, db=False)
    agree(dx[:, 0], want, "dx")


def test_gelu_in_float32_is_good_to_its_value():
    """gelu's negative side is a tail of the normal distribution times z, and its results are small: the error is bounded
    by the result, not by 1.  The tail is a polynomial fitted to 1 unit of 2^-24, with its coefficients' roundings and eight
    multiply-adds of partly alternating terms (3), a reciprocal of 2 that enters 1.5-fold (3), an exponential of 2 with a
    corrected exponent (1) and three products (1.5): 12 units, and 16 = 2^-20 allowed.  The slope adds z times the density,
    within 1.13 in all: 2^-20 of 1."""
    n = 1 << 18
    z = torch.linspace(-12.0, 12.0, n, device=DEV)
    y = ar.ar_linear_forward(z[:, None], torch.ones(1, 1, device=DEV), activation="gelu")[:, 0]
    zz = z.double()
    tail = torch.special.erfc(-zz / math.sqrt(2)) / 2
    worst = ((y.double() - zz * tail).abs() / (zz * tail).abs()).max()
    assert float(worst) <= 2.0 ** -20, float(worst) * 2 ** 24
    few = ar.ar_linear_forward(z[:64, None], torch.ones(1, 1, device=DEV), activation="gelu")[:, 0]
    assert torch.equal(few, y[:64])
    _, _, db = ar.ar_linear_backward(torch.ones(1, n, device=DEV), torch.ones(1, 1, device=DEV), torch.ones(n, 1, device=DEV),
                                     preact=z[None], activation="gelu", dx=False, dw=False)
    want = tail + zz * torch.exp(-zz * zz / 2) / math.sqrt(2 * math.pi)
    assert float((db.double() - want).abs().max()) <= 2.0 ** -20


@pytest.mark.parametrize("dtype", TYPES[:2], ids=IDS[:2])
def test_gelu_of_16_bits_is_good_to_its_value(dtype):
    """From operands of 16 bits the tail is good to 6e-5 of itself and 60 units of 2^-24 (its exponent's rounding at z = -9),
    7e-5 together, and the result is rounded once; below 16 bits' normal numbers by half their smallest step."""
    z = torch.linspace(-9.0, 9.0, 1 << 16, device=DEV).to(dtype)
    zz = z.double()
    want = zz * torch.special.erfc(-zz / math.sqrt(2)) / 2
    one = torch.ones(1, 1, dtype=dtype, device=DEV)
    y = ar.ar_linear_forward(z[:, None], one, activation="gelu")[:, 0].double()
    step = 2.0 ** -25 if dtype == torch.float16 else 2.0 ** -134
    assert bool(((y - want).abs() <= (ref.U[dtype] * (1 + 7e-5) + 7e-5) * want.abs() + step).all())
    y = ar.ar_linear_forward(z[:, None], one, activation="gelu", out_dtype=torch.float32)[:, 0].double()
    assert bool(((y - want).abs() <= 7e-5 * want.abs()).all())


def test_the_widest_matrices():
    """Column counts at which a launch with a thread for each piece of a row would pass 2^32 threads: the bias' gradient, the
    two kernels of few rows and, beyond their widths, tiles."""
    if torch.cuda.mem_get_info()[0] < 40 << 30:
        pytest.skip("needs 30 GB")
    n = (1 << 28) + 21
    dy = torch.empty(1, n, dtype=torch.bfloat16, device=DEV).normal_()
    one = torch.ones(1, 1, dtype=torch.bfloat16, device=DEV)
    w = torch.empty(n, 1, dtype=torch.bfloat16, device=DEV)
    print("[gpu] db", n, flush=True)
    _, _, db = ar.ar_linear_backward(dy, one, w, dx=False, dw=False)
    assert torch.equal(db, dy[0])
    got = torch.ones(n, dtype=torch.float32, device=DEV)
    ar.ar_linear_backward(dy, one, w, dx=False, dw=False, db=got, accumulate=True)
    assert torch.equal(got[:10000], 1 + dy[0, :10000].float()) and torch.equal(got[-10000:], 1 + dy[0, -10000:].float())
    del dy, w, db, got
    torch.cuda.empty_cache()
    for M, N in ((17, (1 << 28) - 64), (17, (1 << 28) + 40), (2, (1 << 30) - 64), (2, 1 << 30)):
        print("[gpu] forward", M, N, flush=True)
        w = torch.empty(N, 8, dtype=torch.bfloat16, device=DEV).normal_()
        x = torch.empty(M, 8, dtype=torch.bfloat16, device=DEV).normal_()
        y = ar.ar_linear_forward(x, w)
        at = torch.cat([torch.arange(200), torch.randint(0, N, (2000,), generator=torch.Generator().manual_seed(1)),
                        torch.arange(N - 200, N)]).to(DEV)
        want = ref.forward(x, w[at])
        ref.close(y[:, at], want[0], want[2], "y")
        del w, y
        torch.cuda.empty_cache()


def test_tensors_that_torch_records():
    """A forward call on a tensor that requires a gradient is refused while torch records and runs where it does not; a custom
    function of the two calls differentiates; what is written in place counts as written."""
    g = torch.Generator().manual_seed(30)
    x, w, b, r = (matrix(g, *s, torch.float32) for s in ((40, 24), (16, 24), (1, 16), (40, 16)))
    b = b[0]
    want = ar.ar_linear_forward(x, w, b, r)
    for i, name in enumerate(("x", "w", "bias", "residual")):
        args = [t.clone().requires_grad_(j == i) for j, t in enumerate((x, w, b, r))]
        with pytest.raises(ar.ArError, match=name + " requires a gradient"):
            ar.ar_linear_forward(*args)
        with torch.no_grad():
            assert torch.equal(ar.ar_linear_forward(*args), want)
    with pytest.raises(ar.ArError, match="out requires a gradient"):
        ar.ar_linear_forward(x, w, b, r, out=torch.zeros(40, 16, device=DEV, requires_grad=True))

    class Linear(torch.autograd.Function):
        @staticmethod
        def forward(ctx, x, w, b):
            y, z = ar.ar_linear_forward(x, w, b, activation="silu", preact=True)
            ctx.save_for_backward(x, w, z)
            return y

        @staticmethod
        def backward(ctx, dy):
            x, w, z = ctx.saved_tensors
            return ar.ar_linear_backward(dy, x, w, preact=z, activation="silu")

    leaves = [t.clone().requires_grad_(True) for t in (x, w, b)]
    c = matrix(g, 40, 16, torch.float32)
    (Linear.apply(*leaves) * c).sum().backward()
    with torch.no_grad():
        z = ar.ar_linear_forward(x, w, b)
        grads = ar.ar_linear_backward(c, *leaves[:2], preact=z, activation="silu")
    for leaf, grad in zip(leaves, grads):
        assert torch.equal(leaf.grad, grad)

    y, z, dx, dw, db, v = (torch.zeros(s, device=DEV) for s in ((40, 16), (40, 16), (40, 24), (16, 24), (16,), (40, 16)))
    before = [t._version for t in (y, z, dx, dw, db, v)]
    ar.ar_linear_forward(x, w, b, out=y, preact=z)
    ar.ar_linear_backward(c, x, w, dx=dx, dw=dw, db=db)
    ar.ar_dropout_forward(c, ar.Dropout(0.5, 1), out=v)
    assert [t._version for t in (y, z, dx, dw, db, v)] == [n + 1 for n in before]
    with torch.inference_mode():
        t = torch.zeros(40, 16, device=DEV)
    ar.ar_linear_forward(x, w, b, r, out=t)
    assert torch.equal(t, want)


def test_no_memory_for_a_result():
    """torch's own error, which programs catch to go on with less."""
    x = torch.ones(1 << 21, 1, dtype=torch.bfloat16, device=DEV)  # 8 TB of results
    with pytest.raises(torch.OutOfMemoryError):
        ar.ar_linear_forward(x, x)
    assert ar.ar_linear_forward(x[:2], x[:3]).shape == (2, 3)
