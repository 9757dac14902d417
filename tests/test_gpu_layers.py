"""The layer operators on the GPU against their definitions in 64 bits
(layer_reference.py): sizes that end inside tiles, batches and 16-byte pieces,
every type, rows at any distance and address, activations, dropout, gradients
(against the formulas and against differences), streams, graphs, NaN and
infinities."""
import math

import pytest
import torch

import layer_reference as ref
from paper_2004_09362_amd import ar

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
TYPES = [torch.bfloat16, torch.float16, torch.float32]
IDS = ["bf16", "f16", "f32"]


def matrix(g, rows, cols, dtype, std=1.0, pad=0, shift=0):
    """rows x cols normal numbers, `pad` elements between rows, the first `shift` elements after an aligned address."""
    t = torch.empty(rows * (cols + pad) + shift + 8, dtype=torch.float32).normal_(0, std, generator=g).to(dtype).to(DEV)
    return t[shift:shift + rows * (cols + pad)].view(rows, cols + pad)[:, :cols]


def seeded(*key):
    return torch.Generator().manual_seed(hash(key) & 0x7FFFFFFF)


# rows, columns, inner length: one of everything, the few-row kernel's three sizes and its edges, tiles of
# 128, whole and ragged, inner lengths that end inside a chunk, a tile, or split over workgroups
SIZES = [(1, 1, 1), (1, 130, 77), (3, 16, 512), (16, 33, 64), (17, 48, 1000), (33, 70, 129), (64, 200, 96), (65, 64, 64),
         (128, 128, 128), (129, 257, 65), (200, 72, 1031), (257, 130, 40), (300, 136, 4096), (1, 24, 9000)]


@pytest.mark.parametrize("dtype", TYPES, ids=IDS)
@pytest.mark.parametrize("size", SIZES, ids=lambda s: "x".join(map(str, s)))
def test_forward(size, dtype):
    M, N, K = size
    g = seeded(1, M, N, K)
    for pad, shift, act, d, out in ((0, 0, "none", None, dtype), (8, 0, "gelu", None, torch.float32),
                                    (3, 1, "silu", (0.3, 99, 4, 1 << 33), dtype),
                                    (0, 0, "gelu_tanh", (0.125, (1 << 63) + 5, 0, 7), dtype), (1, 0, "relu", None, dtype)):
        print("[gpu] forward", size, dtype, pad, shift, act, flush=True)
        x, w = matrix(g, M, K, dtype, pad=pad, shift=shift), matrix(g, N, K, dtype, K ** -0.5, pad, shift)
        bias = matrix(g, 1, N, torch.float32 if act == "silu" else dtype)[0] if act != "none" else None
        res = matrix(g, M, N, out, pad=pad) if act in ("silu", "gelu_tanh") else None
        keep = act != "none"
        got = ar.ar_linear_forward(x, w, bias, res, activation=act, dropout=d and ar.Dropout(*d), out_dtype=out,
                                   preact=keep or None)
        y, z = got if keep else (got, None)
        wy, wz, off, off_z = ref.forward(x, w, bias, res, act, d)
        assert y.dtype == out and y.shape == (M, N)
        ref.close(y, wy, off, "y")
        if keep:
            assert z.dtype == dtype
            ref.close(z, wz, off_z, "z")


@pytest.mark.parametrize("dtype", TYPES, ids=IDS)
def test_forward_large_tiles(dtype):
    """Enough tiles of 256 x 256 that the large shape runs, the last ones ragged in rows, columns and inner length."""
    M, N, K = 256 * 15 + 40, 256 * 13 - 24, 200
    g = seeded(2, M, N)
    x, w = matrix(g, M, K, dtype), matrix(g, N, K, dtype, K ** -0.5)
    bias, res = matrix(g, 1, N, dtype)[0], matrix(g, M, N, dtype)
    d = (0.2, 12345, 1, 0)
    y, z = ar.ar_linear_forward(x, w, bias, res, activation="gelu", dropout=ar.Dropout(*d), preact=True)
    wy, wz, off, off_z = ref.forward(x, w, bias, res, "gelu", d)
    ref.close(y, wy, off, "y")
    ref.close(z, wz, off_z, "z")


BACK = [(1, 1, 1), (5, 64, 64), (16, 40, 24), (63, 65, 130), (128, 128, 128), (130, 264, 72), (257, 96, 1000), (1500, 136, 64),
        (4096, 64, 80), (70, 2100, 33)]


@pytest.mark.parametrize("dtype", TYPES, ids=IDS)
@pytest.mark.parametrize("size", BACK, ids=lambda s: "x".join(map(str, s)))
def test_backward(size, dtype):
    M, N, K = size
    g = seeded(3, M, N, K)
    for pad, shift, act, d, dw_dtype in ((0, 0, "none", None, torch.float32), (8, 0, "gelu", None, dtype),
                                         (3, 1, "silu", (0.25, 7, 1, 3), dtype),
                                         (0, 0, "none", (0.5, 1 << 40, 0, 0), torch.float32), (0, 0, "relu", None, dtype),
                                         (0, 0, "gelu_tanh", None, dtype)):
        print("[gpu] backward", size, dtype, pad, shift, act, flush=True)
        dy, x = matrix(g, M, N, dtype, 0.1, pad, shift), matrix(g, M, K, dtype, pad=pad, shift=shift)
        w = matrix(g, N, K, dtype, K ** -0.5, pad, shift)
        z = matrix(g, M, N, dtype, pad=pad) if act != "none" else None
        dx, dw, db = ar.ar_linear_backward(dy, x, w, preact=z, activation=act, dropout=d and ar.Dropout(*d),
                                           dw_dtype=dw_dtype)
        want = ref.backward(dy, x, w, z, act, d)
        assert dx.dtype == dtype and dw.dtype == dw_dtype and db.dtype == dw_dtype
        for name, t in (("dx", dx), ("dw", dw), ("db", db)):
            ref.close(t, want[name][0], want[name][1], name)


@pytest.mark.parametrize("dtype", TYPES, ids=IDS)
def test_backward_large_tiles(dtype):
    """Products of 256 x 256 tiles in the gradient's two layouts, ragged at their ends."""
    M, N, K = 3400, 3592, 3856
    g = seeded(4, M, N, K)
    dy, x, w = matrix(g, M, N, dtype, 0.1), matrix(g, M, K, dtype), matrix(g, N, K, dtype, K ** -0.5)
    dx, dw, db = ar.ar_linear_backward(dy, x, w, dx_dtype=torch.float32, dw_dtype=torch.float32)
    rows = torch.randint(0, 3400, (40,), generator=g)  # the 64-bit products of some rows
    X, W, D = x.double().cpu(), w.double().cpu(), dy.double().cpu()
    ref.close(dx[rows.to(DEV)], D[rows] @ W, (N + 8) * ref.E32 * (D[rows].abs() @ W.abs()), "dx")
    Dt = D.t()[rows]
    ref.close(dw[rows.to(DEV)], Dt @ X, (M + 8) * ref.E32 * (Dt.abs() @ X.abs()), "dw")
    for t, w_, off in ((dx[-70:], D[-70:] @ W, (N + 8) * ref.E32 * (D[-70:].abs() @ W.abs())),
                       (dw[-70:], D.t()[-70:] @ X, (M + 8) * ref.E32 * (D.t()[-70:].abs() @ X.abs()))):
        ref.close(t, w_, off, "last rows")
    ref.close(db, D.sum(0), (M + 8) * ref.E32 * D.abs().sum(0), "db")


@pytest.mark.parametrize("dtype", TYPES, ids=IDS)
def test_backward_parts_and_accumulation(dtype):
    """Each gradient by itself, a wider dy, and dw and db added to gradient buffers that are views of one vector."""
    M, N, K = 150, 72, 88
    g = seeded(5, 1)
    dy, x, w = matrix(g, M, N, torch.float32, 0.1), matrix(g, M, K, dtype), matrix(g, N, K, dtype, K ** -0.5)
    want = ref.backward(dy, x, w)
    for i, name in enumerate(("dx", "dw", "db")):
        got = ar.ar_linear_backward(dy, x, w, dx=i == 0, dw=i == 1, db=i == 2)
        assert [t is None for t in got] == [j != i for j in range(3)]
        ref.close(got[i], want[name][0], want[name][1], name)
    flat = torch.full((N * K + N + 3,), 0.5, device=DEV)
    dw, db = flat[:N * K].view(N, K), flat[N * K:N * K + N]
    for times in (1, 2):
        got = ar.ar_linear_backward(dy, x, w, dx=False, dw=dw, db=db, accumulate=True)
        assert got[1].data_ptr() == dw.data_ptr()
        for t, name in ((dw, "dw"), (db, "db")):
            ref.close(t, 0.5 + times * want[name][0], times * want[name][1] + 4 * times * ref.E32 * (1 + times * want[name][0].abs()), name)
    assert bool((flat[-3:] == 0.5).all())


def test_gradient_against_differences():
    """The gradient in float32 against differences of the forward pass along random directions.  The sum of
    y * c is smooth here (gelu; the mask is fixed), with y off by about 1e-6 of its unit size in 2500 elements: a
    difference with step h is off by about 1e-6 * sqrt(2500) / h = 5e-3 at h = 1e-2, on derivatives of about
    sqrt(2500) = 50.  Unit steps of the weights move z by sqrt(40) each, so the error of a two-point difference,
    h^2 / 6 of the third derivative, would reach 0.7; the four-point one's, of order h^4, is 5e-3."""
    M, N, K = 50, 50, 40
    g = seeded(6, 6)
    x, w = matrix(g, M, K, torch.float32), matrix(g, N, K, torch.float32, K ** -0.5)
    b, c = matrix(g, 1, N, torch.float32, 0.1)[0], matrix(g, M, N, torch.float32)
    d = ar.Dropout(0.25, 4711, 2)

    def loss(x, w, b):
        return float((ar.ar_linear_forward(x, w, b, activation="gelu", dropout=d).double() * c.double()).sum())

    z = ar.ar_linear_forward(x, w, b, activation="gelu", dropout=d, preact=True)[1]
    grads = ar.ar_linear_backward(c, x, w, preact=z, activation="gelu", dropout=d)
    h = 1e-2
    for i, t in enumerate((x, w, b)):
        v = torch.empty(t.shape).normal_(generator=g).to(DEV)
        v = v * math.sqrt(t.numel()) / v.norm() * (1 if i else 0.3)
        args = [x, w, b]
        at = {}
        for k in (-2, -1, 1, 2):
            args[i] = t + k * h * v
            at[k] = loss(*args)
        diff = (8 * (at[1] - at[-1]) - (at[2] - at[-2])) / (12 * h)
        got = float((grads[i].double() * v.double()).sum())
        assert abs(diff - got) < 0.1 + 5e-3 * abs(got), (i, got, diff)


@pytest.mark.parametrize("dtype", TYPES, ids=IDS)
@pytest.mark.parametrize("out", TYPES, ids=IDS)
def test_dropout(dtype, out):
    for rows, cols, pad, shift, d in ((1, 1, 0, 0, (0.5, 1, 0, 0)), (3, 17, 1, 1, (0.3, 2, 3, 0)),
                                      (5, 4099, 0, 0, (0.1, 3 << 40, 1, (1 << 32) - 2)), (70, 256, 8, 0, (0.9, 5, 0, 0)),
                                      (1000, 8, 0, 0, (0.01, 6, 7, 8))):
        g = seeded(7, rows, cols)
        x, r = matrix(g, rows, cols, dtype, pad=pad, shift=shift), matrix(g, rows, cols, out, pad=pad)
        y = ar.ar_dropout_forward(x, ar.Dropout(*d), r, out_dtype=out)
        want = ref.drop(x.double().cpu(), d)
        ref.close(y, want + r.double().cpu(), 4 * ref.E32 * (want.abs() + r.double().cpu().abs()), "y")
        dx = ar.ar_dropout_backward(x, ar.Dropout(*d), out_dtype=out)
        ref.close(dx, want, 4 * ref.E32 * want.abs(), "dx")
        assert torch.equal(dx.cpu() != 0, (want != 0) & (dx.cpu() != 0)) and int((dx != 0).sum()) >= int((want != 0).sum()) - 1


def test_mask_is_a_function_of_the_place():
    """The linear layer draws dropout's mask; rows of a part draw the whole's; sites and seeds differ; the share kept is 1 - p."""
    rows, cols = 512, 768
    ones = torch.ones(rows, cols, device=DEV)
    d = ar.Dropout(0.3, 77, 5)
    whole = ar.ar_dropout_forward(ones, d)
    assert torch.equal(whole.cpu() != 0, ref.keep_mask(rows, cols, *d))
    part = ar.ar_dropout_forward(ones[200:300], d._replace(row0=200))
    assert torch.equal(part, whole[200:300])
    x, w = torch.ones(rows, 1, device=DEV), torch.ones(cols, 1, device=DEV)
    assert torch.equal(ar.ar_linear_forward(x, w, dropout=d), whole)
    assert torch.equal(ar.ar_linear_forward(x[:20], w, dropout=d), whole[:20])  # the few-row kernel
    for other in (d._replace(seed=78), d._replace(seed=77 + (1 << 32)), d._replace(site=6), d._replace(row0=rows)):
        same = float((ar.ar_dropout_forward(ones, other) == whole).float().mean())
        assert abs(same - (0.7 ** 2 + 0.3 ** 2)) < 6 * 0.5 / math.sqrt(rows * cols)
    kept = float((whole != 0).double().mean())
    assert abs(kept - 0.7) < 6 * math.sqrt(0.21 / (rows * cols))


def test_dropout_of_everything_and_of_nothing():
    x = torch.tensor([[1.0, math.inf, math.nan, -3.0, 5.0]], device=DEV)
    assert torch.equal(ar.ar_dropout_forward(x, ar.Dropout(1.0, 3)), torch.zeros_like(x))
    assert torch.equal(ar.ar_dropout_forward(x, ar.Dropout(0.0, 3)).nan_to_num(nan=9), x.nan_to_num(nan=9))
    big = torch.full((64, 64), math.inf, device=DEV)
    y = ar.ar_dropout_forward(big, ar.Dropout(0.5, 3))
    assert not bool(y.isnan().any()) and bool((y == 0).any()) and bool((y == math.inf).any())
    assert torch.equal(y.cpu() == 0, ~ref.keep_mask(64, 64, 0.5, 3))


@pytest.mark.parametrize("rows", [4, 200], ids=["few", "tiles"])
@pytest.mark.parametrize("dtype", TYPES, ids=IDS)
def test_infinities_and_nan_stay_in_their_rows_and_columns(rows, dtype):
    """K ends inside a chunk and M, N inside tiles, so that what lies behind the operands' ends -- here NaN -- must not count."""
    M, N, K, pad = rows, 70, 77, 11
    bufs = [torch.full((r + 1, K + pad), math.nan, dtype=dtype, device=DEV) for r in (M, N)]
    x, w = bufs[0][:M, :K], bufs[1][:N, :K]
    g = seeded(8, rows)
    x.copy_(matrix(g, M, K, dtype))
    w.copy_(matrix(g, N, K, dtype))
    assert bool(ar.ar_linear_forward(x, w).isfinite().all())
    dy = matrix(g, M, N, dtype)
    assert all(bool(t.isfinite().all()) for t in ar.ar_linear_backward(dy, x, w))
    x[2, 5], w[3, 76] = math.inf, math.nan
    y = ar.ar_linear_forward(x, w, activation="relu")
    want = torch.relu(x.double().cpu() @ w.double().cpu().t())
    assert torch.equal(y.isfinite().cpu(), want.isfinite()) and torch.equal(y.isnan().cpu(), want.isnan())


@pytest.mark.parametrize("dtype", TYPES, ids=IDS)
def test_empty_sizes(dtype):
    z = lambda r, c: torch.zeros(r, c, dtype=dtype, device=DEV)  # noqa: E731
    assert ar.ar_linear_forward(z(0, 5), z(4, 5)).shape == (0, 4)
    assert ar.ar_linear_forward(z(3, 5), z(0, 5)).shape == (3, 0)
    bias, res = torch.arange(4, device=DEV).to(dtype), torch.ones(100, 4, dtype=dtype, device=DEV)
    for M in (3, 100):  # an inner length of 0: a sum of nothing, then the epilogue
        y = ar.ar_linear_forward(z(M, 0), z(4, 0), bias, res[:M])
        assert torch.equal(y, (bias + res[:M]))
    dx, dw, db = ar.ar_linear_backward(z(0, 4), z(0, 5), z(4, 5))
    assert dx.shape == (0, 5) and not dw.any() and not db.any() and dw.shape == (4, 5) and db.shape == (4,)
    dx, dw, db = ar.ar_linear_backward(z(3, 0), z(3, 5), z(0, 5))
    assert dx.shape == (3, 5) and not dx.any() and dw.shape == (0, 5) and db.shape == (0,)
    assert ar.ar_dropout_forward(z(0, 7), ar.Dropout(0.5, 1)).shape == (0, 7)


@pytest.mark.parametrize("dtype", TYPES, ids=IDS)
def test_in_place_and_columns_of_a_wider_matrix(dtype):
    """y onto its residual, dropout onto its input, and operands that are columns of one matrix."""
    M, N, K = 140, 96, 64
    g = seeded(9, 9)
    wide = matrix(g, M, K + N, dtype)
    x, y = wide[:, :K], wide[:, K:]
    w = matrix(g, N, K, dtype, K ** -0.5)
    want = ref.forward(x, w, None, y)
    x0 = x.clone()
    got = ar.ar_linear_forward(x, w, None, y, out=y)
    assert got.data_ptr() == y.data_ptr() and torch.equal(x, x0)
    ref.close(y, want[0], want[2], "y")
    d = (0.4, 8, 0, 0)
    want = ref.drop(x.double().cpu(), d)
    ar.ar_dropout_forward(x, ar.Dropout(*d), out=x)
    ref.close(x, want, 4 * ref.E32 * want.abs(), "x")


def test_rows_further_apart_than_32_bits():
    """Offsets past 2^32 bytes: rows 2^29 elements apart."""
    if torch.cuda.mem_get_info()[0] < 24 << 30:
        pytest.skip("needs 20 GB")
    ld = 1 << 29
    buf = torch.empty(4 * ld + 256, dtype=torch.bfloat16, device=DEV)
    x = buf.as_strided((5, 200), (ld, 1))
    g = seeded(10, 10)
    x.copy_(matrix(g, 5, 200, torch.bfloat16))
    w = matrix(g, 72, 200, torch.bfloat16)
    want = ref.forward(x, w)
    ref.close(ar.ar_linear_forward(x, w), want[0], want[2], "few rows")
    want = ref.forward(w, x)
    ref.close(ar.ar_linear_forward(w, x), want[0], want[2], "tiles")
    dy = matrix(g, 5, 72, torch.bfloat16)
    back = ref.backward(dy, x, w)
    for t, name in zip(ar.ar_linear_backward(dy, x, w), ("dx", "dw", "db")):
        ref.close(t, back[name][0], back[name][1], name)
    d = (0.5, 1, 0, 0)
    want = ref.drop(x.double().cpu(), d)
    ref.close(ar.ar_dropout_forward(x, ar.Dropout(*d)), want, 4 * ref.E32 * want.abs(), "dropout")


def test_results_do_not_depend_on_timing():
    """The same call gives the same bits, alone and next to other work, where the inner length is split over workgroups."""
    g = seeded(11, 11)
    cases = [(4, 64, 8192), (256, 128, 8192)]
    made = [(matrix(g, M, K, torch.bfloat16), matrix(g, N, K, torch.bfloat16), matrix(g, M, N, torch.bfloat16)) for M, N, K in cases]
    first = [(ar.ar_linear_forward(x, w), ar.ar_linear_backward(dy, x, w, dw_dtype=torch.float32)) for x, w, dy in made]
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    for _ in range(5):
        with torch.cuda.stream(s):
            other = [ar.ar_linear_forward(w, w) for x, w, dy in made]
        for (x, w, dy), (y, grads) in zip(made, first):
            assert torch.equal(ar.ar_linear_forward(x, w), y)
            for a, b in zip(ar.ar_linear_backward(dy, x, w, dw_dtype=torch.float32), grads):
                assert torch.equal(a, b)
    torch.cuda.synchronize()
    assert other


def test_stream_argument():
    """Work goes to the stream that is given, in its order, and so does the memory of the results."""
    g = seeded(12, 12)
    x, w = matrix(g, 300, 512, torch.bfloat16), matrix(g, 256, 512, torch.bfloat16)
    want = ar.ar_linear_forward(x, w, activation="gelu")
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    for handle in (s, s.cuda_stream):
        x2 = torch.zeros_like(x)
        torch.cuda.synchronize()
        with torch.cuda.stream(s):
            torch.cuda._sleep(20_000_000)
            x2.copy_(x)
        y = ar.ar_linear_forward(x2, w, activation="gelu", stream=handle)
        z = ar.ar_dropout_forward(y, ar.Dropout(0.0, 1), stream=handle)
        s.synchronize()
        assert torch.equal(y, want) and torch.equal(z, want)


def test_graph_capture_and_replay():
    """A forward and backward pass captured once and replayed on new inputs, with other work between the replays."""
    g = seeded(13, 13)
    M, N, K = 192, 256, 4096  # split over workgroups: the workspace is in the graph's memory
    x, w = torch.zeros(M, K, dtype=torch.bfloat16, device=DEV), matrix(g, N, K, torch.bfloat16, K ** -0.5)
    dy, dw, db = torch.zeros(M, N, dtype=torch.bfloat16, device=DEV), torch.zeros(N, K, device=DEV), torch.zeros(N, device=DEV)
    d = ar.Dropout(0.1, 3)

    def step():
        y, z = ar.ar_linear_forward(x, w, activation="silu", dropout=d, preact=True)
        dx, _, _ = ar.ar_linear_backward(dy, x, w, preact=z, activation="silu", dropout=d, dw=dw, db=db)
        return y, dx

    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        with torch.cuda.graph(graph, stream=s):
            y, dx = step()
    for _ in range(3):
        x.copy_(matrix(g, M, K, torch.bfloat16))
        dy.copy_(matrix(g, M, N, torch.bfloat16))
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in (y, dx, dw, db)]
        wy, wdx = step()
        torch.cuda.synchronize()
        for a, b in zip(got, (wy, wdx, dw, db)):
            assert torch.equal(a, b)


def test_c_call_with_raw_addresses():
    """The C entry points with their own structures, a caller's workspace and an explicit stream."""
    import ctypes

    M, N, K = 100, 64, 8192
    g = seeded(14, 14)
    x, w = matrix(g, M, K, torch.float16), matrix(g, N, K, torch.float16, K ** -0.5)
    y = torch.empty(M, N, device=DEV)
    mat = lambda t, code: ctypes.byref(ar.Matrix(t.data_ptr(), t.stride(0), code))  # noqa: E731
    need = ctypes.c_int64()
    assert ar.lib.ar_linear_forward_workspace(M, N, K, mat(x, ar.AR_FLOAT16), mat(w, ar.AR_FLOAT16), ctypes.byref(need)) == ar.AR_OK
    assert need.value > 0
    ws = torch.empty(need.value, dtype=torch.uint8, device=DEV)
    call = lambda size: ar.lib.ar_linear_forward(  # noqa: E731
        M, N, K, mat(x, ar.AR_FLOAT16), mat(w, ar.AR_FLOAT16), None, None, ar.AR_ACT_NONE, None, mat(y, ar.AR_FLOAT32), None,
        ws.data_ptr(), size, torch.cuda.current_stream().cuda_stream)
    assert call(need.value - 1) == ar.AR_ERR_INVALID_ARG and "workspace" in ar.ar_last_error_message()
    assert call(need.value) == ar.AR_OK
    want = ref.forward(x, w)
    ref.close(y, want[0], want[2], "y")


def test_refusals_of_device_tensors():
    """What is wrong with tensors on the GPU is named before anything is launched."""
    x, w = torch.zeros(4, 8, device=DEV), torch.zeros(6, 8, device=DEV)
    wide = torch.zeros(4, 16, device=DEV)
    d = ar.Dropout(0.5, 1)
    for call, text in ((lambda: ar.ar_linear_forward(x, w[:, :7]), "w is 6 x 7"),
                       (lambda: ar.ar_linear_forward(x, w.half()), "wrong type"),
                       (lambda: ar.ar_linear_forward(x.double(), w.double()), "float32, float16 or bfloat16"),
                       (lambda: ar.ar_linear_forward(x.t(), w), "consecutive"),
                       (lambda: ar.ar_linear_forward(x[0], w), "2 dimensions"),
                       (lambda: ar.ar_linear_forward(x, w, torch.zeros(5, device=DEV)), "bias"),
                       (lambda: ar.ar_linear_forward(x, w, None, torch.zeros(4, 6, device=DEV).half()), "residual"),
                       (lambda: ar.ar_linear_forward(x, w, out=torch.zeros(4, 6, device=DEV).half()), "out|y must"),
                       (lambda: ar.ar_linear_forward(wide[:, :8], w, out=wide[:, 7:13]), "overlaps"),
                       (lambda: ar.ar_linear_forward(x, w, out=w[:4, :6]), "overlaps w"),
                       (lambda: ar.ar_linear_forward(x, w, out=x[:1].expand(4, 8)[:, :6]), "overlap"),
                       (lambda: ar.ar_linear_forward(x, w.cpu()), "not on a GPU"),
                       (lambda: ar.ar_linear_backward(x[:, :6], x, w, activation="gelu"), "preact"),
                       (lambda: ar.ar_linear_backward(x[:, :6], x, w, accumulate=True), "accumulate"),
                       (lambda: ar.ar_linear_backward(x[:, :6], x, w, dx=x), "overlaps"),
                       (lambda: ar.ar_dropout_forward(x, d, out=wide[:, 1:9][:, :7]), "out is 4 x 7"),
                       (lambda: ar.ar_dropout_forward(wide[:, :8], d, out=wide[:, 4:12]), "overlaps"),
                       (lambda: ar.ar_dropout_forward(x, ar.Dropout(1.5, 1)), "p must be"),
                       (lambda: ar.ar_dropout_forward(x, None), "drop is NULL")):
        with pytest.raises(ar.ArError, match=text):
            call()
    torch.cuda.synchronize()
    assert not x.any() and not w.any() and not wide.any()


@pytest.mark.parametrize("dtype", TYPES, ids=IDS)
@pytest.mark.parametrize("out32", [False, True], ids=["same", "f32"])
def test_every_end_of_a_row(dtype, out32):
    """Rows that end after each number of columns of the last group of 8, or are shorter than one, in place on the residual
    and between columns that must stay as they are: whole and split products, the gradient, and dropout."""
    out = torch.float32 if out32 else dtype
    for N in (1, 3, 5, 7, 8, 9, 10, 11, 12, 13, 14, 15, 16, 21):
        g = seeded(20, N)
        for M, K in ((70, 40), (66, 2500)):
            print("[gpu] row ends", dtype, out, M, N, K, flush=True)
            x, w, bias = matrix(g, M, K, dtype), matrix(g, N, K, dtype, K ** -0.5), matrix(g, 1, N, dtype)[0]
            wide = matrix(g, M, N + 5, out)
            before, y = wide.clone(), wide[:, 2:N + 2]
            d = (0.25, 5, 6, 7)
            wy, wz, off, off_z = ref.forward(x, w, bias, before[:, 2:N + 2], "silu", d)
            got, z = ar.ar_linear_forward(x, w, bias, y, activation="silu", dropout=ar.Dropout(*d), out=y, preact=True)
            ref.close(got, wy, off, "y")
            ref.close(z, wz, off_z, "z")
            assert torch.equal(wide[:, :2], before[:, :2]) and torch.equal(wide[:, N + 2:], before[:, N + 2:])
        M, K = 45, N + 2
        dy, x, w, z = matrix(g, M, N, dtype, 0.1), matrix(g, M, K, dtype), matrix(g, N, K, dtype, 0.3), matrix(g, M, N, dtype)
        want = ref.backward(dy, x, w, z, "gelu", d)
        for name, t in zip(("dx", "dw", "db"), ar.ar_linear_backward(dy, x, w, preact=z, activation="gelu",
                                                                     dropout=ar.Dropout(*d), dw_dtype=out)):
            ref.close(t, want[name][0], want[name][1], name)
        wide = matrix(g, 50, N + 3, dtype)
        before, v = wide.clone(), wide[:, 1:N + 1]
        ar.ar_dropout_backward(v, ar.Dropout(*d), out=v)
        kept = ref.drop(before[:, 1:N + 1].double().cpu(), d)
        ref.close(v, kept, 4 * ref.E32 * kept.abs(), "dropped")
        assert torch.equal(wide[:, :1], before[:, :1]) and torch.equal(wide[:, N + 1:], before[:, N + 1:])


@pytest.mark.parametrize("dtype", TYPES[:2], ids=IDS[:2])
def test_forward_large_tiles_to_float32(dtype):
    """256 x 256 tiles with a residual and results of 32 bits, in place, with every stage and with the residual alone."""
    M, N, K = 256 * 15 + 8, 256 * 13 + 40, 136
    g = seeded(21, M, N)
    x, w, bias, r = matrix(g, M, K, dtype), matrix(g, N, K, dtype, K ** -0.5), matrix(g, 1, N, dtype)[0], matrix(g, M, N, torch.float32)
    d = (0.1, 9, 8, 1 << 40)
    for act, drop in (("silu", d), ("none", None)):
        wy, wz, off, _ = ref.forward(x, w, bias, r, act, drop)
        y = r.clone()
        ar.ar_linear_forward(x, w, bias, y, activation=act, dropout=drop and ar.Dropout(*drop), out=y)
        ref.close(y, wy, off, act)


@pytest.mark.parametrize("dtype", TYPES, ids=IDS)
def test_backward_products_together(dtype):
    """Gradients of medium size, whose products share a launch, one of them split, added to what is there."""
    for M, N, K in ((6100, 1000, 1032), (2048, 1280, 768), (700, 2050, 515)):
        print("[gpu] products together", dtype, M, N, K, flush=True)
        g = seeded(22, M)
        dy, x, w = matrix(g, M, N, dtype, 0.1), matrix(g, M, K, dtype), matrix(g, N, K, dtype, K ** -0.5)
        want = ref.backward(dy, x, w)
        dw, db = matrix(g, N, K, torch.float32), matrix(g, 1, N, torch.float32)[0]
        before = {"dw": dw.clone().double().cpu(), "db": db.clone().double().cpu()}
        dx, _, _ = ar.ar_linear_backward(dy, x, w, dw=dw, db=db, accumulate=True)
        ref.close(dx, want["dx"][0], want["dx"][1], "dx")
        for name, t in (("dw", dw), ("db", db)):
            sum_ = before[name] + want[name][0]
            ref.close(t, sum_, want[name][1] + 4 * ref.E32 * (before[name].abs() + want[name][0].abs()), name)
