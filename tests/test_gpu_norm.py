"""Layer norm and its gradient on the GPU against their definitions in 64 bits
(training_reference.py): rows of one column to more than a team of lanes holds,
one row to more than a launch's teams take at once, every type, rows at any
distance and address, columns and rows of very different sizes, gradients
(against the formulas and against differences), in place, streams, graphs, NaN
and infinities."""
import ctypes
import math

import pytest
import torch

import layer_reference as ref
import training_reference as tref
from paper_2004_09362_amd import ar

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
TYPES = [torch.bfloat16, torch.float16, torch.float32]
IDS = ["bf16", "f16", "f32"]


def matrix(g, rows, cols, dtype, std=1.0, mean=0.0, pad=0, shift=0):
    """rows x cols numbers, `pad` elements between rows, the first `shift` elements after an aligned address."""
    t = torch.empty(rows * (cols + pad) + shift + 8, dtype=torch.float32).normal_(mean, std, generator=g).to(dtype).to(DEV)
    return t[shift:shift + rows * (cols + pad)].view(rows, cols + pad)[:, :cols]


def seeded(*key):
    return torch.Generator().manual_seed(hash(key) & 0x7FFFFFFF)


# rows of fewer than 8 columns; teams of 8 to 1024 lanes with one group of columns and with two, whole and ragged; rows
# longer than a team holds; more rows than teams
SIZES = [(1, 1), (3, 2), (40, 7), (2, 8), (9, 9), (4, 63), (7, 64), (33, 65), (6, 130), (300, 256), (3, 511), (130, 512), (5, 513),
         (300, 1000), (4, 1024), (3, 1025), (17, 2047), (2, 2049), (9, 4096), (3, 5001), (5, 8193), (2, 16384), (3, 16385),
         (2, 40000), (1, 70001), (4000, 24), (70000, 9)]


@pytest.mark.parametrize("dtype", TYPES, ids=IDS)
@pytest.mark.parametrize("size", SIZES, ids=lambda s: "x".join(map(str, s)))
def test_forward(size, dtype):
    rows, cols = size
    g = seeded(1, rows, cols)
    for pad, shift, out, wtype, btype in ((0, 0, dtype, torch.float32, dtype), (8, 0, torch.float32, dtype, torch.bfloat16),
                                          (3, 1, torch.bfloat16, torch.float16, None), (1, 0, torch.float16, None, torch.float32)):
        print("[gpu] norm", size, dtype, pad, shift, flush=True)
        x = matrix(g, rows, cols, dtype, 2.0, 0.7, pad, shift)
        w = matrix(g, 1, cols, wtype, mean=1.0, shift=shift)[0] if wtype else None
        b = matrix(g, 1, cols, btype, shift=shift)[0] if btype else None
        y, stats = ar.ar_layer_norm_forward(x, w, b, out_dtype=out, stats=True)
        want = tref.norm(x, w, b)
        assert y.dtype == out and y.shape == (rows, cols) and stats.dtype == torch.float32 and stats.shape == (rows, 2)
        ref.close(y, *want["y"], "y")
        ref.close(stats[:, 0], *want["mean"], "mean")
        ref.close(stats[:, 1], *want["rstd"], "rstd")
        assert torch.equal(ar.ar_layer_norm_forward(x, w, b, out_dtype=out), y)


@pytest.mark.parametrize("dtype", TYPES, ids=IDS)
@pytest.mark.parametrize("size", SIZES, ids=lambda s: "x".join(map(str, s)))
def test_backward(size, dtype):
    rows, cols = size
    g = seeded(2, rows, cols)
    for pad, shift, dytype, wtype, res, dw_dtype in ((0, 0, dtype, torch.float32, True, torch.float32),
                                                     (8, 0, torch.float32, dtype, False, dtype),
                                                     (3, 1, torch.bfloat16, torch.float16, True, torch.float16),
                                                     (1, 0, torch.float16, None, False, torch.bfloat16)):
        print("[gpu] norm gradient", size, dtype, pad, shift, flush=True)
        x, dy = matrix(g, rows, cols, dtype, 2.0, 0.7, pad, shift), matrix(g, rows, cols, dytype, 0.1, 0.0, pad, shift)
        w = matrix(g, 1, cols, wtype, mean=1.0, shift=shift)[0] if wtype else None
        r = matrix(g, rows, cols, dtype, 0.1, 0.0, pad) if res else None
        stats = ar.ar_layer_norm_forward(x, stats=True)[1]
        dx, dw, db = ar.ar_layer_norm_backward(dy, x, stats, w, residual=r, dw_dtype=dw_dtype)
        want = tref.norm_grad(dy, x, stats, w, r)
        assert dx.dtype == dtype and dw.dtype == dw_dtype and db.dtype == dw_dtype
        for name, t in (("dx", dx), ("dw", dw), ("db", db)):
            ref.close(t, *want[name], name)


@pytest.mark.parametrize("cols", [96, 1024, 4096, 9000])
def test_many_rows(cols):
    """Several rows to each team, the last round incomplete; the rows' statistics of 64 bits."""
    rows = 5003 if cols < 9000 else 1301
    g = seeded(3, cols)
    x, dy = matrix(g, rows, cols, torch.bfloat16, 3.0, -1.0), matrix(g, rows, cols, torch.bfloat16, 0.1)
    w, b = matrix(g, 1, cols, torch.bfloat16, 0.1, 1.0)[0], matrix(g, 1, cols, torch.bfloat16)[0]
    y, stats = ar.ar_layer_norm_forward(x, w, b, stats=True)
    want = tref.norm(x, w, b)
    ref.close(y, *want["y"], "y")
    dx, dw, db = ar.ar_layer_norm_backward(dy, x, stats, w, dw_dtype=torch.float32)
    want = tref.norm_grad(dy, x, stats, w)
    for name, t in (("dx", dx), ("dw", dw), ("db", db)):
        ref.close(t, *want[name], name)


@pytest.mark.parametrize("dtype", TYPES, ids=IDS)
@pytest.mark.parametrize("cols", [513, 1000, 1024, 1025, 2047, 2056, 4095, 4097, 6000, 8192, 8199, 16383])
def test_forward_of_many_rows(cols, dtype):
    """Rows of one wave, of two and of four, from half of their columns on to all, more than the chip takes at once, on any
    address; without w, without b, with both."""
    rows = 2048 + 37 + 64 * (cols % 3)
    g = seeded(14, cols)
    for pad, shift, out, w, b in ((0, 0, dtype, True, True), (5, 3, torch.bfloat16, True, False), (8, 0, torch.float32, False, True)):
        print("[gpu] norm of many rows", cols, dtype, pad, shift, flush=True)
        x = matrix(g, rows, cols, dtype, 2.0, 0.7, pad, shift)
        w = matrix(g, 1, cols, torch.float32, mean=1.0)[0] if w else None
        b = matrix(g, 1, cols, torch.float16)[0] if b else None
        y, stats = ar.ar_layer_norm_forward(x, w, b, out_dtype=out, stats=True)
        want = tref.norm(x, w, b)
        ref.close(y, *want["y"], "y")
        ref.close(stats[:, 0], *want["mean"], "mean")
        ref.close(stats[:, 1], *want["rstd"], "rstd")


@pytest.mark.parametrize("cols", [77, 2000, 20000])
def test_rows_far_from_zero_and_outlying_columns(cols):
    """The variance is about the mean: rows whose mean is 10^4 of their deviation, a first column 10^4 times the others, and
    rows of one value."""
    g = seeded(4, cols)
    x = matrix(g, 12, cols, torch.float32)
    x[:4] += 1e4
    x[4:8, 0] *= 1e4
    x[8] = 3.25
    x[9] = 0
    x[10] *= 1e-18  # squares below the smallest number
    x[11] *= 1e14  # the sum of the squares is within 32 bits' range
    y, stats = ar.ar_layer_norm_forward(x, stats=True)
    want = tref.norm(x)
    for name, t in (("y", y), ("mean", stats[:, 0]), ("rstd", stats[:, 1])):
        ref.close(t, *want[name], name)
    assert torch.equal(y[8:10], torch.zeros(2, cols, device=DEV))


def test_gradient_against_differences():
    """The gradient in float32 against central differences, step t = 1e-5, of the forward pass in 64 bits along random
    directions v.  A row's result is sqrt(n) of the unit vector of its deviations u; the third derivative of that along v is
    at most 15 (|v| / |u|)^3, here 15 / 8, so that a difference is off by t^2 / 6 * 15 / 8 * sqrt(203) * |dy| of a row, 14,
    times 9 rows: 6e-8; and by the loss' own rounding, 1500 * 2^-53 * 8 / t = 1e-7."""
    rows, cols = 9, 203
    g = seeded(5, 0)
    x, w, b = matrix(g, rows, cols, torch.float32, 2.0, 0.5), matrix(g, 1, cols, torch.float32, 0.2, 1.0)[0], matrix(g, 1, cols, torch.float32)[0]
    dy = matrix(g, rows, cols, torch.float32)
    stats = ar.ar_layer_norm_forward(x, w, b, stats=True)[1]
    got = ar.ar_layer_norm_backward(dy, x, stats, w)
    off = tref.norm_grad(dy, x, stats, w)

    def loss(X, W, B):
        d = X - X.mean(1, keepdim=True)
        return float((dy.double().cpu() * (d * (d.square().mean(1, keepdim=True) + 1e-5).rsqrt() * W + B)).sum())

    values = [t.double().cpu() for t in (x, w, b)]
    stat_off = tref.norm(x)
    # stats are rounded to 32 bits: what that does to dx and dw, relative, with some room
    rel = 4 * float((stat_off["rstd"][1] / stat_off["rstd"][0]).max()) + 8 * ref.E32
    for i, name in enumerate(("dx", "dw", "db")):
        for _ in range(3):
            v = torch.empty(values[i].shape, dtype=torch.float64).normal_(generator=g)
            t = 1e-5
            up, down = list(values), list(values)
            up[i], down[i] = values[i] + t * v, values[i] - t * v
            diff = (loss(*up) - loss(*down)) / (2 * t)
            along = float((got[i].double().cpu() * v).sum())
            size = float((got[i].double().cpu().abs() * v.abs()).sum())
            bound = float((off[name][1] * v.abs()).sum()) + rel * size + 2e-7
            assert abs(diff - along) <= bound, (name, diff, along, bound)


def test_parts_and_accumulation():
    """Each gradient by itself, and dw and db added to gradient buffers that are views of one vector."""
    rows, cols = 150, 72
    g = seeded(6, 1)
    x, dy = matrix(g, rows, cols, torch.bfloat16), matrix(g, rows, cols, torch.bfloat16, 0.1)
    w = matrix(g, 1, cols, torch.bfloat16, 0.1, 1.0)[0]
    for c in (cols, 5):
        xs, ds, ws = x[:, :c], dy[:, :c], w[:c]
        stats = ar.ar_layer_norm_forward(xs, stats=True)[1]
        whole = ar.ar_layer_norm_backward(ds, xs, stats, ws, dw_dtype=torch.float32)
        for i in range(3):
            got = ar.ar_layer_norm_backward(ds, xs, stats, ws, dx=i == 0, dw=i == 1, db=i == 2, dw_dtype=torch.float32)
            assert [t is None for t in got] == [j != i for j in range(3)]
            assert torch.equal(got[i], whole[i])
        assert ar.ar_layer_norm_backward(ds, xs, stats, ws, dx=False, dw=False, db=False) == (None, None, None)
        flat = torch.full((2 * c + 3,), 0.5, device=DEV)
        want = tref.norm_grad(ds, xs, stats, ws)
        for times in (1, 2):
            got = ar.ar_layer_norm_backward(ds, xs, stats, ws, dx=False, dw=flat[:c], db=flat[c:2 * c], accumulate=True)
            assert got[1].data_ptr() == flat.data_ptr()
            for t, name in ((flat[:c], "dw"), (flat[c:2 * c], "db")):
                ref.close(t, 0.5 + times * want[name][0], times * want[name][1] + 4 * times * ref.E32 * (1 + times * want[name][0].abs()), name)
        assert bool((flat[-3:] == 0.5).all())


@pytest.mark.parametrize("dtype", TYPES, ids=IDS)
@pytest.mark.parametrize("cols", [6, 100, 3001, 17001])
def test_in_place_and_columns_of_a_wider_matrix(cols, dtype):
    g = seeded(7, cols)
    rows = 37
    wide = matrix(g, rows, cols + 21, dtype)
    x, dy = wide[:, 5:5 + cols], matrix(g, rows, cols, dtype, 0.1)
    w = matrix(g, 1, cols, dtype, 0.1, 1.0)[0]
    y, stats = ar.ar_layer_norm_forward(x, w, stats=True)
    dx = ar.ar_layer_norm_backward(dy, x, stats, w, residual=dy, dw=False, db=False)[0]
    kept = wide.clone()
    assert ar.ar_layer_norm_forward(x, w, out=x).data_ptr() == x.data_ptr()
    assert torch.equal(x, y)
    assert torch.equal(wide[:, :5], kept[:, :5]) and torch.equal(wide[:, 5 + cols:], kept[:, 5 + cols:])
    x = kept[:, 5:5 + cols]
    both = dy.clone()
    ar.ar_layer_norm_backward(both, x, stats, w, residual=both, dx=both, dw=False, db=False)
    assert torch.equal(both, dx)
    # dw and db of a gradient whose dx is written over dy
    want = ar.ar_layer_norm_backward(dy, x, stats, w, dx=False)
    over = dy.clone()
    got = ar.ar_layer_norm_backward(over, x, stats, w, dx=over)
    assert torch.equal(got[1], want[1]) and torch.equal(got[2], want[2])
    out = torch.full((rows + 2, cols + 9), 7.0, dtype=dtype, device=DEV)
    ar.ar_layer_norm_forward(x, w, out=out[1:-1, 4:4 + cols])
    assert torch.equal(out[1:-1, 4:4 + cols], y)
    out[1:-1, 4:4 + cols] = 7
    assert bool((out == 7).all())


def test_rows_further_apart_than_32_bits():
    rows, cols, ld = 3, 300, (1 << 31) + 8
    if torch.cuda.mem_get_info()[0] < 40 << 30:
        pytest.skip("needs 20 GB")
    g = seeded(8, 0)
    big = torch.zeros(2 * ld + 1000, dtype=torch.bfloat16, device=DEV)
    x = big.as_strided((rows, cols), (ld, 1))
    small = matrix(g, rows, cols, torch.bfloat16)
    x.copy_(small)
    y, stats = ar.ar_layer_norm_forward(x, stats=True)
    want, ws = ar.ar_layer_norm_forward(small, stats=True)
    assert torch.equal(y, want) and torch.equal(stats, ws)
    dx = ar.ar_layer_norm_backward(x, x, stats, residual=x, dx=big.as_strided((rows, cols), (ld, 1), 600))[0]
    assert torch.equal(dx, ar.ar_layer_norm_backward(small, small, stats, residual=small)[0])
    assert int(big.count_nonzero()) == int(small.count_nonzero() + dx.count_nonzero())


@pytest.mark.parametrize("cols", [5, 50, 1500, 17000])
def test_infinities_and_nan_stay_in_their_rows(cols):
    g = seeded(9, cols)
    x, dy = matrix(g, 6, cols, torch.float32), matrix(g, 6, cols, torch.float32)
    x[1, 0], x[3, cols // 2], x[4, cols - 1] = math.inf, math.nan, -math.inf
    y, stats = ar.ar_layer_norm_forward(x, stats=True)
    assert bool(y[[1, 3, 4]].isnan().all()) and bool(stats[[1, 3, 4], 1].isnan().all())
    assert bool(y[[0, 2, 5]].isfinite().all())
    dx, dw, db = ar.ar_layer_norm_backward(dy, x, stats)
    assert bool(dx[[1, 3, 4]].isnan().all()) and bool(dx[[0, 2, 5]].isfinite().all())
    assert bool(dw.isnan().all()) and bool(db.isfinite().all())
    x = x.nan_to_num(0, 0, 0)
    dy[2, cols - 1] = math.inf
    stats = ar.ar_layer_norm_forward(x, stats=True)[1]
    dx, dw, db = ar.ar_layer_norm_backward(dy, x, stats)
    assert bool(dx[[0, 1, 3, 4, 5]].isfinite().all()) and not bool(dx[2].isfinite().any())
    assert bool(dw[:-1].isfinite().all()) and not bool(dw[-1].isfinite())
    assert bool(db[:-1].isfinite().all()) and bool(db[-1].isinf())
    one = torch.full((1, cols), 2.0, device=DEV)
    assert bool(ar.ar_layer_norm_forward(one, eps=0.0).isnan().all())


def test_empty_sizes():
    x = torch.empty(0, 40, device=DEV)
    y, stats = ar.ar_layer_norm_forward(x, stats=True)
    assert y.shape == (0, 40) and stats.shape == (0, 2)
    dx, dw, db = ar.ar_layer_norm_backward(x, x, stats)
    assert dx.shape == (0, 40) and torch.equal(dw, torch.zeros(40, device=DEV)) and torch.equal(db, dw)
    kept = torch.ones(40, device=DEV)
    ar.ar_layer_norm_backward(x, x, stats, dw=kept, db=False, accumulate=True)
    assert torch.equal(kept, torch.ones(40, device=DEV))
    none = torch.empty(3, 0, device=DEV)
    assert ar.ar_layer_norm_forward(none).shape == (3, 0)
    with pytest.raises(ar.ArError, match="no statistics"):
        ar.ar_layer_norm_forward(none, stats=True)


def test_results_do_not_depend_on_timing_or_stream():
    g = seeded(10, 0)
    x, dy = matrix(g, 3000, 1030, torch.bfloat16), matrix(g, 3000, 1030, torch.bfloat16, 0.1)
    w = matrix(g, 1, 1030, torch.float32, 0.1, 1.0)[0]
    y, stats = ar.ar_layer_norm_forward(x, w, stats=True)
    want = ar.ar_layer_norm_backward(dy, x, stats, w)
    other = torch.cuda.Stream()
    torch.cuda.synchronize()
    for stream in (None, other, other.cuda_stream):
        for _ in range(3):
            y2, stats2 = ar.ar_layer_norm_forward(x, w, stats=True, stream=stream)
            got = ar.ar_layer_norm_backward(dy, x, stats2, w, stream=stream)
            torch.cuda.synchronize()
            assert torch.equal(y, y2) and torch.equal(stats, stats2)
            assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_graph_capture_and_replay():
    """A captured forward and backward pass, replayed with other inputs and eager calls of the same kind between."""
    g = seeded(11, 0)
    rows, cols = 700, 520
    x, dy = matrix(g, rows, cols, torch.bfloat16), matrix(g, rows, cols, torch.bfloat16, 0.1)
    w, b = matrix(g, 1, cols, torch.float32, 0.1, 1.0)[0], matrix(g, 1, cols, torch.float32)[0]

    def run():
        y, stats = ar.ar_layer_norm_forward(x, w, b, stats=True)
        return (y, stats) + ar.ar_layer_norm_backward(dy, x, stats, w, residual=dy, dw_dtype=torch.float32)

    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        run()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = run()
    for i in range(4):
        x.copy_(matrix(g, rows, cols, torch.bfloat16, 1.0 + i))
        dy.copy_(matrix(g, rows, cols, torch.bfloat16, 0.1))
        want = run()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(held, want))


def test_c_call_with_raw_addresses():
    g = seeded(12, 0)
    rows, cols = 21, 333
    x, dy = matrix(g, rows, cols, torch.float16, pad=7), matrix(g, rows, cols, torch.float16, 0.1, pad=2)
    want, stats = ar.ar_layer_norm_forward(x, eps=1e-3, stats=True)
    mat = lambda t, ld: ctypes.byref(ar.Matrix(t.data_ptr(), ld, ar._FLOAT_CODES[t.dtype]))
    y, s = torch.zeros(rows, cols, dtype=torch.float16, device=DEV), torch.zeros(rows, 5, device=DEV)
    stream = ctypes.c_void_p(torch.cuda.current_stream().cuda_stream)
    assert ar.lib.ar_layer_norm_forward(rows, cols, mat(x, 340), None, None, 1e-3, mat(y, cols), mat(s, 5), stream) == ar.AR_OK
    assert torch.equal(y, want) and torch.equal(s[:, :2], stats) and bool((s[:, 2:] == 0).all())
    dw, need = torch.zeros(cols, device=DEV), ctypes.c_int64()
    args = (rows, cols, mat(dy, 335), mat(x, 340), mat(s, 5), None, None, None, mat(dw, 0), None)
    assert ar.lib.ar_layer_norm_backward_workspace(*args, ctypes.byref(need)) == ar.AR_OK and need.value > 0
    ws = torch.full((need.value + 256,), 85, dtype=torch.uint8, device=DEV)
    assert ar.lib.ar_layer_norm_backward(*args, 0, ctypes.c_void_p(ws.data_ptr()), need.value, stream) == ar.AR_OK
    assert torch.equal(dw, ar.ar_layer_norm_backward(dy, x, stats, dx=False, db=False, dw_dtype=torch.float32)[1])
    assert bool((ws[need.value:] == 85).all())


def test_refusals_of_device_tensors():
    x = torch.zeros(4, 8, device=DEV)
    stats = torch.zeros(4, 2, device=DEV)
    for call, text in (
            (lambda: ar.ar_layer_norm_forward(x[0]), "x must have 2 dimensions"),
            (lambda: ar.ar_layer_norm_forward(x.t()), "consecutive"),
            (lambda: ar.ar_layer_norm_forward(x.cpu()), "not on a GPU"),
            (lambda: ar.ar_layer_norm_forward(x.int()), "float32, float16"),
            (lambda: ar.ar_layer_norm_forward(x, torch.zeros(7, device=DEV)), "weight is 1 x 7"),
            (lambda: ar.ar_layer_norm_forward(x, bias=torch.zeros(1, 8, device=DEV)), "bias must have 1 dimension"),
            (lambda: ar.ar_layer_norm_forward(x, eps=-1e-5), "eps must be finite"),
            (lambda: ar.ar_layer_norm_forward(x, eps=math.nan), "eps must be finite"),
            (lambda: ar.ar_layer_norm_forward(x, eps="a"), "eps must be a number"),
            (lambda: ar.ar_layer_norm_forward(x, out=x[:, :7]), "out is 4 x 7"),
            (lambda: ar.ar_layer_norm_forward(x, stats=torch.zeros(4, 3, device=DEV)), "stats is 4 x 3"),
            (lambda: ar.ar_layer_norm_forward(x, stats=stats.half()), "stats must be float32"),
            (lambda: ar.ar_layer_norm_forward(x, stats=x[:, :2]), "stats overlaps x"),
            (lambda: ar.ar_layer_norm_forward(x.clone().requires_grad_(True)), "x requires a gradient"),
            (lambda: ar.ar_layer_norm_backward(x, x[:, :7], stats), "x is 4 x 7"),
            (lambda: ar.ar_layer_norm_backward(x, x, stats[:3]), "stats is 3 x 2"),
            (lambda: ar.ar_layer_norm_backward(x, x, stats, residual=x.half()), "residual must have x's type"),
            (lambda: ar.ar_layer_norm_backward(x, x, stats, dx=x.half()), "dx must have x's type"),
            (lambda: ar.ar_layer_norm_backward(x.clone(), x, stats, dx=x), "dx overlaps x"),
            (lambda: ar.ar_layer_norm_backward(x, x.clone(), stats, dw=x[1]), "dw overlaps dy"),
            (lambda: ar.ar_layer_norm_backward(x, x, stats, accumulate=True), "must be tensors")):
        with pytest.raises(ar.ArError, match=text):
            call()
    with torch.no_grad():
        ar.ar_layer_norm_forward(x.clone().requires_grad_(True))


def test_a_custom_function_differentiates():
    """A torch.autograd.Function of the two calls, and what is written in place counts as written."""
    g = seeded(13, 0)
    x, w, b = matrix(g, 12, 30, torch.float32), matrix(g, 1, 30, torch.float32)[0], matrix(g, 1, 30, torch.float32)[0]

    class Norm(torch.autograd.Function):
        @staticmethod
        def forward(ctx, x, w, b):
            y, stats = ar.ar_layer_norm_forward(x, w, b, stats=True)
            ctx.save_for_backward(x, w, stats)
            return y

        @staticmethod
        def backward(ctx, dy):
            x, w, stats = ctx.saved_tensors
            return ar.ar_layer_norm_backward(dy, x, stats, w)

    leaves = [t.clone().requires_grad_(True) for t in (x, w, b)]
    c = matrix(g, 12, 30, torch.float32)
    (Norm.apply(*leaves) * c).sum().backward()
    stats = ar.ar_layer_norm_forward(x, stats=True)[1]
    for leaf, grad in zip(leaves, ar.ar_layer_norm_backward(c, x, stats, w)):
        assert torch.equal(leaf.grad, grad)
    y, s, dx, dw, db = (torch.zeros(n, device=DEV) for n in ((12, 30), (12, 2), (12, 30), 30, 30))
    before = [t._version for t in (y, s, dx, dw, db)]
    ar.ar_layer_norm_forward(x, w, b, out=y, stats=s)
    ar.ar_layer_norm_backward(c, x, s, w, dx=dx, dw=dw, db=db)
    assert [t._version for t in (y, s, dx, dw, db)] == [n + 1 for n in before]
