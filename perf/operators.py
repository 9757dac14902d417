"""What is measured: the operators that a layer runs around an Allreduce -- the linear layer with its epilogue, its
gradient, and dropout from a counter-based generator -- as programs call them.

``op`` names the operator of a case:

``forward``    y = residual + drop(act(x w^T + bias)), and the pre-activation z = x w^T + bias where training keeps it;
``backward``   dz = act'(z) * drop(dy), dx = dz w, dw = dz^T x, db = the sum of dz over the rows;
``dropout``    y = residual + drop(x);
``dropgrad``   dx = drop(dy).

drop(v) keeps element (i, j) of a matrix, times 1 / (1 - p), where a word of the generator is below
round((1 - p) 2^32), and is 0 elsewhere.  The words are those of the seven-round counter generator on four 32-bit words
(Salmon et al., 2011): word j mod 4 at the counter (j / 4, row mod 2^32, row / 2^32, site), row = row0 + i, with the seed's
halves as key.

The other fields: rows ``M``, columns ``N`` and inner length ``K``; ``dtype`` of the operands and ``out`` of what is
computed from them (y and the residual; the weight's and the bias' gradient; of dropout the result), the activation ``act``, the drop
probability ``p``, whether there is a ``bias``, a ``residual`` and a kept pre-activation (``keep``), and ``pad``, the elements
between the end of a row and the next one's start.
"""
import math

import torch

own = False

DTYPES = {"float32": torch.float32, "float16": torch.float16, "bfloat16": torch.bfloat16}
ACTS = ["none", "relu", "gelu", "gelu_tanh", "silu"]


def _case(name, op, M, N, K=0, *, dtype="bfloat16", out=None, act="none", p=0.0, bias=False, residual=False, keep=False,
          pad=0):
    c = dict(name=name, op=op, M=M, N=N, K=K, dtype=dtype, out=dtype if out is None else out, act=act, p=p, bias=bias,
             residual=residual, keep=keep, pad=pad)
    if name is None:
        del c["name"]
    return c


def listed():
    return [
        # a projection of one new token: the weights are read once, latency counts
        _case("token_4096", "forward", 1, 4096, 4096, bias=True),
        # the widening product of a feed-forward layer for one token of each of 24 sequences
        _case("decode24_up", "forward", 24, 16384, 4096, act="silu", bias=True),
        # a short prompt through a layer of odd sizes, whose rows start on any element
        _case("ragged_f16", "forward", 1537, 2047, 1023, dtype="float16", act="relu", bias=True, residual=True),
        # one rank's part of a product whose inner length is dealt out over ranks, in the Allreduce's own type
        _case("partial_f32", "forward", 2048, 4096, 1024, dtype="float32"),
        # the widening product of a training step, the pre-activation kept for the gradient
        _case("train_up", "forward", 8192, 16384, 4096, act="gelu_tanh", bias=True, keep=True),
        # and the narrowing one, with dropout, onto the residual stream
        _case("train_down", "forward", 8192, 4096, 16384, p=0.1, bias=True, residual=True),
        # the gradient of a small layer of odd sizes
        _case("grad_ragged_f16", "backward", 200, 1001, 777, dtype="float16", bias=True),
        # the gradient of a square layer over many tokens, the weight's part in the type that the Allreduce sums
        _case("grad_long", "backward", 16384, 1024, 1024, out="float32", bias=True),
        # the gradient of the widening product, through the activation
        _case("grad_up", "backward", 8192, 16384, 4096, act="gelu_tanh", bias=True, keep=True),
        # dropout onto the residual stream of 24 tokens: the smallest call
        _case("drop_tokens", "dropout", 24, 4096, p=0.1, residual=True),
        # a summed product of all ranks, dropped and added to the residual stream in its type
        _case("drop_summed", "dropout", 8192, 8192, dtype="float32", out="bfloat16", p=0.1, residual=True),
        # the gradient of dropout on odd rows
        _case("dropgrad_ragged_f16", "dropgrad", 30011, 4099, dtype="float16", p=0.25),
    ]


def _log_uniform(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _size(rng, lo, hi):
    """A length: half of them multiples of 64, as layers have them, the others any."""
    n = _log_uniform(rng, lo, hi)
    return max(64, n // 64 * 64) if rng.random() < 0.5 else n


def draw(rng):
    op = rng.choice(["forward", "forward", "forward", "backward", "backward", "dropout", "dropgrad"])
    dtype = rng.choice(["bfloat16", "bfloat16", "float16", "float32"])
    pad = rng.choice([0, 0, 0, 8, rng.randint(1, 63)])
    p = rng.choice([0.0, 0.1, round(rng.uniform(0.02, 0.6), 3)])
    if op in ("dropout", "dropgrad"):
        N = _size(rng, 64, 16384)
        M = _log_uniform(rng, 1, min(65536, (1 << 27) // N))
        return _case(None, op, M, N, dtype=dtype, out=rng.choice([dtype, "float32", "bfloat16"]), p=max(p, 0.02),
                     residual=op == "dropout" and rng.random() < 0.5, pad=pad)
    N, K = _size(rng, 64, 16384), _size(rng, 64, 16384)
    most = (1 << 39) // (N * K) if dtype != "float32" else (1 << 37) // (N * K)
    M = _log_uniform(rng, 1 if op == "forward" else 16, max(16, min(32768, most)))
    act = rng.choice(["none", "none"] + ACTS[1:])
    if op == "forward":
        return _case(None, op, M, N, K, dtype=dtype, out=rng.choice([dtype, dtype, "float32"]), act=act, p=p,
                     bias=rng.random() < 0.7, residual=rng.random() < 0.5, keep=act != "none" and rng.random() < 0.5, pad=pad)
    out = rng.choice([dtype, "float32"]) if act == "none" and p == 0 else dtype
    return _case(None, op, M, N, K, dtype=dtype, out=out, act=act, p=p, bias=rng.random() < 0.7, keep=act != "none", pad=pad)


def _inputs(case, seed):
    """Activations of unit size, weights that keep it, gradients that are small, as a network in training has them."""
    g = torch.Generator(device="cuda")
    g.manual_seed(seed * 1000003 + 7 * case["M"] + case["N"])
    M, N, K, dt, out = case["M"], case["N"], case["K"], DTYPES[case["dtype"]], DTYPES[case["out"]]

    def normal(rows, cols, dtype, std):
        t = torch.empty(rows, cols + case["pad"], dtype=dtype, device="cuda").normal_(0.0, std, generator=g)
        return t[:, :cols]

    s = {"drop": (case["p"], 20040936 + ((seed & 0xFFFFFFF) << 33), 5, seed) if case["p"] > 0 else None, "act": case["act"],
         "dtype": dt, "out": out, "op": case["op"], "keep": case["keep"], "has_bias": case["bias"]}
    if case["op"] == "forward":
        s["x"], s["w"] = normal(M, K, dt, 1.0), normal(N, K, dt, K ** -0.5)
    elif case["op"] == "backward":
        s["dy"], s["x"], s["w"] = normal(M, N, dt, 0.01), normal(M, K, dt, 1.0), normal(N, K, dt, K ** -0.5)
        s["z"] = normal(M, N, dt, 1.0) if case["act"] != "none" else None
    else:
        s["x"] = normal(M, N, dt, 1.0)
    s["bias"] = normal(1, N, dt, 0.1)[0] if case["op"] == "forward" and case["bias"] else None
    s["residual"] = normal(M, N, out, 1.0) if case["residual"] else None
    return s


def prepare(case, seed):
    s = _inputs(case, seed)
    if own:
        from paper_2004_09362_amd import ar

        s["ar"] = ar
        p, key, site, row0 = s["drop"] or (0.0, 0, 0, 0)
        s["dropout"] = ar.Dropout(p, key, site, row0) if s["drop"] else None
    return s


# ---- the plain form: elementary operations in 32 bits, rounded once at the end ----

_LOW = 0xFFFFFFFF


def _kept(rows, cols, drop):
    """Which elements of a rows x cols matrix drop() keeps."""
    p, key, site, row0 = drop
    groups = (cols + 3) // 4
    c0 = torch.arange(groups, device="cuda").expand(rows, groups)
    row = (torch.arange(rows, device="cuda") + row0)[:, None].expand(rows, groups)
    c1, c2, c3 = row & _LOW, row >> 32, site
    k0, k1 = key & _LOW, key >> 32 & _LOW
    for _ in range(7):
        a, b = c0 * 0xD2511F53, c2 * 0xCD9E8D57  # 64-bit products: their halves are right though the sign may not be
        c0, c1, c2, c3 = (b >> 32 & _LOW) ^ c1 ^ k0, b & _LOW, (a >> 32 & _LOW) ^ c3 ^ k1, a & _LOW
        k0, k1 = (k0 + 0x9E3779B9) & _LOW, (k1 + 0xBB67AE85) & _LOW
    words = torch.stack([c0, c1, c2, c3], dim=-1).view(rows, 4 * groups)[:, :cols]
    return words < math.floor((1 - p) * 2.0 ** 32 + 0.5)


def _dropped(v, drop):
    if drop is None:
        return v
    return torch.where(_kept(v.shape[0], v.shape[1], drop), v * (1 / (1 - drop[0])), torch.zeros((), device=v.device))


def _act(z, act):
    if act == "none":
        return z
    if act == "relu":
        return z.clamp(min=0)
    if act == "gelu":
        return 0.5 * z * (1 + torch.erf(z * math.sqrt(0.5)))
    if act == "gelu_tanh":
        return 0.5 * z * (1 + torch.tanh(math.sqrt(2 / math.pi) * (z + 0.044715 * z * z * z)))
    return z * torch.sigmoid(z)


def _act_slope(z, act):
    if act == "relu":
        return (z > 0).to(z.dtype)
    if act == "gelu":
        return 0.5 * (1 + torch.erf(z * math.sqrt(0.5))) + z * torch.exp(-0.5 * z * z) * (1 / math.sqrt(2 * math.pi))
    if act == "gelu_tanh":
        c = math.sqrt(2 / math.pi)
        t = torch.tanh(c * (z + 0.044715 * z * z * z))
        return 0.5 * (1 + t) + 0.5 * z * (1 - t * t) * c * (1 + 3 * 0.044715 * z * z)
    s = torch.sigmoid(z)
    return s * (1 + z * (1 - s))


def _run_plain(s):
    out = s["out"]
    if s["op"] == "forward":
        z = s["x"].float() @ s["w"].float().t()
        if s["bias"] is not None:
            z = z + s["bias"].float()
        y = _dropped(_act(z, s["act"]), s["drop"])
        if s["residual"] is not None:
            y = y + s["residual"].float()
        return {"y": y.to(out), "z": z.to(s["dtype"])} if s["keep"] else {"y": y.to(out)}
    if s["op"] == "backward":
        dz = _dropped(s["dy"].float(), s["drop"])
        if s["z"] is not None:
            dz = dz * _act_slope(s["z"].float(), s["act"])
        got = {"dx": (dz @ s["w"].float()).to(s["dtype"]), "dw": (dz.t() @ s["x"].float()).to(out)}
        if s["has_bias"]:
            got["db"] = dz.sum(0).to(out)
        return got
    y = _dropped(s["x"].float(), s["drop"])
    if s["residual"] is not None:
        y = y + s["residual"].float()
    return {"y": y.to(out)}


def run(s):
    if not own:
        return _run_plain(s)
    ar = s["ar"]
    if s["op"] == "forward":
        if s["keep"]:
            y, z = ar.ar_linear_forward(s["x"], s["w"], s["bias"], s["residual"], activation=s["act"], preact=True,
                                        out_dtype=s["out"], dropout=s["dropout"])
            return {"y": y, "z": z}
        return {"y": ar.ar_linear_forward(s["x"], s["w"], s["bias"], s["residual"], activation=s["act"],
                                          out_dtype=s["out"], dropout=s["dropout"])}
    if s["op"] == "backward":
        dx, dw, db = ar.ar_linear_backward(s["dy"], s["x"], s["w"], preact=s["z"], activation=s["act"],
                                           dropout=s["dropout"], db=s["has_bias"], dw_dtype=s["out"])
        return {"dx": dx, "dw": dw, "db": db} if s["has_bias"] else {"dx": dx, "dw": dw}
    if s["op"] == "dropout":
        return {"y": ar.ar_dropout_forward(s["x"], s["dropout"], s["residual"], out_dtype=s["out"])}
    return {"y": ar.ar_dropout_backward(s["x"], s["dropout"], out_dtype=s["out"])}


def work(case):
    M, N, K = case["M"], case["N"], case["K"]
    e, o = DTYPES[case["dtype"]].itemsize, DTYPES[case["out"]].itemsize
    if case["op"] == "forward":
        b = (M * K + N * K) * e + M * N * o * (2 if case["residual"] else 1) + (N * e if case["bias"] else 0)
        return {"bytes": b + (M * N * e if case["keep"] else 0), "flops": 2 * M * N * K}
    if case["op"] == "backward":
        b = (M * N * (2 if case["act"] != "none" else 1) + 2 * M * K + N * K) * e + N * K * o
        return {"bytes": b + (N * o if case["bias"] else 0), "flops": 4 * M * N * K}
    return {"bytes": M * N * (e + o * (2 if case["residual"] else 1)), "flops": 2 * M * N}


# ---- the definition in 64 bits, on its own ----

def _exact_keep(case, drop):
    """1 / (1 - p) where an element is kept, 0 where it is not; the generator's products taken in 16-bit parts."""
    p, key, site, row0 = drop
    M, G = case["M"], -(-case["N"] // 4)
    i = torch.arange(M * G, dtype=torch.int64, device="cuda")
    row = row0 + torch.div(i, G, rounding_mode="floor")
    x = [i % G, row % 2 ** 32, torch.div(row, 2 ** 32, rounding_mode="floor"), torch.full_like(i, site)]
    del i, row

    def wide(m, v):
        low = m * (v % 65536)
        high = m * torch.div(v, 65536, rounding_mode="floor") + torch.div(low, 65536, rounding_mode="floor")
        return torch.div(high, 65536, rounding_mode="floor"), high % 65536 * 65536 + low % 65536

    for n in range(7):
        h0, l0 = wide(0xD2511F53, x[0])
        h2, l2 = wide(0xCD9E8D57, x[2])
        ka, kb = (key % 2 ** 32 + n * 0x9E3779B9) % 2 ** 32, (key // 2 ** 32 + n * 0xBB67AE85) % 2 ** 32
        x = [torch.bitwise_xor(torch.bitwise_xor(h2, x[1]), ka), l2, torch.bitwise_xor(torch.bitwise_xor(h0, x[3]), kb), l0]
    limit = int((1 - p) * 2 ** 32 + 0.5)
    keep = torch.empty(M, G, 4, dtype=torch.bool, device="cuda")
    for j in range(4):
        keep[:, :, j] = (x[j] < limit).view(M, G)
    return keep.view(M, 4 * G)[:, :case["N"]].double() / (1 - p)


def exact(case, seed):
    s = _inputs(case, seed)
    d = {k: v.double() for k, v in s.items() if isinstance(v, torch.Tensor)}
    mask = _exact_keep(case, s["drop"]) if s["drop"] else None
    if case["op"] in ("dropout", "dropgrad"):
        y = d["x"] if mask is None else d["x"] * mask
        return {"y": y + d["residual"] if "residual" in d else y}

    def value_and_slope(z):
        act = case["act"]
        if act == "relu":
            return torch.where(z > 0, z, 0.0), torch.where(z > 0, 1.0, 0.0).double()
        if act == "gelu":
            cdf = torch.special.ndtr(z)
            return z * cdf, cdf + z * torch.exp(-z.square() / 2) / math.sqrt(2 * math.pi)
        # both of the others are z times a logistic function of u(z)
        if act == "silu":
            u, du = z, 1.0
        else:
            u = 2 * math.sqrt(2 / math.pi) * (z + 0.044715 * z ** 3)
            du = 2 * math.sqrt(2 / math.pi) * (1 + 0.134145 * z ** 2)
        g = 1 / (1 + torch.exp(-u))
        return z * g, g + z * g * (1 - g) * du

    if case["op"] == "forward":
        z = torch.mm(d["x"], d["w"].T)
        if "bias" in d:
            z += d["bias"]
        y = z if case["act"] == "none" else value_and_slope(z)[0]
        if mask is not None:
            y = y * mask
        if "residual" in d:
            y = y + d["residual"]
        return {"y": y, "z": z} if case["keep"] else {"y": y}
    dz = d["dy"] if mask is None else d["dy"] * mask
    if "z" in d:
        dz = dz * value_and_slope(d["z"])[1]
    got = {"dx": torch.mm(dz, d["w"]), "dw": torch.mm(dz.T.contiguous(), d["x"])}
    if case["bias"]:
        got["db"] = dz.sum(dim=0)
    return got
