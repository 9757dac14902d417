"""The layer operators' definitions in 64 bits, written out for the tests, and
how far the kernels' results may be from them.

A result of type T is rounded once, by at most u(T) of its size (u = 2^-24,
2^-11 and 2^-8 for float32, float16 and bfloat16; below float16's normal range
by half its smallest step).  Before that everything is 32-bit arithmetic: a sum
of n products is off by at most (n + 8) 2^-24 of the sum of their sizes, in any
order, and an activation (slopes are at most 1.13) by 2^-20 (1 + |z|) of its
own evaluation besides what its argument is off by."""
import math

import numpy as np
import torch

U = {torch.float32: 2.0 ** -24, torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}
E32 = 2.0 ** -24


def counter_words(c, k, rounds=7):
    """The generator on lists of four and two 32-bit numbers, in Python's integers."""
    c, k, m = list(c), list(k), 0xFFFFFFFF
    for _ in range(rounds):
        a, b = 0xD2511F53 * c[0], 0xCD9E8D57 * c[2]
        c = [(b >> 32) ^ c[1] ^ k[0], b & m, (a >> 32) ^ c[3] ^ k[1], a & m]
        k = [(k[0] + 0x9E3779B9) & m, (k[1] + 0xBB67AE85) & m]
    return c


def keep_mask(rows, cols, p, seed, site=0, row0=0):
    """The kept elements, drawn with numpy's 64-bit integers."""
    g = -(-cols // 4)
    row = np.arange(rows, dtype=np.uint64)[:, None] + np.uint64(row0)
    m32, s32 = np.uint64(0xFFFFFFFF), np.uint64(32)
    c = [np.broadcast_to(np.arange(g, dtype=np.uint64), (rows, g)), np.broadcast_to(row & m32, (rows, g)),
         np.broadcast_to(row >> s32, (rows, g)), np.full((rows, g), site, dtype=np.uint64)]
    k0, k1 = seed & 0xFFFFFFFF, seed >> 32
    for _ in range(7):
        a, b = c[0] * np.uint64(0xD2511F53), c[2] * np.uint64(0xCD9E8D57)
        c = [(b >> s32) ^ c[1] ^ np.uint64(k0), b & m32, (a >> s32) ^ c[3] ^ np.uint64(k1), a & m32]
        k0, k1 = (k0 + 0x9E3779B9) & 0xFFFFFFFF, (k1 + 0xBB67AE85) & 0xFFFFFFFF
    words = np.stack(c, axis=-1).reshape(rows, 4 * g)[:, :cols]
    return torch.from_numpy(words < np.uint64(math.floor((1 - p) * 2.0 ** 32 + 0.5)))


def drop(v, d):
    """drop() of a 64-bit matrix; d is None or (p, seed, site, row0)."""
    if d is None or d[0] == 0:
        return v
    if d[0] == 1:
        return torch.zeros_like(v)
    mask = keep_mask(v.shape[0], v.shape[1], *d).to(v.device)
    return torch.where(mask, v / (1 - d[0]), torch.zeros_like(v))


def act(z, name):
    if name == "relu":
        return torch.relu(z)
    if name == "gelu":
        return z * 0.5 * torch.erfc(-z / math.sqrt(2))
    if name == "gelu_tanh":
        return 0.5 * z * (1 + torch.tanh(math.sqrt(2 / math.pi) * (z + 0.044715 * z ** 3)))
    if name == "silu":
        return z / (1 + torch.exp(-z))
    return z


def slope(z, name):
    """By torch's differentiation of act (0 at relu's kink)."""
    z = z.detach().clone().requires_grad_(True)
    act(z, name).sum().backward()
    return z.grad


def close(got, want, before, where=""):
    """got within rounding of its type of want, which was off by at most `before` before the rounding."""
    g, w = got.double().cpu(), want.double().cpu()
    u = U[got.dtype]
    tol = before.double().cpu() * (1 + u) + u * w.abs() + (2.0 ** -25 if got.dtype == torch.float16 else 2.0 ** -140)
    bad = ~((g - w).abs() <= tol)
    assert not bad.any(), "%s: %d of %d off, worst %g of the tolerance" % (
        where, int(bad.sum()), bad.numel(), float(((g - w).abs() / tol).nan_to_num(nan=math.inf).max()))


def forward(x, w, bias=None, residual=None, activation="none", d=None):
    """(y, z) in 64 bits and how far 32-bit arithmetic may be off, before rounding."""
    X, W = x.double().cpu(), w.double().cpu()
    z, size = X @ W.t(), X.abs() @ W.abs().t()
    n = X.shape[1] + 8
    if bias is not None:
        z, size = z + bias.double().cpu(), size + bias.double().cpu().abs()
    off_z = n * E32 * size
    a = act(z, activation)
    off = off_z if activation == "none" else 1.13 * off_z + 2.0 ** -20 * (1 + z.abs())
    y = drop(a, d)
    if d is not None and d[0] not in (0, 1):
        off = off / (1 - d[0]) + 4 * E32 * y.abs()
    if residual is not None:
        y = y + residual.double().cpu()
        off = off + 2 * E32 * (y.abs() + residual.double().cpu().abs())
    return y, z, off, off_z


def backward(dy, x, w, z=None, activation="none", d=None):
    """{name: (value, off)} of dx, dw and db, where the products take dz in x's type."""
    dz = drop(dy.double().cpu(), d)
    off = 4 * E32 * dz.abs()
    if activation != "none":
        # a slope is off by 2^-20 (1 + |z|) of its evaluation
        Z = z.double().cpu()
        off = off * 1.13 + 2.0 ** -20 * (1 + Z.abs()) * dz.abs()
        dz = dz * slope(Z, activation)
    rounded = activation != "none" or (d is not None and d[0] > 0) or dy.dtype != x.dtype
    off_in = off
    if rounded:
        off_in = off * 2 + U[x.dtype] * dz.abs() + (2.0 ** -25 if x.dtype == torch.float16 else 0.0)
    X, W = x.double().cpu(), w.double().cpu()
    big = dz.abs() + off_in
    return {"dx": (dz @ W, off_in @ W.abs() + (W.shape[0] + 8) * E32 * (big @ W.abs())),
            "dw": (dz.t() @ X, off_in.t() @ X.abs() + (X.shape[0] + 8) * E32 * (big.t() @ X.abs())),
            "db": (dz.sum(0), off.sum(0) + (X.shape[0] + 8) * E32 * dz.abs().sum(0))}
