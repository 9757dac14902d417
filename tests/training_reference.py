"""The definitions of layer norm and its gradient in 64 bits, written out for the
tests, and how far the kernels' results may be from them before their rounding.

Everything before a store is 32-bit arithmetic, u = 2^-24 of a result's size an
operation.  A sum over a row of n columns adds at most depth(n) numbers one after
the other on any way from an element to the sum: 16 in a lane, 6 exchanges in a
wave, 16 waves, and for rows of more than 16384 columns 8 for each 8192 of them.
So it is off by depth(n) u of the sum of the sizes."""
import torch

from layer_reference import E32


def depth(n):
    return 40 + 8 * (n // 8192)


def norm(x, weight=None, bias=None, eps=1e-5):
    """{name: (value, off)} of y, mean and rstd."""
    X = x.double().cpu()
    n = X.shape[1]
    w = torch.ones(n, dtype=torch.float64) if weight is None else weight.double().cpu()
    b = torch.zeros(n, dtype=torch.float64) if bias is None else bias.double().cpu()
    mean = X.mean(1, keepdim=True)
    d = X - mean
    var = d.square().mean(1, keepdim=True)
    rstd = (var + eps).rsqrt()
    off_mean = (depth(n) + 2) * E32 * X.abs().mean(1, keepdim=True)  # the sum, 1/n and the product with it
    off_d = off_mean + E32 * d.abs()
    # squares of what is off, their own rounding and their sum's; 1/n, its product, eps
    off_var = 2 * (off_d * d.abs()).mean(1, keepdim=True) + off_d.square().mean(1, keepdim=True) + (depth(n) + 4) * E32 * (var + eps)
    part = off_var / (var + eps)
    # of the inverse root half the argument's part (the larger side, where the argument is smaller), the root's and the quotient's
    off_rstd = rstd * ((1 - part).clamp(min=1e-9).rsqrt() - 1 + 3 * E32)
    y = d * rstd * w + b
    off_y = (off_d * rstd + d.abs() * off_rstd + off_d * off_rstd) * w.abs() + 4 * E32 * ((d * rstd * w).abs() + b.abs())
    return {"y": (y, off_y), "mean": (mean[:, 0], off_mean[:, 0]), "rstd": (rstd[:, 0], off_rstd[:, 0])}


def norm_grad(dy, x, stats, weight=None, residual=None):
    """{name: (value, off)} of dx, dw and db, for the stats given."""
    D, X, S = dy.double().cpu(), x.double().cpu(), stats.double().cpu()
    rows, n = X.shape
    w = torch.ones(n, dtype=torch.float64) if weight is None else weight.double().cpu()
    h = (X - S[:, :1]) * S[:, 1:]
    g = D * w
    m0, m1 = g.mean(1, keepdim=True), (g * h).mean(1, keepdim=True)
    dx = S[:, 1:] * (g - m0 - h * m1)
    # h: a difference and a product; g: one; the means: the sum, 1/n and its product
    off_h, off_g = 2.1 * E32 * h.abs(), E32 * g.abs()
    off0 = (depth(n) + 4) * E32 * g.abs().mean(1, keepdim=True)
    off1 = (depth(n) + 8) * E32 * (g * h).abs().mean(1, keepdim=True)
    size = g.abs() + m0.abs() + (h * m1).abs()
    off = S[:, 1:] * (off_g + off0 + h.abs() * off1 + off_h * m1.abs() + off_h * off1 + 5 * E32 * size)
    if residual is not None:
        dx = dx + residual.double().cpu()
        off = off + 2 * E32 * (dx.abs() + residual.double().cpu().abs())
    # over the rows in any order
    return {"dx": (dx, off), "dw": ((D * h).sum(0), (rows + 8) * E32 * (D * h).abs().sum(0)),
            "db": (D.sum(0), (rows + 8) * E32 * D.abs().sum(0))}


def orthogonal(x, steps=5, coefficients=(3.4445, -4.7750, 2.0315), eps=1e-7, dtype=torch.float64, rounded=False):
    """X after the steps, of one matrix or a stack, on the CPU in `dtype`.  rounded: with the operands of the products
    rounded to 11 bits as ar_orthogonalize says that it does towards bfloat16 (X in 22 bits; of Q the diagonal in full)."""
    many = x.double().cpu()
    turned = many.shape[-2] > many.shape[-1]
    many = (many.transpose(-2, -1) if turned else many).reshape(-1, *sorted(many.shape[-2:]))
    triples = [coefficients] * steps if not isinstance(coefficients[0], (tuple, list)) else coefficients

    def bits11(t, scale):
        return (t * scale).half().to(dtype) / scale

    def bits22(t, scale):
        high = bits11(t, scale)
        return high, bits11(t - high, scale)

    got = []
    for X in many:
        X = (X / (X.norm() + eps)).to(dtype)
        for a, b, c in triples:
            if not rounded:
                A = X @ X.t()
                X = a * X + (b * A + c * (A @ A)) @ X
                continue
            high, low = bits22(X, 8192)
            A = bits11(high @ high.t(), 8192)
            Q = b * A + c * (A @ A)
            d = torch.diag(Q)
            X = a * (high + low) + d[:, None] * high + bits11(Q - torch.diag(d), 4096) @ high
        got.append(X.t() if turned else X)
    return torch.stack(got).view(x.shape)
