"""A feed-forward block trained by data-parallel ranks: the layer operators and
the Allreduce together.

    python -m paper_2004_09362_amd.ffn --ranks 8 --tokens 512 --width 1024 --inner 4096 --steps 5 [--norm] [--orthogonal]

The block is y = x + drop(w2 gelu(w1 x + b1) + b2), in bfloat16 with float32
weights behind it.  Each of P virtual ranks holds some of the tokens.  A
training step runs both linear layers forward (the first keeps its
pre-activation, the second drops and adds the residual in its epilogue) and
backward, writes every rank's float32 gradients into its rank buffer, sums the
rank buffers with a Plan, and updates the weights from the sum.  A rank draws
the dropout mask of its rows of the whole batch, so P ranks compute what one
rank with all tokens does.

:meth:`FeedForward.split` runs the block with the inner dimension dealt out over
the ranks instead: float32 partial products, their Allreduce, then dropout and
residual on the sum.

:class:`NormedFeedForward` takes the layer norm of x into the first product, as a
block on a residual stream does; its gradient joins the residual's.  With
``orthogonal`` the two weight matrices are updated by the orthogonalised momentum
of the summed gradients, in place.
"""
from __future__ import annotations

import argparse
import time

import torch

from . import ar


class FeedForward:
    def __init__(self, ranks: int, width: int, inner: int, p: float = 0.1, lr: float = 0.1, seed: int = 0,
                 device="cuda", orthogonal: bool = False, rate: float = 0.02):
        g = torch.Generator(device=device).manual_seed(seed)
        self.ranks, self.p, self.lr, self.seed, self.step_no = ranks, p, lr, seed, 0
        self.orthogonal, self.rate = orthogonal, rate
        shapes = self._shapes(width, inner)
        sizes = [torch.Size(s).numel() for s in shapes]
        n = sum(sizes)
        self.plan = ar.Plan(ranks, n, "float32", "sum")
        # one vector of weights, and one rank buffer of gradients like it per rank (on 256-byte boundaries)
        self.master, self.velocity = torch.zeros(n, device=device), torch.zeros(n, device=device)
        self.buffers = list(torch.zeros(ranks, -(-n // 64) * 64, device=device)[:, :n].unbind(0))
        self.w1, self.b1, self.w2, self.b2, *self.norm = self._views(self.master, shapes, sizes)
        self.momenta = self._views(self.velocity, shapes, sizes)
        self.grads = [self._views(b, shapes, sizes) for b in self.buffers]
        self.w1.normal_(0, width ** -0.5, generator=g)
        self.w2.normal_(0, inner ** -0.5, generator=g)
        self._lower()

    @staticmethod
    def _shapes(width, inner):
        return [(inner, width), (inner,), (width, inner), (width,)]

    @staticmethod
    def _views(flat, shapes, sizes):
        out, at = [], 0
        for shape, size in zip(shapes, sizes):
            out.append(flat[at:at + size].view(shape))
            at += size
        return out

    def _lower(self):
        """The bfloat16 weights that the products take."""
        self.low = [w.to(torch.bfloat16) for w in (self.w1, self.w2)]

    def _drop(self, row0: int) -> ar.Dropout:
        return ar.Dropout(self.p, self.seed + self.step_no, site=1, row0=row0)

    def forward(self, x, row0: int = 0):
        """(y, h, z): the block's result, the hidden values and their pre-activation."""
        h, z = ar.ar_linear_forward(x, self.low[0], self.b1, activation="gelu", preact=True)
        return ar.ar_linear_forward(h, self.low[1], self.b2, x, dropout=self._drop(row0)), h, z

    def backward(self, dy, x, h, z, grads, row0: int = 0):
        """dx, with the weights' gradients written to ``grads`` (w1, b1, w2, b2)."""
        dh, _, _ = ar.ar_linear_backward(dy, h, self.low[1], dropout=self._drop(row0), dw=grads[2], db=grads[3])
        dx, _, _ = ar.ar_linear_backward(dh, x, self.low[0], preact=z, activation="gelu", dw=grads[0], db=grads[1])
        return dx + dy

    def gradients(self, xs, targets):
        """Every rank's gradients in its rank buffer, then their sum in all of
        them; the summed loss, half the mean square over all ranks' tokens."""
        total, losses, row0 = sum(x.numel() for x in xs), [], 0
        for x, target, grads in zip(xs, targets, self.grads):
            y, *kept = self.forward(x, row0)
            diff = y.float() - target.float()
            losses.append(diff.square().sum() / (2 * total))
            self.backward((diff / total).to(torch.bfloat16), x, *kept, grads, row0)
            row0 += x.shape[0]
        self.plan(self.buffers)
        return torch.stack(losses).sum()

    def step(self, xs, targets):
        """One step with momentum, of size lr / inner: the curvature grows with
        the inner dimension; or of size ``rate`` in every direction of a matrix."""
        loss = self.gradients(xs, targets)
        self.velocity.mul_(0.8).add_(self.buffers[0])
        if self.orthogonal:
            for weight, momentum in zip((self.w1, self.b1, self.w2, self.b2, *self.norm), self.momenta):
                if weight.dim() == 2:  # of one size whatever the gradient's, larger for tall matrices
                    scale = self.rate * max(1.0, weight.shape[0] / weight.shape[1]) ** 0.5
                    ar.ar_orthogonalize(momentum, scale=-scale, residual=weight, out=weight)
                else:
                    weight -= self.lr / self.w1.shape[0] * momentum
        else:
            self.master -= self.lr / self.w1.shape[0] * self.velocity
        self._lower()
        self.step_no += 1
        return loss

    def _enter(self, x):
        """What the first product takes."""
        return x

    def split(self, x, row0: int = 0):
        """The block's result with the inner dimension dealt out over the ranks."""
        M, width = x.shape
        n = self._enter(x)
        parts = torch.empty(self.ranks, M, width, device=x.device)
        edges = [r * self.w1.shape[0] // self.ranks for r in range(self.ranks + 1)]
        for r, (lo, hi) in enumerate(zip(edges, edges[1:])):
            h = ar.ar_linear_forward(n, self.low[0][lo:hi], self.b1[lo:hi], activation="gelu")
            # one rank adds the bias
            ar.ar_linear_forward(h, self.low[1][:, lo:hi], self.b2 if r == 0 else None, out=parts[r])
        ar.Plan(self.ranks, M * width, "float32", "sum")(list(parts.view(self.ranks, -1).unbind(0)))
        return ar.ar_dropout_forward(parts[0], self._drop(row0), x, out_dtype=torch.bfloat16)


class NormedFeedForward(FeedForward):
    """y = x + drop(w2 gelu(w1 n + b1) + b2) with n the layer norm of x."""

    def __init__(self, *args, **kwargs):
        super().__init__(*args, **kwargs)
        self.norm[0].fill_(1.0)

    @staticmethod
    def _shapes(width, inner):
        return FeedForward._shapes(width, inner) + [(width,), (width,)]

    def _enter(self, x):
        return ar.ar_layer_norm_forward(x, *self.norm)

    def forward(self, x, row0: int = 0):
        """(y, h, z, n, stats): as the block's without the norm, the norm's result and its rows' statistics."""
        n, stats = ar.ar_layer_norm_forward(x, *self.norm, stats=True)
        h, z = ar.ar_linear_forward(n, self.low[0], self.b1, activation="gelu", preact=True)
        return ar.ar_linear_forward(h, self.low[1], self.b2, x, dropout=self._drop(row0)), h, z, n, stats

    def backward(self, dy, x, h, z, n, stats, grads, row0: int = 0):
        """dx, with the weights' gradients written to ``grads`` (w1, b1, w2, b2, the norm's weight and bias)."""
        dh, _, _ = ar.ar_linear_backward(dy, h, self.low[1], dropout=self._drop(row0), dw=grads[2], db=grads[3])
        dn, _, _ = ar.ar_linear_backward(dh, n, self.low[0], preact=z, activation="gelu", dw=grads[0], db=grads[1])
        return ar.ar_layer_norm_backward(dn, x, stats, self.norm[0], residual=dy, dx=dn, dw=grads[4], db=grads[5])[0]


def main(argv=None):
    ap = argparse.ArgumentParser(description="train a feed-forward block on virtual data-parallel ranks")
    for name, default in (("ranks", 8), ("tokens", 512), ("width", 1024), ("inner", 4096), ("steps", 5)):
        ap.add_argument("--" + name, type=int, default=default)
    ap.add_argument("--norm", action="store_true", help="take the layer norm of x into the first product")
    ap.add_argument("--orthogonal", action="store_true", help="update the matrices by their orthogonalised momentum")
    a = ap.parse_args(argv)
    kind = NormedFeedForward if a.norm else FeedForward
    block = kind(a.ranks, a.width, a.inner, lr=a.width * 0.5, orthogonal=a.orthogonal)
    g = torch.Generator(device="cuda").manual_seed(1)
    xs = [torch.empty(a.tokens, a.width, device="cuda").normal_(generator=g).bfloat16() for _ in range(a.ranks)]
    targets = [x.roll(1, 1) for x in xs]
    for i in range(a.steps):
        torch.cuda.synchronize()
        t = time.perf_counter()
        loss = block.step(xs, targets)
        torch.cuda.synchronize()
        print("step %d: loss %.5f, %.2f ms" % (i, float(loss), 1e3 * (time.perf_counter() - t)), flush=True)


if __name__ == "__main__":
    main()
