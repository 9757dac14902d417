"""The feed-forward example with layer norm and orthogonalised updates, on the GPU: the operators together as a training
step runs them.  Gradients against torch's differentiation of the same block in 64 bits, P ranks against one, a whole step
against its parts."""
import math

import pytest
import torch

import training_reference as tref
from paper_2004_09362_amd import ar
from paper_2004_09362_amd.ffn import FeedForward, NormedFeedForward, main

pytestmark = pytest.mark.gpu

WIDTH, INNER, TOKENS = 200, 520, (70, 33, 97)


def batch(seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    x = (3 * torch.empty(sum(TOKENS), WIDTH, device="cuda").normal_(generator=g) + 0.5).bfloat16()
    return x, x.roll(1, 1)


def started(ranks, seed, **kw):
    """A block whose norm is not the identity."""
    block = NormedFeedForward(ranks, WIDTH, INNER, seed=seed, **kw)
    g = torch.Generator(device="cuda").manual_seed(seed)
    block.norm[0].normal_(1.0, 0.2, generator=g)
    block.norm[1].normal_(0.0, 0.2, generator=g)
    return block


def test_gradients_against_64_bits():
    """A gradient passes at most six tensors that are rounded to bfloat16 on its way (n, z, h, dy, dh and dz's two, dn), each
    off by 2^-8 of its elements at most, and each by itself moves a gradient by about that part of its size; differences that
    add in squares, as roundings do, make 2^-8 * sqrt(6) = 1 %, and twice that is allowed."""
    x, _ = batch(1)
    block = started(1, 7, p=0.0)
    g = torch.Generator(device="cuda").manual_seed(2)
    dy = torch.empty_like(x).normal_(generator=g)
    y, *kept = block.forward(x)
    dx = block.backward(dy, x, *kept, block.grads[0])
    low = [w.double().cpu().requires_grad_(True) for w in (block.low[0], block.b1, block.low[1], block.b2, *block.norm)]
    X = x.double().cpu().requires_grad_(True)
    w1, b1, w2, b2, gain, shift = low
    n = torch.nn.functional.layer_norm(X, (WIDTH,), gain, shift)
    z = n @ w1.t() + b1
    want = X + (z * 0.5 * torch.erfc(-z / math.sqrt(2))) @ w2.t() + b2
    want.backward(dy.double().cpu())
    # y is rounded once more, to bfloat16
    assert float((y.double().cpu() - want.detach()).norm()) < 2 * 2.0 ** -8 * math.sqrt(4) * float(want.detach().norm())
    for name, got, ref in [("dx", dx, X.grad)] + [(n, g, v.grad) for n, g, v in zip(("w1", "b1", "w2", "b2", "gain", "shift"), block.grads[0], low)]:
        far = float((got.double().cpu() - ref).norm() / ref.norm())
        assert far < 2 * 2.0 ** -8 * math.sqrt(6), (name, far)


def test_ranks_compute_what_one_rank_does():
    """As without the norm, whose rows are each one rank's: summed gradients agree to the order of 32-bit sums and the few
    roundings to bfloat16 that fall the other way for it, 2e-4 of their size."""
    x, t = batch(3)
    many, one = started(3, 5), started(1, 5)
    assert torch.equal(many.master, one.master)
    many.gradients(list(x.split(TOKENS)), list(t.split(TOKENS)))
    one.gradients([x], [t])
    for r in range(1, 3):
        assert torch.equal(many.buffers[0], many.buffers[r])
    for got, want in zip(many.grads[0], one.grads[0]):
        assert float((got - want).norm()) < 2e-4 * float(want.norm())


@pytest.mark.parametrize("kind", [FeedForward, NormedFeedForward])
def test_an_orthogonal_step_is_its_parts(kind):
    """The matrices move by -rate times the orthogonalised momentum (2^-20 of it and one rounding to 32 bits off; rate is 0.02,
    weights are below 1), the vectors by the momentum as ever; gradients reach the ranks' buffers before."""
    x, t = batch(4)
    xs, ts = list(x.split(TOKENS)), list(t.split(TOKENS))
    block, plain = kind(3, WIDTH, INNER, seed=9, lr=4.0, orthogonal=True), kind(3, WIDTH, INNER, seed=9, lr=4.0)
    before = block.master.clone()
    for b in (block, plain):
        b.step(xs, ts)
    assert torch.equal(block.velocity, plain.velocity)
    sizes = [w.numel() for w in (block.w1, block.b1, block.w2, block.b2, *block.norm)]
    at = 0
    for w, v, p, size in zip((block.w1, block.b1, block.w2, block.b2, *block.norm), block.momenta, (plain.w1, plain.b1, plain.w2, plain.b2, *plain.norm), sizes):
        old = before[at:at + size].view(w.shape)
        if w.dim() == 2:
            want = old.double().cpu() - 0.02 * max(1.0, w.shape[0] / w.shape[1]) ** 0.5 * tref.orthogonal(v)
            assert float((w.double().cpu() - want).abs().max()) < 2.0 ** -23
        else:
            assert torch.equal(w, old - 4.0 / INNER * v)
            assert torch.equal(w, p)
        at += size
    assert torch.equal(block.low[0], block.w1.bfloat16())
    # a second step runs on what the first left
    block.step(xs, ts)
    assert bool(block.master.isfinite().all())


def test_split_inner_dimension_with_the_norm():
    """As without: one bfloat16 rounding, which may fall the other way, apart."""
    x, _ = batch(5)
    for ranks in (1, 3):
        block = started(ranks, 6)
        want = block.forward(x, row0=11)[0].float()
        got = block.split(x, row0=11).float()
        assert bool(((got - want).abs() <= 2.0 ** -7 * want.abs() + 2.0 ** -12).all())


def test_the_command_runs(capsys):
    for flags in ([], ["--norm"], ["--orthogonal"], ["--norm", "--orthogonal"]):
        main(["--ranks", "2", "--tokens", "40", "--width", "64", "--inner", "136", "--steps", "2"] + flags)
    assert capsys.readouterr().out.count("step 1: loss") == 4
