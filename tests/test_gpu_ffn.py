"""The feed-forward example on the GPU: P data-parallel ranks compute the
gradients that one rank with all tokens does, the loss falls, and the block with
its inner dimension dealt out over ranks gives the same result."""
import pytest
import torch

from paper_2004_09362_amd.ffn import FeedForward

pytestmark = pytest.mark.gpu

WIDTH, INNER, TOKENS = 200, 520, (70, 33, 97)


def batch(seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    x = torch.empty(sum(TOKENS), WIDTH, device="cuda").normal_(generator=g).bfloat16()
    return x, x.roll(1, 1)


def test_ranks_compute_what_one_rank_does():
    """The masks are those of the whole batch's rows, and every y, h and dz of a token is the same number whoever holds it,
    up to the order of 32-bit sums (2^-24 of 520 terms, so that a rounding to bfloat16 falls the other way for about one
    value in 500, by 2^-8 of it): the summed gradients agree to 2^-8 / sqrt(500) of their size, 2e-4."""
    x, t = batch(3)
    many, one = FeedForward(3, WIDTH, INNER, seed=5), FeedForward(1, WIDTH, INNER, seed=5)
    assert torch.equal(many.master, one.master)
    a = many.gradients(list(x.split(TOKENS)), list(t.split(TOKENS)))
    b = one.gradients([x], [t])
    assert abs(float(a) - float(b)) < 1e-4 * float(b)
    for r in range(1, 3):
        assert torch.equal(many.buffers[0], many.buffers[r])
    for got, want in zip(many.grads[0], one.grads[0]):
        assert float((got - want).norm()) < 2e-4 * float(want.norm())


def test_training_lowers_the_loss():
    x, t = batch(4)
    block = FeedForward(3, WIDTH, INNER, p=0.05, lr=WIDTH * 0.5)
    losses = [float(block.step(list(x.split(TOKENS)), list(t.split(TOKENS)))) for _ in range(8)]
    assert losses[-1] < 0.9 * losses[0], losses


def test_split_inner_dimension():
    """Each hidden value is rounded as before; the partial sums are in 32 bits; the result is rounded once: one
    bfloat16 rounding, which may fall the other way, apart."""
    x, _ = batch(5)
    for ranks in (1, 3, 7):
        block = FeedForward(ranks, WIDTH, INNER, seed=6)
        want = block.forward(x, row0=11)[0].float()
        got = block.split(x, row0=11).float()
        assert bool(((got - want).abs() <= 2.0 ** -7 * want.abs() + 2.0 ** -12).all())
