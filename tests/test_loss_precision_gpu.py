"""The loss's errors by their norms, relative to that of the result: what per-element
bounds, which count every rounding at its worst, let pass.

A tensor core cuts a float32 sum off after each product of 16 terms, by half a
spacing on average, 0.72 x 2^-24 of it for sums of any size. Over the 16 such
products of a chunk, whose partial sums grow to the chunk's like sqrt(i / 16), that
is 16 x 0.72 x 2^-24 x 2/3 = 4.6e-7 of the chunk's sum, towards 0 (a chunk of eight
times the length loses 3.7e-6). Chunks are added to each other with errors of 3e-8."""
import pytest
import torch

from paper_2607_21224_gb300 import layers

F32, BF16 = torch.float32, torch.bfloat16


def operands(W, M, D, V, dtype, device="cuda"):
    gen = torch.Generator().manual_seed(W + 3 * M + 5 * D + 7 * V)
    x = torch.randn(W, M, D, generator=gen).to(dtype)
    weight = (torch.randn(W, V, D, generator=gen) * 1.5 / D ** 0.5).to(dtype)
    targets = torch.randint(0, V, (W, M), generator=gen)
    targets[torch.rand(W, M, generator=gen) < 0.05] = -1
    dloss = torch.rand(W, M, generator=gen) / M
    return [t.to(device) for t in (x, weight, targets, dloss)]


def formulas(x, weight, targets, dloss):
    """loss, lse, dx, dweight in 64 bits."""
    a, w = x.double(), weight.double()
    logits = a @ w.transpose(1, 2)
    lse = torch.logsumexp(logits, -1)
    at, real = targets.clamp(min=0)[..., None], targets >= 0
    loss = torch.where(real, lse - logits.gather(-1, at)[..., 0], 0.0)
    d = torch.exp(logits - lse[..., None]).scatter_add_(-1, at, torch.full_like(lse, -1.0)[..., None])
    d *= (dloss.double() * real)[..., None]
    return loss, lse, d @ w, d.transpose(1, 2) @ a


def off(got, want):
    return float((got.double() - want).norm() / want.norm())


# Logits have a deviation of 1.5 and losses are some 8 to 12: 4.6e-7 x 1.5 of the target's logit and, as the words with
# large logits count, 4.6e-7 x 1.5^2 of lse, are 6e-8 and 1e-7 of them; lse and loss are rounded by 3e-8 each.
LOSS_OFF = 2e-7


@pytest.mark.gpu
@pytest.mark.parametrize("W,M,D,V", [(1, 4, 1024, 32768), (2, 300, 2048, 10000), (1, 200, 3001, 4001), (3, 77, 128, 5000)])
def test_losses_of_bfloat16_operands(W, M, D, V):
    x, weight, targets, dloss = operands(W, M, D, V, BF16)
    loss, lse = layers.linear_cross_entropy(x, weight, targets)
    want = formulas(x, weight, targets, dloss)
    assert off(loss, want[0]) < LOSS_OFF and off(lse, want[1]) < LOSS_OFF


# The chunks' 4.6e-7, at a deviation of 0.3 of the logits; lse, which the backward pass takes as float32, is off by up to
# half a spacing, 2.8e-7 on average between 8 and 16, which is a factor of the token's d; powers and planes by 1e-7 each.
GRADIENTS_OFF = 1e-6
# A bfloat16 output that is off by 1e-6 goes to another neighbour than the formula's value with a probability of at most
# 1e-6 / 2^-8, and is a spacing away then, 2^-7.5 on average.
BF16_OFF = (1e-6 * 2 ** 8) ** 0.5 * 2 ** -7.5


@pytest.mark.gpu
@pytest.mark.parametrize("W,M,D,V", [(4, 200, 128, 64), (1, 300, 300, 4096), (1, 300, 300, 4097), (1, 512, 128, 8192), (2, 130, 1027, 20001),
                                     (1, 2000, 96, 1000)])
def test_gradients_of_bfloat16_operands(W, M, D, V):
    x, weight, targets, dloss = operands(W, M, D, V, BF16)
    lse = layers.linear_cross_entropy(x, weight, targets)[1]
    dx, dweight = layers.linear_cross_entropy_backward(dloss, x, weight, targets, lse)
    want = formulas(x, weight, targets, dloss)
    assert dweight.dtype is F32 and off(dweight, want[3]) < GRADIENTS_OFF
    narrow = layers.linear_cross_entropy_backward(dloss, x, weight, targets, lse, dtype=BF16)[1]
    for got, exact in ((dx, want[2]), (narrow, want[3])):
        assert got.dtype is BF16 and off(got, exact.to(BF16).double()) < BF16_OFF


@pytest.mark.gpu
def test_one_large_gradient_beside_small_ones():
    """A token whose dloss is 2^40 times the others' takes nothing from their precision."""
    x, weight, targets, dloss = operands(1, 200, 128, 5000, BF16)
    dloss[0, 0] = 2.0 ** 40
    lse = layers.linear_cross_entropy(x, weight, targets)[1]
    dx = layers.linear_cross_entropy_backward(dloss, x, weight, targets, lse)[0]
    want = formulas(x, weight, targets, dloss)[2]
    assert off(dx[:, 1:], want[:, 1:].to(BF16).double()) < BF16_OFF


@pytest.mark.gpu
def test_an_infinite_gradient_follows_the_formula():
    x, weight, targets, dloss = operands(1, 150, 128, 5000, BF16)
    targets[0, 7], dloss[0, 7] = 3, float("inf")
    lse = layers.linear_cross_entropy(x, weight, targets)[1]
    dx, dweight = layers.linear_cross_entropy_backward(dloss, x, weight, targets, lse)
    _, _, ex, ew = formulas(x, weight, targets, dloss)
    assert torch.isnan(ex[0, 7]).all() and torch.isinf(ew).all()  # x has no zeros
    for got, want in ((dx, ex), (dweight, ew)):
        assert torch.equal(torch.isnan(got), torch.isnan(want)) and torch.equal(got[torch.isinf(want)].double(), want[torch.isinf(want)])


@pytest.mark.gpu
@pytest.mark.parametrize("W,M,D,V", [(1, 25, 771, 5000), (2, 200, 300, 4001), (1, 130, 64, 70), (1, 300, 1024, 9000)])
def test_float32_operands(W, M, D, V):
    x, weight, targets, dloss = operands(W, M, D, V, F32)
    loss, lse = layers.linear_cross_entropy(x, weight, targets)
    got = loss, lse, *layers.linear_cross_entropy_backward(dloss, x, weight, targets, lse)
    want = formulas(x, weight, targets, dloss)
    for g, w, most in zip(got, want, (LOSS_OFF, LOSS_OFF, GRADIENTS_OFF, GRADIENTS_OFF)):
        assert off(g, w) < most


@pytest.mark.gpu
def test_the_largest_float32_numbers():
    """3.4e38 is nearer to 2^128 than to bfloat16's largest number."""
    x, weight, targets, dloss = operands(1, 60, 100, 300, F32)
    x[0, :, 0], x[0, 7, 0] = 0, torch.finfo(F32).max
    weight[0, :, 0] = 0
    loss, lse = layers.linear_cross_entropy(x, weight, targets)
    dx, dweight = layers.linear_cross_entropy_backward(dloss * 1e-3, x, weight, targets, lse)
    want = formulas(x, weight, targets, dloss * 1e-3)
    assert off(loss, want[0]) < LOSS_OFF and off(lse, want[1]) < LOSS_OFF
    assert off(dx, want[2]) < GRADIENTS_OFF and off(dweight[..., 0], want[3][..., 0]) < GRADIENTS_OFF
    assert off(dweight[..., 1:], want[3][..., 1:]) < GRADIENTS_OFF
    x, weight, targets, dloss = operands(1, 60, 100, 300, F32)  # and as weights
    weight[0, 5, 0], weight[0, 6, 0] = torch.finfo(F32).max, -torch.finfo(F32).max
    x[0, :, 0] = 0
    loss, lse = layers.linear_cross_entropy(x, weight, targets)
    assert off(loss, formulas(x, weight, targets, dloss)[0]) < LOSS_OFF


@pytest.mark.gpu
@pytest.mark.parametrize("W,M,D,V,dtype", [(1, 900, 40, 220001, F32), (2, 450, 70, 200300, BF16)])
def test_a_vocabulary_in_pieces(W, M, D, V, dtype):
    """Three parts of d for 900 tokens stay below 1 GiB up to 198,841 words: two pieces, the second off every border."""
    x, weight, targets, dloss = operands(W, M, D, V, dtype)
    loss, lse = layers.linear_cross_entropy(x, weight, targets)
    dx, dweight = layers.linear_cross_entropy_backward(dloss, x, weight, targets, lse)
    want = formulas(x, weight, targets, dloss)
    assert off(loss, want[0]) < LOSS_OFF and off(lse, want[1]) < LOSS_OFF
    half = V // 2 + 1000
    for part in (slice(0, half), slice(half, V), slice(V - 100, V)):
        assert off(dweight[:, part], want[3][:, part]) < GRADIENTS_OFF
    assert off(dx, want[2]) < GRADIENTS_OFF if dtype is F32 else off(dx, want[2].to(BF16).double()) < BF16_OFF
    assert (dx[targets < 0] == 0).all()


def test_a_lost_plane_is_seen():
    """Three products of two planes each, on the CPU: what they leave out is above the limits."""
    x, weight, targets, dloss = operands(1, 130, 300, 1000, F32, "cpu")

    def planes(t, count):
        held = torch.zeros_like(t)
        for _ in range(count):
            held = held + (t - held).to(BF16).float()
        return held

    want = formulas(x, weight, targets, dloss)
    two = formulas(planes(x, 2), planes(weight, 2), targets, dloss)
    assert all(off(t, w) > 2 * GRADIENTS_OFF for t, w in zip(two[2:], want[2:]))
    three = formulas(planes(x, 3), planes(weight, 3), targets, dloss)
    assert all(off(t, w) < 1e-7 for t, w in zip(three, want))
