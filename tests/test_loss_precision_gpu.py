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
