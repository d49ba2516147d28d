"""The loss, the clipping, the convolution and the scan on arrays of more than 2^32
elements: their last parts against the same calls on those parts alone, or against
the formulas in 64 bits."""
import pytest
import torch

from paper_2607_21224_gb300 import layers
from test_layers_gpu import near

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16
T, D = (1 << 20) + 35, 4100  # T D = 2^32 + 4.3 million


def many(*shape, seed=0, std=1.0):
    return torch.empty(shape, dtype=BF16, device="cuda").normal_(0.0, std, generator=torch.Generator(device="cuda").manual_seed(seed))


def test_conv():
    x, dy = many(1, T, D), many(1, T, D, seed=1)
    weight, bias = torch.randn(1, D, 4, device="cuda"), torch.randn(1, D, device="cuda")
    y, last = layers.causal_conv(x, weight, bias)
    dx = layers.causal_conv_backward(dy, x, weight, bias)[0]
    assert torch.equal(last, x[:, -3:])
    # the last 50 steps, from the inputs before them
    tail, state = x[:, -50:].contiguous(), x[:, -53:-50].contiguous()
    assert torch.equal(layers.causal_conv(tail, weight, bias, state)[0], y[:, -50:])
    assert torch.equal(layers.causal_conv_backward(dy[:, -50:].contiguous(), tail, weight, bias, state)[0], dx[:, -50:])


def test_scan():
    N = 4
    u, delta = many(1, T, D), many(1, T, D, seed=1)
    b, c = many(1, T, N, seed=2), many(1, T, N, seed=3)
    a_log, skip, bias = torch.randn(1, D, N, device="cuda"), torch.randn(1, D, device="cuda"), torch.randn(1, D, device="cuda")
    y, last, carry = layers.selective_scan(u, delta, a_log, b, c, skip, bias)
    at = T // layers.CARRY_STEPS * layers.CARRY_STEPS  # the last chunk, of 3 steps
    cut = [t[:, at:].contiguous() for t in (u, delta, b, c)]
    tail = layers.selective_scan(cut[0], cut[1], a_log, cut[2], cut[3], skip, bias, h0=carry[:, -1].contiguous())
    assert T - at == 3 and torch.equal(tail[0], y[:, at:]) and torch.equal(tail[1], last)
    dlast = torch.randn_like(last)
    grads = layers.selective_scan_backward(y, u, delta, a_log, b, c, skip, bias, carry, dlast=dlast)
    want = layers.selective_scan_backward(y[:, at:].contiguous(), cut[0], cut[1], a_log, cut[2], cut[3], skip, bias, tail[2], dlast=dlast)
    for i in (0, 1, 3, 4):  # du, ddelta, db, dc
        assert torch.equal(grads[i][:, at:], want[i])


def test_clip():
    g = many(2, (1 << 32) + 77)
    tail = g[1, -1000:].clone()
    norms = layers.clip_gradients(g, 1.0)
    # 2^32 squares with mean 1 and deviation sqrt(2): 6 deviations are 1.3e-4 of their sum, half of that of the root
    assert (norms / 2.0 ** 16 - 1).abs().max() < 1e-4
    want = tail.double() / norms[1].double()
    near(g[1, -1000:], want.cpu(), want.abs().cpu() * 2.0 ** -22)


def test_loss():
    M, D, V = 40, 2048, (1 << 21) + 5
    x, weight = many(1, M, D), many(1, V, D, seed=1, std=0.05)
    targets = torch.arange(M, device="cuda")[None] * 50000 + (V - 1 - 39 * 50000)
    loss, lse = layers.linear_cross_entropy(x, weight, targets)
    dloss = torch.full((1, M), 0.3, device="cuda")
    dw = layers.linear_cross_entropy_backward(dloss, x, weight, targets, lse, dtype=BF16)[1]
    words = torch.arange(V - 70, V, device="cuda")
    logits = x[0].double() @ weight[0, words].double().T
    # logits are sums of 2,048 products of about 0.05 each: cut off by at most 2 * 2048 * 2^-24 of their magnitudes' sum
    size = float((x[0].double().abs() @ weight[0, words].double().abs().T).amax()) * 2 * 2064 * 2.0 ** -24
    assert abs(float(loss[0, -1]) - float(lse[0, -1] - logits[-1, -1])) <= 2 * size + 1e-5
    hot = (targets[0][:, None] == words).double()
    d = 0.3 * (torch.exp(logits - lse[0].double()[:, None]) - hot)
    want = d.T @ x[0].double()
    # d: its rounding to bfloat16, and the logits' error
    bound = (2.0 ** -8 + 2 * size) * (d.abs().T @ x[0].double().abs())
    near(dw[0, words], want.cpu(), bound.cpu())
