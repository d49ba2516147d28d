"""The loss, the clipping, the convolution and the scan together, as a training
program uses them (examples/recurrent_lm.py with the scan as its mixer): the whole
model's gradients against autograd on the same model in float32, a short run, and
tokens generated by single steps against the same model's passes over sequences."""
import importlib.util
from pathlib import Path

import pytest
import torch
import torch.nn.functional as F

from paper_2607_21224_gb300 import layers

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def lm():
    path = Path(__file__).resolve().parents[1] / "examples" / "recurrent_lm.py"
    spec = importlib.util.spec_from_file_location("recurrent_lm", path)
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


def plain_loss(model, theta, tokens):
    """The model of one worker in float32, without 8 bits: its mean loss, and each block's delta, whose gradient is that
    of the step sizes token by token."""
    deltas = []
    B, T, D, N, K = tokens.shape[0], tokens.shape[1] - 1, model.width, model.states, model.taps
    norm = lambda s, w: w * s / torch.sqrt(s.square().mean(-1, keepdim=True) + 1e-6)  # noqa: E731
    part = lambda n: model.view(theta, n)  # noqa: E731
    s = x = part("embed")[tokens[:, :-1]]
    for b in range(model.blocks):
        s = x if b == 0 else s + x
        both = norm(s, part(f"norm{b}")) @ part(f"in{b}").T
        x, z = F.pad(both[..., :D], (0, 0, K - 1, 0)), both[..., D:]
        u = F.silu(part(f"conv_bias{b}") + sum(x[:, k:k + T] * part(f"conv{b}")[:, k] for k in range(K)))
        delta, bs, cs = (u @ part(f"mix{b}").T).split((D, N, N), -1)
        delta.retain_grad()
        deltas.append(delta)
        dt, rate = F.softplus(delta + part(f"dt_bias{b}")), torch.exp(part(f"a_log{b}"))
        h, ys = torch.zeros(B, D, N, device=theta.device), []
        for t in range(T):
            h = torch.exp(-dt[:, t, :, None] * rate) * h + (dt * u)[:, t, :, None] * bs[:, t, None]
            ys.append((h * cs[:, t, None]).sum(-1) + part(f"skip{b}") * u[:, t])
        x = (torch.stack(ys, 1) * F.silu(z)) @ part(f"out{b}").T
    logits = norm(s + x, part("norm")) @ part("head").T
    return F.cross_entropy(logits.flatten(0, 1), tokens[:, 1:].flatten()), deltas


def test_gradients_of_the_whole_model(lm):
    W, B, T = 3, 4, 37
    model = lm.RecurrentLM(vocab=41, width=72, blocks=2, mixer="scan", states=8)
    gen = torch.Generator(device="cuda").manual_seed(5)
    params = torch.stack([model.init(gen) for _ in range(W)])
    tokens = lm.counting(gen, (W, B), T + 1, model.vocab)
    grads = torch.full((W, model.N), float("nan"), device="cuda")
    loss = model.step(params, grads, tokens)
    assert torch.isfinite(grads).all()  # every parameter has its gradient
    for w in range(W):
        theta = params[w].clone().requires_grad_()
        want, deltas = plain_loss(model, theta, tokens[w])
        want.backward()
        assert abs(float(loss[w]) - float(want.detach())) <= 0.02 * float(want.detach())
        for name in model.shapes:
            got, ref = model.view(grads[w], name).flatten(), model.view(theta.grad, name).flatten()
            # 8-bit activations (0.7 % each, three per block), bfloat16 activations and products (0.4 % each), over two blocks
            size = ref.norm()
            if name.startswith("dt_bias"):
                # the sum over 148 tokens of g_t, the gradients of delta, of both signs: where each is off by at most a
                # share r of |g_t|, the sum is off by at most r sum(|g_t|), which is not small beside it as the sum itself is
                size = deltas[int(name[-1])].grad.abs().sum((0, 1)).norm()
            assert float((got - ref).norm() / size) <= 0.08, name


def test_a_step_with_clipping(lm):
    model = lm.RecurrentLM(vocab=17, width=40, blocks=1, mixer="scan")
    gen = torch.Generator(device="cuda").manual_seed(6)
    params = torch.stack([model.init(gen) for _ in range(2)])
    grads = torch.zeros((2, model.N), device="cuda")
    model.step(params, grads, lm.counting(gen, (2, 3), 20, model.vocab))
    want = grads.double()
    norms = layers.clip_gradients(grads, 0.5 * float(want.norm(dim=1).min()))
    assert torch.allclose(norms.double(), want.norm(dim=1), rtol=1e-5)
    assert torch.allclose(grads.double().norm(dim=1), 0.5 * want.norm(dim=1).min().expand(2), rtol=1e-5)


@pytest.mark.parametrize("mixer", ["recurrence", "scan"])
def test_training_and_generation_run(lm, mixer):
    model, st, losses = lm.train(steps=8, mixer=mixer)
    assert all(0 < x < 10 for x in losses)
    prompt = lm.counting(torch.Generator(device="cuda").manual_seed(7), (3,), 6, model.vocab)
    made = model.generate(st.anchor, prompt, 4)
    st.close()
    assert made.shape == (3, 4) and ((made >= 0) & (made < model.vocab)).all()
    assert layers.wait_timeouts() == 0


def test_mixer_steps_are_the_pass(lm):
    """A sequence through the mixer at once, and token by token."""
    model = lm.RecurrentLM(vocab=17, width=48, blocks=1, mixer="scan")
    gen = torch.Generator(device="cuda").manual_seed(8)
    theta = model.init(gen)
    B, T = 3, 21
    both = torch.randn(B, T, 2 * model.width, generator=gen, device="cuda").bfloat16()
    h, _ = model._mix(theta[None], {k: v[None] for k, v in model._products(theta).items()}, 0, both)
    state, weight = model._mix_state(B, theta.device), model._products(theta)
    for t in range(T):
        y = model._mix_step(theta, weight, 0, both[:, t], state)
        # one rounding to bfloat16 each, and products of bfloat16 that torch may sum in another order
        assert torch.allclose(y.float(), h[:, t].float(), rtol=2.0 ** -6, atol=2.0 ** -7 * float(h.abs().max()))
