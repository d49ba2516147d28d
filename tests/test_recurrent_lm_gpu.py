"""The layers together, as a training program uses them (examples/recurrent_lm.py):
the whole model's gradients against autograd on the same model in float32, then a
short CPDP run whose loss falls, whose replicas agree, and whose model continues
the sequences that it was trained on."""
import importlib.util
from pathlib import Path

import pytest
import torch
import torch.nn.functional as F

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def lm():
    path = Path(__file__).resolve().parents[1] / "examples" / "recurrent_lm.py"
    spec = importlib.util.spec_from_file_location("recurrent_lm", path)
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


def plain_loss(model, theta, tokens):
    """The model of one worker in float32, without 8 bits: its mean loss."""
    B, T, D = tokens.shape[0], tokens.shape[1] - 1, model.width
    norm = lambda s, w: w * s / torch.sqrt(s.square().mean(-1, keepdim=True) + 1e-6)  # noqa: E731
    s = x = model.view(theta, "embed")[tokens[:, :-1]]
    for b in range(model.blocks):
        s = x if b == 0 else s + x
        both = norm(s, model.view(theta, f"norm{b}")) @ model.view(theta, f"in{b}").T
        a, v = torch.sigmoid(both[..., :D]), both[..., D:]
        h, hs = torch.zeros(B, D, device=theta.device), []
        for t in range(T):
            h = a[:, t] * h + (1 - a[:, t]) * v[:, t]
            hs.append(h)
        x = torch.stack(hs, 1) @ model.view(theta, f"out{b}").T
    logits = norm(s + x, model.view(theta, "norm")) @ model.view(theta, "head").T
    return F.cross_entropy(logits.flatten(0, 1), tokens[:, 1:].flatten())


def test_gradients_of_the_whole_model(lm):
    W, B, T = 3, 4, 37
    model = lm.RecurrentLM(vocab=41, width=72, blocks=2)
    gen = torch.Generator(device="cuda").manual_seed(5)
    params = torch.stack([model.init(gen) for _ in range(W)])
    tokens = lm.counting(gen, (W, B), T + 1, model.vocab)
    grads = torch.full((W, model.N), float("nan"), device="cuda")
    loss = model.step(params, grads, tokens)
    assert torch.isfinite(grads).all()  # every parameter has its gradient
    for w in range(W):
        theta = params[w].clone().requires_grad_()
        want = plain_loss(model, theta, tokens[w])
        want.backward()
        assert abs(float(loss[w]) - float(want.detach())) <= 0.02 * float(want.detach())
        for name in model.shapes:
            got, ref = model.view(grads[w], name).flatten(), model.view(theta.grad, name).flatten()
            # 8-bit activations (0.7 % each), bfloat16 activations and products (0.4 % each), over two blocks
            assert float((got - ref).norm() / ref.norm()) <= 0.06, name


def test_workers_train_and_the_model_generates(lm):
    model, st, losses = lm.train(steps=240)
    with st:
        assert losses[0] > 3.5 and sum(losses[-10:]) / 10 < 0.6
        assert all(torch.equal(st.params[0], st.params[w]) for w in range(st.W))  # the last step synchronizes
        prompt = lm.counting(torch.Generator(device="cuda").manual_seed(9), (32,), 24, model.vocab)
        made = model.generate(st.anchor, prompt[:, :16], 8)
        assert float((made == prompt[:, 16:]).float().mean()) > 0.9
