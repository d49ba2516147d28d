"""W simulated workers train a small recurrent language model with CPDP, all on
one GPU, and the trained model generates tokens.

Every worker's layers run in the same calls (paper_2607_21224_gb300.layers); the
products between them are torch.bmm. Weights are views into ``CPDPState.params``
and the backward pass writes its gradients straight into the [W][N] gradient
buffer that ``CPDPState.step`` takes. What the backward pass needs of the
activations is held in 8 bits.

The model: an embedding, blocks of (norm, product, gated recurrence, product)
on a residual stream, a norm and a head. The data: sequences that count up by a
step of their own, modulo the vocabulary.

    python examples/recurrent_lm.py [--steps 200]
"""
from __future__ import annotations

import argparse
import math
import sys
from pathlib import Path

import torch

sys.path.insert(0, str(Path(__file__).resolve().parents[1]))
from paper_2607_21224_gb300 import layers  # noqa: E402
from paper_2607_21224_gb300.state import CPDPState  # noqa: E402

BF16 = torch.bfloat16


class RecurrentLM:
    """The model's layout in a flat parameter vector, and its passes."""

    def __init__(self, vocab: int = 64, width: int = 128, blocks: int = 2):
        self.vocab, self.width, self.blocks = vocab, width, blocks
        D = width
        shapes = [("embed", (vocab, D))]
        for b in range(blocks):
            shapes += [(f"norm{b}", (D,)), (f"in{b}", (2 * D, D)), (f"out{b}", (D, D))]
        shapes += [("norm", (D,)), ("head", (vocab, D))]
        self.shapes, self.offsets = dict(shapes), {}
        n = 0
        for name, shape in shapes:
            self.offsets[name] = n
            n += math.prod(shape)
        self.N = n

    @property
    def tensor_offsets(self) -> list[int]:
        return [*self.offsets.values(), self.N]

    def init(self, gen: torch.Generator) -> torch.Tensor:
        theta = torch.empty(self.N, device=gen.device)
        for name, shape in self.shapes.items():
            part = self.view(theta, name)
            if len(shape) == 1:
                part.fill_(1.0)
            else:
                part.normal_(0.0, 0.02 if name in ("embed", "head") else shape[1] ** -0.5, generator=gen)
        return theta

    def view(self, rows: torch.Tensor, name: str) -> torch.Tensor:
        """Tensor `name` in a flat vector (N,) or in each worker's row (W, N)."""
        shape, a = self.shapes[name], self.offsets[name]
        return rows[..., a:a + math.prod(shape)].unflatten(-1, shape)

    def step(self, params: torch.Tensor, grads: torch.Tensor, tokens: torch.Tensor) -> torch.Tensor:
        """Each worker's mean loss on tokens (W, B, T + 1); its gradients go to its row of `grads` (W, N)."""
        W, B, T = tokens.shape[0], tokens.shape[1], tokens.shape[2] - 1
        M, D = B * T, self.width
        inputs, targets = tokens[..., :-1].reshape(W, M), tokens[..., 1:].reshape(W, M)
        weight = {n: self.view(params, n).to(BF16) for n, shape in self.shapes.items() if len(shape) == 2}
        worker = torch.arange(W, device=tokens.device)[:, None]

        x, s, held = weight["embed"][worker, inputs], None, []
        for b in range(self.blocks):
            y, s, normed = layers.add_rmsnorm(x, self.view(params, f"norm{b}"), s, checkpoint=True)
            both = torch.bmm(y, weight[f"in{b}"].transpose(1, 2)).view(W * B, T, 2 * D)
            gate, value = both[..., :D], both[..., D:]
            h, _, carry = layers.gated_recurrence(gate, value)
            states, h = layers.checkpoint(h.view(W, M, D))
            x = torch.bmm(h, weight[f"out{b}"].transpose(1, 2))
            held.append((s, normed, gate, value, carry, states))
        y, s, normed = layers.add_rmsnorm(x, self.view(params, "norm"), s, checkpoint=True)
        logp = torch.bmm(y, weight["head"].transpose(1, 2)).float().log_softmax(-1)
        loss = -logp.gather(-1, targets[..., None]).mean((1, 2))

        dlogits = logp.exp()
        dlogits.scatter_add_(-1, targets[..., None], torch.full_like(logp[..., :1], -1.0))
        dlogits = (dlogits / M).to(BF16)
        layers.weight_gradient(dlogits, normed, out=self.view(grads, "head"))
        dy = torch.bmm(dlogits, weight["head"])
        ds, _ = layers.add_rmsnorm_backward(dy, s, self.view(params, "norm"), dweight=self.view(grads, "norm"))
        for b in reversed(range(self.blocks)):
            s, normed, gate, value, carry, states = held[b]
            layers.weight_gradient(ds, states, out=self.view(grads, f"out{b}"))
            dh = torch.bmm(ds, weight[f"out{b}"]).view(W * B, T, D)
            dboth = torch.empty((W * B, T, 2 * D), dtype=BF16, device=dh.device)
            layers.gated_recurrence_backward(dh, gate, value, carry, out=dboth)
            dboth = dboth.view(W, M, 2 * D)
            layers.weight_gradient(dboth, normed, out=self.view(grads, f"in{b}"))
            ds, _ = layers.add_rmsnorm_backward(torch.bmm(dboth, weight[f"in{b}"]), s, self.view(params, f"norm{b}"), ds,
                                                dweight=self.view(grads, f"norm{b}"))
        dembed = torch.zeros((W, self.vocab, D), device=ds.device)
        dembed.index_put_((worker.expand(W, M), inputs), ds.float(), accumulate=True)
        self.view(grads, "embed").copy_(dembed)
        return loss

    def generate(self, theta: torch.Tensor, prompt: torch.Tensor, count: int) -> torch.Tensor:
        """`count` tokens after prompt (B, T), the likeliest each time, by single steps of the recurrences."""
        B, D = prompt.shape[0], self.width
        weight = {n: self.view(theta, n).to(BF16) for n, shape in self.shapes.items() if len(shape) == 2}
        states = [torch.zeros((B, D), device=theta.device) for _ in range(self.blocks)]
        tokens = list(prompt.unbind(1))
        for t in range(prompt.shape[1] + count - 1):
            x, s = weight["embed"][tokens[t]], None
            for b in range(self.blocks):
                y, s, _ = layers.add_rmsnorm(x, self.view(theta, f"norm{b}"), s)
                both = y @ weight[f"in{b}"].T
                x = layers.gated_recurrence_step(both[:, :D], both[:, D:], states[b]) @ weight[f"out{b}"].T
            if t >= prompt.shape[1] - 1:
                y, _, _ = layers.add_rmsnorm(x, self.view(theta, "norm"), s)
                tokens.append((y @ weight["head"].T).argmax(-1))
        return torch.stack(tokens[prompt.shape[1]:], 1)


def counting(gen: torch.Generator, shape: tuple, length: int, vocab: int) -> torch.Tensor:
    """Sequences that count up by 1 to 4, modulo the vocabulary, from anywhere."""
    start = torch.randint(0, vocab, shape, generator=gen, device=gen.device)
    by = torch.randint(1, 5, shape, generator=gen, device=gen.device)
    return (start[..., None] + by[..., None] * torch.arange(length, device=gen.device)) % vocab


def train(steps: int = 200, W: int = 4, B: int = 16, T: int = 48, K: int = 4, seed: int = 1):
    """Returns (model, state, mean losses)."""
    gen = torch.Generator(device="cuda").manual_seed(seed)
    model = RecurrentLM()
    st = CPDPState(W, model.N, model.tensor_offsets, lr=2e-3, momentum=0.0, weight_decay=0.01, K=K, beta=0.3)
    st.set_adamw(beta1=0.9, beta2=0.99)
    st.init_params(model.init(gen))
    grads = torch.zeros((W, model.N), device="cuda")
    losses = []
    for t in range(1, steps + 1):
        losses.append(model.step(st.params, grads, counting(gen, (W, B), T + 1, model.vocab)).mean())
        st.step(grads, t, steps)
    return model, st, torch.stack(losses).tolist()


def main() -> None:
    parser = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    parser.add_argument("--steps", type=int, default=200)
    args = parser.parse_args()
    model, st, losses = train(args.steps)
    for t in range(0, len(losses), max(1, len(losses) // 10)):
        print(f"step {t + 1:4d}  loss {losses[t]:.3f}")
    print(f"step {len(losses):4d}  loss {losses[-1]:.3f}")
    prompt = counting(torch.Generator(device="cuda").manual_seed(7), (4,), 8, model.vocab)
    made = model.generate(st.anchor, prompt, 8)
    for p, m in zip(prompt.tolist(), made.tolist()):
        print(p, "->", m)
    st.close()


if __name__ == "__main__":
    main()
