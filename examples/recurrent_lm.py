"""W simulated workers train a small recurrent language model with CPDP, all on
one GPU, and the trained model generates tokens.

Every worker's layers run in the same calls (paper_2607_21224_gb300.layers); the
products between them are torch.bmm. Weights are views into ``CPDPState.params``
and the backward pass writes its gradients straight into the [W][N] gradient
buffer that ``CPDPState.step`` takes. The inputs of the blocks' products are held
in 8 bits for their weight gradients, the head's input and the rest in bfloat16.

The model: an embedding, blocks of (norm, product, mixer, product) on a residual
stream, a norm and a head, whose loss is taken without the logits. The mixer is a
gated recurrence, or a short convolution and a selective scan. Each worker's
gradients are clipped to a norm. The data: sequences that count up by a step of
their own, modulo the vocabulary.

    python examples/recurrent_lm.py [--steps 200] [--mixer scan]
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

    def __init__(self, vocab: int = 64, width: int = 128, blocks: int = 2, mixer: str = "recurrence", states: int = 16, taps: int = 4):
        self.vocab, self.width, self.blocks, self.mixer, self.states, self.taps = vocab, width, blocks, mixer, states, taps
        D = width
        shapes = [("embed", (vocab, D))]
        for b in range(blocks):
            shapes += [(f"norm{b}", (D,)), (f"in{b}", (2 * D, D)), (f"out{b}", (D, D))]
            if mixer == "scan":  # what the scan takes of a token (step size, b, c) is a product of the convolution's output
                shapes += [(f"conv{b}", (D, taps)), (f"conv_bias{b}", (D,)), (f"mix{b}", (D + 2 * states, D)), (f"a_log{b}", (D, states)),
                           (f"skip{b}", (D,)), (f"dt_bias{b}", (D,))]
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
            if name.startswith("a_log"):
                part.copy_(torch.arange(1, shape[1] + 1, device=theta.device).log().expand(shape))
            elif name.startswith("dt_bias"):  # steps of about 0.1
                part.fill_(math.log(math.expm1(0.1)))
            elif name.startswith("conv_bias"):
                part.zero_()
            elif len(shape) == 1:
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
        weight = self._products(params)
        worker = torch.arange(W, device=tokens.device)[:, None]

        x, s, held = weight["embed"][worker, inputs], None, []
        for b in range(self.blocks):
            y, s, normed = layers.add_rmsnorm(x, self.view(params, f"norm{b}"), s, checkpoint=True)
            both = torch.bmm(y, weight[f"in{b}"].transpose(1, 2)).view(W * B, T, 2 * D)
            h, mixed = self._mix(params, weight, b, both)
            states, h = layers.checkpoint(h.view(W, M, D))
            x = torch.bmm(h, weight[f"out{b}"].transpose(1, 2))
            held.append((s, normed, both, mixed, states))
        y, s, _ = layers.add_rmsnorm(x, self.view(params, "norm"), s)
        losses, lse = layers.linear_cross_entropy(y, weight["head"], targets)
        loss = losses.mean(1)

        dy, _ = layers.linear_cross_entropy_backward(torch.full_like(losses, 1.0 / M), y, weight["head"], targets, lse,
                                                     dweight=self.view(grads, "head"))
        ds, _ = layers.add_rmsnorm_backward(dy, s, self.view(params, "norm"), dweight=self.view(grads, "norm"))
        for b in reversed(range(self.blocks)):
            s, normed, both, mixed, states = held[b]
            layers.weight_gradient(ds, states, out=self.view(grads, f"out{b}"))
            dh = torch.bmm(ds, weight[f"out{b}"]).view(W * B, T, D)
            dboth = self._mix_backward(params, weight, grads, b, both, mixed, dh).view(W, M, 2 * D)
            layers.weight_gradient(dboth, normed, out=self.view(grads, f"in{b}"))
            ds, _ = layers.add_rmsnorm_backward(torch.bmm(dboth, weight[f"in{b}"]), s, self.view(params, f"norm{b}"), ds,
                                                dweight=self.view(grads, f"norm{b}"))
        dembed = torch.zeros((W, self.vocab, D), device=ds.device)
        dembed.index_put_((worker.expand(W, M), inputs), ds.float(), accumulate=True)
        self.view(grads, "embed").copy_(dembed)
        return loss

    def _products(self, params: torch.Tensor) -> dict:
        """The weights of the products, in bfloat16."""
        return {n: self.view(params, n).to(BF16) for n in self.shapes if n.startswith(("embed", "head", "in", "out", "mix"))}

    def _scan_weights(self, params: torch.Tensor, b: int) -> tuple:
        return tuple(self.view(params, f"{n}{b}") for n in ("a_log", "skip", "dt_bias"))

    def _mix(self, params: torch.Tensor, weight: dict, b: int, both: torch.Tensor) -> tuple:
        """The mixer's output (W B, T, D) from the two halves of `both`, and what its backward pass needs."""
        D, N = self.width, self.states
        if self.mixer == "recurrence":
            h, _, carry = layers.gated_recurrence(both[..., :D], both[..., D:])
            return h, carry
        W, T = params.shape[0], both.shape[1]
        u, _ = layers.causal_conv(both[..., :D], self.view(params, f"conv{b}"), self.view(params, f"conv_bias{b}"))
        held, u = layers.checkpoint(u.view(W, -1, D))
        per = torch.bmm(u, weight[f"mix{b}"].transpose(1, 2)).view(-1, T, D + 2 * N)
        delta, bs, cs = per.split((D, N, N), -1)
        a_log, skip, bias = self._scan_weights(params, b)
        h, _, carry = layers.selective_scan(u.view(-1, T, D), delta, a_log, bs, cs, skip, bias, both[..., D:])
        return h, (held, per, carry)

    def _mix_backward(self, params: torch.Tensor, weight: dict, grads: torch.Tensor, b: int, both: torch.Tensor, mixed, dh: torch.Tensor):
        """The gradient of `both`; the mixer's weights' go to their parts of `grads`."""
        D, N = self.width, self.states
        dboth = torch.empty_like(both)
        if self.mixer == "recurrence":
            layers.gated_recurrence_backward(dh, both[..., :D], both[..., D:], mixed, out=dboth)
            return dboth
        held, per, carry = mixed
        W, T, part = params.shape[0], both.shape[1], lambda n: self.view(grads, f"{n}{b}")
        u = layers.restore(held)
        delta, bs, cs = per.split((D, N, N), -1)
        a_log, skip, bias = self._scan_weights(params, b)
        du, ddelta, _, db, dc, _, _, dz, _ = layers.selective_scan_backward(
            dh, u.view(-1, T, D), delta, a_log, bs, cs, skip, bias, carry, both[..., D:], da_log=part("a_log"), dskip=part("skip"),
            dbias=part("dt_bias"))
        dper = torch.cat((ddelta, db, dc), -1).view(W, -1, D + 2 * N)
        layers.weight_gradient(dper, held, out=part("mix"))
        du = torch.baddbmm(du.view(W, -1, D), dper, weight[f"mix{b}"]).view(-1, T, D)
        dx, _, _ = layers.causal_conv_backward(du, both[..., :D], self.view(params, f"conv{b}"), self.view(params, f"conv_bias{b}"),
                                               dweight=part("conv"), dbias=part("conv_bias"))
        dboth[..., :D], dboth[..., D:] = dx, dz
        return dboth

    def _mix_step(self, theta: torch.Tensor, weight: dict, b: int, both: torch.Tensor, state: tuple) -> torch.Tensor:
        """The mixer's output (B, D) for one token; its states are moved on."""
        D, N = self.width, self.states
        if self.mixer == "recurrence":
            return layers.gated_recurrence_step(both[:, :D], both[:, D:], *state)
        u = layers.causal_conv_step(both[:, :D], self.view(theta, f"conv{b}"), self.view(theta, f"conv_bias{b}"), state[0])
        u = layers.checkpoint(u[None])[1][0]  # the values that training sees
        delta, bs, cs = (u @ weight[f"mix{b}"].T).split((D, N, N), -1)
        a_log, skip, bias = self._scan_weights(theta, b)
        return layers.selective_scan_step(u, delta, a_log, bs, cs, skip, bias, state[1], both[:, D:])

    def _mix_state(self, B: int, device) -> tuple:
        if self.mixer == "recurrence":
            return (torch.zeros((B, self.width), device=device),)
        return (torch.zeros((B, self.taps - 1, self.width), dtype=BF16, device=device), torch.zeros((B, self.width, self.states), device=device))

    def generate(self, theta: torch.Tensor, prompt: torch.Tensor, count: int) -> torch.Tensor:
        """`count` tokens after prompt (B, T), the likeliest each time, by single steps of the mixers."""
        B = prompt.shape[0]
        weight = self._products(theta)
        states = [self._mix_state(B, theta.device) for _ in range(self.blocks)]
        tokens = list(prompt.unbind(1))
        for t in range(prompt.shape[1] + count - 1):
            x, s = weight["embed"][tokens[t]], None
            for b in range(self.blocks):
                y, s, _ = layers.add_rmsnorm(x, self.view(theta, f"norm{b}"), s)
                both = y @ weight[f"in{b}"].T
                x = self._mix_step(theta, weight, b, both, states[b]) @ weight[f"out{b}"].T
            if t >= prompt.shape[1] - 1:
                y, _, _ = layers.add_rmsnorm(x, self.view(theta, "norm"), s)
                tokens.append((y @ weight["head"].T).argmax(-1))
        return torch.stack(tokens[prompt.shape[1]:], 1)


def counting(gen: torch.Generator, shape: tuple, length: int, vocab: int) -> torch.Tensor:
    """Sequences that count up by 1 to 4, modulo the vocabulary, from anywhere."""
    start = torch.randint(0, vocab, shape, generator=gen, device=gen.device)
    by = torch.randint(1, 5, shape, generator=gen, device=gen.device)
    return (start[..., None] + by[..., None] * torch.arange(length, device=gen.device)) % vocab


def train(steps: int = 200, W: int = 4, B: int = 16, T: int = 48, K: int = 4, seed: int = 1, mixer: str = "recurrence", max_norm: float = 10.0):
    """Returns (model, state, mean losses)."""
    gen = torch.Generator(device="cuda").manual_seed(seed)
    model = RecurrentLM(mixer=mixer)
    st = CPDPState(W, model.N, model.tensor_offsets, lr=2e-3, momentum=0.0, weight_decay=0.01, K=K, beta=0.3)
    st.set_adamw(beta1=0.9, beta2=0.99)
    st.init_params(model.init(gen))
    grads = torch.zeros((W, model.N), device="cuda")
    losses = []
    for t in range(1, steps + 1):
        losses.append(model.step(st.params, grads, counting(gen, (W, B), T + 1, model.vocab)).mean())
        layers.clip_gradients(grads, max_norm)
        st.step(grads, t, steps)
    return model, st, torch.stack(losses).tolist()


def main() -> None:
    parser = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    parser.add_argument("--steps", type=int, default=200)
    parser.add_argument("--mixer", choices=("recurrence", "scan"), default="recurrence")
    args = parser.parse_args()
    model, st, losses = train(args.steps, mixer=args.mixer)
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
