"""The operators of worker-batched layers that are timed, with their plain forms.

W simulated workers train replicas of one model in one GPU's memory. Next to the optimizer and reconcile steps they
need the layers that make their gradients, for all workers at once: a root-mean-square norm with the residual's
addition and an 8-bit output, activation checkpoints in 8 bits with the weight gradient that reads them, and a gated
linear recurrence. Weights are slices of the workers' parameter rows and weight gradients slices of their gradient
rows, so both have the row's stride and whatever alignment the slice has.

- norm: s = x + residual, in x's type; y = weight * s / sqrt(mean(s^2) + eps). With a checkpoint y is held in 8 bits
  and returned as the values that these stand for. Backward: the gradients of x (with the residual stream's added) and
  of the weight.
- 8 bits: blocks of 32 neighbouring features share the exponent e, the least with max|x| <= 127 * 2^e; a value is held as
  the nearest whole number of 2^e (ties to even). Those values are exact in bfloat16.
- weight gradient: dW[w] = dy[w]^T x^[w], x^ the values held in 8 bits.
- recurrence: h_t = a_t h_(t-1) + (1 - a_t) v_t with a = sigmoid(gate), over each sequence's length; beyond it h is 0.
"""
from __future__ import annotations

import math

import torch

own = False

EPS = 1e-6
BLOCK = 32
DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


# -- cases ---------------------------------------------------------------------------------------------------------------

def _norm(W, M, D, dtype="bf16", train=True, checkpoint=True, residual=True, grad="f32", shift=0, **more):
    return dict(more, op="norm", W=W, M=M, D=D, dtype=dtype, train=train, checkpoint=checkpoint, residual=residual,
                grad=grad, shift=shift)


def _weight(W, M, I, O, dtype="bf16", grad="f32", shift=0, **more):
    return dict(more, op="weight", W=W, M=M, I=I, O=O, dtype=dtype, grad=grad, shift=shift)


def _rec(B, T, D, dtype="bf16", mode="train", ragged=False, **more):
    return dict(more, op="recurrence", B=B, T=T, D=D, dtype=dtype, mode=mode, ragged=ragged)


def listed():
    return [
        # One generated token for each of 4 sequences at width 384 (ViT-S/16's), served from one model: latency.
        _norm(1, 4, 384, train=False, checkpoint=False, name="norm_decode"),
        # A training step's norm: 8 workers, 16 images of 197 tokens each (ViT-S/16), bf16 gradients.
        _norm(8, 16 * 197, 384, grad="bf16", name="norm_train_w8"),
        # Odd width and token count in float32, the weight at an odd place of the worker's row, no checkpoint.
        _norm(2, 1021, 2731, dtype="f32", checkpoint=False, shift=3, name="norm_train_odd_f32"),
        # Long batches of a wide model: 4 workers, 8,192 tokens of width 4,096.
        _norm(4, 8192, 4096, name="norm_train_wide"),
        # A small network's layer (64 x 64) for 4 workers and 32 samples: the smallest training call.
        _weight(4, 32, 64, 64, name="weight_small"),
        # ViT-S/16's first MLP weight (1536 x 384) for 8 workers of 16 images, gradients in bf16.
        _weight(8, 16 * 197, 384, 1536, grad="bf16", name="weight_mlp_w8"),
        # Odd sizes in every direction, float32 activations, the gradient at an odd place of the row.
        _weight(2, 1999, 1003, 517, dtype="f32", shift=5, name="weight_odd_f32"),
        # A wide model's MLP weight for 2 workers and 16,384 tokens: bound by the tensor cores.
        _weight(2, 16384, 2048, 8192, grad="bf16", name="weight_wide"),
        # One generated token for each of 4 sequences: the state's step.
        _rec(4, 1, 384, mode="step", name="recurrence_decode"),
        # A training step over 8 workers' 16 sequences of 197 tokens.
        _rec(8 * 16, 197, 384, name="recurrence_train_w8"),
        # Sequences of differing length (none, one and odd ones among them), odd width, float32.
        _rec(6, 1500, 771, dtype="f32", ragged=True, name="recurrence_ragged_f32"),
        # One long document: 65,536 tokens; few rows, so the time axis has to be shared out.
        _rec(1, 65536, 1024, name="recurrence_long"),
    ]


def draw(rng):
    """Workers 1 to 32, tokens 1 to 65,536, widths 16 to 8,192; half of the sizes are odd or ragged. A case moves and
    computes at most what the largest listed one of its operator does."""
    def size(lo, hi, multiple):
        n = int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
        return n if rng.random() < 0.5 else max(multiple, n // multiple * multiple)

    while True:
        op = rng.choice(["norm", "weight", "recurrence"])
        dtype = rng.choice(["bf16", "bf16", "f32"])
        grad, shift = rng.choice(["f32", "bf16"]), rng.choice([0, 0, 0, 8, 1, 3])
        if op == "norm":
            train = rng.random() < 0.7
            c = _norm(size(1, 32, 1), size(1, 16384, 8), size(16, 8192, 32), dtype, train, rng.random() < 0.6,
                      rng.random() < 0.8, grad, shift)
        elif op == "weight":
            c = _weight(size(1, 32, 1), size(1, 32768, 64), size(16, 8192, 64), size(16, 8192, 64), dtype, grad, shift)
        else:
            mode = rng.choice(["train", "train", "forward", "step"])
            c = _rec(size(1, 256, 1), 1 if mode == "step" else size(1, 65536, 16), size(16, 8192, 32), dtype, mode,
                     mode != "step" and rng.random() < 0.4)
        largest = [work(x) for x in listed() if x["op"] == op]
        w = work(c)
        if w["bytes"] <= max(x["bytes"] for x in largest) and w["flops"] <= max(x["flops"] for x in largest):
            return c


def work(case):
    """Inputs read once and outputs written once; what a checkpoint holds is written by the forward pass and read by the
    backward pass."""
    e = 2 if case["dtype"] == "bf16" else 4
    if case["op"] == "norm":
        n = case["W"] * case["M"] * case["D"]
        row = e * (4 if case["residual"] else 2)  # x and the residual in, s and y out
        if case["checkpoint"]:
            row += 2 - e + 1 + 1 / BLOCK  # y in bf16, its codes and exponents
        flops = 8 * n
        params = 4 * case["W"] * case["D"]
        if case["train"]:
            row += 4 * e  # dy, s and the residual stream's gradient in, dx out
            flops += 14 * n
            params += (4 + (4 if case["grad"] == "f32" else 2)) * case["W"] * case["D"]
        return {"bytes": n * row + params, "flops": flops}
    if case["op"] == "weight":
        W, M, I, O = case["W"], case["M"], case["I"], case["O"]
        codes = 2 * (1 + 1 / BLOCK)
        return {"bytes": W * M * I * (e + 2 + codes) + W * M * O * 2 + W * I * O * (4 if case["grad"] == "f32" else 2),
                "flops": 2 * W * M * I * O}
    B, T, D = case["B"], case["T"], case["D"]
    read = B * T  # the tokens inside the lengths, on average
    if case["ragged"]:
        read = T + 1 + (B - 3) * T / 2 if B > 2 else T + (B - 1) * T / 2
    state = 4 * B * D
    if case["mode"] == "train":  # forward: gate and value in, h out; backward: gate, value and dh in, two gradients out
        return {"bytes": e * D * (5 * read + 3 * B * T) + 4 * state, "flops": 30 * read * D}
    return {"bytes": e * D * (2 * read + B * T) + 2 * state, "flops": 10 * read * D}


# -- inputs --------------------------------------------------------------------------------------------------------------

def _lengths(case, gen, dev):
    """Sequence lengths: anything from none to T, with an empty and a one-token sequence where there is room."""
    if not case["ragged"]:
        return None
    n = torch.randint(0, case["T"] + 1, (case["B"],), generator=gen, device=dev, dtype=torch.int32)
    n[0] = case["T"]
    if case["B"] > 2:
        n[1], n[2] = 0, 1
    return n


def prepare(case, seed):
    dev = torch.device("cuda")
    gen = torch.Generator(device=dev)
    gen.manual_seed(int(seed) * 1_000_003 + 17)
    dt = DTYPES[case["dtype"]]

    def normal(*shape, std=1.0, mean=0.0, to=dt):
        return torch.empty(shape, device=dev).normal_(mean, std, generator=gen).to(to)

    st = dict(case)
    if case["op"] == "norm":
        W, M, D, k = case["W"], case["M"], case["D"], case["shift"]
        st["x"] = normal(W, M, D, std=0.7)
        st["residual"] = normal(W, M, D, std=2.0) if case["residual"] else None
        params = normal(W, D + 2 * k, std=0.2, mean=1.0, to=torch.float32)
        st["weight"] = params[:, k:k + D]
        if case["train"]:
            st["dy"], st["ds"] = normal(W, M, D, std=1e-3), normal(W, M, D, std=1e-3)
            st["dweight"] = torch.zeros((W, D + 2 * k), device=dev, dtype=DTYPES[case["grad"]])[:, k:k + D]
    elif case["op"] == "weight":
        W, M, I, O, k = case["W"], case["M"], case["I"], case["O"], case["shift"]
        # activations after a norm: unit size, some features larger than others
        st["x"] = (normal(W, M, I, to=torch.float32) * normal(1, 1, I, std=0.5, to=torch.float32).exp_()).to(dt)
        st["dy"] = normal(W, M, O, std=1e-3, to=torch.bfloat16)
        st["dW"] = torch.zeros((W, O * I + 2 * k), device=dev, dtype=DTYPES[case["grad"]])[:, k:k + O * I].view(W, O, I)
    else:
        B, T, D = case["B"], case["T"], case["D"]
        both = torch.empty((B, T, 2 * D), device=dev, dtype=dt)  # one product's output: gates, then values
        both[..., :D].normal_(2.0, 1.5, generator=gen)
        both[..., D:].normal_(0.0, 1.0, generator=gen)
        if case["mode"] == "step":
            both = both[:, 0]
        st["gate"], st["value"] = both[..., :D], both[..., D:]
        st["h0"] = normal(B, D, std=0.5, to=torch.float32)
        st["lengths"] = _lengths(case, gen, dev)
        if case["mode"] == "train":
            st["dh"] = normal(B, T, D, std=1e-3)
            st["dh_last"] = normal(B, D, std=1e-3, to=torch.float32)
    return st


# -- one pass ------------------------------------------------------------------------------------------------------------

def run(state):
    return (_run_own if own else _run_plain)(state)


def _run_own(s):
    from paper_2607_21224_gb300 import layers

    if s["op"] == "norm":
        y, res, _ = layers.add_rmsnorm(s["x"], s["weight"], s["residual"], eps=EPS, checkpoint=s["checkpoint"])
        out = {"y": y, "s": res}
        if s["train"]:
            out["dx"], out["dweight"] = layers.add_rmsnorm_backward(s["dy"], res, s["weight"], s["ds"], eps=EPS,
                                                                    dweight=s["dweight"])
        return out
    if s["op"] == "weight":
        saved, values = layers.checkpoint(s["x"])
        return {"values": values, "dW": layers.weight_gradient(s["dy"], saved, out=s["dW"])}
    if s["mode"] == "step":
        return {"h": layers.gated_recurrence_step(s["gate"], s["value"], s["h0"]), "state": s["h0"]}
    h, last, carry = layers.gated_recurrence(s["gate"], s["value"], s["h0"], s["lengths"])
    out = {"h": h, "last": last}
    if s["mode"] == "train":
        out["dgate"], out["dvalue"], out["dh0"] = layers.gated_recurrence_backward(
            s["dh"], s["gate"], s["value"], carry, s["dh_last"], s["lengths"])
    return out


def _held(x):
    """The values that 8 bits hold of the float32 x, blocks of 32 along the last axis."""
    n = x.shape[-1]
    blocks = torch.nn.functional.pad(x, (0, -n % BLOCK)).unflatten(-1, (-1, BLOCK))
    top = blocks.abs().amax(-1, keepdim=True)
    fraction, power = torch.frexp(top)  # top = fraction * 2^power, fraction in [0.5, 1)
    e = (power - 7 + (fraction > 127 / 128)).clamp(-126, 121)
    unit = torch.ldexp(torch.ones_like(top), e)
    return ((blocks / unit).round() * unit).flatten(-2)[..., :n]


def _scan(a, b):
    """h_t = a_t h_(t-1) + b_t along axis 1 with h_0 = 0: spans double until they reach the start."""
    a, b, span = a.clone(), b.clone(), 1
    while span < a.shape[1]:
        b[:, span:] = b[:, span:] + a[:, span:] * b[:, :-span]
        a[:, span:] = a[:, span:] * a[:, :-span]
        span *= 2
    return b


def _run_plain(s):
    if s["op"] == "norm":
        x, weight = s["x"], s["weight"][:, None]
        res = (x.float() + s["residual"].float()).to(x.dtype) if s["residual"] is not None else x
        r = res.float()
        scale = (r.square().mean(-1, keepdim=True) + EPS).rsqrt()
        y = r * scale * weight
        out = {"y": _held(y).to(torch.bfloat16) if s["checkpoint"] else y.to(x.dtype), "s": res}
        if s["train"]:
            g = s["dy"].float()
            n = r * scale
            gw = g * weight
            dx = s["ds"].float() + scale * (gw - n * (gw * n).mean(-1, keepdim=True))
            s["dweight"].copy_((g * n).sum(1))
            out["dx"], out["dweight"] = dx.to(x.dtype), s["dweight"]
        return out
    if s["op"] == "weight":
        values = _held(s["x"].float())
        s["dW"].copy_(s["dy"].float().transpose(1, 2) @ values)
        return {"values": values.to(torch.bfloat16), "dW": s["dW"]}
    gate, v, h0 = s["gate"].float(), s["value"].float(), s["h0"]
    a, keep = torch.sigmoid(gate), torch.sigmoid(-gate)
    if s["mode"] == "step":
        h0.copy_(a * h0 + keep * v)
        return {"h": h0.to(s["value"].dtype), "state": h0}
    dt, lengths = s["value"].dtype, s["lengths"]
    inside = None
    if lengths is not None:  # beyond its length a sequence keeps its state and answers 0
        inside = (torch.arange(a.shape[1], device=a.device) < lengths[:, None])[..., None]
        a, keep, v = torch.where(inside, a, 1.0), torch.where(inside, keep, 0.0), torch.where(inside, v, 0.0)
    b = keep * v
    b[:, 0] += a[:, 0] * h0
    h = _scan(a, b)
    last = h[:, -1].clone()
    out = {"h": (h if inside is None else torch.where(inside, h, 0.0)).to(dt), "last": last}
    if s["mode"] == "train":
        dh = s["dh"].float() if inside is None else torch.where(inside, s["dh"].float(), 0.0)
        dh = torch.cat([dh[:, :-1], dh[:, -1:] + s["dh_last"][:, None]], 1)
        after = torch.cat([a[:, 1:], torch.ones_like(a[:, :1])], 1)  # what carries h_t's gradient back from t + 1
        g = _scan(after.flip(1), dh.flip(1)).flip(1)
        before = torch.cat([h0[:, None], h[:, :-1]], 1)
        out["dgate"] = (g * (before - v) * a * keep).to(dt)
        out["dvalue"] = (g * keep).to(dt)
        out["dh0"] = a[:, 0] * g[:, 0]
    return out


# -- in 64 bits ----------------------------------------------------------------------------------------------------------

def _held_exact(x):
    n = x.shape[-1]
    out = torch.zeros(x.shape[:-1] + (-(-n // BLOCK) * BLOCK,), dtype=torch.float64, device=x.device)
    out[..., :n] = x
    out = out.reshape(x.shape[:-1] + (-1, BLOCK))
    top = out.abs().max(-1, keepdim=True).values
    k = torch.frexp(top)[1].double() - 7  # top < 2^(k + 7), so the unit is 2^k or, above 127 of these, 2^(k + 1)
    unit = torch.ldexp(torch.ones_like(top), k)
    unit = torch.where(top > 127.0 * unit, 2.0 * unit, unit).clamp(2.0 ** -126, 2.0 ** 121)
    return (torch.round(out / unit) * unit).reshape(x.shape[:-1] + (-1,))[..., :n]


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "norm":
        x = s["x"]
        if s["residual"] is not None:
            x = (x.double() + s["residual"].double()).to(x.dtype)  # the residual stream as it is held
        r, w = x.double(), s["weight"].double().unsqueeze(1)
        rms = torch.sqrt((r * r).mean(dim=-1, keepdim=True) + EPS)
        y = w * r / rms
        out = {"y": _held_exact(y) if case["checkpoint"] else y, "s": r}
        if case["train"]:
            g = s["dy"].double()
            dot = (g * w * r).mean(dim=-1, keepdim=True)
            out["dx"] = s["ds"].double() + g * w / rms - r * dot / rms ** 3
            out["dweight"] = torch.einsum("wmd,wmd->wd", g, r / rms)
        return out
    if case["op"] == "weight":
        values = _held_exact(s["x"].double())
        return {"values": values, "dW": torch.einsum("wmo,wmi->woi", s["dy"].double(), values)}
    x, v, h = s["gate"].double(), s["value"].double(), s["h0"].double()
    if case["mode"] == "step":
        h = h / (1.0 + torch.exp(-x)) + v / (1.0 + torch.exp(x))
        return {"h": h, "state": h}
    B, T, D = case["B"], case["T"], case["D"]
    a = 1.0 / (1.0 + torch.exp(-x))
    rest = 1.0 / (1.0 + torch.exp(x))
    if s["lengths"] is not None:
        beyond = (torch.arange(T, device=v.device)[None] >= s["lengths"][:, None])[..., None]
        a.masked_fill_(beyond, 1.0)
        rest.masked_fill_(beyond, 0.0)
    b = rest * v
    states = torch.empty((T + 1, B, D), dtype=torch.float64, device=v.device)
    states[0] = h
    for t in range(T):  # the definition, a step at a time
        torch.addcmul(b[:, t], a[:, t], states[t], out=states[t + 1])
    h = states[1:].transpose(0, 1)
    out = {"h": h.masked_fill(beyond, 0.0) if s["lengths"] is not None else h, "last": states[T]}
    if case["mode"] == "train":
        dh = s["dh"].double()
        if s["lengths"] is not None:
            dh.masked_fill_(beyond, 0.0)
        g, totals = s["dh_last"].double(), torch.empty_like(dh)
        for t in range(T - 1, -1, -1):
            torch.add(g, dh[:, t], out=totals[:, t])
            g = totals[:, t] * a[:, t]
        out["dvalue"] = totals * rest
        out["dgate"] = out["dvalue"] * (states[:-1].transpose(0, 1) - v) * a
        out["dh0"] = g
    return out
