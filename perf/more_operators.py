"""Operators of a language model's training step around the worker-batched layers, timed, with their plain forms.

W simulated workers train replicas of one language model in one GPU's memory. Next to the layers between its products a
training step needs the loss over the vocabulary with its gradients, the gradients' norm with their clipping before the
optimizer's step, and a block that mixes tokens: a short causal convolution and a selective state space scan, with their
steps for one generated token. Weights are slices of the workers' parameter rows.

- loss: logits = x weight^T, lse = log(sum(exp(logits))), loss = lse - logits[target], for every token; 0 where the target
  is negative. Backward: with d = dloss * (exp(logits - lse) - onehot(target)), dx = d weight and dweight = d^T x. The logits
  are kept nowhere.
- clip: norm = sqrt(sum(g^2)) over a worker's row, g * min(1, max_norm / norm).
- conv: y_t = silu(bias + sum_k weight[k] x_(t - K + 1 + k)), what lies before the first token taken from a state of the
  K - 1 inputs before it; that state after the last token. Beyond a sequence's length y is 0.
- scan: dt = softplus(delta + bias), h_t = exp(-dt exp(a_log)) h_(t-1) + dt u_t b_t with N states per channel,
  y_t = (sum_n c_t h_t + skip u_t) * silu(z_t). Beyond a sequence's length y is 0 and the state stays.
"""
from __future__ import annotations

import math

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


# -- cases ---------------------------------------------------------------------------------------------------------------

def _loss(W, M, D, V, dtype="bf16", train=True, **more):
    return dict(more, op="loss", W=W, M=M, D=D, V=V, dtype=dtype, train=train)


def _clip(W, N, dtype="f32", shift=0, **more):
    return dict(more, op="clip", W=W, N=N, dtype=dtype, shift=shift)


def _conv(W, B, T, D, K=4, dtype="bf16", mode="train", ragged=False, **more):
    return dict(more, op="conv", W=W, B=B, T=T, D=D, K=K, dtype=dtype, mode=mode, ragged=ragged)


def _scan(W, B, T, D, N=16, dtype="bf16", mode="train", ragged=False, **more):
    return dict(more, op="scan", W=W, B=B, T=T, D=D, N=N, dtype=dtype, mode=mode, ragged=ragged)


def listed():
    return [
        # The example's step: 4 workers, 16 sequences of 48 tokens, width 128, 64 words: launches and latency.
        _loss(4, 16 * 48, 128, 64, name="loss_small"),
        # The likelihood of four tokens under one model: bound by reading the head's weight.
        _loss(1, 4, 1024, 32768, train=False, name="loss_score"),
        # Odd sizes in every direction, float32.
        _loss(2, 517, 771, 10007, dtype="f32", name="loss_odd_f32"),
        # A training step of two workers, 4,096 tokens each, over a large vocabulary: bound by the tensor cores.
        _loss(2, 4096, 2048, 50000, name="loss_wide"),
        # A small model's gradients (the example's size) for 4 workers.
        _clip(4, 115000, name="clip_small"),
        # ResNet-50's gradient rows for 8 workers.
        _clip(8, 23712932, name="clip_resnet50"),
        # One generated token for each of 4 sequences, twice ViT-S/16's width.
        _conv(1, 4, 1, 768, mode="step", name="conv_decode"),
        # A training step over 8 workers' 16 sequences of 197 tokens.
        _conv(8, 8 * 16, 197, 768, name="conv_train_w8"),
        # One generated token for each of 4 sequences.
        _scan(1, 4, 1, 768, mode="step", name="scan_decode"),
        # A training step over 8 workers' 16 sequences of 197 tokens.
        _scan(8, 8 * 16, 197, 768, name="scan_train_w8"),
        # Sequences of differing length (none, one and odd ones among them), odd width, float32.
        _scan(2, 6, 1500, 387, dtype="f32", ragged=True, name="scan_ragged_f32"),
        # One long prompt: few channels' worth of work side by side, so the time axis has to be shared out.
        _scan(1, 1, 16384, 1024, mode="forward", name="scan_long"),
    ]


def draw(rng):
    """Workers 1 to 8, tokens 1 to 16,384, widths 16 to 4,096, vocabularies 16 to 65,536, rows of 1,000 to 30 million
    gradients, 1 to 32 states; half of the sizes are odd or ragged. A case moves and computes at most what the largest
    listed one of its operator does."""
    def size(lo, hi, multiple):
        n = int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
        return n if rng.random() < 0.5 else max(multiple, n // multiple * multiple)

    while True:
        op = rng.choice(["loss", "loss", "clip", "conv", "scan", "scan"])
        dtype = rng.choice(["bf16", "bf16", "f32"])
        W = size(1, 8, 1)
        mode = rng.choice(["train", "train", "forward", "step"])
        T = 1 if mode == "step" else size(1, 16384, 16)
        ragged = mode != "step" and rng.random() < 0.4
        if op == "loss":
            c = _loss(W, size(1, 8192, 64), size(16, 4096, 64), size(16, 65536, 256), dtype, rng.random() < 0.7)
        elif op == "clip":
            c = _clip(W, size(1000, 30000000, 64), dtype, rng.choice([0, 0, 1, 3, 8]))
        elif op == "conv":
            c = _conv(W, W * size(1, 32, 1), T, size(16, 4096, 64), rng.choice([2, 3, 4, 4]), dtype, mode, ragged)
        else:
            c = _scan(W, W * size(1, 32, 1), T, size(16, 4096, 64), rng.choice([1, 4, 7, 8, 16, 16, 16, 32]), dtype, mode, ragged)
        largest = [work(x) for x in listed() if x["op"] == op]
        w = work(c)
        if w["bytes"] <= max(x["bytes"] for x in largest) and w["flops"] <= max(x["flops"] for x in largest):
            return c


def _tokens_read(case):
    """The tokens inside the lengths, on average."""
    B, T = case["B"], case["T"]
    if not case["ragged"]:
        return B * T
    return T + 1 + (B - 3) * T / 2 if B > 2 else T + (B - 1) * T / 2


def work(case):
    """Inputs read once and outputs written once. A training step counts the forward pass and the backward pass, each
    input once for both; a loss counts its three products (the logits, dx, dweight)."""
    e = 2 if case["dtype"] == "bf16" else 4
    W = case["W"]
    if case["op"] == "loss":
        M, D, V = case["M"], case["D"], case["V"]
        once = e * (W * M * D + W * V * D)
        if not case["train"]:
            return {"bytes": once + 16 * W * M, "flops": 2 * W * M * V * D}
        return {"bytes": 2 * once + 20 * W * M, "flops": 6 * W * M * V * D}
    if case["op"] == "clip":
        return {"bytes": 2 * e * W * case["N"] + 4 * W, "flops": 3 * W * case["N"]}
    B, T, D = case["B"], case["T"], case["D"]
    read, train = _tokens_read(case), case["mode"] == "train"
    if case["op"] == "conv":
        K = case["K"]
        params, state = 4 * W * D * (K + 1), e * B * (K - 1) * D
        if train:  # x and dy in, y and dx out
            return {"bytes": e * D * (2 * read + 2 * B * T) + 2 * params + 2 * state, "flops": (6 * K + 16) * read * D}
        return {"bytes": e * D * (read + B * T) + params + 2 * state, "flops": (2 * K + 5) * read * D}
    N = case["N"]
    params, state = 4 * W * D * (N + 2), 4 * B * D * N
    if train:  # u, delta, z, dy and b, c in; y, three gradients, db and dc out
        return {"bytes": e * (D * (4 * read + 4 * B * T) + N * (2 * read + 2 * B * T)) + 2 * params + 4 * state,
                "flops": 24 * read * D * N + 60 * read * D}
    return {"bytes": e * (D * (3 * read + B * T) + N * 2 * read) + params + 2 * state, "flops": 8 * read * D * N + 20 * read * D}


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
    gen.manual_seed(int(seed) * 1_000_003 + 29)
    dt = DTYPES[case["dtype"]]

    def normal(*shape, std=1.0, mean=0.0, to=dt):
        return torch.empty(shape, device=dev).normal_(mean, std, generator=gen).to(to)

    def params(*shape, std=1.0, mean=0.0):
        """Float32 weights inside longer rows, as those of the parameter rows."""
        n = math.prod(shape[1:])
        return normal(shape[0], n + 3, std=std, mean=mean, to=torch.float32)[:, :n].view(shape)

    st, W = dict(case), case["W"]
    if case["op"] == "loss":
        M, D, V = case["M"], case["D"], case["V"]
        st["x"] = normal(W, M, D)
        st["weight"] = normal(W, V, D, std=1.5 / math.sqrt(D))  # logits of a spread that training reaches
        st["targets"] = torch.randint(0, V, (W, M), generator=gen, device=dev)
        padded = torch.rand((W, M), generator=gen, device=dev) < 0.05
        st["targets"][padded] = -1
        if case["train"]:
            st["dloss"] = torch.full((W, M), 1.0 / M, device=dev)
            st["dweight"] = torch.zeros((W, V, D), dtype=dt, device=dev)
        return st
    if case["op"] == "clip":
        N, k = case["N"], case["shift"]
        rows = torch.empty((W, N + 2 * k), dtype=dt, device=dev)
        for w in range(W):  # a row at a time: the workers' gradients differ in size, and not all of them are above the norm
            rows[w] = normal(N + 2 * k, std=(0.3 + 0.5 * (w % 4)) / math.sqrt(N))
        st["grads"] = rows[:, k:k + N]
        st["out"] = torch.zeros((W, N + 2 * k), dtype=dt, device=dev)[:, k:k + N]
        st["max_norm"] = 1.0
        return st
    B, T, D = case["B"], case["T"], case["D"]
    st["lengths"] = _lengths(case, gen, dev)
    if case["op"] == "conv":
        K = case["K"]
        st["x"] = normal(B, T, D) if case["mode"] != "step" else normal(B, D)
        st["weight"], st["bias"] = params(W, D, K, std=1.0 / math.sqrt(K)), params(W, D, std=0.1)
        st["state"] = normal(B, K - 1, D)
        if case["mode"] == "train":
            st["dy"] = normal(B, T, D, std=1e-3)
        return st
    N = case["N"]
    many = (B, D) if case["mode"] == "step" else (B, T, D)
    few = many[:-1] + (N,)
    st["u"], st["delta"], st["z"] = normal(*many, std=0.7), normal(*many, std=0.5), normal(*many)
    st["b"], st["c"] = normal(*few), normal(*few)
    steps = torch.arange(1, N + 1, device=dev, dtype=torch.float32).log()
    st["a_log"] = params(W, D, N, std=0.1).add_(steps)  # decays from slow to fast, as such models start
    st["skip"] = params(W, D, std=0.2, mean=1.0)
    size = torch.empty((W, D), device=dev).uniform_(math.log(1e-3), math.log(1e-1), generator=gen).exp_()
    st["bias"] = params(W, D)
    st["bias"].copy_(size.expm1().log())  # softplus(bias) = size
    st["h0"] = normal(B, D, N, std=0.5, to=torch.float32)
    if case["mode"] == "train":
        st["dy"] = normal(B, T, D, std=1e-3)
        st["dlast"] = normal(B, D, N, std=1e-3, to=torch.float32)
    return st


# -- one pass ------------------------------------------------------------------------------------------------------------

def run(state):
    return (_run_own if own else _run_plain)(state)


def _run_own(s):
    from paper_2607_21224_gb300 import layers

    if s["op"] == "loss":
        loss, lse = layers.linear_cross_entropy(s["x"], s["weight"], s["targets"])
        out = {"loss": loss, "lse": lse}
        if s["train"]:
            out["dx"], out["dweight"] = layers.linear_cross_entropy_backward(s["dloss"], s["x"], s["weight"], s["targets"], lse,
                                                                             dweight=s["dweight"])
        return out
    if s["op"] == "clip":
        return {"norms": layers.clip_gradients(s["grads"], s["max_norm"], out=s["out"]), "clipped": s["out"]}
    if s["op"] == "conv":
        if s["mode"] == "step":
            return {"y": layers.causal_conv_step(s["x"], s["weight"], s["bias"], s["state"]), "state": s["state"]}
        y, last = layers.causal_conv(s["x"], s["weight"], s["bias"], s["state"], s["lengths"])
        out = {"y": y, "last": last}
        if s["mode"] == "train":
            out["dx"], out["dweight"], out["dbias"] = layers.causal_conv_backward(s["dy"], s["x"], s["weight"], s["bias"], s["state"],
                                                                                  s["lengths"])
        return out
    inputs = s["u"], s["delta"], s["a_log"], s["b"], s["c"], s["skip"], s["bias"]
    if s["mode"] == "step":
        return {"y": layers.selective_scan_step(*inputs, s["h0"], s["z"]), "state": s["h0"]}
    y, last, carry = layers.selective_scan(*inputs, s["z"], s["h0"], s["lengths"], carry=s["mode"] == "train")
    out = {"y": y, "last": last}
    if s["mode"] == "train":
        grads = layers.selective_scan_backward(s["dy"], *inputs, carry, s["z"], s["dlast"], s["lengths"])
        out.update(zip(("du", "ddelta", "da_log", "db", "dc", "dskip", "dbias", "dz", "dh0"), grads))
    return out


def _along(a, b):
    """h_t = a_t h_(t-1) + b_t along axis 1 with h_0 = 0: spans double until they reach the start."""
    a, span = a.clone(), 1
    while span < a.shape[1]:
        b = torch.cat([b[:, :span], torch.addcmul(b[:, span:], a[:, span:], b[:, :-span])], 1)
        a[:, span:] = a[:, span:] * a[:, :-span]
        span *= 2
    return b


def _inside(s, like):
    """Which tokens (B, T, 1) lie within the lengths; None: all."""
    if s["lengths"] is None:
        return None
    return (torch.arange(like.shape[1], device=like.device) < s["lengths"][:, None])[..., None]


def _of_sequences(t, B):
    """A worker's parameters (W, ...) for each of its sequences: (B, 1, ...)."""
    return t.repeat_interleave(B // t.shape[0], 0)[:, None]


def _run_plain(s):
    return {"loss": _plain_loss, "clip": _plain_clip, "conv": _plain_conv, "scan": _plain_scan}[s["op"]](s)


def _plain_loss(s):
    x, weight, targets = s["x"].float(), s["weight"].float(), s["targets"]
    real = targets >= 0
    at = targets.clamp(min=0)[..., None]
    logits = x @ weight.transpose(1, 2)
    top = logits.amax(-1, keepdim=True)
    lse = (logits - top).exp_().sum(-1).log() + top[..., 0]
    loss = torch.where(real, lse - logits.gather(-1, at)[..., 0], 0.0)
    out = {"loss": loss, "lse": lse}
    if s["train"]:
        d = logits.sub_(lse[..., None]).exp_()
        d.scatter_add_(-1, at, torch.full_like(lse, -1.0)[..., None])
        d.mul_(torch.where(real, s["dloss"], 0.0)[..., None])
        out["dx"] = (d @ weight).to(s["x"].dtype)
        s["dweight"].copy_(d.transpose(1, 2) @ x)
        out["dweight"] = s["dweight"]
    return out


def _plain_clip(s):
    g = s["grads"].float()
    norms = g.square().sum(-1, dtype=torch.float64).sqrt().float()
    scale = (s["max_norm"] / norms).clamp(max=1.0)
    s["out"].copy_(g * scale[:, None])
    return {"norms": norms, "clipped": s["out"]}


def _silu_slope(v):
    gate = torch.sigmoid(v)
    return gate * (1.0 + v * (1.0 - gate))


def _plain_conv(s):
    K, B = s["K"], s["x"].shape[0]
    x, dt = s["x"].float(), s["x"].dtype
    step = x.dim() == 2
    if step:
        x = x[:, None]
    T = x.shape[1]
    weight, bias = _of_sequences(s["weight"], B), _of_sequences(s["bias"], B)
    inside = None if step else _inside(s, x)
    before = torch.cat([s["state"].float(), x], 1)  # input t is at K - 1 + t
    spans = before.unfold(1, K, 1)  # (B, T, D, K)
    v = bias + (spans * weight).sum(-1)
    y = v * torch.sigmoid(v)
    if inside is not None:
        y = torch.where(inside, y, 0.0)
    n = torch.full((B,), T, device=x.device) if inside is None else s["lengths"].long()
    at = (n[:, None] + torch.arange(K - 1, device=x.device))[..., None].expand(-1, -1, x.shape[2])
    last = before.gather(1, at).to(dt)
    if step:
        s["state"].copy_(last)
        return {"y": y[:, 0].to(dt), "state": s["state"]}
    out = {"y": y.to(dt), "last": last}
    if s["mode"] == "train":
        dv = s["dy"].float() * _silu_slope(v)
        if inside is not None:
            dv = torch.where(inside, dv, 0.0)
        after = torch.cat([dv, dv.new_zeros(B, K - 1, dv.shape[2])], 1)
        out["dx"] = (after.unfold(1, K, 1) * weight.flip(-1)).sum(-1).to(dt)
        workers = lambda t: t.unflatten(0, (s["W"], -1)).sum(1)  # noqa: E731
        out["dweight"] = workers((dv[..., None] * spans).sum(1))
        out["dbias"] = workers(dv.sum(1))
    return out


def _plain_scan(s):
    dt, step = s["u"].dtype, s["u"].dim() == 2
    u, delta, z, b, c = (t.float()[:, None] if step else t.float() for t in (s["u"], s["delta"], s["z"], s["b"], s["c"]))
    B, T, D = u.shape
    A, skip, bias = -_of_sequences(s["a_log"], B).exp(), _of_sequences(s["skip"], B), _of_sequences(s["bias"], B)
    inside = None if step else _inside(s, u)
    raw = delta + bias
    size = raw.clamp(min=0.0) + torch.log1p(torch.exp(-raw.abs()))  # softplus
    if inside is not None:  # beyond its length a sequence keeps its state
        size = torch.where(inside, size, 0.0)
    a = (size[..., None] * A).exp()
    h = (size * u)[..., None] * b[:, :, None]
    h[:, 0] += a[:, 0] * s["h0"]
    h = _along(a, h)
    sums = (h * c[:, :, None]).sum(-1) + skip * u
    gate = torch.sigmoid(z)
    y = sums * z * gate
    if inside is not None:
        y = torch.where(inside, y, 0.0)
    last = h[:, -1].clone()
    if step:
        s["h0"].copy_(last)
        return {"y": y[:, 0].to(dt), "state": s["h0"]}
    out = {"y": y.to(dt), "last": last}
    if s["mode"] == "train":
        dy = s["dy"].float()
        if inside is not None:
            dy = torch.where(inside, dy, 0.0)
        out["dz"] = (dy * sums * _silu_slope(z)).to(dt)
        gy = dy * z * gate
        reach = gy[..., None] * c[:, :, None]
        reach[:, -1] += s["dlast"]
        after = torch.cat([a[:, 1:], torch.ones_like(a[:, :1])], 1)  # what carries h_t's gradient back from t + 1
        g = _along(after.flip(1), reach.flip(1)).flip(1)
        del reach, after
        workers = lambda t: t.unflatten(0, (s["W"], -1)).sum(1)  # noqa: E731
        before = torch.cat([s["h0"][:, None], h[:, :-1]], 1)
        decay = g * before * a * A  # per unit of the step's size
        through = (g * b[:, :, None]).sum(-1)
        dsize = decay.sum(-1) + through * u
        dbase = dsize * torch.sigmoid(raw)
        if inside is not None:
            dbase = torch.where(inside, dbase, 0.0)
        out["du"] = (through * size + skip * gy).to(dt)
        out["ddelta"] = dbase.to(dt)
        out["da_log"] = workers((decay * size[..., None]).sum(1))
        out["db"] = (g * (size * u)[..., None]).sum(2).to(dt)
        out["dc"] = (h * gy[..., None]).sum(2).to(dt)
        out["dskip"], out["dbias"] = workers((gy * u).sum(1)), workers(dbase.sum(1))
        out["dh0"] = a[:, 0] * g[:, 0]
    return out


# -- in 64 bits ----------------------------------------------------------------------------------------------------------

def exact(case, seed):
    s = prepare(case, seed)
    return {"loss": _exact_loss, "clip": _exact_clip, "conv": _exact_conv, "scan": _exact_scan}[case["op"]](case, s)


def _exact_loss(case, s):
    """Tokens in groups, so that their logits fit."""
    W, M, D, V = (case[k] for k in "WMDV")
    out = {"loss": torch.zeros((W, M), dtype=torch.float64, device="cuda"), "lse": torch.zeros((W, M), dtype=torch.float64, device="cuda")}
    if case["train"]:
        out["dx"] = torch.zeros((W, M, D), dtype=torch.float64, device="cuda")
        out["dweight"] = torch.zeros((W, V, D), dtype=torch.float64, device="cuda")
    for w in range(W):
        weight = s["weight"][w].double()
        for m in range(0, M, 4096):
            rows = slice(m, min(M, m + 4096))
            x, t = s["x"][w, rows].double(), s["targets"][w, rows]
            logits = torch.einsum("md,vd->mv", x, weight)
            lse = torch.logsumexp(logits, -1)
            chosen = torch.zeros_like(logits)
            chosen[torch.nonzero(t >= 0)[:, 0], t[t >= 0]] = 1.0
            out["lse"][w, rows] = lse
            out["loss"][w, rows] = torch.where(t >= 0, lse - (logits * chosen).sum(-1), torch.zeros_like(lse))
            if case["train"]:
                logits.sub_(lse.unsqueeze(-1)).exp_().sub_(chosen)
                logits.mul_((s["dloss"][w, rows].double() * (t >= 0)).unsqueeze(-1))
                out["dx"][w, rows] = torch.einsum("mv,vd->md", logits, weight)
                out["dweight"][w] += torch.einsum("mv,md->vd", logits, x)
    return out


def _exact_clip(case, s):
    norms, clipped = [], torch.empty(s["grads"].shape, dtype=torch.float64, device="cuda")
    for w in range(case["W"]):
        g = s["grads"][w].double()
        norms.append(torch.linalg.vector_norm(g))
        clipped[w] = g * min(1.0, s["max_norm"] / float(norms[-1]))
    return {"norms": torch.stack(norms), "clipped": clipped}


def _each(case, t):
    """Per-sequence float64 copies of a worker's parameters."""
    return torch.stack([t[i * case["W"] // case["B"]].double() for i in range(case["B"])])


def _exact_conv(case, s):
    B, T, D, K = (case[k] for k in "BTDK")
    x = s["x"].double().reshape(B, T, D)
    n = torch.full((B,), T, device="cuda") if s["lengths"] is None else s["lengths"].long()
    on = (torch.arange(T, device="cuda")[None, :] < n[:, None]).unsqueeze(-1).double()
    w, bias = _each(case, s["weight"]), _each(case, s["bias"])
    held = torch.zeros((B, T + K - 1, D), dtype=torch.float64, device="cuda")
    held[:, :K - 1], held[:, K - 1:] = s["state"].double(), x
    v = torch.zeros_like(x) + bias.unsqueeze(1)
    for k in range(K):
        v += held[:, k:k + T] * w[:, None, :, k]
    gate = 1.0 / (1.0 + torch.exp(-v))
    last = torch.stack([held[i, int(n[i]):int(n[i]) + K - 1] for i in range(B)])
    if case["mode"] == "step":
        return {"y": (v * gate)[:, 0], "state": last}
    out = {"y": v * gate * on, "last": last}
    if case["mode"] == "train":
        dv = s["dy"].double() * (gate + v * gate * (1.0 - gate)) * on
        dheld, dw = torch.zeros_like(held), torch.zeros_like(w)
        for k in range(K):
            dheld[:, k:k + T] += dv * w[:, None, :, k]
            dw[..., k] = (dv * held[:, k:k + T]).sum(1)
        out["dx"] = dheld[:, K - 1:]
        out["dweight"] = dw.reshape(case["W"], -1, D, K).sum(1)
        out["dbias"] = dv.sum(1).reshape(case["W"], -1, D).sum(1)
    return out


def _exact_scan(case, s):
    """The definition, a step at a time; the backward pass goes through the states again from one in sixteen."""
    B, T, D, N, W = (case[k] for k in "BTDNW")
    if case["mode"] == "train" and B * D * N * (T / 16 + 40) * 8 > 60e9:
        return None
    u, delta, z = (s[k].double().reshape(B, T, D) for k in ("u", "delta", "z"))
    b, c = (s[k].double().reshape(B, T, N) for k in ("b", "c"))
    n = torch.full((B,), T, device="cuda") if s["lengths"] is None else s["lengths"].long()
    on = (torch.arange(T, device="cuda")[None, :] < n[:, None]).unsqueeze(-1)
    rate, skip, bias = -torch.exp(_each(case, s["a_log"])), _each(case, s["skip"]), _each(case, s["bias"])
    raw = delta + bias.unsqueeze(1)
    size = torch.where(on, torch.logaddexp(raw, torch.zeros_like(raw)), torch.zeros_like(raw))
    move = size * u

    def forward(h, t):
        return torch.exp(size[:, t].unsqueeze(-1) * rate) * h + move[:, t].unsqueeze(-1) * b[:, t].unsqueeze(1)

    h, sums, kept = s["h0"].double(), torch.empty_like(u), []
    for t in range(T):
        if t % 16 == 0 and case["mode"] == "train":
            kept.append(h)
        h = forward(h, t)
        sums[:, t] = torch.einsum("bdn,bn->bd", h, c[:, t])
    sums += skip.unsqueeze(1) * u
    gate = 1.0 / (1.0 + torch.exp(-z))
    y = torch.where(on, sums * z * gate, torch.zeros_like(u))
    if case["mode"] == "step":
        return {"y": y[:, 0], "state": h}
    out = {"y": y, "last": h}
    if case["mode"] != "train":
        return out
    dy = torch.where(on, s["dy"].double(), torch.zeros_like(u))
    out["dz"] = dy * sums * (gate + z * gate * (1.0 - gate))
    gy = dy * z * gate
    flow, drate = s["dlast"].double(), torch.zeros_like(rate)
    du, dsize, db, dc = torch.empty_like(u), torch.empty_like(u), torch.empty_like(b), torch.empty_like(c)
    for first in range((T - 1) // 16 * 16, -1, -16):
        states = [kept[first // 16]]
        for t in range(first, min(T, first + 16)):
            states.append(forward(states[-1], t))
        for t in range(min(T, first + 16) - 1, first - 1, -1):
            before, now = states[t - first], states[t - first + 1]
            flow = flow + gy[:, t].unsqueeze(-1) * c[:, t].unsqueeze(1)
            dc[:, t] = torch.einsum("bdn,bd->bn", now, gy[:, t])
            db[:, t] = torch.einsum("bdn,bd->bn", flow, move[:, t])
            through = torch.einsum("bdn,bn->bd", flow, b[:, t])
            back = flow * torch.exp(size[:, t].unsqueeze(-1) * rate)
            reach = back * before
            du[:, t] = through * size[:, t]
            dsize[:, t] = (reach * rate).sum(-1) + through * u[:, t]
            drate += reach * size[:, t].unsqueeze(-1)
            flow = back
    dbase = torch.where(on, dsize / (1.0 + torch.exp(-raw)), torch.zeros_like(raw))
    workers = lambda t: t.reshape((W, -1) + t.shape[1:]).sum(1)  # noqa: E731
    out.update(du=du + skip.unsqueeze(1) * gy, ddelta=dbase, da_log=workers(drate * rate), db=db, dc=dc,
               dskip=workers((gy * u).sum(1)), dbias=workers(dbase.sum(1)), dh0=flow)
    return out
