"""The loss, the clipping, the convolution and the selective scan of
include/cpdp_layers.h in 64 bits, written from their formulas (torch float64 on
the CPU), with bounds on what float32 arithmetic may add. Bounds are per element,
as in layers_reference.py: a count of float32 roundings times the magnitudes that
the formula adds up."""
import torch

from layers_reference import HALF_SPACING, U32, rounding  # noqa: F401

BF16 = torch.bfloat16


def product_bound(magnitudes, terms, dtype):
    """What a sum of `terms` products may be off, given the sum of their magnitudes: additions that may round towards
    zero (2 U32 each, one after another at worst). float32 operands are three bfloat16 parts: six times as many terms,
    and what is left out of each product is at most 2 x 2^-8 x 2^-16 + 2^-32 + 2 x 2^-27 of it, below 4 U32."""
    if dtype is torch.float32:
        return (2 * (6 * terms + 16) + 4) * U32 * magnitudes
    return 2 * (terms + 16) * U32 * magnitudes


def loss(x, weight, targets):
    """A dict of loss, lse and their bounds, with the logits and theirs, for (W, M, D) and (W, V, D)."""
    a, w = x.double(), weight.double()
    logits = a @ w.transpose(1, 2)
    elogits = product_bound(a.abs() @ w.abs().transpose(1, 2), a.shape[-1], x.dtype)
    lse = torch.logsumexp(logits, -1)
    top = logits.amax(-1)
    # exponents (l - top) log2(e): two roundings of what is at most |l| + |top|, powers to 4 U32, the sums of V terms
    # in an order of at most 128 + 64 + V / 256 additions, their logarithm, the last addition
    count = logits.shape[-1] / 256 + 256
    else_ = elogits.amax(-1) + U32 * (count + 4 * (logits.abs().amax(-1) + top.abs()) + 4 * lse.abs() + 16)
    real = targets >= 0
    at = targets.clamp(min=0)[..., None]
    value = torch.where(real, lse - logits.gather(-1, at)[..., 0], 0.0)
    evalue = torch.where(real, else_ + elogits.gather(-1, at)[..., 0] + U32 * value.abs(), 0.0)
    return {"loss": value, "eloss": evalue, "lse": lse, "else": else_, "logits": logits, "elogits": elogits}


def loss_backward(dloss, x, weight, targets):
    """dx, dweight and their bounds."""
    f = loss(x, weight, targets)
    a, w, real = x.double(), weight.double(), targets >= 0
    a = torch.where(real[..., None], a, 0.0)  # ignored tokens reach nothing
    hot = torch.zeros_like(f["logits"]).scatter_(-1, targets.clamp(min=0)[..., None], 1.0)
    p = torch.exp(f["logits"] - f["lse"][..., None])
    r = torch.where(real, dloss.double(), 0.0)[..., None]
    d = r * (p - hot)
    # p's exponent is off by what logit and lse are, and by the roundings of their difference and its product
    ep = p * (f["elogits"] + f["else"][..., None] + U32 * (8 * (f["logits"].abs() + f["lse"].abs()[..., None]) + 16))
    ed = r.abs() * (ep + 4 * U32 * (p + hot))
    if x.dtype is BF16:  # d is rounded to bfloat16
        ed = ed + d.abs() * HALF_SPACING[BF16] * 1.01 + r.abs() * 1e-30
    else:
        ed = ed + 4 * U32 * d.abs()
    M, V = d.shape[1], d.shape[2]
    size, top = d.abs() + ed, 4 * U32
    dx, dweight = d @ w, d.transpose(1, 2) @ a
    edx = ed @ w.abs() + product_bound(size @ w.abs(), V, x.dtype) + top * dx.abs()
    edw = ed.transpose(1, 2) @ a.abs() + product_bound(size.transpose(1, 2) @ a.abs(), M, x.dtype) + top * dweight.abs()
    return dx, dweight, edx, edw


def clip(grads, max_norm):
    """norms, the clipped rows and their bounds, for (W, N)."""
    g = grads.double()
    norms = g.square().sum(-1).sqrt()
    scale = torch.clamp(max_norm / norms, max=1.0)
    # squares and sums of positive terms in an order of at most 512 + 40 additions, then the parts (at most 1,216); half
    # of it through the root. The ratio, the product.
    enorms = 1024 * U32 * norms
    out = g * scale[:, None]
    return norms, out, enorms, (1024 + 4) * U32 * out.abs()


def per_sequence(t, B):
    """A worker's weights (W, ...) for each of its sequences, in 64 bits."""
    return t.double().repeat_interleave(B // t.shape[0], 0)


def silu_slope(v):
    a = torch.sigmoid(v)
    return a * (1 + v * (1 - a))


# A sigmoid to a few roundings; its exponent's rounding grows with |v|, in bfloat16 without a correction: 2^-24 log2(e) |v|.
def gate_error(v):
    return (12 + 3 * v.abs()) * U32


def conv(x, weight, bias, state, lengths):
    """A dict of y, last and what the backward pass needs, with bounds. x (B, T, D), weight (W, D, K)."""
    B, T, D = x.shape
    K = weight.shape[2]
    w, b = per_sequence(weight, B), per_sequence(bias, B)[:, None]
    n = torch.full((B,), T) if lengths is None else lengths.long().clamp(0, T)
    on = (torch.arange(T)[None] < n[:, None])[..., None]
    before = torch.zeros(B, K - 1, D, dtype=torch.float64) if state is None else state.double()
    ext = torch.cat([before, torch.where(on, x.double(), 0.0)], 1)
    v, size = b.expand(B, T, D).clone(), b.abs().expand(B, T, D).clone()
    for k in range(K):
        v += w[:, None, :, k] * ext[:, k:k + T]
        size += (w[:, None, :, k] * ext[:, k:k + T]).abs()
    ev = (K + 2) * U32 * size
    y = torch.where(on, v * torch.sigmoid(v), 0.0)
    ey = torch.where(on, 1.1 * ev + (y.abs() + ev) * gate_error(v), 0.0)  # |silu'| <= 1.1
    last = torch.stack([ext[i, n[i]:n[i] + K - 1] for i in range(B)]) if B else before
    return {"y": y, "ey": ey, "last": last, "ext": ext, "v": v, "ev": ev, "on": on, "n": n, "w": w}


def conv_backward(dy, x, weight, bias, state, lengths, dlast):
    """dx, dweight, dbias, dstate in a dict with bounds (names with an e in front)."""
    f = conv(x, weight, bias, state, lengths)
    B, T, D = x.shape
    W, K = weight.shape[0], weight.shape[2]
    v, on, ext, w, n = f["v"], f["on"], f["ext"], f["w"], f["n"]
    dy = torch.where(on, dy.double(), 0.0)
    dv = dy * silu_slope(v)
    # |silu''| <= 0.5; the slope's own products: at most 1.1 and |v| (1 - a) a <= 0.3 each
    edv = dy.abs() * (0.5 * f["ev"] + 2 * gate_error(v))
    dext, edext = torch.zeros_like(ext), torch.zeros_like(ext)
    size = torch.zeros_like(ext)
    dw, edw = torch.zeros_like(w), torch.zeros_like(w)
    for k in range(K):
        dext[:, k:k + T] += w[:, None, :, k] * dv
        edext[:, k:k + T] += w[:, None, :, k].abs() * edv
        size[:, k:k + T] += (w[:, None, :, k] * dv).abs()
        dw[..., k] = (dv * ext[:, k:k + T]).sum(1)
        # sums over a stretch, a thread's stretches, teams, parts: at most B T additions one after another
        edw[..., k] = ((edv + (B * T + 8) * U32 * dv.abs()) * ext[:, k:k + T].abs()).sum(1)
    if dlast is not None:
        for i in range(B):
            dext[i, n[i]:n[i] + K - 1] += dlast[i].double()
            size[i, n[i]:n[i] + K - 1] += dlast[i].double().abs()
    edext += (K + 2) * U32 * size
    workers = lambda t: t.unflatten(0, (W, B // W)).sum(1)  # noqa: E731
    edb = edv + (B * T + 8) * U32 * dv.abs()
    return {"dx": dext[:, K - 1:], "edx": edext[:, K - 1:], "dstate": dext[:, :K - 1], "edstate": edext[:, :K - 1],
            "dweight": workers(dw), "edweight": workers(edw), "dbias": workers(dv.sum(1)), "edbias": workers(edb.sum(1))}
