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
