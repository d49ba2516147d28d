"""The layers of include/cpdp_layers.h in 64 bits, written from their formulas
(torch float64 on the CPU), with bounds on what float32 arithmetic may add.

A bound is per element: `u` times the magnitudes that the formula adds up, u the
float32 unit roundoff 2^-24 times a count of roundings, plus half a spacing of
the output's type."""
import torch

U32 = 2.0 ** -24
HALF_SPACING = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8}
BLOCK = 32


def rounding(x, dtype):
    """What storing x in dtype may add (subnormal spacings included)."""
    return x.abs() * HALF_SPACING[dtype] + 2.0 ** -133


def units(x):
    """The power of two that each value of x (float64, last axis in blocks of 32) is held in."""
    n = x.shape[-1]
    b = torch.nn.functional.pad(x.abs(), (0, -n % BLOCK)).unflatten(-1, (-1, BLOCK))
    top = b.amax(-1)
    e = torch.full(top.shape, -126, dtype=torch.int64)
    for k in range(-126, 121):  # the least e with top <= 127 * 2^e
        e = torch.where(top > 127.0 * 2.0 ** k, k + 1, e)
    return e


def held(x):
    """(values, exponents) of x in 8 bits."""
    n = x.shape[-1]
    e = units(x)
    unit = torch.ldexp(torch.ones_like(e, dtype=torch.float64), e).repeat_interleave(BLOCK, -1)[..., :n]
    return torch.clamp(torch.round(x / unit), -127, 127) * unit, e


def norm(x, weight, residual, eps):
    """(y, s, what float32 may add to y) for (W, M, D) tensors of the kernels' types."""
    s = x if residual is None else (x.float() + residual.float()).to(x.dtype)
    r = s.double()
    y = weight.double()[:, None] * r / torch.sqrt(r.square().mean(-1, keepdim=True) + eps)
    # the mean of positive squares: at most 32 + 10 additions deep; then a reciprocal root, two products
    return y, s, 64 * U32 * y.abs()


def norm_backward(dy, s, weight, ds, eps):
    """(dx, dweight) and their bounds."""
    g, r, w = dy.double(), s.double(), weight.double()[:, None]
    k = 1.0 / torch.sqrt(r.square().mean(-1, keepdim=True) + eps)
    through = torch.zeros_like(r) if ds is None else ds.double()
    dx = through + k * g * w - r * k ** 3 * (g * w * r).mean(-1, keepdim=True)
    size = through.abs() + k * (g * w).abs() + r.abs() * k ** 3 * (g * w * r).abs().mean(-1, keepdim=True)
    dweight = (g * r * k).sum(1)
    depth = 64 + g.shape[1]  # a sum of M terms in any order
    return dx, dweight, 128 * U32 * size, depth * U32 * (g * r * k).abs().sum(1)


def weight_gradient(dy, values):
    """dW and its bound: products of bfloat16 are exact in float32; M additions that may round towards zero."""
    g, v = dy.to(torch.bfloat16).double(), values.double()
    dW = torch.einsum("wmo,wmi->woi", g, v)
    return dW, 2 * (g.shape[1] + 16) * U32 * torch.einsum("wmo,wmi->woi", g.abs(), v.abs())


STEP = 16 * U32  # roundings per step of the recurrence: the gate's sigmoid to a few ulps, a product, an addition


def recurrence(gate, value, h0, lengths):
    """A dict of h, last, the states before each step, and bounds (eh of the states, elast)."""
    x, v = gate.double(), value.double()
    B, T, D = x.shape
    a, rest = torch.sigmoid(x), torch.sigmoid(-x)
    n = torch.full((B,), T) if lengths is None else lengths.long().clamp(0, T)
    h = torch.zeros(B, D, dtype=torch.float64) if h0 is None else h0.double()
    size, err = h.abs(), torch.zeros_like(h)
    out = {"h": torch.zeros_like(v), "eh": torch.zeros_like(v), "before": torch.zeros_like(v), "ebefore": torch.zeros_like(v),
           "a": a, "rest": rest, "n": n}
    for t in range(T):
        on = (t < n)[:, None]
        out["before"][:, t], out["ebefore"][:, t] = h, err
        grown = a[:, t] * size + rest[:, t] * torch.where(on, v[:, t].abs(), 0.0)
        err = torch.where(on, a[:, t] * err + STEP * grown, err)
        h = torch.where(on, a[:, t] * h + rest[:, t] * torch.where(on, v[:, t], 0.0), h)
        size = torch.where(on, grown, size)
        out["h"][:, t] = torch.where(on, h, 0.0)
        out["eh"][:, t] = torch.where(on, err, 0.0)
    return {**out, "last": h, "elast": err}


def recurrence_backward(dh, gate, value, h0, dh_last, lengths):
    """dgate, dvalue, dh0 with their bounds."""
    f = recurrence(gate, value, h0, lengths)
    a, rest, n, v, o = f["a"], f["rest"], f["n"], value.double(), dh.double()
    B, T, D = v.shape
    flow = torch.zeros(B, D, dtype=torch.float64) if dh_last is None else dh_last.double()
    size, err = flow.abs(), torch.zeros_like(flow)
    r = {k: torch.zeros_like(v) for k in ("dgate", "dvalue", "edgate", "edvalue")}
    for t in range(T - 1, -1, -1):
        on = (t < n)[:, None]
        g, gs = flow + o[:, t], size + o[:, t].abs()
        eg = err + STEP * gs
        diff, spread = f["before"][:, t] - v[:, t], f["before"][:, t].abs() + v[:, t].abs()
        slope = a[:, t] * rest[:, t]
        for k, x in (("dvalue", rest[:, t] * g), ("edvalue", rest[:, t] * (eg + STEP * g.abs())), ("dgate", slope * g * diff),
                     ("edgate", slope * (eg * diff.abs() + g.abs() * (f["ebefore"][:, t] + 4 * STEP * spread) + eg * f["ebefore"][:, t]))):
            r[k][:, t] = torch.where(on, x, 0.0)
        flow, size = torch.where(on, a[:, t] * g, flow), torch.where(on, a[:, t] * gs, size)
        err = torch.where(on, a[:, t] * eg + STEP * size, err)
    return {**r, "dh0": flow, "edh0": err}
