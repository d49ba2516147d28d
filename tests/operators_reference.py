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


def scan(u, delta, a_log, b, c, skip, bias, z, h0, lengths):
    """A dict of y, last, the states before each step, and what the backward pass needs, with bounds (an e in front; an s
    in front of a magnitude that the formula adds up). u (B, T, D), b (B, T, N), a_log (W, D, N)."""
    B, T, D = u.shape
    N = a_log.shape[2]
    n = torch.full((B,), T) if lengths is None else lengths.long().clamp(0, T)
    on = (torch.arange(T)[None] < n[:, None])[..., None]
    inside = lambda t: torch.where(on, t.double(), 0.0)  # noqa: E731
    u, delta, b, c = inside(u), inside(delta), inside(b), inside(c)
    rate = torch.exp(per_sequence(a_log, B))
    skips, biases = per_sequence(skip, B)[:, None], per_sequence(bias, B)[:, None]
    raw = delta + biases
    # the addition's rounding reaches dt through a slope of sigmoid(raw); then the power, a division, seven terms
    slip = (delta.abs() + biases.abs()) * U32
    dt = torch.where(on, torch.logaddexp(raw, torch.zeros_like(raw)), 0.0)
    edt = torch.where(on, dt * (24 + 4 * raw.abs()) * U32 + torch.sigmoid(raw) * slip, 0.0)
    x, ex = dt * u, u.abs() * edt + 2 * U32 * (dt * u).abs()
    f = {"u": u, "b": b, "c": c, "rate": rate, "skip": skips, "raw": raw, "slip": slip, "dt": dt, "edt": edt, "x": x, "ex": ex, "on": on, "n": n,
         "z": None if z is None else inside(z), "delta": delta}
    h = torch.zeros(B, D, N, dtype=torch.float64) if h0 is None else h0.double()
    sh, eh = h.abs(), torch.zeros_like(h)
    for k in ("before", "sbefore", "ebefore", "after", "safter", "eafter", "a", "ea"):
        f[k] = torch.zeros(B, T, D, N, dtype=torch.float64)
    sums, esums = torch.zeros_like(u), torch.zeros_like(u)
    for t in range(T):
        p = dt[:, t, :, None] * rate
        a = torch.exp(-p)
        # exponent: the rate (a power, a product), the product with dt; segments compose decays of sums of dt
        ea = a * ((16 + 16 * p) * U32 + edt[:, t, :, None] * rate)
        f["before"][:, t], f["sbefore"][:, t], f["ebefore"][:, t], f["a"][:, t], f["ea"][:, t] = h, sh, eh, a, ea
        add = x[:, t, :, None] * b[:, t, None]
        eh = a * eh + ea * sh + ex[:, t, :, None] * b[:, t, None].abs()
        h, sh = a * h + add, a * sh + add.abs()
        eh = eh + 3 * U32 * sh
        off = ~on[:, t, :, None]
        eh = torch.where(off, f["ebefore"][:, t], eh)
        f["after"][:, t], f["safter"][:, t], f["eafter"][:, t] = h, sh, eh
        sums[:, t] = (h * c[:, t, None]).sum(-1)
        esums[:, t] = (c[:, t, None].abs() * (eh + (N + 4) * U32 * sh)).sum(-1)
    v = sums + skips * u
    ev = esums + 2 * U32 * ((f["safter"] * c[:, :, None].abs()).sum(-1) + (skips * u).abs())
    f.update(v=v, ev=ev, last=h, elast=eh)
    if z is None:
        f.update(y=torch.where(on, v, 0.0), ey=torch.where(on, ev, 0.0))
    else:
        gate = f["z"] * torch.sigmoid(f["z"])
        f.update(y=torch.where(on, v * gate, 0.0), ey=torch.where(on, gate.abs() * (ev + (v.abs() + ev) * gate_error(f["z"])), 0.0))
    return f


def scan_backward(dy, u, delta, a_log, b, c, skip, bias, z, h0, dlast, lengths):
    """A dict of the gradients with bounds."""
    f = scan(u, delta, a_log, b, c, skip, bias, z, h0, lengths)
    B, T, D = u.shape
    W, N = a_log.shape[0], a_log.shape[2]
    on, u, b, c, dt, edt, x, ex, rate, v = (f[k] for k in ("on", "u", "b", "c", "dt", "edt", "x", "ex", "rate", "v"))
    dy = torch.where(on, dy.double(), 0.0)
    r = {}
    if z is None:
        gy, egy = dy, torch.zeros_like(dy)
    else:
        gate = f["z"] * torch.sigmoid(f["z"])
        gy = dy * gate
        egy = gy.abs() * (gate_error(f["z"]) + 3 * U32)
        slope = silu_slope(f["z"])
        r["dz"] = dy * v * slope
        r["edz"] = dy.abs() * (f["ev"] * slope.abs() + (v.abs() + f["ev"]) * 2 * gate_error(f["z"]))
    g = torch.zeros(B, D, N, dtype=torch.float64) if dlast is None else dlast.double()
    sg, eg = g.abs(), torch.zeros_like(g)
    for k in ("through", "ethrough", "sthrough", "reach", "ereach", "sreach"):
        r[k] = torch.zeros_like(u)
    for k in ("db", "edb", "dc", "edc"):
        r[k] = torch.zeros_like(b)
    da, eda = torch.zeros_like(rate), torch.zeros_like(rate)
    depth, long = (D / 32 + 24) * U32, (B // W * T + 40) * U32
    for t in range(T - 1, -1, -1):
        off = ~on[:, t, :, None]
        a, ea, cs, bs = f["a"][:, t], f["ea"][:, t], c[:, t, None], b[:, t, None]
        gyt, egyt, xt, ext = gy[:, t, :, None], egy[:, t, :, None], x[:, t, :, None], ex[:, t, :, None]
        h, sh, eh = f["after"][:, t], f["safter"][:, t], f["eafter"][:, t]
        old, sold, eold = f["before"][:, t], f["sbefore"][:, t], f["ebefore"][:, t]
        flow, sflow = g + gyt * cs, sg + (gyt * cs).abs()
        eflow = eg + egyt * cs.abs() + 2 * U32 * sflow
        r["dc"][:, t] = (gyt * h).sum(1)
        r["edc"][:, t] = (egyt * sh + gyt.abs() * eh + depth * gyt.abs() * sh).sum(1)
        r["db"][:, t] = (flow * xt).sum(1)
        r["edb"][:, t] = (eflow * xt.abs() + (sflow + eflow) * ext + depth * sflow * xt.abs()).sum(1)
        r["through"][:, t] = (flow * bs).sum(-1)
        r["sthrough"][:, t] = (sflow * bs.abs()).sum(-1)
        r["ethrough"][:, t] = (eflow * bs.abs()).sum(-1) + (N + 8) * U32 * r["sthrough"][:, t]
        k, sk = a * flow * old, a * sflow * sold
        ek = a * (eflow * sold + (sflow + eflow) * eold) + ea * (sflow + eflow) * (sold + eold) + 4 * U32 * sk
        r["reach"][:, t] = (k * rate).sum(-1)
        r["sreach"][:, t] = (sk * rate).sum(-1)
        r["ereach"][:, t] = (ek * rate).sum(-1) + (N + 16) * U32 * r["sreach"][:, t]
        da -= k * dt[:, t, :, None] * rate
        eda += rate * (ek * dt[:, t, :, None] + sk * edt[:, t, :, None] + long * sk * dt[:, t, :, None])
        new, enew = a * flow, a * eflow + ea * (sflow + eflow) + 2 * U32 * a * sflow
        g, sg, eg = torch.where(off, g, new), torch.where(off, sg, a * sflow), torch.where(off, eg, enew)
    sig = torch.sigmoid(f["raw"])
    dsize = r["through"] * u - r["reach"]
    ssize = r["sthrough"] * u.abs() + r["sreach"]
    esize = r["ethrough"] * u.abs() + r["ereach"] + 6 * U32 * ssize
    dbase = torch.where(on, dsize * sig, 0.0)
    edbase = torch.where(on, sig * (esize + ssize * (gate_error(f["raw"]) + f["slip"])), 0.0)
    workers = lambda t: t.unflatten(0, (W, B // W)).sum(1)  # noqa: E731
    skips = f["skip"]
    r["du"] = r["through"] * dt + skips * gy
    r["edu"] = r["ethrough"] * dt + r["sthrough"] * edt + skips.abs() * egy + 4 * U32 * (r["sthrough"] * dt + (skips * gy).abs())
    r.update(ddelta=dbase, eddelta=edbase, da_log=workers(da), eda_log=workers(eda), dskip=workers((gy * u).sum(1)),
             edskip=workers((egy * u.abs() + long * (gy * u).abs()).sum(1)), dbias=workers(dbase.sum(1)),
             edbias=workers((edbase + long * (dbase.abs() + edbase)).sum(1)), dh0=g, edh0=eg)
    return r
