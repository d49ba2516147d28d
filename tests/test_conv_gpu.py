"""The causal convolution on the GPU against 64-bit references: sequences of no
steps, one and many, widths that are not whole pieces, lengths, initial states
and their gradients, unaligned weights, single steps that continue a pass."""
import pytest
import torch

import operators_reference as ref
from paper_2607_21224_gb300 import cpdp, layers
from test_layers_gpu import near, normal, rng, slices, strided

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16


def inputs(shape, dtype, ragged, seed=0):
    W, B, T, D, K = shape
    gen = rng(seed + 13 * T + D)
    x, dy = normal(gen, B, T, D, std=2.0, dtype=dtype), normal(gen, B, T, D, dtype=dtype)
    weight, bias = normal(gen, W, D, K), normal(gen, W, D, std=0.3)
    state, dlast = normal(gen, B, K - 1, D, dtype=dtype), normal(gen, B, K - 1, D, dtype=dtype)
    lengths = None
    if ragged:
        lengths = torch.randint(-1, T + 3, (B,), generator=gen, dtype=torch.int32)
        for i, n in enumerate((T, 0, 1, min(2, T))[:B]):
            lengths[i] = n
    return x, dy, weight, bias, state, dlast, lengths


SHAPES = [(1, 1, 1, 1, 4), (2, 4, 1, 64, 2), (1, 3, 2, 33, 4), (2, 4, 3, 8, 3), (1, 5, 17, 40, 4), (4, 8, 197, 96, 4), (2, 2, 300, 771, 3),
          (1, 1, 1025, 24, 4), (3, 6, 64, 129, 2), (1, 40, 33, 260, 4), (8, 8, 50, 16, 4)]


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("shape", SHAPES)
@pytest.mark.parametrize("ragged", [False, True])
@pytest.mark.parametrize("layout", ["plain", "strided"])
def test_conv(shape, dtype, ragged, layout):
    W, B, T, D, K = shape
    x, dy, weight, bias, state, dlast, lengths = inputs(shape, dtype, ragged)
    put = (lambda t: t.cuda()) if layout == "plain" else strided
    ws, bs = slices(weight, 0 if layout == "plain" else 3)[0], slices(bias, 0 if layout == "plain" else 1)[0]
    ns = None if lengths is None else lengths.cuda()
    for s in (None, state):
        at = None if s is None else s.cuda()
        f = ref.conv(x, weight, bias, s, lengths)
        xs = put(x)
        if ragged and layout == "strided":  # nothing beyond a length is read
            xs.masked_fill_(~f["on"].cuda(), float("nan"))
        y, last = layers.causal_conv(xs, ws, bs, at, ns)
        near(y, f["y"], f["ey"])
        assert torch.equal(last.double().cpu(), f["last"])
        dys = put(dy)
        if ragged and layout == "strided":
            dys.masked_fill_(~f["on"].cuda(), float("inf"))
        g = ref.conv_backward(dy, x, weight, bias, s, lengths, None if s is None else dlast)
        grad = dtype if layout == "plain" else F32
        dw, wrows = slices(torch.zeros(W, D, K, dtype=grad), 5)
        db, brows = slices(torch.zeros(W, D, dtype=grad), 2)
        dstate = torch.full((B, K - 1, D), float("nan"), dtype=dtype, device="cuda")
        dx, got_w, got_b = layers.causal_conv_backward(dys, xs, ws, bs, at, ns, None if s is None else dlast.cuda(), dweight=dw, dbias=db,
                                                       dstate=dstate)
        assert got_w.data_ptr() == dw.data_ptr() and got_b.data_ptr() == db.data_ptr()
        for got, name in ((dx, "dx"), (dw, "dweight"), (db, "dbias"), (dstate, "dstate")):
            near(got, g[name], g["e" + name])
        assert torch.isnan(wrows).sum() == wrows.numel() - dw.numel() and torch.isnan(brows).sum() == brows.numel() - db.numel()
        again = layers.causal_conv_backward(dys, xs, ws, bs, at, ns, None if s is None else dlast.cuda(), dtype=grad)
        assert all(torch.equal(a, b) for a, b in zip(again, (dx, dw, db)))


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("K", [2, 3, 4])
def test_steps_continue_a_pass(dtype, K):
    shape = (2, 6, 9, 72, K)
    x, _, weight, bias, state, _, _ = inputs(shape, dtype, False, 3)
    f = ref.conv(x, weight, bias, state, None)
    xs, ws, bs = strided(x), weight.cuda(), bias.cuda()
    y, s = layers.causal_conv(xs[:, :4], ws, bs, state.cuda())
    near(y, f["y"][:, :4], f["ey"][:, :4])
    for t in range(4, 9):
        near(layers.causal_conv_step(xs[:, t], ws, bs, s), f["y"][:, t], f["ey"][:, t])
    assert torch.equal(s.double().cpu(), f["last"])
    one = layers.causal_conv_step(xs[:, 0], ws[1], bs[1], state.cuda())
    assert torch.equal(one[3:], layers.causal_conv_step(xs[:, 0], ws, bs, state.cuda())[3:])


def test_gradients_against_differences():
    shape = (2, 4, 21, 10, 4)
    x, dy, weight, bias, state, dlast, lengths = inputs(shape, F32, True, 8)
    gen, h = rng(2), 1e-6
    us = [normal(gen, *t.shape).double() for t in (x, weight, bias, state)]

    def total(s):
        f = ref.conv(*(t.double() + s * u for t, u in zip((x, weight, bias, state), us)), lengths)
        return (f["y"] * dy).sum() + (f["last"] * dlast).sum()

    dstate = torch.empty_like(state, device="cuda")
    dx, dw, db = layers.causal_conv_backward(*(t.cuda() for t in (dy, x, weight, bias, state, lengths, dlast)), dstate=dstate)
    parts = [(g.double().cpu() * u) for g, u in zip((dx, dw, db, dstate), us)]
    want = (total(h) - total(-h)) / (2 * h)
    assert abs(sum(p.sum() for p in parts) - want) <= 1e-5 * sum(float(p.abs().sum()) for p in parts)


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_large_activations(dtype):
    """silu far from 0: v and 0; its slope 1 and 0."""
    x = torch.tensor([-3e4, -200.0, -90.0, -40.0, 40.0, 90.0, 200.0, 3e4]).to(dtype).view(1, 8, 1).expand(1, 8, 16).contiguous()
    weight, bias = torch.zeros(1, 16, 2), torch.zeros(1, 16)
    weight[..., 1] = 1.0
    f = ref.conv(x, weight, bias, None, None)
    near(layers.causal_conv(x.cuda(), weight.cuda(), bias.cuda())[0], f["y"], f["ey"] + 1e-30)
    g = ref.conv_backward(torch.ones_like(x), x, weight, bias, None, None, None)
    dx, dw, db = layers.causal_conv_backward(torch.ones_like(x).cuda(), x.cuda(), weight.cuda(), bias.cuda())
    near(dx, g["dx"], g["edx"] + 1e-30)
    near(dw, g["dweight"], g["edweight"] + 1e-30)


def test_no_sequences_no_steps_many_sequences():
    w, b = torch.ones(2, 16, 4, device="cuda"), torch.zeros(2, 16, device="cuda")
    x = torch.empty(0, 5, 16, device="cuda")
    y, last = layers.causal_conv(x, w, b)
    assert y.shape == (0, 5, 16) and last.shape == (0, 3, 16)
    dx, dw, db = layers.causal_conv_backward(x, x, w, b, dweight=torch.full((2, 16, 4), 7.0, device="cuda"))
    assert (dw == 0).all() and (db == 0).all()
    assert layers.causal_conv_step(x[:, 0], w, b, last).shape == (0, 16)
    x, state = torch.empty(4, 0, 16, device="cuda"), torch.randn(4, 3, 16, device="cuda")
    y, last = layers.causal_conv(x, w, b, state)
    assert y.shape == (4, 0, 16) and torch.equal(last, state)
    dstate = torch.empty_like(state)
    dx, dw, db = layers.causal_conv_backward(x, x, w, b, state, dlast=last, dstate=dstate)
    assert (dw == 0).all() and (db == 0).all() and torch.equal(dstate, state)
    shape = (1, 70000, 2, 3, 4)
    x, dy, weight, bias, state, _, _ = inputs(shape, F32, False)
    f, g = ref.conv(x, weight, bias, state, None), ref.conv_backward(dy, x, weight, bias, state, None, None)
    near(layers.causal_conv(x.cuda(), weight.cuda(), bias.cuda(), state.cuda())[0], f["y"], f["ey"])
    got = layers.causal_conv_backward(*(t.cuda() for t in (dy, x, weight, bias, state)))
    for a, name in zip(got, ("dx", "dweight", "dbias")):
        near(a, g[name], g["e" + name])


def test_streams_and_graphs():
    x, dy, weight, bias, state, dlast, lengths = (t.cuda() for t in inputs((2, 4, 60, 40, 4), BF16, True))

    def step():
        return *layers.causal_conv(x, weight, bias, state, lengths), *layers.causal_conv_backward(dy, x, weight, bias, state, lengths, dlast)

    want = step()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = *layers.causal_conv(x, weight, bias, state, lengths, stream=side), *layers.causal_conv_backward(
        dy, x, weight, bias, state, lengths, dlast, stream=side)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(want, got))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = step()
    x.copy_(x.flip(0))
    graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(held, step())) and not torch.equal(held[0], want[0])


def test_refusals():
    x, dy, weight, bias, state, dlast, lengths = (t.cuda() for t in inputs((2, 4, 10, 16, 4), BF16, True))
    for bad in (lambda: layers.causal_conv(x.half(), weight, bias), lambda: layers.causal_conv(x, weight.bfloat16(), bias),
                lambda: layers.causal_conv(x, weight, bias, state.float()), lambda: layers.causal_conv(x, weight, bias, state, lengths.long()),
                lambda: layers.causal_conv_backward(dy.float(), x, weight, bias), lambda: layers.causal_conv_step(x[:, 0].float(), weight, bias, state),
                lambda: layers.causal_conv_backward(dy, x, weight, bias, dweight=torch.zeros(2, 16, 4, device="cuda"),
                                                    dbias=torch.zeros(2, 16, device="cuda", dtype=BF16))):
        with pytest.raises(TypeError):
            bad()
    for bad in (lambda: layers.causal_conv(x[0], weight, bias), lambda: layers.causal_conv(x[:3], weight, bias),
                lambda: layers.causal_conv(x, weight[..., :15, :], bias), lambda: layers.causal_conv(x, weight, bias[:1]),
                lambda: layers.causal_conv(x[..., ::2], weight[:, ::2], bias[:, ::2]), lambda: layers.causal_conv(x, weight, bias, state[:, :2]),
                lambda: layers.causal_conv(x, weight.transpose(1, 2).contiguous().transpose(1, 2), bias),
                lambda: layers.causal_conv(x, weight, bias, None, lengths[:2]), lambda: layers.causal_conv(x, weight.clone().requires_grad_(), bias),
                lambda: layers.causal_conv_backward(dy[:, :5], x, weight, bias),
                lambda: layers.causal_conv_backward(dy, x, weight, bias, dbias=torch.zeros(1, 16, device="cuda").expand(2, 16)),
                lambda: layers.causal_conv_step(x[:, 0], weight, bias, state[:, :2]), lambda: layers.causal_conv_step(x[:3, 0], weight, bias, state)):
        with pytest.raises(ValueError):
            bad()
    for taps in (1, 5):
        with pytest.raises(cpdp.CPDPError):
            layers.causal_conv(x, torch.ones(2, 16, taps, device="cuda"), bias)
