"""The selective scan on the GPU against 64-bit references: every padded number of
states, widths that are not whole columns, lengths, initial states, sequences
shared out among segments, missing gates, single steps that continue a pass."""
import pytest
import torch

import operators_reference as ref
from paper_2607_21224_gb300 import cpdp, layers
from test_layers_gpu import near, normal, rng, slices, strided

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16
GRADS = ("du", "ddelta", "da_log", "db", "dc", "dskip", "dbias", "dz", "dh0")


def inputs(shape, dtype, ragged, seed=0):
    """u, delta, a_log, b, c, skip, bias; then z, h0, lengths, dy, dlast."""
    W, B, T, D, N = shape
    gen = rng(seed + 17 * T + D + N)
    u, delta, z, dy = (normal(gen, B, T, D, std=s, dtype=dtype) for s in (0.7, 1.5, 2.0, 1.0))
    b, c = normal(gen, B, T, N, dtype=dtype), normal(gen, B, T, N, dtype=dtype)
    a_log = normal(gen, W, D, N, std=0.3) + torch.arange(1, N + 1).log()
    skip, bias = 1 + normal(gen, W, D, std=0.3), normal(gen, W, D) - 2.5
    h0, dlast = normal(gen, B, D, N), normal(gen, B, D, N)
    lengths = None
    if ragged:
        lengths = torch.randint(-1, T + 3, (B,), generator=gen, dtype=torch.int32)
        for i, n in enumerate((T, 0, 1, min(16, T), min(17, T))[:B]):
            lengths[i] = n
    return (u, delta, a_log, b, c, skip, bias), (z, h0, lengths, dy, dlast)


def on_gpu(tensors, layout):
    """The seven inputs on the GPU; weights as slices of longer rows."""
    put = (lambda t: t.cuda()) if layout == "plain" else strided
    k = 0 if layout == "plain" else 3
    u, delta, a_log, b, c, skip, bias = tensors
    return put(u), put(delta), slices(a_log, k)[0], put(b), put(c), slices(skip, k)[0], slices(bias, k)[0]


SHAPES = [(1, 1, 1, 1, 1), (2, 4, 1, 64, 16), (1, 3, 15, 33, 16), (2, 2, 16, 32, 8), (1, 2, 17, 40, 7), (1, 5, 18, 130, 4), (2, 6, 70, 96, 16),
          (1, 1, 33, 24, 32), (3, 3, 50, 37, 13), (1, 2, 40, 20, 17), (4, 8, 20, 16, 2), (1, 1, 400, 33, 16), (1, 2, 515, 20, 8),
          (1, 1, 300, 18, 32), (2, 2, 290, 70, 5)]


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("shape", SHAPES)
@pytest.mark.parametrize("ragged", [False, True])
@pytest.mark.parametrize("layout", ["plain", "strided"])
def test_scan(shape, dtype, ragged, layout):
    W, B, T, D, N = shape
    tensors, (z, h0, lengths, dy, dlast) = inputs(shape, dtype, ragged)
    xs = on_gpu(tensors, layout)
    put = (lambda t: t.cuda()) if layout == "plain" else strided
    zs, dys, ns = put(z), put(dy), None if lengths is None else lengths.cuda()
    if ragged and layout == "strided":  # nothing beyond a length is read
        off = torch.arange(T)[None] >= lengths.clamp(0, T)[:, None]
        for t in (xs[0], xs[1], xs[3], xs[4], zs, dys):
            t.masked_fill_(off[..., None].cuda(), float("nan"))
    for gate, start in ((True, True), (False, False)):
        if not gate and shape[2] > 100:
            continue
        zr, zg = (z, zs) if gate else (None, None)
        h, hg = (h0, h0.cuda()) if start else (None, None)
        dl, dlg = (dlast, dlast.cuda()) if start else (None, None)
        f = ref.scan(*tensors, zr, h, lengths)
        y, last, carry = layers.selective_scan(*xs, zg, hg, ns)
        near(y, f["y"], f["ey"])
        near(last, f["last"], f["elast"])
        for k in range(0, T, 16):
            inside = f["n"] > k
            near(carry[:, k // 16][inside.cuda()], f["before"][:, k][inside], f["ebefore"][:, k][inside])
        y2, last2, none = layers.selective_scan(*xs, zg, hg, ns, carry=False)
        assert none is None and torch.equal(y2, y) and torch.equal(last2, last)
        g = ref.scan_backward(dy, *tensors, zr, h, dl, lengths)
        grad = dtype if layout == "plain" else F32
        (da, r0), (ds, r1), (db, r2) = (slices(torch.zeros(W, *s, dtype=grad), k) for s, k in (((D, N), 5), ((D,), 2), ((D,), 1)))
        out = layers.selective_scan_backward(dys, *xs, carry, zg, dlg, ns, da_log=da, dskip=ds, dbias=db)
        assert out[2].data_ptr() == da.data_ptr() and out[5].data_ptr() == ds.data_ptr() and out[6].data_ptr() == db.data_ptr()
        for got, name in zip(out, GRADS):
            if name == "dz" and not gate:
                assert got is None
                continue
            assert got.dtype == (F32 if name == "dh0" else grad if name in ("da_log", "dskip", "dbias") else dtype)
            try:
                near(got, g[name], g["e" + name])
            except AssertionError as e:
                raise AssertionError(f"{name}: {e}") from None
        for rows, part in ((r0, da), (r1, ds), (r2, db)):
            assert torch.isnan(rows).sum() == rows.numel() - part.numel()
        again = layers.selective_scan_backward(dys, *xs, carry, zg, dlg, ns, dtype=grad)
        assert all(p is None and q is None or torch.equal(p, q) for p, q in zip(again, out))


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("N", [1, 8, 16, 19, 32])
def test_steps_continue_a_pass(dtype, N):
    shape = (2, 6, 9, 72, N)
    tensors, (z, h0, _, _, _) = inputs(shape, dtype, False, 3)
    f = ref.scan(*tensors, z, h0, None)
    u, delta, a_log, b, c, skip, bias = on_gpu(tensors, "strided")
    zs = strided(z)
    y, state, _ = layers.selective_scan(u[:, :4], delta[:, :4], a_log, b[:, :4], c[:, :4], skip, bias, zs[:, :4], h0.cuda())
    near(y, f["y"][:, :4], f["ey"][:, :4])
    for t in range(4, 9):
        y = layers.selective_scan_step(u[:, t], delta[:, t], a_log, b[:, t], c[:, t], skip, bias, state, zs[:, t])
        near(y, f["y"][:, t], f["ey"][:, t])
    near(state, f["last"], f["elast"])
    plain = ref.scan(*tensors, None, h0, None)
    state = h0.cuda()
    one = layers.selective_scan_step(u[:, 0], delta[:, 0], a_log, b[:, 0], c[:, 0], skip, bias, state)
    near(one, plain["y"][:, 0], plain["ey"][:, 0])
    state = h0.cuda()[3:].contiguous()
    half = layers.selective_scan_step(u[3:, 0], delta[3:, 0], a_log[1], b[3:, 0], c[3:, 0], skip[1], bias[1], state)
    assert torch.equal(half, one[3:])


def test_gradients_against_differences():
    shape = (2, 4, 21, 10, 6)
    tensors, (z, h0, lengths, dy, dlast) = inputs(shape, F32, True, 8)
    gen, h = rng(2), 1e-6
    everything = (*tensors, z, h0)
    us = [normal(gen, *t.shape).double() for t in everything]

    def total(s):
        f = ref.scan(*(t.double() + s * u for t, u in zip(everything, us)), lengths)
        return (f["y"] * dy).sum() + (f["last"] * dlast).sum()

    xs = [t.cuda() for t in everything]
    carry = layers.selective_scan(*xs[:7], xs[7], xs[8], lengths.cuda())[2]
    out = layers.selective_scan_backward(dy.cuda(), *xs[:7], carry, xs[7], dlast.cuda(), lengths.cuda())
    parts = [g.double().cpu() * u for g, u in zip(out, us)]
    want = (total(h) - total(-h)) / (2 * h)
    assert abs(sum(p.sum() for p in parts) - want) <= 1e-5 * sum(float(p.abs().sum()) for p in parts)


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_steps_of_very_small_and_large_size(dtype):
    """dt from 1e-30 (a state that stays) to 100 (one that is forgotten), gates far from 0."""
    B, T, D, N = 1, 20, 9, 16
    tensors, (z, h0, _, dy, dlast) = inputs((1, B, T, D, N), dtype, False, 4)
    u, delta, a_log, b, c, skip, bias = tensors
    bias = torch.tensor([[-70.0, -30.0, -10.0, -3.0, 0.0, 3.0, 10.0, 30.0, 100.0]])
    z = z * 20
    tensors = (u, delta, a_log, b, c, skip, bias)
    f, g = ref.scan(*tensors, z, h0, None), ref.scan_backward(dy, *tensors, z, h0, dlast, None)
    xs = on_gpu(tensors, "plain")
    y, last, carry = layers.selective_scan(*xs, z.cuda(), h0.cuda())
    tiny = 2.0 ** -120  # powers below 2^-126 count as 0
    near(y, f["y"], f["ey"] + tiny)
    near(last, f["last"], f["elast"] + tiny)
    out = layers.selective_scan_backward(dy.cuda(), *xs, carry, z.cuda(), dlast.cuda())
    for got, name in zip(out, GRADS):
        near(got, g[name], g["e" + name] + tiny)


def test_no_sequences_no_steps_and_very_many_sequences():
    w = dict(a_log=torch.zeros(2, 16, 4, device="cuda"), skip=torch.ones(2, 16, device="cuda"), bias=torch.zeros(2, 16, device="cuda"))
    u, b = torch.empty(0, 5, 16, device="cuda"), torch.empty(0, 5, 4, device="cuda")
    y, last, carry = layers.selective_scan(u, u, b=b, c=b, z=u, **w)
    assert y.shape == (0, 5, 16) and last.shape == (0, 16, 4)
    out = layers.selective_scan_backward(u, u, u, b=b, c=b, carry=carry, z=u, **w)
    assert all((out[i] == 0).all() for i in (2, 5, 6))
    assert layers.selective_scan_step(u[:, 0], u[:, 0], b=b[:, 0], c=b[:, 0], state=last, **w).shape == (0, 16)
    u, b, h0 = torch.empty(4, 0, 16, device="cuda"), torch.empty(4, 0, 4, device="cuda"), torch.randn(4, 16, 4, device="cuda")
    y, last, carry = layers.selective_scan(u, u, b=b, c=b, h0=h0, **w)
    assert torch.equal(last, h0) and carry.shape == (4, 0, 16, 4)
    out = layers.selective_scan_backward(u, u, u, b=b, c=b, carry=carry, dlast=h0, **w)
    assert all((out[i] == 0).all() for i in (2, 5, 6)) and torch.equal(out[8], h0)
    shape = (1, 70000, 2, 3, 2)
    tensors, (z, h0, lengths, dy, dlast) = inputs(shape, F32, True)
    f, g = ref.scan(*tensors, z, h0, lengths), ref.scan_backward(dy, *tensors, z, h0, dlast, lengths)
    xs = on_gpu(tensors, "plain")
    y, last, carry = layers.selective_scan(*xs, z.cuda(), h0.cuda(), lengths.cuda())
    near(y, f["y"], f["ey"])
    out = layers.selective_scan_backward(dy.cuda(), *xs, carry, z.cuda(), dlast.cuda(), lengths.cuda())
    for got, name in zip(out, GRADS):
        near(got, g[name], g["e" + name])


def test_streams_and_graphs():
    tensors, (z, h0, lengths, dy, dlast) = inputs((1, 2, 400, 40, 16), BF16, True)
    xs, (z, h0, lengths, dy, dlast) = on_gpu(tensors, "plain"), (t.cuda() for t in (z, h0, lengths, dy, dlast))

    def step(**kw):
        y, last, carry = layers.selective_scan(*xs, z, h0, lengths, **kw)
        return y, last, *layers.selective_scan_backward(dy, *xs, carry, z, dlast, lengths, **kw)

    want = step()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = step(stream=side)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(want, got))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = step()
    xs[0].copy_(xs[0].flip(1))
    graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(held, step())) and not torch.equal(held[0], want[0])


def test_refusals():
    tensors, (z, h0, lengths, dy, dlast) = inputs((2, 4, 10, 16, 8), BF16, True)
    xs, (z, h0, lengths, dy, dlast) = list(on_gpu(tensors, "plain")), (t.cuda() for t in (z, h0, lengths, dy, dlast))
    carry = layers.selective_scan(*xs, z, h0, lengths)[2]

    def swapped(i, t, *rest, **kw):
        return layers.selective_scan(*xs[:i], t, *xs[i + 1:], *rest, **kw)

    for bad in (lambda: swapped(0, xs[0].half()), lambda: swapped(1, xs[1].float()), lambda: swapped(2, xs[2].bfloat16()),
                lambda: swapped(3, xs[3].float()), lambda: layers.selective_scan(*xs, z.float()), lambda: layers.selective_scan(*xs, z, h0.bfloat16()),
                lambda: layers.selective_scan(*xs, z, h0, lengths.long()),
                lambda: layers.selective_scan_backward(dy, *xs, carry, z, dskip=torch.zeros(2, 16, dtype=BF16, device="cuda"),
                                                       dbias=torch.zeros(2, 16, device="cuda"))):
        with pytest.raises(TypeError):
            bad()
    for bad in (lambda: swapped(0, xs[0][0]), lambda: swapped(1, xs[1][:, :5]), lambda: swapped(2, xs[2][:, :15]), lambda: swapped(2, xs[2][..., ::2]),
                lambda: swapped(3, xs[3][..., :4]), lambda: swapped(5, xs[5][:1]), lambda: swapped(6, xs[6][:, None]),
                lambda: layers.selective_scan(*xs, z[..., :8]), lambda: layers.selective_scan(*xs, z, h0[:, :8]),
                lambda: layers.selective_scan(*xs, z, h0, lengths[:2]), lambda: swapped(2, torch.zeros(3, 16, 8, device="cuda")),
                lambda: swapped(2, xs[2].clone().requires_grad_()), lambda: layers.selective_scan_backward(dy, *xs, carry[:, :0], z),
                lambda: layers.selective_scan_backward(dy, *xs, carry, z, da_log=torch.zeros(1, 16, 8, device="cuda").expand(2, 16, 8)),
                lambda: layers.selective_scan_step(*(t[:, 0] if t.dim() == 3 and t.dtype == BF16 else t for t in xs), h0[:, :8]),
                lambda: layers.selective_scan_step(*xs, h0)):
        with pytest.raises(ValueError):
            bad()
    with pytest.raises(cpdp.CPDPError):
        layers.selective_scan(*xs[:2], torch.zeros(2, 16, 33, device="cuda"), *(torch.zeros(4, 10, 33, dtype=BF16, device="cuda"),) * 2, *xs[5:])
