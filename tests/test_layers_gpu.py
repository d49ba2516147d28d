"""The worker-batched layers on the GPU against 64-bit references
(layers_reference.py), at the sizes, strides, masks and types where they can go
wrong: one row and none, odd widths and unaligned slices, rows of zeros,
infinities and NaN, sequences of length zero and one, streams other than the
current one. Tolerances are the references' own bounds."""
import itertools

import pytest
import torch

import layers_reference as ref
from paper_2607_21224_gb300 import layers
from paper_2607_21224_gb300.cpdp import CPDPError

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16
EPS = 1e-6


def rng(seed):
    return torch.Generator().manual_seed(seed)


def normal(gen, *shape, std=1.0, dtype=F32):
    return (torch.randn(shape, generator=gen) * std).to(dtype)


def slices(t, shift):
    """A CUDA copy of t (W, ...) whose worker parts lie `shift` elements into longer rows, as in the [W][N] buffers."""
    W, n = t.shape[0], t[0].numel()
    rows = torch.full((W, n + 2 * shift + 5), float("nan"), dtype=t.dtype, device="cuda")
    part = rows[:, shift:shift + n].view(t.shape)
    part.copy_(t)
    return part, rows


def strided(t):
    """A CUDA copy of t (A, B, D) with longer rows and parts in between."""
    A, B, D = t.shape
    big = torch.full((A, B + 2, 2 * D + 3), float("nan"), dtype=t.dtype, device="cuda")
    view = big[:, 1:B + 1, D:2 * D]
    view.copy_(t)
    return view


def near(got, want, bound, dtype=None):
    dtype = dtype or got.dtype
    got = got.double().cpu()
    err = (got - want).abs()
    room = bound + ref.rounding(want, dtype) + bound * ref.HALF_SPACING[dtype]
    bad = ~(err <= room)
    assert not bad.any(), f"{int(bad.sum())} of {bad.numel()} off, worst {float((err / room).nan_to_num(9e9).max()):.3g} times its bound"


NORM_SHAPES = [(1, 1, 384), (3, 5, 64), (1, 3, 1), (2, 7, 31), (2, 4, 33), (1, 9, 771), (4, 2, 1024), (2, 3, 1032), (1, 2, 2731),
               (2, 300, 40), (1, 2, 4096), (3, 1, 4104), (1, 3, 8192), (1, 2, 16384), (1, 1, 16383)]


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("shape", NORM_SHAPES)
@pytest.mark.parametrize("layout", ["plain", "strided"])
def test_norm_forward(shape, dtype, layout):
    W, M, D = shape
    gen = rng(D)
    x, r = normal(gen, *shape, dtype=dtype), normal(gen, *shape, std=3.0, dtype=dtype)
    w = 1 + 0.3 * normal(gen, W, D)
    weight, _ = slices(w, 0 if layout == "plain" else 3)
    put = (lambda t: t.cuda()) if layout == "plain" else strided
    for residual in (None, r):
        want, s, bound = ref.norm(x, w, residual, EPS)
        y, got_s, saved = layers.add_rmsnorm(put(x), weight, None if residual is None else put(residual), eps=EPS)
        assert saved is None and y.dtype == dtype and torch.equal(got_s.cpu(), s)
        near(y, want, bound)

        y8, got_s, saved = layers.add_rmsnorm(put(x), weight, None if residual is None else put(residual), eps=EPS, checkpoint=True)
        assert y8.dtype == BF16 and torch.equal(got_s.cpu(), s)
        e = saved.exponents.cpu().long() - 127
        lo, hi = ref.units(want - bound * want.sign()), ref.units(want + bound * want.sign())
        assert ((e >= lo) & (e <= hi)).all()
        unit = torch.ldexp(torch.ones(e.shape, dtype=torch.float64), e).repeat_interleave(32, -1)
        values = saved.codes.cpu().double() * unit
        assert (values[..., D:] == 0).all()
        assert torch.equal(values[..., :D], y8.double().cpu())
        assert ((values[..., :D] - want).abs() <= unit[..., :D] * 0.5 + bound).all()
        assert torch.equal(layers.restore(saved), y8)


@pytest.mark.parametrize("dtype,grad", [(F32, F32), (BF16, BF16), (BF16, F32)])
@pytest.mark.parametrize("shape", NORM_SHAPES + [(2, 4000, 96), (1, 700, 2056), (5, 63, 512)])
@pytest.mark.parametrize("layout", ["plain", "strided"])
def test_norm_backward(shape, dtype, grad, layout):
    W, M, D = shape
    gen = rng(D + 1)
    dy, s, ds = (normal(gen, *shape, std=k, dtype=dtype) for k in (1.0, 2.0, 0.5))
    w = 1 + 0.3 * normal(gen, W, D)
    weight, _ = slices(w, 0 if layout == "plain" else 1)
    put = (lambda t: t.cuda()) if layout == "plain" else strided
    for through in (None, ds):
        dx, dw, edx, edw = ref.norm_backward(dy, s, w, through, EPS)
        out, rows = slices(torch.zeros(W, D, dtype=grad), 0 if layout == "plain" else 5)
        got, got_w = layers.add_rmsnorm_backward(put(dy), put(s), weight, None if through is None else put(through), eps=EPS, dweight=out)
        assert got_w.data_ptr() == out.data_ptr()
        near(got, dx, edx)
        near(got_w, dw, edw)
        assert torch.isnan(rows).sum() == rows.numel() - W * D  # nothing beside the slices is written
        again, again_w = layers.add_rmsnorm_backward(put(dy), put(s), weight, None if through is None else put(through), eps=EPS, dtype=grad)
        assert torch.equal(again, got) and torch.equal(again_w, got_w)


def test_norm_rows_of_zeros_infinity_and_nan():
    x = torch.zeros(1, 5, 64)
    x[0, 1] = 1.0
    x[0, 2, 7], x[0, 3, 7] = float("inf"), float("nan")
    x[0, 4] = 1e-30
    w = torch.ones(1, 64)
    for dtype, saved in itertools.product((F32, BF16), (False, True)):
        y, s, held = layers.add_rmsnorm(x.to(dtype).cuda(), w.cuda(), eps=EPS, checkpoint=saved)
        y = y[0].float().cpu()
        assert (y[0] == 0).all() and torch.allclose(y[1], torch.ones(64), rtol=1e-2)
        assert torch.isnan(y[2, 7]) and torch.isnan(y[3]).all()
        assert torch.allclose(y[4], torch.full((64,), 1e-27), rtol=1e-2, atol=0)
        if saved:  # the NaN's block reads back as NaN, the row's other block (0: divided by infinity) as 0
            assert held.exponents.cpu()[0, 2].tolist() == [255, 1] and torch.isnan(y[2, :32]).all() and (y[2, 32:] == 0).all()
            assert held.exponents.cpu()[0, 3].tolist() == [255, 255]


def test_norm_without_rows():
    w = torch.ones(2, 40, device="cuda")
    x = torch.empty(2, 0, 40, device="cuda")
    y, s, saved = layers.add_rmsnorm(x, w, x, checkpoint=True)
    assert y.shape == (2, 0, 40) and saved.codes.shape == (2, 0, 64)
    dx, dw = layers.add_rmsnorm_backward(x, x, w, dweight=torch.full((2, 40), 7.0, device="cuda"))
    assert dx.shape == (2, 0, 40) and (dw == 0).all()


def test_norm_takes_one_model_and_repeated_rows():
    gen = rng(5)
    x, w = normal(gen, 6, 96).cuda(), normal(gen, 96).cuda()
    y, s, _ = layers.add_rmsnorm(x, w)
    assert s is x and torch.equal(y, layers.add_rmsnorm(x[None], w[None])[0][0])
    row = normal(gen, 1, 1, 96).cuda()
    y = layers.add_rmsnorm(row.expand(2, 4, 96), w.expand(2, 96))[0]
    assert torch.equal(y, y[:1, :1].expand(2, 4, 96))
    dx, dw = layers.add_rmsnorm_backward(x, x, w)
    assert dx.shape == x.shape and dw.shape == w.shape


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("shape", [(1, 1, 1), (2, 3, 32), (1, 5, 33), (3, 7, 384), (1, 2, 1003), (1, 1, 20000), (2, 65, 256)])
@pytest.mark.parametrize("layout", ["plain", "strided"])
def test_checkpoint(shape, dtype, layout):
    gen = rng(shape[-1])
    x = normal(gen, *shape) * torch.exp(3 * normal(gen, *shape))
    x.view(-1)[::7] = 0.0
    x = x.to(dtype)
    saved, values = layers.checkpoint(x.cuda() if layout == "plain" else strided(x))
    want, e = ref.held(x.double())
    assert torch.equal(saved.exponents.cpu().long() - 127, e)
    assert torch.equal(values.double().cpu(), want)
    assert torch.equal(layers.restore(saved), values)
    again, none = layers.checkpoint(x.cuda(), values=False)
    assert none is None and torch.equal(again.codes, saved.codes) and torch.equal(again.exponents, saved.exponents)
    assert (saved.codes[..., shape[-1]:] == 0).all()


def test_checkpoint_at_the_edges_of_the_types():
    top = torch.finfo(F32).max
    rows = [[0.0] * 32, [127.0] * 32, [127.00001] * 32, [top] * 32, [-top] + [top * 0.9] * 31, [1e-45] * 32, [2.0 ** -126] * 32,
            [-126.5] + [0.5] * 31, [1.5, 2.5, -0.5, -1.5, 127.0] + [0.0] * 27]
    x = torch.tensor(rows, dtype=F32)[None]
    saved, values = layers.checkpoint(x.cuda())
    want, e = ref.held(x.double())
    assert torch.equal(values.double().cpu(), want) and torch.isfinite(values).all()
    assert torch.equal(saved.exponents.cpu().long()[..., 0] - 127, e[..., 0])
    assert saved.codes[0, 8, :5].tolist() == [2, 2, 0, -2, 127]  # ties to even
    for bad in (float("inf"), float("-inf"), float("nan")):
        y = torch.ones(1, 2, 64)
        y[0, 0, 40] = bad
        saved, values = layers.checkpoint(y.cuda())
        assert saved.exponents[0].tolist() == [[121, 255], [121, 121]]
        assert torch.isnan(values[0, 0, 32:]).all() and (values[0, 0, :32] == 1).all() and (values[0, 1] == 1).all()
        assert torch.isnan(layers.restore(saved)[0, 0, 32:]).all()


WEIGHT_SHAPES = [(1, 1, 1, 1), (4, 32, 64, 64), (2, 33, 17, 31), (1, 100, 128, 256), (3, 65, 130, 257), (1, 1999, 100, 51),
                 (2, 128, 129, 512), (1, 64, 384, 40), (2, 5, 8, 1000), (1, 4500, 64, 72), (8, 200, 96, 160), (1, 777, 260, 300)]


@pytest.mark.parametrize("grad", [F32, BF16])
@pytest.mark.parametrize("shape", WEIGHT_SHAPES)
@pytest.mark.parametrize("layout", ["plain", "strided", "f32"])
def test_weight_gradient(shape, grad, layout):
    W, M, I, O = shape
    gen = rng(M)
    x, dy = normal(gen, W, M, I), normal(gen, W, M, O, dtype=F32 if layout == "f32" else BF16)
    saved, values = layers.checkpoint(x.cuda())
    dW, bound = ref.weight_gradient(dy, values.cpu())
    out, rows = slices(torch.zeros(W, O, I, dtype=grad), 3 if layout == "strided" else 0)
    got = layers.weight_gradient(strided(dy) if layout == "strided" else dy.cuda(), saved, out=out)
    assert got.data_ptr() == out.data_ptr()
    near(got, dW, bound)
    assert torch.isnan(rows).sum() == rows.numel() - W * O * I
    assert torch.equal(layers.weight_gradient(dy.cuda(), saved, dtype=grad), got)


def test_weight_gradient_of_repeated_and_shifted_dy():
    """dy whose rows repeat, overlap or start between words, against the same values laid out anew."""
    gen = rng(21)
    saved, _ = layers.checkpoint(normal(gen, 2, 70, 96).cuda())
    row = normal(gen, 1, 1, 40, dtype=BF16).cuda()
    long = normal(gen, 2 * 5000, dtype=BF16).cuda()
    def laid(t, worker, step, first=0):
        return t.as_strided((2, 70, 40), (worker, step, 1), first)

    for dy in (row.expand(2, 70, 40), laid(long, 3000, 8), laid(long, 0, 48), laid(long, 3000, 41, 1), laid(long, 4096, 48, 3),
               laid(long.float(), 3000, 41, 1)):
        want = layers.weight_gradient(dy.contiguous().clone(), saved)
        assert torch.equal(layers.weight_gradient(dy, saved), want)


def test_weight_gradient_of_many_tokens_keeps_its_precision():
    """128 tiles of 16,384 tokens, so no split of the tokens: one chain of 1,024 products would cut dW by 6e-6.
    Chunks of 128 products, each cutting at most 2^-25 of a sum that is two thirds of the last on average: 2.5e-6."""
    gen = torch.Generator(device="cuda").manual_seed(3)
    x = torch.randn(16, 16384, 512, generator=gen, device="cuda")
    dy = torch.randn(16, 16384, 512, generator=gen, device="cuda").to(BF16)
    saved, values = layers.checkpoint(x)
    dW = layers.weight_gradient(dy, saved)
    again = layers.weight_gradient(dy, saved)
    want = torch.einsum("wmo,wmi->woi", dy.double(), values.double())
    assert float((dW.double() - want).norm() / want.norm()) <= 2.5e-6
    assert torch.equal(dW, again)
    half = layers.weight_gradient(dy, saved, dtype=BF16)
    near(half, want.cpu(), 2e-4 * want.abs().cpu() + 2e-3)


def test_arrays_of_more_than_two_to_the_31_elements():
    """The last rows of arrays past 32-bit offsets, against the same rows alone."""
    M, D, tail = 540_000, 4096, 64
    gen = torch.Generator(device="cuda").manual_seed(4)
    x = torch.empty(1, M, D, dtype=BF16, device="cuda").normal_(generator=gen)
    assert x.numel() > 2 ** 31
    w = torch.rand(1, D, generator=gen, device="cuda")
    last = x[:, -tail:].contiguous()
    y, _, saved = layers.add_rmsnorm(x, w, x, checkpoint=True)
    y2, s2, saved2 = layers.add_rmsnorm(last, w, last, checkpoint=True)
    assert torch.equal(y[:, -tail:], y2) and torch.equal(saved.codes[:, -tail:], saved2.codes)
    assert torch.equal(layers.restore(saved)[:, -tail:], y2)
    del y
    dx, dw = layers.add_rmsnorm_backward(x, x, w)
    assert torch.equal(dx[:, -tail:], layers.add_rmsnorm_backward(last, last, w)[0]) and torch.isfinite(dw).all()
    del dx
    held, values = layers.checkpoint(x)
    assert torch.equal(values[:, -tail:], layers.checkpoint(last)[1])
    del values
    dy = torch.zeros(1, M, 16, dtype=BF16, device="cuda")
    dy[:, -tail:] = 1
    part = layers.weight_gradient(dy[:, -tail:].contiguous(), layers.checkpoint(last)[0])
    assert torch.allclose(layers.weight_gradient(dy, held), part, rtol=1e-5, atol=1e-3)
    del held
    h, end, carry = layers.gated_recurrence(x, x)
    h2, end2, carry2 = layers.gated_recurrence(last, last, carry[:, (M - tail) // layers.CARRY_STEPS])
    assert torch.allclose(h[:, -tail:].float(), h2.float(), rtol=1e-2, atol=1e-5) and torch.allclose(end, end2, rtol=1e-5, atol=1e-6)
    dgate, dvalue, _ = layers.gated_recurrence_backward(x, x, x, carry)
    dgate2, dvalue2, _ = layers.gated_recurrence_backward(last, last, last, carry2)
    assert torch.allclose(dgate[:, -tail:].float(), dgate2.float(), rtol=1e-2, atol=1e-5)
    assert torch.allclose(dvalue[:, -tail:].float(), dvalue2.float(), rtol=1e-2, atol=1e-5)


def test_weight_gradient_of_no_tokens_and_of_nan():
    saved, _ = layers.checkpoint(torch.empty(2, 0, 40, device="cuda"))
    out = torch.full((2, 24, 40), 3.0, device="cuda")
    assert (layers.weight_gradient(torch.empty(2, 0, 24, device="cuda", dtype=BF16), saved, out=out) == 0).all()
    x = torch.ones(1, 8, 64)
    x[0, 3, 5] = float("nan")
    saved, _ = layers.checkpoint(x.cuda())
    dW = layers.weight_gradient(torch.ones(1, 8, 16, dtype=BF16, device="cuda"), saved)[0]
    assert torch.isnan(dW[:, :32]).all() and (dW[:, 32:] == 8).all()


RECURRENCE_SHAPES = [(1, 1, 1), (4, 1, 384), (2, 5, 31), (3, 64, 64), (2, 65, 66), (1, 200, 33), (128, 3, 8), (2, 197, 384), (1, 1000, 70),
                     (3, 1025, 2), (1, 5000, 64)]


def recurrence_inputs(shape, dtype, ragged):
    B, T, D = shape
    gen = rng(T * 1000 + D)
    gate, value, dh = normal(gen, *shape, std=2.0) + 2.0, normal(gen, *shape), normal(gen, *shape)
    h0, dh_last = normal(gen, B, D), normal(gen, B, D)
    lengths = None
    if ragged:
        lengths = torch.randint(0, T + 1, (B,), generator=gen).to(torch.int32)
        lengths[0] = 0
        if B > 1:
            lengths[1] = 1
    return gate.to(dtype), value.to(dtype), dh.to(dtype), h0, dh_last, lengths


def on_gpu(t):
    return None if t is None else t.cuda()


@pytest.mark.parametrize("ragged", [False, True])
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("shape", RECURRENCE_SHAPES)
@pytest.mark.parametrize("layout", ["plain", "strided"])
def test_recurrence(shape, dtype, ragged, layout):
    gate, value, dh, h0, dh_last, lengths = recurrence_inputs(shape, dtype, ragged)
    put = on_gpu if layout == "plain" else strided
    n = on_gpu(lengths)
    for start, end in ((h0, dh_last), (None, None)):
        f = ref.recurrence(gate, value, start, lengths)
        h, last, carry = layers.gated_recurrence(put(gate), put(value), on_gpu(start), n)
        near(h, f["h"], f["eh"])
        near(last, f["last"], f["elast"])
        b = ref.recurrence_backward(dh, gate, value, start, end, lengths)
        dgate, dvalue, dh0 = layers.gated_recurrence_backward(put(dh), put(gate), put(value), carry, on_gpu(end), n)
        near(dvalue, b["dvalue"], b["edvalue"])
        near(dgate, b["dgate"], b["edgate"])
        near(dh0, b["dh0"], b["edh0"])
    # without the carries, and twice: the same bits
    h2, last2, none = layers.gated_recurrence(put(gate), put(value), None, n, carry=False)
    assert none is None and torch.equal(h2, h) and torch.equal(last2, last)
    again = layers.gated_recurrence_backward(put(dh), put(gate), put(value), carry, None, n)
    assert all(torch.equal(p, q) for p, q in zip(again, (dgate, dvalue, dh0)))


def test_recurrence_of_long_ragged_sequences():
    """A long sequence next to shorter ones: many segments, ends inside and between them, the same bits each time."""
    shape = (3, 20000, 200)
    gate, value, dh, h0, dh_last, _ = recurrence_inputs(shape, F32, False)
    lengths = torch.tensor([20000, 4097, 15000], dtype=torch.int32)
    f = ref.recurrence(gate, value, h0, lengths)
    b = ref.recurrence_backward(dh, gate, value, h0, dh_last, lengths)
    layers.wait_timeouts()
    for _ in range(3):
        h, last, carry = layers.gated_recurrence(gate.cuda(), value.cuda(), h0.cuda(), lengths.cuda())
        grads = layers.gated_recurrence_backward(dh.cuda(), gate.cuda(), value.cuda(), carry, dh_last.cuda(), lengths.cuda())
        assert layers.wait_timeouts() == 0
    near(h, f["h"], f["eh"])
    near(last, f["last"], f["elast"])
    for got, name in zip(grads, ("dgate", "dvalue", "dh0")):
        near(got, b[name], b["e" + name])


def test_recurrence_reads_nothing_beyond_a_length():
    gate, value, dh, h0, dh_last, _ = recurrence_inputs((3, 90, 40), F32, False)
    lengths = torch.tensor([0, 17, 200], dtype=torch.int32)  # clamped to T
    f = ref.recurrence(gate, value, h0, lengths)
    b = ref.recurrence_backward(dh, gate, value, h0, dh_last, lengths)
    for t in (gate, value, dh):
        t[0], t[1, 17:] = float("nan"), float("nan")
    h, last, carry = layers.gated_recurrence(gate.cuda(), value.cuda(), h0.cuda(), lengths.cuda())
    near(h, f["h"], f["eh"])
    near(last, f["last"], f["elast"])
    dgate, dvalue, dh0 = layers.gated_recurrence_backward(dh.cuda(), gate.cuda(), value.cuda(), carry, dh_last.cuda(), lengths.cuda())
    near(dvalue, b["dvalue"], b["edvalue"])
    near(dgate, b["dgate"], b["edgate"])
    near(dh0, b["dh0"], b["edh0"])
    lengths[:] = -3
    h, last, _ = layers.gated_recurrence(gate.cuda(), value.cuda(), h0.cuda(), lengths.cuda())
    assert (h == 0).all() and torch.equal(last.cpu(), h0)


def test_recurrence_with_open_and_closed_gates():
    T, big = 100, 300.0
    gate = torch.full((3, T, 8), big)
    gate[1], gate[2] = -big, float("inf")
    value, h0 = normal(rng(1), 3, T, 8), normal(rng(2), 3, 8)
    h, last, carry = layers.gated_recurrence(gate.cuda(), value.cuda(), h0.cuda())
    assert torch.equal(last[0].cpu(), h0[0]) and torch.equal(last[2].cpu(), h0[2]) and torch.equal(h[1].cpu(), value[1])
    dh = torch.ones(3, T, 8)
    dgate, dvalue, dh0 = layers.gated_recurrence_backward(dh.cuda(), gate.cuda(), value.cuda(), carry)
    assert (dgate == 0).all() and (dvalue[0] == 0).all() and (dvalue[1] == 1).all() and (dh0[0] == T).all() and (dh0[1] == 0).all()


def test_recurrence_without_steps_or_sequences():
    h0 = normal(rng(3), 2, 16).cuda()
    x = torch.empty(2, 0, 16, device="cuda", dtype=BF16)
    h, last, carry = layers.gated_recurrence(x, x, h0)
    assert h.shape == (2, 0, 16) and torch.equal(last, h0) and carry.shape == (2, 0, 16)
    dgate, dvalue, dh0 = layers.gated_recurrence_backward(x, x, x, carry, h0)
    assert dgate.shape == (2, 0, 16) and torch.equal(dh0, h0)
    x = torch.empty(0, 4, 16, device="cuda")
    h, last, carry = layers.gated_recurrence(x, x)
    assert h.shape == (0, 4, 16) and last.shape == (0, 16)
    assert layers.gated_recurrence_step(x[:, 0], x[:, 0], torch.empty(0, 16, device="cuda")).shape == (0, 16)


def test_recurrence_of_very_many_sequences():
    """More than 65,535, the limit of a grid's second and third sizes."""
    B = 70_000
    gate, value, dh, h0, dh_last, lengths = recurrence_inputs((B, 2, 3), F32, True)
    f = ref.recurrence(gate, value, h0, lengths)
    h, last, carry = layers.gated_recurrence(gate.cuda(), value.cuda(), h0.cuda(), lengths.cuda())
    near(h, f["h"], f["eh"])
    b = ref.recurrence_backward(dh, gate, value, h0, dh_last, lengths)
    grads = layers.gated_recurrence_backward(dh.cuda(), gate.cuda(), value.cuda(), carry, dh_last.cuda(), lengths.cuda())
    for got, name in zip(grads, ("dgate", "dvalue", "dh0")):
        near(got, b[name], b["e" + name])
    state = h0.cuda()
    near(layers.gated_recurrence_step(gate.cuda()[:, 0], value.cuda()[:, 0], state), *[ref.recurrence(gate[:, :1], value[:, :1], h0, None)[k][:, 0] for k in ("h", "eh")])


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("B,D", [(1, 1), (4, 384), (3, 33), (65, 1024)])
def test_recurrence_step_continues_a_sequence(B, D, dtype):
    gate, value, _, h0, _, _ = recurrence_inputs((B, 6, D), dtype, False)
    f = ref.recurrence(gate, value, h0, None)
    state = h0.cuda()
    for t in range(6):
        h = layers.gated_recurrence_step(gate.cuda()[:, t], value.cuda()[:, t], state)
        near(h, f["h"][:, t], f["eh"][:, t])
    near(state, f["last"], f["elast"])


def test_gradients_against_differences():
    """Directional derivatives of the 64-bit forward formulas, by central differences."""
    gen = rng(11)
    h = 1e-6

    def slope(f, *args):
        us = [normal(gen, *a.shape).double() for a in args]
        up, down = f(*[a + h * u for a, u in zip(args, us)]), f(*[a - h * u for a, u in zip(args, us)])
        return float((up - down) / (2 * h)), us

    x, w, dy = normal(gen, 2, 9, 70), 1 + 0.3 * normal(gen, 2, 70), normal(gen, 2, 9, 70)
    f = lambda a, b: (b[:, None] * a / torch.sqrt(a.square().mean(-1, keepdim=True) + EPS) * dy.double()).sum()  # noqa: E731
    want, (ux, uw) = slope(f, x.double(), w.double())
    dx, dw = layers.add_rmsnorm_backward(dy.cuda(), x.cuda(), w.cuda(), eps=EPS)
    got = float((dx.double().cpu() * ux).sum() + (dw.double().cpu() * uw).sum())
    scale = float((dx.double().cpu() * ux).abs().sum() + (dw.double().cpu() * uw).abs().sum())
    assert abs(got - want) <= 1e-5 * scale

    gate, value, dh, h0, dh_last, lengths = recurrence_inputs((4, 70, 9), F32, True)

    def g(*a):
        r = ref.recurrence(*a, lengths)
        return (r["h"] * dh.double()).sum() + (r["last"] * dh_last.double()).sum()

    want, us = slope(g, gate.double(), value.double(), h0.double())
    _, _, carry = layers.gated_recurrence(gate.cuda(), value.cuda(), h0.cuda(), lengths.cuda())
    grads = layers.gated_recurrence_backward(dh.cuda(), gate.cuda(), value.cuda(), carry, dh_last.cuda(), lengths.cuda())
    parts = [float((p.double().cpu() * u).sum()) for p, u in zip(grads, us)]
    scale = sum(float((p.double().cpu() * u).abs().sum()) for p, u in zip(grads, us))
    assert abs(sum(parts) - want) <= 1e-5 * scale


def test_calls_on_another_stream():
    gen = rng(13)
    x, w, r = normal(gen, 2, 50, 64).cuda(), normal(gen, 2, 64).cuda(), normal(gen, 2, 50, 64).cuda()
    gate, value = normal(gen, 2, 300, 64).cuda(), normal(gen, 2, 300, 64).cuda()
    dy = normal(gen, 2, 50, 24, dtype=BF16).cuda()

    def everything(stream=None):
        y, s, saved = layers.add_rmsnorm(x, w, r, checkpoint=True, stream=stream)
        dx, dw = layers.add_rmsnorm_backward(x, s, w, r, stream=stream)
        held, values = layers.checkpoint(x, stream=stream)
        dW = layers.weight_gradient(dy, held, stream=stream)
        h, last, carry = layers.gated_recurrence(gate, value, stream=stream)
        dg, dv, dh0 = layers.gated_recurrence_backward(h, gate, value, carry, stream=stream)
        state = last.clone() if stream is None else None
        return [y, s, dx, dw, values, layers.restore(held, stream=stream), dW, h, last, dg, dv, dh0], state

    want, _ = everything()
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    for stream in (side, side.cuda_stream):
        got, _ = everything(stream)
        side.synchronize()
        assert all(torch.equal(p, q) for p, q in zip(got, want))
    assert torch.cuda.current_stream() != side


def test_calls_can_be_captured():
    gen = rng(17)
    gate, value = normal(gen, 2, 700, 64, dtype=BF16).cuda(), normal(gen, 2, 700, 64, dtype=BF16).cuda()
    x, w, dy = normal(gen, 2, 70, 64).cuda(), normal(gen, 2, 64).cuda(), normal(gen, 2, 70, 24, dtype=BF16).cuda()

    def step():
        y, s, saved = layers.add_rmsnorm(x, w, x, checkpoint=True)
        dx, dw = layers.add_rmsnorm_backward(x, s, w, x)
        dW = layers.weight_gradient(dy, saved)
        h, last, carry = layers.gated_recurrence(gate, value)
        return [y, dx, dw, dW, h, last, *layers.gated_recurrence_backward(h, gate, value, carry)]

    want = step()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = step()
    for _ in range(3):
        graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(p, q) for p, q in zip(got, want))


def test_refusals():
    x, w = torch.zeros(2, 3, 32, device="cuda"), torch.ones(2, 32, device="cuda")
    for call, error in [
        (lambda: layers.add_rmsnorm(x.cpu(), w), ValueError),
        (lambda: layers.add_rmsnorm(x, w[:1]), ValueError),
        (lambda: layers.add_rmsnorm(x, w.bfloat16()), TypeError),
        (lambda: layers.add_rmsnorm(x.half(), w), TypeError),
        (lambda: layers.add_rmsnorm(x, w, x.bfloat16()), TypeError),
        (lambda: layers.add_rmsnorm(x, w, x[:, :2]), ValueError),
        (lambda: layers.add_rmsnorm(x.transpose(1, 2).contiguous().transpose(1, 2), w), ValueError),
        (lambda: layers.add_rmsnorm(x, w, eps=0.0), CPDPError),
        (lambda: layers.add_rmsnorm(x, w, eps=float("nan")), CPDPError),
        (lambda: layers.add_rmsnorm(torch.zeros(1, 1, 16385, device="cuda"), torch.ones(1, 16385, device="cuda")), CPDPError),
        (lambda: layers.add_rmsnorm_backward(x.bfloat16(), x, w), TypeError),
        (lambda: layers.add_rmsnorm_backward(x, x, w, dweight=w[:, :31]), ValueError),
        (lambda: layers.add_rmsnorm_backward(x, x, w, dtype=torch.float16), TypeError),
        (lambda: layers.checkpoint(x[0, 0]), ValueError),
        (lambda: layers.checkpoint(x.int()), TypeError),
        (lambda: layers.weight_gradient(x[:, :2], layers.checkpoint(x)[0]), ValueError),
        (lambda: layers.weight_gradient(x.half(), layers.checkpoint(x)[0]), TypeError),
        (lambda: layers.weight_gradient(x, layers.checkpoint(x)[0], out=torch.zeros(2, 32, 31, device="cuda")), ValueError),
        (lambda: layers.weight_gradient(x, layers.Checkpoint(x, x, 32)), TypeError),
        (lambda: layers.gated_recurrence(x, x.bfloat16()), TypeError),
        (lambda: layers.gated_recurrence(x, x, w.double()), TypeError),
        (lambda: layers.gated_recurrence(x, x, None, torch.zeros(2, device="cuda", dtype=torch.int64)), TypeError),
        (lambda: layers.gated_recurrence(x, x, None, torch.zeros(2, dtype=torch.int32)), ValueError),
        (lambda: layers.gated_recurrence_backward(x, x, x, w), ValueError),
        (lambda: layers.gated_recurrence_step(w, w, w.bfloat16()), TypeError),
        (lambda: layers.gated_recurrence_step(w, w, torch.ones(32, 2, device="cuda").T), ValueError),
    ]:
        with pytest.raises(error):
            call()
    torch.cuda.synchronize()
