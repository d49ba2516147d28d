"""The loss over a vocabulary on the GPU against 64-bit references
(operators_reference.py): sizes around its tiles, odd widths and unaligned rows,
ignored and impossible targets, infinities and NaN in ignored rows, pieces of the
vocabulary, streams and graphs. Tolerances are the references' own bounds."""
import math

import pytest
import torch

import operators_reference as ref
from paper_2607_21224_gb300 import layers
from test_layers_gpu import near, normal, rng, slices, strided

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16


def problem(shape, dtype, seed=0):
    W, M, D, V = shape
    gen = rng(seed + 7 * M + V)
    x, weight = normal(gen, W, M, D, dtype=dtype), normal(gen, W, V, D, std=1.5 / D ** 0.5, dtype=dtype)
    targets = torch.randint(0, V, (W, M), generator=gen)
    targets[torch.rand((W, M), generator=gen) < 0.2] = -1
    dloss = torch.rand((W, M), generator=gen) / max(M, 1)
    return x, weight, targets, dloss


SHAPES = [(1, 1, 1, 1), (1, 1, 64, 2), (4, 32, 128, 64), (2, 33, 17, 31), (1, 128, 64, 256), (1, 129, 72, 257), (3, 65, 130, 511),
          (1, 257, 40, 1000), (2, 5, 771, 1023), (1, 3, 2056, 384), (1, 1000, 16, 65), (2, 70, 96, 4099), (8, 9, 24, 300)]


@pytest.mark.parametrize("dtype,grad", [(F32, F32), (BF16, BF16), (BF16, F32)])
@pytest.mark.parametrize("shape", SHAPES)
@pytest.mark.parametrize("layout", ["plain", "strided"])
def test_loss(shape, dtype, grad, layout):
    W, M, D, V = shape
    x, weight, targets, dloss = problem(shape, dtype)
    put = (lambda t: t.cuda()) if layout == "plain" else strided
    xs, ws, ts = put(x), put(weight), targets.cuda()
    f = ref.loss(x, weight, targets)
    loss, lse = layers.linear_cross_entropy(xs, ws, ts)
    near(loss, f["loss"], f["eloss"])
    near(lse, f["lse"], f["else"])
    dx, dweight, edx, edw = ref.loss_backward(dloss, x, weight, targets)
    out, rows = slices(torch.zeros(W, V, D, dtype=grad), 3 if layout == "strided" else 0)
    got, got_w = layers.linear_cross_entropy_backward(dloss.cuda(), xs, ws, ts, lse, dweight=out)
    assert got_w.data_ptr() == out.data_ptr() and got.dtype == dtype
    near(got, dx, edx)
    near(got_w, dweight, edw)
    assert (got[targets.cuda() < 0] == 0).all()
    assert torch.isnan(rows).sum() == rows.numel() - W * V * D
    again, again_w = layers.linear_cross_entropy_backward(dloss.cuda(), xs, ws, ts, lse, dtype=grad)
    assert torch.equal(again, got) and torch.equal(again_w, got_w)
    assert layers.wait_timeouts() == 0


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_ignored_tokens_reach_nothing(dtype):
    x, weight, targets, dloss = problem((2, 150, 72, 333), dtype, 5)
    targets[:, 1] = 4
    f, g = ref.loss(x, weight, targets), ref.loss_backward(dloss, x, weight, targets)
    ignored = targets < 0
    bad, dl = x.clone(), dloss.clone()
    for k, value in enumerate((float("nan"), float("inf"), -float("inf"))):
        bad[ignored] = torch.where(torch.arange(bad[ignored].shape[0])[:, None] % 3 == k, value, bad[ignored])
    dl[ignored] = float("nan")
    loss, lse = layers.linear_cross_entropy(bad.cuda(), weight.cuda(), targets.cuda())
    assert (loss.cpu()[ignored] == 0).all()
    near(loss[~ignored.cuda()], f["loss"][~ignored], f["eloss"][~ignored])
    dx, dw = layers.linear_cross_entropy_backward(dl.cuda(), bad.cuda(), weight.cuda(), targets.cuda(), lse)
    near(dx, g[0], g[2])
    near(dw, g[1], g[3])
    # all of them, and none of their gradients
    targets[:] = -100
    loss, lse = layers.linear_cross_entropy(bad.cuda(), weight.cuda(), targets.cuda())
    dx, dw = layers.linear_cross_entropy_backward(dl.cuda(), bad.cuda(), weight.cuda(), targets.cuda(), lse)
    assert (loss == 0).all() and (dx == 0).all() and (dw == 0).all()


def test_impossible_targets_and_infinite_logits():
    x, weight, targets, dloss = problem((1, 9, 64, 300), BF16, 2)
    targets[0, :] = torch.tensor([5, 299, 300, 1 << 40, 2 ** 62, 0, 1, 2, 3])
    loss, lse = layers.linear_cross_entropy(x.cuda(), weight.cuda(), targets.cuda())
    wrong = torch.tensor([False, False, True, True, True, False, False, False, False])
    assert torch.equal(torch.isnan(loss.cpu())[0], wrong) and torch.isfinite(lse).all()
    dx, dw = layers.linear_cross_entropy_backward(dloss.cuda(), x.cuda(), weight.cuda(), targets.cuda(), lse)
    assert torch.equal(torch.isnan(dx.cpu()).all(-1)[0], wrong) and torch.equal(torch.isnan(dx.cpu()).any(-1)[0], wrong)
    # a word whose logit is -infinity has the probability 0; one of +infinity leaves no probabilities
    x[..., 0], weight[0, 7, 0] = 1.0, -float("inf")
    targets[0, :] = 5
    near(layers.linear_cross_entropy(x.cuda(), weight.cuda(), targets.cuda())[0], *without(x, weight, targets, 7))
    weight[0, 7, 0] = float("inf")
    loss, lse = layers.linear_cross_entropy(x.cuda(), weight.cuda(), targets.cuda())
    assert not torch.isfinite(loss).any() and not torch.isfinite(lse).any()


def without(x, weight, targets, word):
    keep = [v for v in range(weight.shape[1]) if v != word]
    f = ref.loss(x, weight[:, keep], targets)
    return f["loss"], f["eloss"]


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_large_and_equal_logits(dtype):
    """Logits of +-1e4 (one probability of 1), and all equal (lse = l + log(V))."""
    M, V, D = 40, 700, 64
    x, weight = torch.zeros(1, M, D), torch.zeros(1, V, D)
    x[..., 0] = 128.0
    weight[0, :, 0] = torch.linspace(-80, 80, V).to(torch.bfloat16).float()
    x[0, 20:] = 0.0
    targets = torch.full((1, M), V - 1)
    f = ref.loss(x.to(dtype), weight.to(dtype), targets)
    loss, lse = layers.linear_cross_entropy(x.to(dtype).cuda(), weight.to(dtype).cuda(), targets.cuda())
    near(loss, f["loss"], f["eloss"])
    near(lse, f["lse"], f["else"])


@pytest.mark.parametrize("level", [-300.0, -90.0, 90.0, 300.0])
@pytest.mark.parametrize("V", [3, 128, 129, 300, 4000])
def test_all_logits_far_from_zero(V, level):
    x, weight = torch.zeros(1, 5, 16), normal(rng(V), 1, V, 16)
    x[..., 0], weight[..., 0] = 1.0, level
    x[..., 1] = 1.0
    targets = torch.arange(5)[None] % V
    f = ref.loss(x, weight, targets)
    loss, lse = layers.linear_cross_entropy(x.cuda(), weight.cuda(), targets.cuda())
    near(loss, f["loss"], f["eloss"])
    near(lse, f["lse"], f["else"])


@pytest.mark.parametrize("M", [1, 7, 8, 9, 24, 25])
@pytest.mark.parametrize("D,V", [(4, 1), (3, 127), (128, 128), (200, 129), (132, 391), (1028, 1000), (517, 2049)])
@pytest.mark.parametrize("shift", [0, 1])
def test_few_tokens(M, D, V, shift):
    """Float32 products without planes, and the first size with them; rows at 16 bytes and off them."""
    x, weight, targets, dloss = problem((2, M, D, V), F32, shift)
    targets[0, 0], targets[1, M - 1] = V - 1, 0
    each = (V * D + 7) // 4 * 4  # a worker's part, from a multiple of 16 bytes or one element on
    ws = torch.full((2 * each + 1,), float("nan"), device="cuda").as_strided((2, V, D), (each, D, 1), shift)
    ws.copy_(weight)
    xs, ts = x.cuda(), targets.cuda()
    f = ref.loss(x, weight, targets)
    loss, lse = layers.linear_cross_entropy(xs, ws, ts)
    near(loss, f["loss"], f["eloss"])
    near(lse, f["lse"], f["else"])
    again = layers.linear_cross_entropy(xs, ws, ts)
    assert torch.equal(again[0], loss) and torch.equal(again[1], lse)
    dx, dw, edx, edw = ref.loss_backward(dloss, x, weight, targets)
    got, got_w = layers.linear_cross_entropy_backward(dloss.cuda(), xs, ws, ts, lse)
    near(got, dx, edx)
    near(got_w, dw, edw)


def test_few_tokens_with_infinities():
    """Float32 products keep an infinite word's logit infinite: all other words have the probability 0."""
    x, weight = torch.ones(1, 3, 8), torch.zeros(1, 300, 8)
    weight[0, 200, 3] = -float("inf")
    targets = torch.tensor([[200, 5, -1]])
    loss, lse = layers.linear_cross_entropy(x.cuda(), weight.cuda(), targets.cuda())
    assert loss[0, 0] == float("inf") and loss[0, 2] == 0 and (lse - math.log(299)).abs().max() < 1e-5 and abs(float(loss[0, 1]) - math.log(299)) < 1e-5


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_one_word(dtype):
    """Its probability is 1 whatever the logit: the loss and both gradients are 0."""
    gen = rng(2)
    x, weight = normal(gen, 3, 50, 40, std=9.0, dtype=dtype).cuda(), normal(gen, 3, 1, 40, std=3.0, dtype=dtype).cuda()
    targets = torch.zeros(3, 50, dtype=torch.int64, device="cuda")
    loss, lse = layers.linear_cross_entropy(x, weight, targets)
    dx, dw = layers.linear_cross_entropy_backward(torch.ones_like(loss), x, weight, targets, lse)
    assert (loss == 0).all() and (lse != 0).all() and (dx == 0).all() and (dw == 0).all()


def test_several_pieces_of_the_vocabulary_and_splits():
    """More probabilities than are held at a time, a last piece of another size, and long sums split among blocks. The
    gradients of rows and words picked out are compared."""
    W, M, D, V = 2, 3000, 40, 33001
    x, weight, targets, dloss = problem((W, M, D, V), BF16, 3)
    xs, ws, ts, dl = x.cuda(), weight.cuda(), targets.cuda(), dloss.cuda()
    loss, lse = layers.linear_cross_entropy(xs, ws, ts)
    dx, dw = layers.linear_cross_entropy_backward(dl, xs, ws, ts, lse)
    rows = torch.tensor([0, 1, 127, 128, 1500, 2999])
    f = ref.loss(x[:, rows], weight, targets[:, rows])
    near(loss[:, rows.cuda()], f["loss"], f["eloss"])
    g = ref.loss_backward(dloss[:, rows], x[:, rows], weight, targets[:, rows])
    near(dx[:, rows.cuda()], g[0], g[2])
    # dweight: the words' rows from all tokens, with lse from all words
    words = torch.tensor([0, 255, 256, 16383, 16384, 22015, 22016, 33000])
    p = torch.exp(xs.double() @ ws[:, words.cuda()].double().transpose(1, 2) - lse.double()[..., None])
    hot = (ts[..., None] == words.cuda()).double()
    d = torch.where(ts[..., None] >= 0, dl.double()[..., None] * (p - hot), 0.0)
    want = d.transpose(1, 2) @ xs.double()
    size = d.abs().transpose(1, 2) @ xs.double().abs()
    # d's rounding to bfloat16 and float32's in the exponents (|l - lse| below 16), then the sum of M products
    bound = (2.0 ** -8 * 1.01 + 2.0 ** -18) * size + ref.product_bound(size, M, BF16)
    near(dw[:, words.cuda()], want.cpu(), bound.cpu())


@pytest.mark.parametrize("each", [1 / 7, 0.3, 1.0, 1e-20, 3e30])
def test_a_weight_that_all_tokens_share_is_not_rounded(each):
    """Logits near 0 over 5,000 words: d of a target is dloss (p - 1) with p at most 1.1 / 5,000, and bfloat16 holds 1 - p as
    1. So a word that one token has for its target gets -dloss x within p; nothing adds up to more, since another token's
    share of the word is p x at most."""
    W, M, D, V = 2, 5, 64, 5000
    gen = rng(3)
    x, weight = normal(gen, W, M, D).bfloat16(), (normal(gen, W, V, D) * 1e-4).bfloat16()
    targets = torch.arange(M).repeat(W, 1) * 900
    dloss = torch.full((W, M), each)
    dloss[1, 0] = 0.0
    lse = layers.linear_cross_entropy(x.cuda(), weight.cuda(), targets.cuda())[1]
    dx, dw = layers.linear_cross_entropy_backward(dloss.cuda(), x.cuda(), weight.cuda(), targets.cuda(), lse)
    share = 1.1 / V
    got = dw.cpu().double().gather(1, targets[..., None].expand(W, M, D))
    size = x.double().abs().sum(1, keepdim=True)
    assert ((got + dloss.double()[..., None] * x.double()).abs() <= 1.001 * each * share * size).all()
    want = ref.loss_backward(dloss, x, weight, targets)[0]
    # 1 - p held as 1, the other p rounded, and the sum of V products
    most, every = weight.double().abs().amax(1, keepdim=True), weight.double().abs().sum(1, keepdim=True)
    bound = each * share * (most + 2.0 ** -8 * every) + ref.product_bound(each * (most + share * every), V, BF16)
    near(dx, want, bound.expand(W, M, D))


@pytest.mark.parametrize("M", [8192, 8193, 30001])
def test_weights_of_many_tokens(M):
    """The largest weight of a worker may be any token's; a worker whose weights are all 0, and infinite and NaN ones of
    ignored tokens."""
    W, D, V = 3, 8, 4100
    gen = rng(M)
    x, weight = normal(gen, W, M, D, dtype=BF16), normal(gen, W, V, D, std=0.3, dtype=BF16)
    targets = torch.randint(0, V, (W, M), generator=gen)
    targets[:, 5:7] = -1
    dloss = torch.rand((W, M), generator=gen) * 1e-3
    dloss[0, M - 1], dloss[1] = 37.0, 0.0
    dloss[:, 5], dloss[:, 6] = float("inf"), float("nan")
    lse = layers.linear_cross_entropy(x.cuda(), weight.cuda(), targets.cuda())[1]
    dx, dw = layers.linear_cross_entropy_backward(dloss.cuda(), x.cuda(), weight.cuda(), targets.cuda(), lse)
    assert (dx[1] == 0).all() and (dw[1] == 0).all() and torch.isfinite(dw).all()
    rows = torch.tensor([0, 5, 6, 100, 8191, M - 1])
    dloss[:, 5:7] = 0.0
    g = ref.loss_backward(dloss[:, rows], x[:, rows], weight, targets[:, rows])
    near(dx[:, rows.cuda()], g[0], g[2])


def test_gradients_against_differences():
    W, M, D, V = 2, 37, 24, 90
    x, weight, targets, dloss = problem((W, M, D, V), F32, 9)
    gen = rng(1)
    u, v, h = normal(gen, W, M, D).double(), normal(gen, W, V, D).double(), 1e-5

    def total(s):
        f = ref.loss((x.double() + s * u), (weight.double() + s * v), targets)
        return (f["loss"] * dloss).sum()

    lse = layers.linear_cross_entropy(x.cuda(), weight.cuda(), targets.cuda())[1]
    dx, dw = layers.linear_cross_entropy_backward(dloss.cuda(), x.cuda(), weight.cuda(), targets.cuda(), lse)
    got = (dx.cpu().double() * u).sum() + (dw.cpu().double() * v).sum()
    want = (total(h) - total(-h)) / (2 * h)
    size = (dx.cpu().double() * u).abs().sum() + (dw.cpu().double() * v).abs().sum()
    assert abs(got - want) <= 1e-5 * size


def test_loss_without_tokens_of_one_model_and_repeated_rows():
    weight = torch.ones(2, 50, 16, device="cuda")
    x, targets = torch.empty(2, 0, 16, device="cuda"), torch.empty((2, 0), dtype=torch.int64, device="cuda")
    loss, lse = layers.linear_cross_entropy(x, weight, targets)
    assert loss.shape == lse.shape == (2, 0)
    dx, dw = layers.linear_cross_entropy_backward(loss, x, weight, targets, lse, dweight=torch.full((2, 50, 16), 7.0, device="cuda"))
    assert dx.shape == x.shape and (dw == 0).all()
    x, weight, targets, dloss = (t.cuda() for t in problem((1, 30, 64, 200), BF16, 4))
    loss, lse = layers.linear_cross_entropy(x[0], weight[0], targets[0])
    both = layers.linear_cross_entropy(x, weight, targets)
    assert torch.equal(loss, both[0][0]) and torch.equal(lse, both[1][0])
    dx, dw = layers.linear_cross_entropy_backward(dloss[0], x[0], weight[0], targets[0], lse, dtype=BF16)
    assert dx.shape == (30, 64) and dw.shape == (200, 64) and dw.dtype == BF16
    # rows and workers that repeat in memory
    row = x[:, :1].expand(3, 5, 64)
    t = targets[:, :1].clamp(min=0).expand(3, 5).contiguous()
    loss, lse = layers.linear_cross_entropy(row, weight.expand(3, 200, 64), t)
    assert torch.equal(loss, loss[:1, :1].expand(3, 5))


def test_another_stream_and_a_graph():
    x, weight, targets, dloss = (t.cuda() for t in problem((2, 200, 72, 1000), BF16, 6))

    def step():
        loss, lse = layers.linear_cross_entropy(x, weight, targets)
        return loss, *layers.linear_cross_entropy_backward(dloss, x, weight, targets, lse)

    want = step()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    loss, lse = layers.linear_cross_entropy(x, weight, targets, stream=side)
    dx, dw = layers.linear_cross_entropy_backward(dloss, x, weight, targets, lse, stream=side)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(want, (loss, dx, dw)))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = step()
    new = x.roll(1, 1)
    x.copy_(new)
    for t in held:
        t.fill_(float("nan"))
    graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(held, step()))
    assert not torch.equal(held[0], want[0])


def test_refused_tensors():
    x, weight, targets, dloss = (t.cuda() for t in problem((2, 20, 16, 50), BF16))
    loss, lse = layers.linear_cross_entropy(x, weight, targets)
    for bad in (lambda: layers.linear_cross_entropy(x.half(), weight, targets), lambda: layers.linear_cross_entropy(x, weight.float(), targets),
                lambda: layers.linear_cross_entropy(x, weight, targets.int()),
                lambda: layers.linear_cross_entropy_backward(dloss.bfloat16(), x, weight, targets, lse),
                lambda: layers.linear_cross_entropy_backward(dloss, x, weight, targets, lse, dtype=torch.half)):
        with pytest.raises(TypeError):
            bad()
    for bad in (lambda: layers.linear_cross_entropy(x, weight[:, :, :8], targets), lambda: layers.linear_cross_entropy(x, weight[:1], targets),
                lambda: layers.linear_cross_entropy(x, weight, targets[:, :5]), lambda: layers.linear_cross_entropy(x, weight[0], targets),
                lambda: layers.linear_cross_entropy(x, weight.transpose(1, 2).contiguous().transpose(1, 2), targets),
                lambda: layers.linear_cross_entropy(x, weight, targets.cpu()),
                lambda: layers.linear_cross_entropy(x, weight.clone().requires_grad_(), targets),
                lambda: layers.linear_cross_entropy_backward(dloss[:, ::2], x, weight, targets, lse),
                lambda: layers.linear_cross_entropy_backward(dloss, x, weight, targets, lse,
                                                             dweight=torch.zeros(1, 50, 16, device="cuda").expand(2, 50, 16))):
        with pytest.raises(ValueError):
            bad()
