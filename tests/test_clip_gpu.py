"""Gradient norms and clipping on the GPU against 64-bit references: rows of none
to millions of values at every alignment, values whose squares leave float32,
infinities and NaN, in place and into other rows."""
import pytest
import torch

import operators_reference as ref
from paper_2607_21224_gb300 import cpdp, layers
from test_layers_gpu import near, normal, rng

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16


def rows(t, shift, extra):
    """A CUDA copy of t (W, N) inside longer rows of NaN, and those rows."""
    W, N = t.shape
    long = torch.full((W, N + shift + extra), float("nan"), dtype=t.dtype, device="cuda")
    long[:, shift:shift + N] = t.cuda()
    return long[:, shift:shift + N], long


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("N", [1, 2, 3, 7, 8, 9, 255, 1024, 4096, 4097, 16385, 70001, 700003])
@pytest.mark.parametrize("shifts", [(0, 0), (1, 1), (3, 0), (0, 5), (2, 10), (7, 8)])
def test_clip(N, dtype, shifts):
    W, gen = 4, rng(N)
    g = normal(gen, W, N) * torch.tensor([0.3, 0.9, 1.6, 40.0])[:, None] / N ** 0.5
    g = g.to(dtype)
    norms, out, enorms, eout = ref.clip(g, 1.0)
    grads, long = rows(g, shifts[0], 3)
    to, beside = rows(torch.zeros_like(g), shifts[1], 6)
    got = layers.clip_gradients(grads, 1.0, out=to)
    near(got, norms, enorms, F32)
    near(to, out, eout)
    assert torch.equal(grads.cpu(), g)
    for t in (long, beside):
        assert int(torch.isnan(t).sum()) == t.numel() - g.numel()
    assert torch.equal(layers.clip_gradients(grads, 1.0), got) and torch.equal(grads, to)  # over grads
    assert int(torch.isnan(long).sum()) == long.numel() - g.numel()
    keep = grads.clone()
    layers.clip_gradients(grads, float("inf"))
    assert torch.equal(grads, keep)


@pytest.mark.parametrize("size", [1e-38, 1e-30, 1e-23, 1e-19, 1e-10, 1e10, 1e18, 1e20, 1e30, 1e35])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_sizes_whose_squares_leave_float32(size, dtype):
    g = (normal(rng(1), 2, 3001) * size).to(dtype)
    for most in (1.0, size):
        norms, out, enorms, eout = ref.clip(g, most)
        to = torch.empty_like(g, device="cuda")
        near(layers.clip_gradients(g.cuda(), most, out=to), norms, enorms + 2.0 ** -140, F32)
        near(to, out, eout + 2.0 ** -133)


def test_rows_of_zeros_infinity_and_nan():
    g = torch.ones(4, 5000)
    g[0] = 0.0
    g[1, 77], g[2, 4999] = -float("inf"), float("nan")
    out = torch.empty(4, 5000, device="cuda")
    norms = layers.clip_gradients(g.cuda(), 1.0, out=out).cpu()
    assert norms[0] == 0 and torch.isinf(norms[1]) and torch.isnan(norms[2]) and abs(norms[3] - 5000 ** 0.5) < 1e-4
    out = out.cpu()
    assert (out[0] == 0).all() and torch.isnan(out[1, 77]) and int(torch.isnan(out[1]).sum()) == 1 and (out[1][:77] == 0).all()
    assert torch.isnan(out[2]).all() and torch.allclose(out[3], torch.full((5000,), 5000 ** -0.5))


def test_large_rows_one_model_no_values_and_repeats():
    gen = torch.Generator(device="cuda").manual_seed(3)
    g = torch.randn(3, 30000001, generator=gen, device="cuda") * torch.tensor([[1e-4], [1.0], [1e-3]], device="cuda")
    norms, out, enorms, eout = ref.clip(g, 2.0)
    to = torch.empty_like(g)
    got = layers.clip_gradients(g, 2.0, out=to)
    near(got, norms.cpu(), enorms.cpu())
    assert ((to.double() - out).abs() <= eout + ref.rounding(out, F32)).all()
    again = torch.empty_like(g)
    assert torch.equal(layers.clip_gradients(g, 2.0, out=again), got) and torch.equal(again, to)
    one = layers.clip_gradients(g[1], 2.0, out=again[1])
    assert one.shape == () and abs(float(one) / float(norms[1]) - 1) < 1e-4
    assert torch.equal(layers.clip_gradients(torch.empty(3, 0, device="cuda"), 1.0), torch.zeros(3, device="cuda"))
    assert layers.clip_gradients(torch.empty(0, 5, device="cuda"), 1.0).shape == (0,)
    same = layers.clip_gradients(g[:1, :999].expand(4, 999), 1.0, out=torch.empty(4, 999, device="cuda"))
    assert torch.equal(same, same[:1].expand(4))


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("first,second", [(0, 1000), (1000, 0), (3, 1003)])
def test_rows_between_those_of_the_gradients(first, second, dtype):
    long = normal(rng(5), 3, 2003).to(dtype).cuda()
    grads, out = long[:, first:first + 1000], long[:, second:second + 1000]
    want = torch.empty(3, 1000, dtype=dtype, device="cuda")
    norms = layers.clip_gradients(grads.clone(), 1.0, out=want)
    before = grads.clone()
    near(layers.clip_gradients(grads, 1.0, out=out), norms.double().cpu(), norms.double().cpu() * 1000 * 2.0 ** -24, F32)
    assert torch.equal(grads, before)
    near(out, want.double().cpu(), want.double().cpu().abs() * (1000 * 2.0 ** -24 + torch.finfo(dtype).eps / 2))
    with pytest.raises(cpdp.CPDPError):
        layers.clip_gradients(grads, 1.0, out=long[:, first + 1:first + 1001])


def test_streams_and_graphs():
    g = torch.randn(2, 50000, device="cuda")
    out, other = torch.empty_like(g), torch.empty_like(g)
    want = layers.clip_gradients(g, 1.0, out=out)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = layers.clip_gradients(g, 1.0, out=other, stream=side)
    side.synchronize()
    assert torch.equal(got, want) and torch.equal(out, other)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = layers.clip_gradients(g, 1.0, out=out)
    g.mul_(0.5)
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(held, layers.clip_gradients(g, 1.0, out=other)) and torch.equal(out, other) and not torch.equal(held, want)


def test_refusals():
    g = torch.ones(3, 40, device="cuda")
    for bad in (lambda: layers.clip_gradients(g.half(), 1.0), lambda: layers.clip_gradients(g, 1.0, out=g.bfloat16())):
        with pytest.raises(TypeError):
            bad()
    for bad in (lambda: layers.clip_gradients(g[None], 1.0), lambda: layers.clip_gradients(g[:, ::2], 1.0),
                lambda: layers.clip_gradients(g, 1.0, out=g[:2]), lambda: layers.clip_gradients(g.clone().requires_grad_(), 1.0),
                lambda: layers.clip_gradients(g.cpu(), 1.0), lambda: layers.clip_gradients(torch.empty(2 ** 32 + 1, 0, device="cuda"), 1.0)):
        with pytest.raises(ValueError):
            bad()
    for bad in (lambda: layers.clip_gradients(g, 0.0), lambda: layers.clip_gradients(g, float("nan")), lambda: layers.clip_gradients(g, -1.0),
                lambda: layers.clip_gradients(g[:1].expand(3, 40), 1.0),
                lambda: layers.clip_gradients(g.as_strided((3, 30), (40, 1)), 1.0, out=g.as_strided((3, 30), (35, 1)))):
        with pytest.raises(cpdp.CPDPError):
            bad()
    assert (g == 1).all()
