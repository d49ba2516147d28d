"""Clipping at the ends of the float32 range: limits of infinity, and of sizes far
from the norms'."""
import pytest
import torch

import operators_reference as ref
from paper_2607_21224_gb300 import layers
from test_layers_gpu import near

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16


def bits(t):
    return t.view(torch.int32 if t.dtype is F32 else torch.int16)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("N,shift,to", [(1, 0, 0), (5001, 0, 0), (5001, 3, 3), (5001, 1, 2), (300007, 0, 1)])
def test_an_infinite_limit_leaves_every_row_as_it_is(N, shift, to, dtype):
    gen = torch.Generator().manual_seed(N)
    rows = torch.randn(6, N + 8, generator=gen).to(dtype)
    g = rows[:, shift:shift + N]
    g[1, N // 2] = float("inf")
    g[2, 0] = -float("inf")
    bits(g)[3, N - 1] = 0x7fc12345 if dtype is F32 else -0x3b  # NaN, with bits of its own
    g[4] = 1e38  # a finite row, whose norm is not
    g[5, N // 3], g[5, N - 1] = float("inf"), float("nan")
    rows = rows.cuda()
    g, before = rows[:, shift:shift + N], rows.clone()
    out = torch.full((6, N + 8), 7.0, dtype=dtype, device="cuda")
    norms = layers.clip_gradients(g, float("inf"), out=out[:, to:to + N])
    assert torch.isinf(norms[[1, 2]]).all() and torch.isnan(norms[[3, 5]]).all() and torch.isfinite(norms[0])
    assert torch.equal(bits(out[:, to:to + N]), bits(g)) and (out[:, :to] == 7).all() and (out[:, to + N:] == 7).all()
    again = layers.clip_gradients(g, float("inf"))
    assert torch.equal(bits(again), bits(norms)) and torch.equal(bits(rows), bits(before))
    assert N == 1 or torch.isinf(norms[4])


@pytest.mark.parametrize("most", [1.0, 1e-3, 1e-10, 1e-25])
@pytest.mark.parametrize("size", [1e35, 1e36, 3e36])
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("N,to", [(2001, 0), (2000, 1)])
def test_limits_that_are_tiny_beside_the_norm(size, most, N, to, dtype):
    """Ratios from 2e-37 down to 7e-64, where float32 has few bits (below 1.2e-38) or none (below 1.4e-45)."""
    g = (torch.randn(2, N, generator=torch.Generator().manual_seed(5)) * size).to(dtype)
    norms, out, enorms, eout = ref.clip(g, most)
    got = torch.full((2, N + 8), 7.0, dtype=dtype, device="cuda")
    near(layers.clip_gradients(g.cuda(), most, out=got[:, to:to + N]), norms, enorms, F32)
    near(got[:, to:to + N], out, eout + 2.0 ** -133)


@pytest.mark.parametrize("dtype,N", [(F32, 11000003), (BF16, 22000005)])
@pytest.mark.parametrize("W", [3, 5])
def test_a_last_group_of_fewer_rows(W, N, dtype):
    """Rows of 44 MB pass two at a time."""
    gen = torch.Generator(device="cuda").manual_seed(W)
    g = torch.empty(W, N, device="cuda").normal_(0.0, 1.0, generator=gen)
    g = (g * torch.tensor([0.5, 40.0, 1.0, 3.0, 7.0], device="cuda")[:W, None] / N ** 0.5).to(dtype)
    norms, out, enorms, eout = ref.clip(g, 1.0)
    for to in (torch.empty_like(g), g):
        near(layers.clip_gradients(g, 1.0, out=to), norms.cpu(), enorms.cpu(), F32)
        assert ((to.double() - out).abs() <= eout + ref.rounding(out, dtype)).all()
