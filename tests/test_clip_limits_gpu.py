"""Clipping at the ends of the float32 range: limits of infinity, and of sizes far
from the norms'."""
import pytest
import torch

from paper_2607_21224_gb300 import layers

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
