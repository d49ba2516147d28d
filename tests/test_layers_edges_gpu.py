"""The worker-batched layers on the GPU at the ends of their ranges: very many
tokens in one sum, activations and eps far from 1, gates far from 0, buffers
that change between calls. References are the formulas in 64 bits; a tolerance
is what the stated order of the operations may add."""
import pytest
import torch

import layers_reference as ref
from paper_2607_21224_gb300 import layers

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16


def gpu_rng(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def near(got, want, bound):
    """got against the 64-bit want: `bound` and half a spacing of got's type."""
    room = bound + ref.rounding(want, got.dtype) + bound * ref.HALF_SPACING[got.dtype]
    err = (got.double() - want).abs()
    bad = ~(err <= room)
    assert not bad.any(), f"{int(bad.sum())} of {bad.numel()} off, worst {float((err / room).nan_to_num(9e9).max()):.3g} times its bound"


CHUNK = 2048  # tokens that the tensor core sums in one go


def sum_error(tokens):
    """Relative to the sum of the products' sizes: a chunk is 128 products of 16 tokens, each of which may cut its running
    sum by 2^-22; then the chunks are added up, rounded to nearest."""
    return min(tokens, CHUNK) / 16 * 2.0 ** -22 + -(-tokens // CHUNK) * ref.U32


# 152 workers of one tile each: as many blocks as the GPU has SMs, so the tokens are not split among blocks.
UNSPLIT = 152


@pytest.mark.parametrize("grad", [F32, BF16])
@pytest.mark.parametrize("tokens", [1, CHUNK - 1, CHUNK, CHUNK + 1, 2 * CHUNK, 2 * CHUNK + 65, 3 * CHUNK, 4 * CHUNK + 1, 9000])
@pytest.mark.parametrize("sign", ["both", "one"])
def test_weight_gradient_of_one_to_many_chunks(tokens, grad, sign):
    gen = gpu_rng(tokens)
    x = torch.randn(UNSPLIT, tokens, 40, generator=gen, device="cuda")
    dy = torch.randn(UNSPLIT, tokens, 24, generator=gen, device="cuda").to(BF16)
    if sign == "one":
        x, dy = x.abs(), dy.abs()
    saved, values = layers.checkpoint(x)
    got = layers.weight_gradient(dy, saved, dtype=grad)
    want = torch.einsum("wmo,wmi->woi", dy.double(), values.double())
    size = torch.einsum("wmo,wmi->woi", dy.double().abs(), values.double().abs())
    near(got, want, sum_error(tokens) * size)
    assert torch.equal(got, layers.weight_gradient(dy, saved, dtype=grad))


def test_weight_gradient_in_bfloat16_of_a_million_tokens():
    """Products of one sign: a sum that the tensor core takes in one go comes out 1.2 % too small."""
    M = 1 << 20
    saved, _ = layers.checkpoint(torch.full((1, 1, 8), 127 / 128, device="cuda").expand(UNSPLIT, M, 8), values=False)
    dy = torch.full((1, 1, 8), 129 / 128, dtype=BF16, device="cuda").expand(UNSPLIT, M, 8)
    want = torch.full((UNSPLIT, 8, 8), M * 127 * 129 / 2.0 ** 14, dtype=torch.float64, device="cuda")
    for grad in (F32, BF16):
        near(layers.weight_gradient(dy, saved, dtype=grad), want, sum_error(M) * want)
