"""The worker-batched layers on the GPU at the ends of their ranges: very many
tokens in one sum, activations and eps far from 1, gates far from 0, buffers
that change between calls. References are the formulas in 64 bits; a tolerance
is what the stated order of the operations may add."""
import json
import os
import subprocess
import sys
from pathlib import Path

import pytest
import torch

import layers_reference as ref
from paper_2607_21224_gb300 import build, layers

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16


@pytest.fixture(autouse=True)
def no_wait_runs_out():
    yield
    assert layers.wait_timeouts() == 0


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


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("eps", [1e-6, 1e-30])
@pytest.mark.parametrize("size", [1e-15, 1e-8, 1.0, 1e12, 1e14, 1e15, 1e16, 1e17])
@pytest.mark.parametrize("shape", [(2, 5, 64), (1, 3, 771), (1, 2, 4096), (1, 2, 16384)])
def test_norm_backward_of_small_and_large_rows(shape, size, eps, dtype):
    """dy has a part along s, which the projection takes away: the term that rows of 1e13 and more used to lose."""
    gen = gpu_rng(shape[2])
    s = (torch.randn(shape, generator=gen, device="cuda") * size).to(dtype)
    dy = (torch.randn(shape, generator=gen, device="cuda") + s.float() / size).to(dtype)
    ds = (torch.randn(shape, generator=gen, device="cuda") * 0.1 / size).to(dtype)
    w = 1 + 0.3 * torch.randn(shape[0], shape[2], generator=gen, device="cuda")
    for through in (None, ds):
        want, dweight, bound, bound_w = (t.cuda() for t in ref.norm_backward(dy.cpu(), s.cpu(), w.cpu(), None if through is None else ds.cpu(), eps))
        dx, dw = layers.add_rmsnorm_backward(dy, s, w, through, eps=eps)
        near(dx, want, bound)
        near(dw, dweight, bound_w)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("eps", [1e-6, 1e-26, 1e-30, 1e-37])
@pytest.mark.parametrize("D", [64, 771, 4096, 16384])
def test_norm_backward_of_rows_of_zeros(D, eps, dtype):
    """k = 1 / sqrt(eps) there: dx is ds + k dy weight, with nothing to take away."""
    gen = gpu_rng(D)
    s = torch.zeros(1, 3, D, dtype=dtype, device="cuda")
    dy, ds = (torch.randn(1, 3, D, generator=gen, device="cuda").to(dtype) for _ in range(2))
    w = torch.rand(1, D, generator=gen, device="cuda")
    dx, dw = layers.add_rmsnorm_backward(dy, s, w, ds, eps=eps)
    k = torch.tensor(eps, dtype=F32).double().item() ** -0.5
    want = ds.double() + k * dy.double() * w.double()
    near(dx, want, 16 * ref.U32 * (ds.double().abs() + k * (dy.double() * w.double()).abs()))
    assert (dw == 0).all()


def test_outputs_that_overlap_themselves_are_refused():
    x, w = torch.ones(2, 3, 32, device="cuda"), torch.ones(2, 32, device="cuda")
    saved, _ = layers.checkpoint(x)
    carry = layers.gated_recurrence(x, x)[2]
    long = torch.full((500,), 7.0, device="cuda")
    for call in (lambda: layers.add_rmsnorm_backward(x, x, w, dweight=long[:32].expand(2, 32)),
                 lambda: layers.add_rmsnorm_backward(x, x, w, dweight=long.as_strided((2, 32), (31, 1))),
                 lambda: layers.weight_gradient(x, saved, out=torch.zeros(1, 32, 32, device="cuda").expand(2, 32, 32)),
                 lambda: layers.gated_recurrence_backward(x, x, x, carry, out=long[:64].expand(2, 3, 64)),
                 lambda: layers.gated_recurrence_backward(x, x, x, carry, out=long.as_strided((2, 3, 64), (64 * 3, 63, 1)))):
        with pytest.raises(ValueError, match="overlap"):
            call()
    assert (long == 7).all()


@pytest.mark.parametrize("D", [32, 33])
def test_recurrence_gradients_into_arrays_with_the_steps_outside(D):
    gen = gpu_rng(D)
    gate, value, dh = (torch.randn(3, 70, D, generator=gen, device="cuda") for _ in range(3))
    carry = layers.gated_recurrence(gate, value)[2]
    want = layers.gated_recurrence_backward(dh, gate, value, carry)
    out = torch.full((70, 3, 2 * D), float("nan"), device="cuda").transpose(0, 1)
    got = layers.gated_recurrence_backward(dh, gate, value, carry, out=out)
    assert all(torch.equal(p, q) for p, q in zip(got, want)) and torch.equal(out, torch.cat(want[:2], 2))


def test_weight_gradient_is_nan_where_a_wait_ran_out():
    """In the debug build, where a copy can be left out: its slot never fills, every role's wait ends by its limit, and what
    the blocks write is NaN, through the sum of split tokens too. The next call is whole again."""
    program = Path(__file__).resolve().parent / "checked_layers.py"
    env = dict(os.environ, CPDP_LIBRARY=str(build.build_library(checked=True)))
    proc = subprocess.run([sys.executable, str(program)], env=env, capture_output=True, text=True, timeout=300)
    assert proc.returncode == 0, proc.stderr[-3000:]
    for name, r in json.loads(proc.stdout.strip().splitlines()[-1]).items():
        assert r["before"] == 0 and r["finite"], name
        assert r["ran_out"] > 0 and r["all_nan"] and r["beside"], name
        assert r["same_after"] and r["after"] == 0, name


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("D", [384, 771])
def test_what_one_launch_writes_the_next_one_reads(D, dtype):
    """Chains of calls over the same few buffers, whose contents change from turn to turn, with nothing waited for: each call
    reads what the launch just before it wrote. The same chains with a wait after every call give the same bits."""
    W, M = 4, 700
    gen = gpu_rng(D)
    turns = [[torch.randn(W, M, D, generator=gen, device="cuda").to(dtype) for _ in range(2)] for _ in range(3)]
    first = 1 + 0.1 * torch.randn(W, D, generator=gen, device="cuda")

    def chain(wait):
        def done(x):
            if wait:
                torch.cuda.synchronize()
            return x

        results = []
        w = torch.empty_like(first)
        w.copy_(first)
        for i in range(24):
            x, dy = turns[i % 3]
            # the weight is what the backward pass of the turn before wrote, the last thing on the stream
            y, s, saved = done(layers.add_rmsnorm(x, w, dy, checkpoint=True))
            values = done(layers.restore(saved))
            dW = done(layers.weight_gradient(dy, saved))
            held, _ = done(layers.checkpoint(s))
            dW2 = done(layers.weight_gradient(dy, held, dtype=BF16))
            h, last, carry = done(layers.gated_recurrence(s, x, w))
            dg, dv, dh0 = done(layers.gated_recurrence_backward(h, s, x, carry, last))
            state = last.clone()
            one = done(layers.gated_recurrence_step(dg[:, 0], dv[:, 0], state))
            dx, _ = done(layers.add_rmsnorm_backward(dv, dg, w, dx_before(results), dweight=w))
            results.append([y, values, dW, dW2, h, dg, one, dx, w.clone()])
            w.mul_(1e-2).add_(1.0) if i % 2 else done(layers.add_rmsnorm_backward(dx, dx, first, dweight=w))
        torch.cuda.synchronize()
        return results

    def dx_before(results):
        return results[-1][7] if results else None

    got, want = chain(False), chain(True)
    for i, (a, b) in enumerate(zip(got, want)):
        assert all(torch.equal(p.nan_to_num(7.0), q.nan_to_num(7.0)) for p, q in zip(a, b)), i


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_gates_far_from_zero_keep_their_precision(dtype):
    """a and 1 - a at every gate: one step from a state of 0 and of 1, and its gradients. float32 gates have 16 roundings to
    spare, as in ref.STEP; with bfloat16 gates the power's exponent is a product that is rounded once, with a constant that is:
    2 U32 |x| more."""
    gate = torch.cat([torch.linspace(-86, 86, 4097), torch.tensor([0.0, 16.0, -16.0, 1e-30, -1e-30])]).to(dtype).cuda()[None, None]
    D = gate.shape[2]
    one, zero = torch.ones(1, 1, D, dtype=dtype, device="cuda"), torch.zeros(1, 1, D, dtype=dtype, device="cuda")
    state = torch.ones(1, D, device="cuda")
    x = gate[0].double()
    a, rest = 1 / (1 + torch.exp(-x)), 1 / (1 + torch.exp(x))
    room = ref.STEP + (0 if dtype == F32 else 2 * ref.U32 * x.abs())
    for value, start, want in ((one, None, rest), (zero, state, a)):
        h, last, carry = layers.gated_recurrence(gate, value, start)
        near(last, want, room * want)
        near(h[0], want, room * want)
        step = torch.zeros(1, D, device="cuda") if start is None else start.clone()
        near(layers.gated_recurrence_step(gate[0], value[0], step), want, room * want)
        near(step, want, room * want)
    dgate, dvalue, dh0 = layers.gated_recurrence_backward(one, gate, zero, carry)
    near(dvalue[0], rest, room * rest)
    near(dh0, a, room * a)
    near(dgate[0], a * rest, 2 * room * a * rest)


def test_gates_that_hold_a_state_for_long():
    """Gates of 14 to 18 over 20,000 steps: what leaks in is 1 - a, 1e-7 a step, and its error stays that of the roundings."""
    gen = gpu_rng(3)
    T, D = 20000, 64
    gate = 14 + 4 * torch.rand(1, T, D, generator=gen, device="cuda")
    value = torch.ones(1, T, D, device="cuda")
    h, last, _ = layers.gated_recurrence(gate, value)
    rest = 1 / (1 + torch.exp(gate.double()))
    want = torch.zeros(D, dtype=torch.float64, device="cuda")
    for t in range(T):
        want = want + rest[0, t] * (1 - want)
    # each step adds 1e-7 with 16 roundings of its own and rounds the state, whose own error is at most U32 of it a step
    near(last[0], want, (ref.STEP + T * ref.U32 / 2) * want)


def test_calls_inside_an_autograd_function():
    """Gradients are not recorded inside one, so tensors that require them are taken, and the gradients arrive."""
    class Norm(torch.autograd.Function):
        @staticmethod
        def forward(ctx, x, w):
            ctx.save_for_backward(x, w)
            return layers.add_rmsnorm(x, w)[0]

        @staticmethod
        def backward(ctx, dy):
            x, w = ctx.saved_tensors
            return layers.add_rmsnorm_backward(dy.contiguous(), x, w)

    gen = gpu_rng(1)
    x, dy = (torch.randn(2, 9, 96, generator=gen, device="cuda") for _ in range(2))
    w = torch.rand(2, 96, generator=gen, device="cuda")
    want = layers.add_rmsnorm_backward(dy, x, w)
    x.requires_grad_(), w.requires_grad_()
    Norm.apply(x, w).backward(dy)
    assert torch.equal(x.grad, want[0]) and torch.equal(w.grad, want[1])
    with pytest.raises(ValueError, match="requires a gradient"):
        layers.add_rmsnorm(x, w)


class Guarded:
    """Device memory for an output, `shift` bytes past an allocation's start, with 4 KB around it that must not change."""

    def __init__(self, nbytes, shift=0):
        self.first, self.nbytes = 4096 + shift, nbytes
        self.all = torch.full((2 * 4096 + shift + nbytes,), 0xA5, dtype=torch.uint8, device="cuda")
        self.ptr = self.all.data_ptr() + self.first

    def whole(self):
        return bool((self.all[:self.first] == 0xA5).all() and (self.all[self.first + self.nbytes:] == 0xA5).all())


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("shift", [0, 4])
@pytest.mark.parametrize("W,M,D", [(1, 1, 1), (3, 5, 33), (2, 7, 64), (1, 3, 129), (2, 33, 384), (1, 17, 771), (3, 2, 1024), (1, 5, 2056), (2, 3, 4099),
                                   (1, 2, 8200), (1, 1, 16384)])
def test_nothing_beside_an_output_is_written(W, M, D, shift, dtype):
    """Every output of every call, from C, at sizes that fill their last tile and at others, aligned and not."""
    lib, gen = layers.lib(), gpu_rng(D)
    e, code, n = (4, 0, W * M * D) if dtype == F32 else (2, 1, W * M * D)
    blocks = -(-D // 32)
    x, r, dy = (torch.randn(n, generator=gen, device="cuda").to(dtype) for _ in range(3))
    w = torch.rand(W, D, generator=gen, device="cuda")
    s3 = [M * D, D]
    stream = torch.cuda.current_stream().cuda_stream
    made = []

    def out(nbytes, at=shift):
        made.append(Guarded(nbytes, at))
        return made[-1].ptr

    def work(nbytes):
        return out(nbytes, 0) if nbytes else None

    y, s = out(n * e), out(n * e)
    assert lib.cpdp_add_rmsnorm(x.data_ptr(), *s3, r.data_ptr(), *s3, w.data_ptr(), D, code, W, M, D, 1e-6, y, s, None, None, stream) == 0
    codes, exponents = out(W * M * blocks * 32, 0), out(W * M * blocks)
    assert lib.cpdp_add_rmsnorm(x.data_ptr(), *s3, None, 0, 0, w.data_ptr(), D, code, W, M, D, 1e-6, out(n * 2), None, codes, exponents, stream) == 0
    assert lib.cpdp_restore(codes, exponents, W, M, D, out(n * 2), stream) == 0
    size = lib.cpdp_add_rmsnorm_backward_workspace(W, M, D)
    assert lib.cpdp_add_rmsnorm_backward(dy.data_ptr(), *s3, x.data_ptr(), *s3, r.data_ptr(), *s3, w.data_ptr(), D, code, W, M, D, 1e-6, out(n * e),
                                         out(W * D * e), D, code, work(size), size, stream) == 0
    codes, exponents = out(W * M * blocks * 32, 0), out(W * M * blocks)
    assert lib.cpdp_checkpoint(x.data_ptr(), *s3, code, W, M, D, codes, exponents, out(n * 2), stream) == 0
    O = 300 if D < 100 else 7
    g = torch.randn(W * M * O, generator=gen, device="cuda").to(dtype)
    size = lib.cpdp_weight_gradient_workspace(g.data_ptr(), M * O, O, code, W, M, O, D)
    assert lib.cpdp_weight_gradient(g.data_ptr(), M * O, O, code, codes, exponents, W, M, O, D, out(W * O * D * e), O * D, code, work(size), size, stream) == 0
    # W sequences of M steps
    carry, size = out(W * -(-M // 16) * D * 4), lib.cpdp_gated_recurrence_workspace(W, M, D)
    assert lib.cpdp_gated_recurrence(x.data_ptr(), *s3, r.data_ptr(), *s3, code, W, M, D, None, None, out(n * e), out(W * D * 4), carry, work(size), size,
                                     stream) == 0
    assert lib.cpdp_gated_recurrence_backward(dy.data_ptr(), *s3, x.data_ptr(), *s3, r.data_ptr(), *s3, code, W, M, D, carry, None, None, out(n * e),
                                              out(n * e), *s3, out(W * D * 4), work(size), size, stream) == 0
    state = Guarded(W * D * 4, shift)
    state.all[state.first:state.first + state.nbytes] = 0
    made.append(state)
    assert lib.cpdp_gated_recurrence_step(x.data_ptr(), M * D, r.data_ptr(), M * D, code, W, D, state.ptr, out(W * D * e), stream) == 0
    torch.cuda.synchronize()
    assert [i for i, m in enumerate(made) if not m.whole()] == []


@pytest.mark.parametrize("D", [8, 64, 200, 1000, 3000])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_split_recurrences_repeat_themselves(D, dtype):
    """Ragged sequences whose steps are split into none, a few and many segments: the same bits each time."""
    gen = gpu_rng(D)
    B, T = 3, 5000
    gate, value, dh = (torch.randn(B, T, D, generator=gen, device="cuda").to(dtype) for _ in range(3))
    h0 = torch.randn(B, D, generator=gen, device="cuda")
    lengths = torch.tensor([T, 1234, 0], dtype=torch.int32, device="cuda")
    first = None
    for _ in range(4):
        h, last, carry = layers.gated_recurrence(gate, value, h0, lengths)
        got = (h, last, *layers.gated_recurrence_backward(dh, gate, value, carry, h0, lengths))
        first = first or got
        assert all(torch.equal(p, q) for p, q in zip(got, first))


@pytest.mark.parametrize("T", [50, 5000])
def test_recurrence_with_infinities(T):
    """What is not finite by the formulas is not finite, nothing else is touched: an infinite state, value and gradient in
    channels of their own."""
    gen = gpu_rng(T)
    B, D = 2, 40
    gate, value, dh = (torch.randn(B, T, D, generator=gen, device="cuda") for _ in range(3))
    h0 = torch.randn(B, D, generator=gen, device="cuda")
    h0[0, 3] = float("inf")
    value[0, T // 3, 7], value[1, T // 2, 8] = float("-inf"), float("nan")
    dh[0, T // 2, 11], gate[1, T // 4, 12] = float("inf"), float("nan")
    h, last, carry = layers.gated_recurrence(gate, value, h0)
    bad = torch.zeros(B, T, D, dtype=torch.bool, device="cuda")
    bad[0, :, 3] = True
    bad[0, T // 3:, 7], bad[1, T // 2:, 8], bad[1, T // 4:, 12] = True, True, True
    assert torch.equal(~torch.isfinite(h), bad) and torch.equal(~torch.isfinite(last), bad[:, -1])
    dgate, dvalue, dh0 = layers.gated_recurrence_backward(dh, gate, value, carry)
    back = torch.zeros_like(bad)
    back[0, :T // 2 + 1, 11], back[1, :T // 4 + 1, 12] = True, True
    assert torch.equal(~torch.isfinite(dvalue), back)
    before = torch.cat([~torch.isfinite(h0)[:, None], bad[:, :-1]], 1)
    assert torch.equal(~torch.isfinite(dgate), back | before | ~torch.isfinite(value))
    assert torch.equal(~torch.isfinite(dh0), back[:, 0])
