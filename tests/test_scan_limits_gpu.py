"""The selective scan at the ends of its ranges: rates beyond float32, steps that stay
where they are, long segments, sequences that end inside one."""
import pytest
import torch

import operators_reference as ref
from layers_reference import U32
from paper_2607_21224_gb300 import layers
from test_layers_gpu import near
from test_scan_gpu import GRADS, inputs, on_gpu

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16
# Powers below 2^-126 count as 0, and products below it keep fewer bits: at most 2^-126 of each of the states or gradients
# that decay, which are below 2^6 here.
TINY = 2.0 ** -120


def check(tensors, z, h0, lengths, dy, dlast):
    """Both passes against the references, and again to the bit."""
    f, g = ref.scan(*tensors, z, h0, lengths), ref.scan_backward(dy, *tensors, z, h0, dlast, lengths)
    xs, (z, h0, lengths, dy, dlast) = on_gpu(tensors, "plain"), (t.cuda() for t in (z, h0, lengths, dy, dlast))
    y, last, carry = layers.selective_scan(*xs, z, h0, lengths)
    near(y, f["y"], f["ey"] + TINY)
    near(last, f["last"], f["elast"] + TINY)
    out = layers.selective_scan_backward(dy, *xs, carry, z, dlast, lengths)
    for got, name in zip(out, GRADS):
        try:
            near(got, g[name], g["e" + name] + TINY)
        except AssertionError as e:
            raise AssertionError(f"{name}: {e}") from None
    assert all(torch.equal(a, b) for a, b in zip(out, layers.selective_scan_backward(dy, *xs, carry, z, dlast, lengths)))


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("shape", [(1, 4, 17, 40, 7), (2, 4, 31, 24, 16), (1, 3, 400, 20, 30)])
def test_rates_beyond_float32(shape, dtype):
    """exp(a_log) from 1e38 to 1e60: nothing is left of a state after a step, and gradients stay finite."""
    tensors, rest = inputs(shape, dtype, True, 5)
    W, B, T, D, N = shape
    a_log = tensors[2]
    a_log[:, ::3, 0] = torch.tensor([88.0, 89.0, 100.0, 140.0]).repeat(D)[:a_log[:, ::3, 0].shape[1]]
    a_log[:, 1, :] = 95.0
    check(tensors, *rest)
    u, delta, a_log, b, c, skip, bias = on_gpu(tensors, "plain")
    state = torch.ones(B, D, N, device="cuda")
    layers.selective_scan_step(u[:, 0], delta[:, 0], a_log, b[:, 0], c[:, 0], skip, bias, state)
    one = layers.selective_scan(*(t[:, :1].contiguous() if i in (0, 1, 3, 4) else t for i, t in enumerate((u, delta, a_log, b, c, skip, bias))),
                                h0=torch.ones(B, D, N, device="cuda"))[1]
    assert torch.isfinite(state).all() and (state - one).abs().max() <= 2.0 ** -20 * one.abs().max()
    # a step of no size: the state stays, whatever the rate
    kept = torch.ones(B, D, N, device="cuda")
    layers.selective_scan_step(u[:, 0], torch.full_like(delta[:, 0], -300.0), a_log, b[:, 0], c[:, 0], skip, bias, kept)
    assert (kept == 1).all()


@pytest.mark.parametrize("T", [20, 300])
def test_steps_of_no_size_leave_the_state(T):
    tensors, (z, h0, _, dy, dlast) = inputs((1, 2, T, 24, 16), F32, False, 6)
    xs = list(on_gpu(tensors, "plain"))
    xs[1] = torch.full_like(xs[1], -300.0)
    y, last, carry = layers.selective_scan(*xs, z.cuda(), h0.cuda())
    assert torch.equal(last.cpu(), h0) and torch.equal(carry[:, -1].cpu(), h0)
    dh0 = layers.selective_scan_backward(torch.zeros_like(y), *xs, carry, z.cuda(), dlast.cuda())[8]
    assert torch.equal(dh0.cpu(), dlast)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("N", [3, 8, 16, 29])
def test_steps_move_states_as_a_pass_does(N, dtype):
    """To the bit: what single steps lose of slow states is what a pass loses."""
    T = 100
    tensors, (z, h0, _, _, _) = inputs((1, 3, T, 50, N), dtype, False, 7)
    u, delta, a_log, b, c, skip, bias = on_gpu(tensors, "plain")
    _, last, carry = layers.selective_scan(u, delta, a_log, b, c, skip, bias, h0=h0.cuda())
    state = h0.cuda()
    for t in range(T):
        if t % layers.CARRY_STEPS == 0:
            assert torch.equal(state, carry[:, t // layers.CARRY_STEPS])
        layers.selective_scan_step(u[:, t], delta[:, t], a_log, b[:, t], c[:, t], skip, bias, state)
    assert torch.equal(state, last)


def test_decays_across_long_segments():
    """600 columns of 24,000 equal steps, in segments of 8,000: a segment's decay is that of its summed step sizes. The
    half of the steps that the walk comes to last is of no size, so that the result is made of segments' decays alone."""
    B, T, D = 600, 24000, 32
    delta = torch.empty(D).uniform_(-6, 0, generator=torch.Generator().manual_seed(1))
    dt = torch.log1p(torch.exp(delta.double()))
    a_log = (2 / (dt * (T // 2))).log().float()  # exp(-2) of a state is left
    want = torch.exp(-torch.exp(a_log.double()) * dt * (T // 2))
    p = -want.log()
    # of three segments' decays: dt's own error, sums of 16 steps rounded at most 15 times, each decay's
    bound = want * (p * (24 + 4 * delta.double().abs()) * U32 + (3 * 2 + 10 * p) * 2 * U32)
    early = torch.full((1, T, D), -300.0)
    early[0, : T // 2] = delta
    zero = torch.zeros(1, 1, D, device="cuda").expand(B, T, D)
    weights = dict(a_log=a_log.cuda()[None, :, None], skip=torch.zeros(1, D, device="cuda"), bias=torch.zeros(1, D, device="cuda"))
    few, one = zero[..., :1], torch.ones(B, D, 1, device="cuda")
    last = layers.selective_scan(zero, early.cuda().expand(B, T, D), b=few, c=few, h0=one, carry=False, **weights)[1]
    assert ((last[..., 0].double().cpu() - want).abs() <= bound).all()
    carry = torch.zeros(B, T // layers.CARRY_STEPS, D, 1, device="cuda")
    dh0 = layers.selective_scan_backward(zero, zero, early.flip(1).cuda().expand(B, T, D), b=few, c=few, carry=carry, dlast=one, **weights)[8]
    assert ((dh0[..., 0].double().cpu() - want).abs() <= bound).all()


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("shape", [(1, 7, 300, 21, 16), (2, 8, 200, 34, 5), (1, 6, 333, 16, 32)])
def test_sequences_that_end_inside_a_segment(shape, dtype):
    """Few columns, so that time is split from 128 steps on, with lengths at and around every kind of border."""
    tensors, (z, h0, _, dy, dlast) = inputs(shape, dtype, False, 8)
    W, B, T, D, N = shape
    lengths = torch.tensor([T, 0, 1, 64, 65, 130, 191, T - 1])[:B].to(torch.int32)
    check(tensors, z, h0, lengths, dy, dlast)
