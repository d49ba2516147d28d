"""Host-side tests of the C ABI of the loss, the clipping, the convolution and the
scan that need no GPU: every refusal is made before anything is launched, sizes of
workspaces are consistent, and the 64-bit references agree with differences."""
import struct

import pytest
import torch

import operators_reference as ref
from paper_2607_21224_gb300 import cpdp, layers

P = 1 << 20  # an address that no refused call reads
BIG = 1 << 40

# x, weight, ... as declared; float32, 2 workers
SCAN = dict(u=(P, 320, 32), delta=(P, 320, 32), z=(P, 320, 32), b=(P, 80, 8), c=(P, 80, 8), a_log=(P, 256), skip=(P, 32), bias=(P, 32), lengths=(0,))


def scan(**change):
    fields = {**SCAN, **change}
    return struct.pack("=22q", *(v for f in fields.values() for v in f))


GOOD = {
    "cpdp_linear_cross_entropy": [P, 320, 32, P, 1600, 32, P, 0, 2, 10, 50, 32, P, P, P, BIG, None],
    "cpdp_linear_cross_entropy_backward": [P, P, 320, 32, P, 1600, 32, P, P, 0, 2, 10, 50, 32, P, P, 1600, 0, P, BIG, None],
    "cpdp_clip_gradients": [P, 100, 0, 2, 100, 1.0, P, P, 100, P, BIG, None],
    "cpdp_causal_conv": [P, 320, 32, P, 128, P, 32, None, None, 0, 2, 4, 10, 32, 4, P, P, None],
    "cpdp_causal_conv_backward": [P, 320, 32, P, 320, 32, P, 128, P, 32, None, None, None, 0, 2, 4, 10, 32, 4, P, None, P, 128, P, 32, 0,
                                  P, BIG, None],
    "cpdp_causal_conv_step": [P, 32, P, 128, P, 32, 0, 2, 4, 32, 4, P, P, None],
    "cpdp_selective_scan": [scan(), 0, 2, 4, 10, 32, 8, None, P, P, None, P, BIG, None],
    "cpdp_selective_scan_backward": [P, 320, 32, scan(), 0, 2, 4, 10, 32, 8, P, None, P, P, P, P, P, None, P, 256, P, 32, P, 32, 0, P,
                                     BIG, None],
    "cpdp_selective_scan_step": [scan(), 0, 2, 4, 32, 8, P, P, None],
}
# entry point -> {argument: refused values}, all CPDP_EINVAL
REFUSED = {
    "cpdp_linear_cross_entropy": {0: [None], 1: [-1], 2: [-1], 3: [None], 4: [-1], 5: [-1], 6: [None], 7: [2, -1], 8: [0, 4097, -1],
                                  9: [-1, 1 << 31, 1 << 62], 10: [0, -1], 11: [0, -5], 12: [None], 13: [None], 14: [None], 15: [0, 8]},
    "cpdp_linear_cross_entropy_backward": {0: [None], 1: [None], 4: [None], 7: [None], 8: [None], 9: [5], 10: [0], 11: [-1], 12: [0], 13: [0],
                                           14: [None], 15: [None], 16: [-1, 1599], 17: [2], 18: [None], 19: [0]},
    "cpdp_clip_gradients": {0: [None], 1: [-1], 2: [2], 3: [0, 4097], 4: [-1, 1 << 40], 5: [0.0, -1.0, float("nan")], 6: [None], 7: [None],
                            8: [-1, 99], 9: [None], 10: [0]},
    "cpdp_causal_conv": {0: [None], 1: [-1], 2: [-1], 3: [None], 4: [-1], 5: [None], 6: [-1], 9: [3], 10: [0, 3, 4097], 11: [-1, 1 << 30],
                         12: [-1, 1 << 31], 13: [0], 14: [1, 5], 15: [None]},
    "cpdp_causal_conv_backward": {0: [None], 3: [None], 6: [None], 8: [None], 13: [2], 14: [0, 3], 15: [-1], 16: [-1], 17: [0], 18: [0, 5],
                                  19: [None], 21: [None], 22: [127], 23: [None], 24: [31], 25: [9], 26: [None], 27: [0]},
    "cpdp_causal_conv_step": {0: [None], 1: [-1], 2: [None], 4: [None], 6: [2], 7: [3], 8: [-1], 9: [0], 10: [5], 11: [None], 12: [None]},
    "cpdp_selective_scan": {0: [None] + [scan(**{k: (0,) + SCAN[k][1:]}) for k in ("u", "delta", "b", "c", "a_log", "skip", "bias")]
                            + [scan(**{k: (P, -1) + SCAN[k][2:]}) for k in ("u", "delta", "z", "b", "c", "a_log", "skip", "bias")]
                            + [scan(**{k: (P, 320, 1 << 28)}) for k in ("u", "delta", "z", "b", "c")],
                            1: [2], 2: [0, 3], 3: [-1], 4: [-1, 1 << 31], 5: [0, 1 << 31], 6: [0, 33], 8: [None], 9: [None]},
    "cpdp_selective_scan_backward": {0: [None], 1: [-1], 2: [1 << 28], 3: [None, scan(u=(0, 320, 32))], 4: [7], 5: [0, 3], 6: [-1], 7: [-1],
                                     8: [0], 9: [33], 10: [None], 12: [None], 13: [None], 14: [None], 15: [None], 16: [None], 18: [None],
                                     19: [255], 20: [None], 21: [31], 22: [None], 23: [31], 24: [2], 25: [None], 26: [0]},
    "cpdp_selective_scan_step": {0: [None, scan(delta=(0, 32, 0))], 1: [4], 2: [3], 3: [-1], 4: [0], 5: [33], 6: [None], 7: [None]},
}
MISALIGNED = {
    "cpdp_linear_cross_entropy": [0, 3, 6, 12, 13, 14], "cpdp_linear_cross_entropy_backward": [0, 1, 4, 7, 8, 14, 15, 18],
    "cpdp_clip_gradients": [0, 6, 7, 9], "cpdp_causal_conv": [0, 3, 5, 15, 16], "cpdp_causal_conv_backward": [0, 3, 6, 8, 19, 21, 23, 26],
    "cpdp_causal_conv_step": [0, 2, 4, 11, 12], "cpdp_selective_scan": [8, 9],
    "cpdp_selective_scan_backward": [0, 10, 12, 13, 14, 15, 16, 18, 20, 22, 25], "cpdp_selective_scan_step": [6, 7],
}


@pytest.mark.parametrize("name,i,value", [(n, i, v) for n, c in REFUSED.items() for i, vs in c.items() for v in vs])
def test_refused_arguments(name, i, value):
    arguments = list(GOOD[name])
    arguments[i] = value
    assert layers._entry(name)(*arguments) == cpdp.CPDP_EINVAL
    assert cpdp.cpdp_last_error(None)


@pytest.mark.parametrize("name,i", [(n, i) for n, c in MISALIGNED.items() for i in c])
def test_refused_alignment(name, i):
    arguments = list(GOOD[name])
    arguments[i] = P + 1
    assert layers._entry(name)(*arguments) == cpdp.CPDP_EALIGN


@pytest.mark.parametrize("field", ["u", "delta", "z", "b", "c", "a_log", "skip", "bias", "lengths"])
def test_refused_alignment_of_the_scans_inputs(field):
    arguments = list(GOOD["cpdp_selective_scan"])
    arguments[0] = scan(**{field: (P + 1,) + SCAN[field][1:]})
    assert layers._entry("cpdp_selective_scan")(*arguments) == cpdp.CPDP_EALIGN


def test_an_output_that_is_the_input_with_another_stride_is_refused():
    arguments = list(GOOD["cpdp_clip_gradients"])
    arguments[8] = 101
    assert layers._entry("cpdp_clip_gradients")(*arguments) == cpdp.CPDP_EINVAL


@pytest.mark.parametrize("out,stride", [(P + 4 * k, 100) for k in (1, 99, 100, -1, -99, -100)] + [(P + 4 * 150, 160), (P - 4 * 150, 160)])
def test_outputs_that_overlap_other_gradients_are_refused(out, stride):
    arguments = list(GOOD["cpdp_clip_gradients"])
    arguments[7:9] = out, stride
    assert layers._entry("cpdp_clip_gradients")(*arguments) == cpdp.CPDP_EINVAL
    assert "overlap" in cpdp.cpdp_last_error(None)


@pytest.mark.parametrize("at,inner", [(50, 150), (150, 150), (-50, 150), (-150, 150), (50, 199), (-100, 199)])
def test_outputs_that_cut_into_gradients_of_the_same_stride_are_refused(at, inner):
    arguments = list(GOOD["cpdp_clip_gradients"])
    arguments[1], arguments[7], arguments[8] = inner, P + 4 * at, inner
    assert layers._entry("cpdp_clip_gradients")(*arguments) == cpdp.CPDP_EINVAL
    assert "overlap" in cpdp.cpdp_last_error(None)


def test_workspace_sizes():
    L = layers.lib()
    assert L.cpdp_linear_cross_entropy_workspace(P, 320, 32, P, 1600, 32, 0, 0, 10, 50, 32) == 0
    assert L.cpdp_linear_cross_entropy_backward_workspace(P, 320, 32, P, 1600, 32, 0, 2, -1, 50, 32) == 0
    assert L.cpdp_clip_gradients_workspace(0, 5) == 0
    assert L.cpdp_causal_conv_backward_workspace(3, 4, 10, 32, 4) == 0
    assert L.cpdp_selective_scan_workspace(1, 1 << 50, 32, 8) == 0
    assert L.cpdp_selective_scan_backward_workspace(1, 10, 32, 33) == 0
    # the probabilities of a large vocabulary are held a piece at a time
    one = L.cpdp_linear_cross_entropy_backward_workspace(P, 1 << 24, 1024, P, 1 << 28, 1024, 1, 1, 1 << 14, 1 << 18, 1024)
    assert one < 3 << 30 < (1 << 14) * (1 << 18) * 2
    # a split scan's maps are small beside its inputs
    assert L.cpdp_selective_scan_workspace(1, 1 << 20, 1024, 16) < 1 << 24


def test_tensors_without_a_gpu_are_refused():
    x, w, t = torch.zeros(2, 3, 32), torch.ones(2, 5, 32), torch.zeros(2, 3, dtype=torch.int64)
    conv, bias = torch.ones(2, 32, 4), torch.ones(2, 32)
    few = torch.zeros(2, 3, 8)
    weights = dict(a_log=torch.zeros(2, 32, 8), skip=bias, bias=bias)
    for call in (lambda: layers.linear_cross_entropy(x, w, t), lambda: layers.linear_cross_entropy_backward(bias[:, :3], x, w, t, bias[:, :3]),
                 lambda: layers.clip_gradients(bias, 1.0), lambda: layers.causal_conv(x, conv, bias),
                 lambda: layers.causal_conv_backward(x, x, conv, bias), lambda: layers.causal_conv_step(bias, conv, bias, x),
                 lambda: layers.selective_scan(x, x, b=few, c=few, **weights),
                 lambda: layers.selective_scan_backward(x, x, x, b=few, c=few, carry=few, **weights),
                 lambda: layers.selective_scan_step(bias, bias, b=few[:, 0], c=few[:, 0], state=weights["a_log"], **weights)):
        with pytest.raises(ValueError, match="CUDA"):
            call()


def test_axes_beyond_the_arguments_are_refused():
    for t in (torch.zeros(1).expand(2 ** 32 + 1, 1, 1), torch.zeros(1).expand(1, 1, 2 ** 32 + 64)):
        with pytest.raises(ValueError, match="axis"):
            layers._sequence_shape(t, "x")
    x, w, t = torch.zeros(1, 1, 1), torch.zeros(1).expand(1, 2 ** 32 + 5, 1), torch.zeros(1, 1, dtype=torch.int64)
    with pytest.raises(ValueError, match="axis"):
        layers._head(x, w, t)
    with pytest.raises(ValueError, match="axis"):
        layers._per_worker(1, torch.zeros(1).expand(1, 1, 2 ** 32 + 4), "weight", 3)


def differences(f, tensors, gradients, gen, h=1e-6):
    us = [torch.randn(t.shape, generator=gen, dtype=torch.float64) for t in tensors]
    want = (f(*(t + h * u for t, u in zip(tensors, us))) - f(*(t - h * u for t, u in zip(tensors, us)))) / (2 * h)
    parts = [g * u for g, u in zip(gradients, us)]
    assert abs(sum(p.sum() for p in parts) - want) <= 1e-6 * sum(float(p.abs().sum()) for p in parts)


def test_reference_gradients_against_differences():
    gen = torch.Generator().manual_seed(3)
    f64 = lambda *s: torch.randn(s, generator=gen, dtype=torch.float64)  # noqa: E731
    targets = torch.tensor([[0, 4, -1], [2, 2, 1]])
    x, w, dloss = f64(2, 3, 7), f64(2, 5, 7), f64(2, 3)
    dx, dw, _, _ = ref.loss_backward(dloss, x, w, targets)
    differences(lambda a, b: (ref.loss(a, b, targets)["loss"] * dloss).sum(), (x, w), (dx, dw), gen)
    lengths = torch.tensor([0, 1, 7, 9], dtype=torch.int32)
    x, weight, bias, state, dy, dlast = f64(4, 9, 5), f64(2, 5, 4), f64(2, 5), f64(4, 3, 5), f64(4, 9, 5), f64(4, 3, 5)
    g = ref.conv_backward(dy, x, weight, bias, state, lengths, dlast)

    def conv(*t):
        r = ref.conv(*t, lengths)
        return (r["y"] * dy).sum() + (r["last"] * dlast).sum()

    differences(conv, (x, weight, bias, state), [g[k] for k in ("dx", "dweight", "dbias", "dstate")], gen)
    ts = (f64(4, 9, 5), f64(4, 9, 5), f64(2, 5, 3), f64(4, 9, 3), f64(4, 9, 3), f64(2, 5), f64(2, 5), f64(4, 9, 5), f64(4, 5, 3))
    dlast = f64(4, 5, 3)
    g = ref.scan_backward(dy, *ts, dlast, lengths)

    def scan_of(*t):
        r = ref.scan(*t, lengths)
        return (r["y"] * dy).sum() + (r["last"] * dlast).sum()

    differences(scan_of, ts, [g[k] for k in ("du", "ddelta", "da_log", "db", "dc", "dskip", "dbias", "dz", "dh0")], gen)
