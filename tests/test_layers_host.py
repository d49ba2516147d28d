"""Host-side tests of the layers' C ABI (include/cpdp_layers.h) that need no
GPU: header, binding and library agree, and every refusal is made before
anything is launched. The 64-bit references are checked against differences."""
import ctypes
import re
from pathlib import Path

import pytest
import torch

import layers_reference as ref
from paper_2607_21224_gb300 import cpdp, layers

HEADER = Path(__file__).resolve().parents[1] / "include" / "cpdp_layers.h"
P = 1 << 20  # an address that no refused call reads


def test_header_binding_and_library_agree():
    text = re.sub(r"/\*.*?\*/", "", HEADER.read_text(), flags=re.S)
    declared = dict(re.findall(r"\b(cpdp_[a-z_]+)\s*\(([^)]*)\)", text))
    assert set(declared) == set(layers.SIGNATURES)
    for name, arguments in declared.items():
        assert len(arguments.split(",")) == len(layers.SIGNATURES[name][1]), name
        assert ctypes.cast(getattr(layers.lib(), name), ctypes.c_void_p).value
    constants = dict(re.findall(r"#define (CPDP_[A-Z_]+) (\d+)", HEADER.read_text()))
    assert int(constants["CPDP_NORM_MAX_FEATURES"]) == layers.NORM_MAX_FEATURES
    assert int(constants["CPDP_CARRY_STEPS"]) == layers.CARRY_STEPS


GOOD = {
    "cpdp_add_rmsnorm": [P, 320, 32, None, 0, 0, P, 32, 0, 2, 10, 32, 1e-6, P, None, None, None, None],
    "cpdp_add_rmsnorm_backward": [P, 320, 32, P, 320, 32, None, 0, 0, P, 32, 0, 2, 10, 32, 1e-6, P, P, 32, 0, P, 1 << 40, None],
    "cpdp_checkpoint": [P, 320, 32, 0, 2, 10, 32, P, P, P, None],
    "cpdp_restore": [P, P, 2, 10, 32, P, None],
    "cpdp_weight_gradient": [P, 320, 32, 1, P, P, 2, 10, 32, 32, P, 1024, 0, P, 1 << 40, None],
    "cpdp_gated_recurrence": [P, 320, 32, P, 320, 32, 0, 2, 10, 32, None, None, P, P, None, P, 1 << 40, None],
    "cpdp_gated_recurrence_backward": [P, 320, 32, P, 320, 32, P, 320, 32, 0, 2, 10, 32, P, None, None, P, P, 640, 64, None, P,
                                       1 << 40, None],
    "cpdp_gated_recurrence_step": [P, 32, P, 32, 0, 2, 32, P, P, None],
}
# entry point -> {argument: refused values}, all CPDP_EINVAL
REFUSED = {
    "cpdp_add_rmsnorm": {0: [None], 1: [-1], 2: [-1], 6: [None], 7: [-1], 8: [2, -1], 9: [0, 4097, -1], 10: [-1, 1 << 31, 1 << 62],
                         11: [0, -5, 16385], 12: [0.0, -1.0, float("nan"), float("inf")], 13: [None], 14: [P], 15: [P], 16: [P]},
    "cpdp_add_rmsnorm_backward": {0: [None], 3: [None], 9: [None], 11: [7], 12: [0], 13: [-1], 14: [0, 16385], 15: [0.0], 16: [None],
                                  17: [None], 18: [-1], 19: [9], 20: [None], 21: [0, 8]},
    "cpdp_checkpoint": {0: [None], 3: [5], 4: [0], 5: [-1], 6: [0, (1 << 30) + 1], 7: [None], 8: [None]},
    "cpdp_restore": {0: [None], 1: [None], 2: [4097], 4: [-1], 5: [None]},
    "cpdp_weight_gradient": {0: [None], 1: [-1], 3: [3], 4: [None], 5: [None], 6: [0], 7: [-1], 8: [0], 9: [0], 10: [None], 11: [-1],
                             12: [4]},
    "cpdp_gated_recurrence": {0: [None], 3: [None], 6: [2], 7: [-1, 1 << 30], 8: [-1, 1 << 40], 9: [0], 12: [None], 13: [None]},
    "cpdp_gated_recurrence_backward": {0: [None], 3: [None], 6: [None], 9: [2], 10: [-1], 11: [-1], 12: [0], 13: [None], 16: [None],
                                       17: [None], 18: [-1], 19: [-1]},
    "cpdp_gated_recurrence_step": {0: [None], 1: [-1], 2: [None], 4: [2], 5: [-1], 6: [0], 7: [None], 8: [None]},
}
# arguments refused as misaligned: one byte off for 4-byte elements
MISALIGNED = {
    "cpdp_add_rmsnorm": [0, 6, 13], "cpdp_add_rmsnorm_backward": [0, 3, 9, 16, 17, 20], "cpdp_checkpoint": [0, 9], "cpdp_restore": [5],
    "cpdp_weight_gradient": [0, 10], "cpdp_gated_recurrence": [0, 3, 12, 13], "cpdp_gated_recurrence_backward": [0, 3, 6, 13, 16, 17],
    "cpdp_gated_recurrence_step": [0, 2, 7, 8],
}


@pytest.mark.parametrize("name,i,value", [(n, i, v) for n, c in REFUSED.items() for i, vs in c.items() for v in vs])
def test_refused_arguments(name, i, value):
    arguments = list(GOOD[name])
    arguments[i] = value
    assert getattr(layers.lib(), name)(*arguments) == cpdp.CPDP_EINVAL
    assert cpdp.cpdp_last_error(None)


@pytest.mark.parametrize("name,i", [(n, i) for n, c in MISALIGNED.items() for i in c])
def test_refused_alignment(name, i):
    arguments = list(GOOD[name])
    arguments[i] = P + 1
    assert getattr(layers.lib(), name)(*arguments) == cpdp.CPDP_EALIGN


def test_workspace_sizes_of_refused_sizes_are_zero():
    L = layers.lib()
    assert L.cpdp_add_rmsnorm_backward_workspace(0, 5, 32) == 0
    assert L.cpdp_weight_gradient_workspace(P, 320, 32, 1, 1, -1, 32, 32) == 0
    assert L.cpdp_gated_recurrence_workspace(1, 1 << 50, 32) == 0


def test_tensors_without_a_gpu_are_refused():
    x, w = torch.zeros(2, 3, 32), torch.ones(2, 32)
    for call in (lambda: layers.add_rmsnorm(x, w), lambda: layers.add_rmsnorm_backward(x, x, w), lambda: layers.checkpoint(x),
                 lambda: layers.gated_recurrence(x, x), lambda: layers.gated_recurrence_step(w, w, w)):
        with pytest.raises(ValueError, match="CUDA"):
            call()


def test_reference_gradients_against_differences():
    gen = torch.Generator().manual_seed(3)
    f64 = lambda *s: torch.randn(s, generator=gen, dtype=torch.float64)  # noqa: E731
    h = 1e-6
    x, w, dy, ds = f64(2, 3, 40), 1 + 0.2 * f64(2, 40), f64(2, 3, 40), f64(2, 3, 40)
    dx, dw, _, _ = ref.norm_backward(dy, x, w, ds, 1e-6)
    f = lambda a, b: (b[:, None] * a / torch.sqrt(a.square().mean(-1, keepdim=True) + 1e-6) * dy + ds * a).sum()  # noqa: E731
    u, v = f64(2, 3, 40), f64(2, 40)
    want = (f(x + h * u, w + h * v) - f(x - h * u, w - h * v)) / (2 * h)
    assert abs((dx * u).sum() + (dw * v).sum() - want) <= 1e-7 * float((dx * u).abs().sum())
    lengths = torch.tensor([0, 1, 7, 9], dtype=torch.int32)
    gate, value, dh, h0, last = f64(4, 9, 5), f64(4, 9, 5), f64(4, 9, 5), f64(4, 5), f64(4, 5)

    def g(a, b, c):
        r = ref.recurrence(a, b, c, lengths)
        return (r["h"] * dh).sum() + (r["last"] * last).sum()

    r = ref.recurrence_backward(dh, gate, value, h0, last, lengths)
    us = f64(4, 9, 5), f64(4, 9, 5), f64(4, 5)
    want = (g(*(a + h * u for a, u in zip((gate, value, h0), us))) - g(*(a - h * u for a, u in zip((gate, value, h0), us)))) / (2 * h)
    got = sum((r[k] * u).sum() for k, u in zip(("dgate", "dvalue", "dh0"), us))
    assert abs(got - want) <= 1e-7 * sum(float((r[k] * u).abs().sum()) for k, u in zip(("dgate", "dvalue", "dh0"), us))


def test_axes_beyond_the_arguments_are_refused():
    """Sizes that would be cut to 32 bits on their way into the library."""
    with pytest.raises(ValueError, match="axis"):
        layers._three(torch.zeros(1).expand(1, 1, 2 ** 32 + 64), "x")
    with pytest.raises(ValueError, match="axis"):
        layers._sequences(torch.zeros(1).expand(2 ** 32 + 1, 1, 1))


def test_held_values_are_within_half_a_unit():
    x = torch.randn(4, 70, dtype=torch.float64) * 100
    values, e = ref.held(x)
    unit = torch.ldexp(torch.ones_like(e, dtype=torch.float64), e).repeat_interleave(32, -1)[..., :70]
    assert ((values - x).abs() <= unit / 2).all() and (values / unit).abs().max() <= 127
    assert (x.abs().max() > 63 * unit.min())
