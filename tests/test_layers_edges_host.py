"""Host-side tests of the layers that need no GPU: refusals of outputs that
overlap themselves and of tensors that require gradients, and how the kernels
load."""
import re
from pathlib import Path

import pytest
import torch

from paper_2607_21224_gb300 import cpdp, layers

P = 1 << 20  # an address that no refused call reads
L40 = 1 << 40


def norm_backward(W, stride, D=32):
    return "cpdp_add_rmsnorm_backward", [P, 10 * D, D, P, 10 * D, D, None, 0, 0, P, D, 0, W, 10, D, 1e-6, P, P, stride, 0, P, L40, None]


def weight_gradient(W, stride, O=32, I=32):
    return "cpdp_weight_gradient", [P, 10 * O, O, 1, P, P, W, 10, O, I, P, stride, 0, P, L40, None]


def recurrence_backward(B, T, seq, step, D=32):
    return "cpdp_gated_recurrence_backward", [P, T * D, D, P, T * D, D, P, T * D, D, 0, B, T, D, P, None, None, P, P, seq, step, None,
                                              P, L40, None]


OVERLAPPING = [norm_backward(2, 0), norm_backward(2, 31), norm_backward(4096, 1), weight_gradient(2, 0), weight_gradient(2, 1023),
               recurrence_backward(1, 10, 0, 0), recurrence_backward(1, 10, 0, 31), recurrence_backward(2, 10, 0, 32),
               recurrence_backward(2, 10, 319, 32), recurrence_backward(2, 1, 31, 0), recurrence_backward(2, 10, 32, 63),
               recurrence_backward(3, 10, 32, 95), recurrence_backward(2, 10, L40, 0), recurrence_backward(2, 1 << 20, 1 << 30, 1 << 11)]


@pytest.mark.parametrize("name,arguments", OVERLAPPING, ids=lambda v: v if isinstance(v, str) else None)
def test_overlapping_outputs_are_refused(name, arguments):
    assert getattr(layers.lib(), name)(*arguments) == cpdp.CPDP_EINVAL
    assert "overlap" in cpdp.cpdp_last_error(None)


def test_python_refuses_overlapping_outputs():
    cpu = torch.device("cpu")
    for shape, view in [((2, 8), torch.zeros(1, 8).expand(2, 8)), ((2, 8), torch.zeros(20).as_strided((2, 8), (7, 1))),
                        ((3, 4, 8), torch.zeros(1, 4, 8).expand(3, 4, 8)), ((2, 4, 8), torch.zeros(99).as_strided((2, 4, 8), (31, 8, 1)))]:
        with pytest.raises(ValueError, match="overlap"):
            layers._gradient_out(view, "out", shape, torch.float32, cpu)
    for shape, view in [((2, 8), torch.zeros(20).as_strided((2, 8), (8, 1))), ((1, 8), torch.zeros(8).as_strided((1, 8), (0, 1))),
                        ((2, 4, 8), torch.zeros(2, 40)[:, 3:35].view(2, 4, 8)), ((2, 1), torch.zeros(2, 9)[:, :1])]:
        assert layers._gradient_out(view, "out", shape, torch.float32, cpu) is view
    long = torch.zeros(4000)
    for shape, strides in [((2, 5, 8), (40, 0, 1)), ((2, 5, 8), (0, 8, 1)), ((2, 5, 8), (39, 8, 1)), ((1, 5, 8), (0, 7, 1)),
                           ((2, 5, 8), (8, 15, 1)), ((5, 1, 8), (7, 0, 1))]:
        with pytest.raises(ValueError, match="overlap"):
            layers._rows_apart(long.as_strided(shape, strides), "out")
    # sequences outside, steps outside, gaps, axes of one or none
    for shape, strides in [((2, 5, 8), (40, 8, 1)), ((2, 5, 8), (8, 16, 1)), ((2, 5, 8), (100, 11, 1)), ((1, 5, 8), (0, 8, 1)),
                           ((5, 1, 8), (8, 0, 1)), ((1, 1, 8), (0, 0, 1)), ((0, 5, 8), (0, 0, 1)), ((5, 0, 8), (0, 8, 1)), ((2, 5, 8), (32 + 8, 8, 1))]:
        layers._rows_apart(long.as_strided(shape, strides), "out")


CSRC = Path(layers.__file__).resolve().parent / "csrc"


@pytest.mark.parametrize("name", ["cpdp_layers.cuh", "cpdp_norm.cu", "cpdp_checkpoint.cu", "cpdp_weight_gradient.cu", "cpdp_recurrence.cu"])
def test_loads_stay_below_the_wait_for_the_launch_before(name):
    """Under programmatic dependent launch a block may be there while the launch before still writes what it will read. Loads
    that a compiler may move or merge (the read-only and hinted builtins, assembly that is not volatile or does not clobber
    memory) or that need not be coherent are not used."""
    text = re.sub(r"//[^\n]*", "", (CSRC / name).read_text())
    assert not re.findall(r"__ld(?:g|cs|cg|ca|lu|cv)\b", text)
    assert "__restrict__" not in text
    statements = re.findall(r"\basm\b(\s*volatile)?\s*\((.*?)\)\s*;", text, flags=re.S)
    loads = [(volatile, body) for volatile, body in statements if re.search(r"\b(?:ld|st|red|atom|cp)\.[\w.:]*(?:global|shared)", body)]
    assert all(volatile and '"memory"' in body and ".nc" not in body for volatile, body in loads), loads
    if name == "cpdp_layers.cuh":
        assert len(loads) >= 6


def test_tensors_that_require_a_gradient_are_refused():
    """Their gradient would be lost without a word. Under no_grad, as inside an autograd.Function, they are taken (and refused
    here for being on the CPU)."""
    x, w = torch.zeros(2, 3, 32), torch.ones(2, 32)
    saved = layers.Checkpoint(torch.zeros(2, 3, 32, dtype=torch.int8), torch.zeros(2, 3, 1, dtype=torch.uint8), 32)
    calls = {"add_rmsnorm": [x, w, x.clone()], "add_rmsnorm_backward": [x, x.clone(), w, x.clone()], "checkpoint": [x],
             "weight_gradient": [x, saved], "gated_recurrence": [x, x.clone(), w], "gated_recurrence_backward": [x, x.clone(), x.clone(), w, w.clone()],
             "gated_recurrence_step": [w, w.clone(), w.clone()]}
    for name, arguments in calls.items():
        for i, t in enumerate(arguments):
            if not isinstance(t, torch.Tensor):
                continue
            given = list(arguments)
            given[i] = t.clone().requires_grad_()
            with pytest.raises(ValueError, match="requires a gradient"):
                getattr(layers, name)(*given)
            with torch.no_grad(), pytest.raises(ValueError, match="CUDA"):
                getattr(layers, name)(*given)
    for name, arguments, key, out in [("add_rmsnorm_backward", [x, x, w], "dweight", w), ("weight_gradient", [x, saved], "out", torch.zeros(2, 32, 32)),
                                      ("gated_recurrence_backward", [x, x, x, w], "out", torch.zeros(2, 3, 64))]:
        with pytest.raises(ValueError, match="requires a gradient"):
            getattr(layers, name)(*arguments, **{key: out.clone().requires_grad_()})
    with pytest.raises(ValueError, match="requires a gradient"):  # one model's
        layers.add_rmsnorm(x[0], w[0].clone().requires_grad_())


def test_a_stream_of_another_device_is_refused():
    """The call would have run on the current stream of its tensors' device instead."""
    class Stream:
        device = torch.device("cuda", 1)

    with pytest.raises(ValueError, match="stream"):
        layers._there(torch.device("cuda", 0), Stream())
