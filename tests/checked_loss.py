"""Runs the loss in the debug build (CPDP_LIBRARY names it) with a copy that never
happens, so that waits run out, and prints one JSON line of what came of it.
tests/test_loss_waits_gpu.py runs it; not a test module itself."""
import ctypes
import json
import sys
from pathlib import Path

sys.path.insert(0, str(Path(__file__).resolve().parents[1]))

import torch  # noqa: E402

from paper_2607_21224_gb300 import layers  # noqa: E402


def main() -> None:
    drop = layers.lib().cpdp_layer_drop_loss_step
    drop.restype, drop.argtypes = ctypes.c_int, [ctypes.c_int]
    gen = torch.Generator(device="cuda").manual_seed(1)
    out = {}
    # one tile; several tiles per block, of several chunks; float32
    for name, (W, M, D, V, dtype) in {"tile": (1, 60, 300, 200, torch.bfloat16), "tiles": (2, 3000, 2200, 9000, torch.bfloat16),
                                      "planes": (1, 200, 130, 700, torch.float32)}.items():
        x = torch.randn(W, M, D, generator=gen, device="cuda").to(dtype)
        weight = (torch.randn(W, V, D, generator=gen, device="cuda") / D ** 0.5).to(dtype)
        targets = torch.randint(0, V, (W, M), generator=gen, device="cuda")
        dloss = torch.full((W, M), 1.0 / M, device="cuda")

        def both(dweight=None):
            loss, lse = layers.linear_cross_entropy(x, weight, targets)
            return loss, lse, *layers.linear_cross_entropy_backward(dloss, x, weight, targets, lse, dweight=dweight)

        want = both()
        before = layers.wait_timeouts()
        assert drop(2) == 0
        rows = torch.full((W, V * D + 7), 5.0, device="cuda")
        got = both(rows[:, 3:3 + V * D].view(W, V, D))
        ran_out = layers.wait_timeouts()
        assert drop(-1) == 0
        again = both()
        out[name] = {"before": before, "ran_out": ran_out, "all_nan": all(bool(torch.isnan(t).all()) for t in got),
                     "beside": bool((rows[:, :3] == 5).all() and (rows[:, 3 + V * D:] == 5).all()),
                     "finite": all(bool(torch.isfinite(t).all()) for t in want),
                     "same_after": all(torch.equal(a, b) for a, b in zip(want, again)), "after": layers.wait_timeouts()}
    print(json.dumps(out))


if __name__ == "__main__":
    main()
