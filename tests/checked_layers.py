"""Runs the weight gradient in the debug build (CPDP_LIBRARY names it) with a
copy that never happens, so that waits run out, and prints one JSON line of what
came of it. tests/test_layers_edges_gpu.py runs it; not a test module itself."""
import ctypes
import json
import sys
from pathlib import Path

sys.path.insert(0, str(Path(__file__).resolve().parents[1]))

import torch  # noqa: E402

from paper_2607_21224_gb300 import layers  # noqa: E402


def main() -> None:
    lib = layers.lib()
    drop = lib.cpdp_layer_drop_step
    drop.restype, drop.argtypes = ctypes.c_int, [ctypes.c_int]
    gen = torch.Generator(device="cuda").manual_seed(1)
    out = {}
    # one tile of 10 steps; several tiles and chunks; tokens split among blocks
    for name, (W, M, I, O) in {"tile": (1, 600, 100, 72), "chunks": (80, 4200, 128, 300), "parts": (1, 4000, 64, 64)}.items():
        saved, _ = layers.checkpoint(torch.randn(W, M, I, generator=gen, device="cuda"))
        dy = torch.randn(W, M, O, generator=gen, device="cuda").to(torch.bfloat16)
        for dtype in (torch.float32, torch.bfloat16):
            want = layers.weight_gradient(dy, saved, dtype=dtype)
            before = layers.wait_timeouts()
            assert drop(2) == 0
            rows = torch.full((W, O * I + 7), 5.0, dtype=dtype, device="cuda")
            layers.weight_gradient(dy, saved, out=rows[:, 3:3 + O * I].view(W, O, I))
            ran_out = layers.wait_timeouts()
            assert drop(-1) == 0
            again = layers.weight_gradient(dy, saved, dtype=dtype)
            out[f"{name}/{str(dtype)[6:]}"] = {
                "before": before, "ran_out": ran_out, "all_nan": bool(torch.isnan(rows[:, 3:3 + O * I]).all()),
                "beside": bool((rows[:, :3] == 5).all() and (rows[:, 3 + O * I:] == 5).all()),
                "finite": bool(torch.isfinite(want).all()), "same_after": torch.equal(again, want), "after": layers.wait_timeouts()}
    print(json.dumps(out))


if __name__ == "__main__":
    main()
