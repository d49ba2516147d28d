"""A wait of the loss's kernels that runs out (in the debug build, where a copy is
left out) ends in NaN and a count, and leaves the GPU as it was."""
import json
import os
import subprocess
import sys
from pathlib import Path

import pytest

from paper_2607_21224_gb300 import build

pytestmark = pytest.mark.gpu


def test_a_copy_that_never_happens():
    library = build.build_library(checked=True)
    script = Path(__file__).resolve().parent / "checked_loss.py"
    r = subprocess.run([sys.executable, str(script)], env={**os.environ, "CPDP_LIBRARY": str(library)}, capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stderr[-2000:]
    for name, o in json.loads(r.stdout.splitlines()[-1]).items():
        assert o["before"] == 0 and o["ran_out"] > 0 and o["after"] == 0, (name, o)
        assert o["finite"] and o["all_nan"] and o["beside"] and o["same_after"], (name, o)
