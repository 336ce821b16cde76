"""The device-checked build (libssm_debug.so) runs the 8-bit projections and the token
scores without a failed check, and gives the same outputs as the release library, bit
for bit (the checks change no arithmetic)."""
import os
import subprocess
import sys

import numpy as np
import pytest

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
DEBUG_LIB = os.path.join(ROOT, "paper_2608_23167_amd", "libssm_debug.so")


def test_debug_build_matches_release(gpu, tmp_path):
    assert os.path.exists(DEBUG_LIB), "libssm_debug.so is missing: run __graft_entry__.build()"
    out = tmp_path / "debug.npz"
    print(f"[debug build] child process with {DEBUG_LIB}", flush=True)
    r = subprocess.run([sys.executable, os.path.join(ROOT, "tests", "_debug_i8_child.py"), DEBUG_LIB,
                        str(out)], capture_output=True, text=True, timeout=300, cwd=ROOT)
    assert r.returncode == 0, r.stdout[-2000:] + r.stderr[-4000:]
    from _debug_i8_child import run_cases
    release = run_cases()
    debug = np.load(out)
    assert set(debug.files) == set(release)
    for key, ref in release.items():
        assert np.array_equal(debug[key], ref, equal_nan=True), key
