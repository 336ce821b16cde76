"""How many rows one launch of a row operator takes (no GPU: the debug library says)."""
import ctypes as C
import os

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.mark.parametrize("threads,rows_per_wg", [(64, 1), (256, 4), (256, 1), (1024, 1)])
def test_a_launch_stays_below_2_to_the_32_threads(threads, rows_per_wg):
    lib = C.CDLL(os.path.join(ROOT, "paper_2608_23167_amd", "libssm_debug.so"))
    lib.ssm_debug_rows_a_launch.restype = C.c_int64
    most = lib.ssm_debug_rows_a_launch(threads, rows_per_wg)
    assert -(-most // rows_per_wg) * threads < 2 ** 32 <= -(-(most + 1) // rows_per_wg) * threads
