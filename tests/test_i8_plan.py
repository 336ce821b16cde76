"""Which launch an 8-bit product gets: the choice is made on the host from the sizes
alone, so these tests need no GPU; they ask the debug library, which exports it."""
import ctypes as C
import os

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
TILES = {(64, 32), (64, 64), (64, 96), (128, 64), (128, 96), (128, 128), (128, 160), (128, 192), (256, 128),
         (128, 256), (256, 192), (256, 256)}
FEW, ANY = (16, 16), (0, 0)


def plan(m, n, k):
    """(tile rows, tile columns, K splits)."""
    lib = C.CDLL(os.path.join(ROOT, "paper_2608_23167_amd", "libssm_debug.so"))
    out = (C.c_int32 * 3)()
    assert lib.ssm_debug_gemm_i8_plan(m, n, k, out) == 0
    return tuple(out)


def test_gpu_sizes_reach_every_launch():
    from test_gpu_i8 import SIZES, TILE_SIZES
    seen = {plan(*s) for s in SIZES + TILE_SIZES}
    assert {s[:2] for s in seen} == TILES | {FEW, ANY}
    assert {s[2] for s in seen} == {1, 2, 3, 4, 6, 8}


def test_sizes_in_use_reach_every_tile():
    """Every tile is the choice for some step of the 8B and 7B shapes."""
    pairs = [(12288, 4096), (4096, 4096), (24576, 4096), (4096, 12288), (126464, 4096),
             (4608, 3584), (3584, 3584), (37888, 3584), (3584, 18944), (152064, 3584)]
    seen = {plan(m, n, k)[:2] for n, k in pairs for m in (1, 16, 32, 64, 120, 136, 240, 376, 648, 960, 1264, 1776, 3840)}
    assert seen == TILES | {FEW}


@pytest.mark.parametrize("m,n,k", [(17, 64, 64), (1000, 4096, 112), (5, 64, 100), (4096, 4096, 4095)])
def test_sizes_without_whole_steps(m, n, k):
    assert plan(m, n, k) == (*ANY, 1)


def test_workspace_is_that_of_the_choice():
    from paper_2608_23167_amd.api import ssm_gemm_i8_workspace_size
    for m, n, k in ((1, 4096, 4096), (120, 4096, 12288), (240, 4096, 12288), (68, 186, 2608), (30, 1008, 352)):
        s = plan(m, n, k)[2]
        assert ssm_gemm_i8_workspace_size(m, n, k) == (s * m * (-(-n // 16) * 16) * 4 if s > 1 else 0)
