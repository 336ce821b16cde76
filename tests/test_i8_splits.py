"""Every tile and number of K splits of an 8-bit product that is chosen in use is a
case of tests/test_gpu_i8_splits.py or tests/test_gpu_i8.py (no GPU: the choice is
made on the host)."""
import random

from test_gpu_i8 import SIZES, TILE_SIZES
from test_gpu_i8_splits import MODEL_SIZES, SPLIT_SIZES
from test_i8_plan import plan


def test_gpu_sizes_reach_every_pair_in_use():
    tested = {plan(*s) for s in SIZES + TILE_SIZES + SPLIT_SIZES + MODEL_SIZES}
    pairs = [(12288, 4096), (4096, 4096), (24576, 4096), (4096, 12288), (126464, 4096),
             (4608, 3584), (3584, 3584), (37888, 3584), (3584, 18944), (152064, 3584)]
    used = {plan(m, n, k): (m, n, k) for n, k in pairs for m in range(1, 4337, 3)}
    assert not {p: s for p, s in used.items() if p not in tested}


def test_gpu_sizes_reach_the_pairs_of_any_sizes():
    """Sizes over the whole range: what they get is tested."""
    tested = {plan(*s) for s in SIZES + TILE_SIZES + SPLIT_SIZES + MODEL_SIZES}
    rng = random.Random(2)

    def draw(lo, hi):
        return int(round(lo * (hi / lo) ** rng.random()))
    missing = {}
    for _ in range(60000):
        s = draw(1, 20000), draw(1, 160000), 16 * draw(1, 8191)
        if plan(*s) not in tested:
            missing[plan(*s)] = s
    assert not missing


def test_split_tiles_of_alternating_waves_have_ragged_sizes():
    """The tiles of 256 columns and of 256 x 192, in splits, with rows and columns that end
    inside a tile and K that ends inside a K-step."""
    ragged = {plan(m, n, k) for m, n, k in SPLIT_SIZES if k % 128}
    for tile in ((256, 192), (256, 256)):
        assert {(*tile, s) for s in (3, 4)} <= ragged
        assert any(plan(m, n, k)[:2] == tile and plan(m, n, k)[2] > 1 and m % tile[0] and n % tile[1] and k % 128
                   for m, n, k in SPLIT_SIZES)
