"""The verification's launches against what its handle allocated: no block has a place past the end."""
import ctypes
import random

import pytest

from paper_2607_11951_gb300 import grid as G
from tests import fakes
from tests.test_operators_host import step

STAT, BEST, PER_POSITION = 16, 8, 16  # bytes of an entry of the first two allocations; of the drafted ids'


@pytest.fixture(scope="module")
def fake(tmp_path_factory):
    return fakes.link(tmp_path_factory.mktemp("fake"))


@pytest.mark.parametrize("B,K,V", [(1, 0, 1), (1, 0, 4096), (1, 8, 151_937), (7, 3, 33_000), (300, 4, 151_936), (65_535, 0, 33),
                                   (40, 64, 70_000)])
def test_every_block_has_a_place_in_the_scratch(fake, B, K, V):
    rng = random.Random(B + K + V)
    with fakes.use(fake) as rt:
        rt.reset()
        d = G.Drafts(B, K, V)
        stats, best, rows, drafted, done = rt.allocations()
        calls = [(B, K, V), (1, K, V), (B, 0, V), (1, 0, V)] + [(rng.randint(1, B), rng.randint(0, K), rng.randint(1, V)) for _ in range(60)]
        for b, k, v in calls:
            rt.reset()
            assert G.lib().grid_draft_verify(d.h, ctypes.byref(step(B=b, K=k, V=v, noise_stride=v)), None) == 0
            (_, g0, *_), *draw = rt.launches()
            assert g0[0] % (b * (k + 1)) == 0 and g0[0] * STAT <= stats and b * k * PER_POSITION <= max(drafted, 16)
            for _, g1, *_ in draw:
                assert g1[0] % b == 0 and g1[0] * BEST <= best
