"""grid_pages_update whose new lengths take the place of what was asked for."""
import pytest

from tests.test_gpu_pages import State

pytestmark = pytest.mark.gpu

NAMES = ("table", "held", "copies", "refs", "status")


@pytest.mark.parametrize("A,B,page,longest", [(4, 6, 16, 100), (200, 256, 16, 700), (3, 2000, 8, 40), (1100, 1030, 32, 90), (200, 256, 16, 12_000)])
@pytest.mark.parametrize("spare,bad", [(1.0, 0.0), (0.4, 0.0), (0.7, 0.3)])
@pytest.mark.parametrize("place", ["want", "keep"])
def test_lengths_in_place(A, B, page, longest, spare, bad, place):
    """By one block and by a cluster of them."""
    for seed in range(2):
        s = State(A, B, page, longest, seed, spare, bad, width_out=30 if seed else None)
        want = s.expect()
        s.out["held_out"] = s.t["want"] if place == "want" else s.more["keep"]
        for name, got, w in zip(NAMES, [x.tolist() for x in s.run()], want):
            assert got == w, name
