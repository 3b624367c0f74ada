"""Rows of a `start` that is not in order, each of them in order by itself: more work together than the host's check
of the chunk's tokens foresees."""
import pytest

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("rows", [17, 33])  # (2.3 and 4.4 billion tiles and ends of units: past 31 bits, and past 32)
def test_overlapping_rows_past_the_plans_room_all_fail(rows):
    import torch
    from paper_2607_11951_gb300 import grid as G
    N, H, D, page, cached = 8192, 16, 64, 1024, 1 << 25
    i32 = dict(dtype=torch.int32, device="cuda")
    pool = torch.zeros((1, page, H, D), dtype=torch.bfloat16, device="cuda")
    kv = G.PagedKV(pool, pool.clone(), H)
    B = 2 * rows - 1  # [0, N), [N, 0), [0, N) ..: every other row is in order
    start = torch.tensor([0, N] * rows, **i32)
    table = torch.zeros((B, (cached + N) // page), **i32)
    q = torch.ones((N, H, D), dtype=torch.bfloat16, device="cuda")
    out, lse = torch.full_like(q, 7.0), torch.full((N, H), 7.0, device="cuda")
    status = torch.full((B,), -1, **i32)
    G.grid_kv_attend(kv, table, torch.full((B,), cached, **i32), q, out, status, lse=lse, start=start)
    assert status.tolist() == [7] * B
    assert bool((out == 0).all()) and bool((lse == -float("inf")).all())
