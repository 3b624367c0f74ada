"""grid_kv_attend where a lost share of the values shows in the result: keys far below the largest; and what is not a
number in a query."""
import math

import pytest

from tests.test_gpu_kv import TINY, UNIT, Batch

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("old,new,heads,kv_heads,D", [
    ([2_000], [1], 4, 1, 128), ([2_000], [1], 8, 2, 64), ([16_000], [1], 2, 2, 128), ([16_000], [1], 2, 2, 64),
    ([2_000, 300], [200, 150], 4, 2, 128), ([2_000, 300], [200, 150], 4, 2, 64), ([0], [2_000], 2, 1, 64), ([0], [2_000], 2, 1, 128)])
@pytest.mark.parametrize("below,sink", [(14.28125, 0.0), (17.46875, 0.0), (14.28125, 0.5), (3.0, 0.0)])
def test_f16_values_of_many_keys_far_below_one(old, new, heads, kv_heads, D, below, sink):
    """The first key outweighs every other by e^below and has (almost) no value; the others' values are 1.  A probability
    that f16 holds below its normal range is off by 2^-25 of 2^7, which the largest one is at least, so n of them by n 2^-32."""
    import torch
    b = Batch(old, new, heads, kv_heads, D, 16, "f16", scale=0.0)
    b.qkv[:] = 0
    b.qkv[:, :, 0] = 1.0  # (queries; keys of the chunk are zero)
    b.nk[:] = 0
    b.nv[:] = 1
    for i, n in enumerate(b.old):
        k, v = b.cached[i]
        k[:], v[:] = 0, 1
        if n:
            k[0, :, 0], v[0] = below, sink
            b.put(i, 0, k, v)
    a = 0
    for i, n in enumerate(b.new):
        if not b.old[i]:
            b.nk[a, :, 0], b.nv[a] = below, sink
        a += n
    b.fill()
    b.attend(scale=1.0)
    a, unit = 0, UNIT["f16"]
    for i, n in enumerate(b.new):
        others = (torch.arange(n, device="cuda") + b.old[i]).double()
        small = math.exp(-below)
        z = 1 + others * small
        share = others * small / z
        want = share + sink / z
        # rounded probabilities, scores and exponentials in fp32, the result's own rounding
        near = (unit + 2.0 ** -18) * want * 2 + others * 2.0 ** -32 + TINY
        off = (b.out[a:a + n].double() - want[:, None, None]).abs() - near[:, None, None]
        assert float(off.max()) <= 0, (i, float(off.max()), float(want.min()))
        lse = below + z.log()
        assert float(((b.lse[a:a + n].double() - lse[:, None]).abs() - 2.0 ** -18 * (1 + lse[:, None])).max()) <= 0
        assert int(b.status[i]) == 0
        a += n


@pytest.mark.parametrize("bad", [math.nan, math.inf])
@pytest.mark.parametrize("old,new,heads,kv_heads,D", [([400, 90, 5], [1, 1, 1], 8, 2, 64), ([9_000, 90, 700], [2, 5, 1], 8, 2, 128),
                                                       ([100, 3_000, 0], [40, 700, 300], 4, 1, 128), ([100, 0, 7], [400, 300, 20], 14, 2, 64)])
def test_what_is_not_a_number_in_a_query_stays_in_its_own_result(bad, old, new, heads, kv_heads, D):
    import torch
    b = Batch(old, new, heads, kv_heads, D, 16)
    b.fill()
    b.attend()
    out, lse = b.out.clone(), b.lse.clone()
    at = b.start.tolist()
    places = [(at[1], heads - 1), (at[2] - 1, 0)]  # of row 1
    for i, h in places:
        b.q[i, h, :] = bad  # (infinite: scores of both signs, or infinity less infinity)
    b.attend()
    assert b.status.tolist() == [0, 0, 0]
    for i, h in places:
        assert bool(b.out[i, h].isnan().all()) and bool(b.lse[i, h].isnan()), (i, h)
        b.out[i, h], b.lse[i, h] = out[i, h], lse[i, h]
    for r in (0, 2):  # nothing of these rows is shared with row 1
        assert torch.equal(b.out[at[r]:at[r + 1]], out[at[r]:at[r + 1]])
    assert float((b.out - out).abs().max()) <= 2.0 ** -6 * float(out.abs().max()) and float((b.lse - lse).abs().max()) < 1e-4
