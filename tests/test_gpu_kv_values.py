"""grid_kv_attend where a wrong key or a lost share of the values shows in the result: every key found at its own place,
keys far below the largest, and what is not a number in a query."""
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


class Coded(Batch):
    """Keys are signs, all different; a query that repeats a key's signs three times as large finds that key alone."""

    def __init__(self, *a, **kw):
        super().__init__(*a, scale=0.0, **kw)
        sign = lambda x: (self.rand(*x.shape) > 0).to(x.dtype) * 2 - 1
        for i, (k, v) in enumerate(self.cached):
            k[:] = sign(k)
            self.put(i, 0, k, v)
        self.nk[:] = sign(self.nk)
        self.fill()

    def find(self, pick):
        """Attend with the query of token t of row b and head h at position pick(b, t, h), and compare bit for bit.  The
        position's score is 3 D; no two keys here agree in all but 6 of their signs, so that any other's is below 3 (D - 12)
        and its share below e^-36: times the number of keys that is less than fp32 keeps beside 1."""
        import torch
        group, a, want = self.H // self.Hk, 0, []
        h = torch.arange(self.H, device="cuda")
        for b, n in enumerate(self.new):
            k = torch.cat([self.cached[b][0], self.nk[a:a + n]])
            v = torch.cat([self.cached[b][1], self.nv[a:a + n]])
            if n:
                t = torch.arange(n, device="cuda")
                j = pick(b, t[:, None], h[None]).clamp(min=0)
                j = torch.minimum(j, self.old[b] + t[:, None])
                self.q[a:a + n] = 3 * k[j, h // group]
                want.append(v[j, h // group])
            a += n
        self.out.fill_(7.0)
        self.attend(scale=1.0)
        assert torch.equal(self.out[:self.N], torch.cat(want)) and not bool(self.status.any())


SHAPES = [([260], [1], 4, 2, 128, 16), ([130, 1, 400, 255], [1] * 4, 8, 1, 64, 8), ([3_000], [1], 16, 4, 128, 64),
          ([3_000], [2], 14, 2, 64, 32), ([1_500] * 3, [1] * 3, 32, 8, 128, 128), ([700, 0, 90], [40, 300, 1], 14, 2, 128, 16),
          ([300, 5], [500, 131], 4, 2, 64, 1024), ([60] * 20, [1] * 20, 16, 8, 64, 16), ([4_000, 9], [700, 3], 4, 1, 128, 32)]


@pytest.mark.parametrize("old,new,heads,kv_heads,D,page", SHAPES)
@pytest.mark.parametrize("dt,order", [("bf16", "token"), ("f16", "head")])
def test_every_key_is_found_at_its_own_place(old, new, heads, kv_heads, D, page, dt, order):
    import torch
    b = Coded(old, new, heads, kv_heads, D, page, dt, order=order, seed=len(old))
    longest = max(o + n for o, n in zip(old, new))
    spread = heads // kv_heads * min(new)  # positions that one pass finds of a row, whatever the key head
    for first in range(0, longest, spread):
        b.find(lambda r, t, h: first + t % min(new) * (heads // kv_heads) + h % (heads // kv_heads))
    b.find(lambda r, t, h: b.old[r] + t)           # the token's own key
    b.find(lambda r, t, h: b.old[r] + t - 1 - h)   # and those just before it
    b.find(lambda r, t, h: (b.old[r] + t) // 128 * 128 - h % 2)  # the ends of tiles
    g = torch.Generator(device="cuda")
    g.manual_seed(1)
    b.find(lambda r, t, h: torch.randint(0, b.old[r] + new[r], (t.shape[0], heads), generator=g, device="cuda"))


@pytest.mark.parametrize("heads,kv_heads", [(17, 1), (24, 1), (64, 2), (33, 3), (128, 1), (160, 1)])
@pytest.mark.parametrize("D,dt", [(64, "f16"), (128, "bf16")])
def test_many_query_heads_to_a_key_head(heads, kv_heads, D, dt):
    b = Batch([300, 0, 127, 2_000], [1, 9, 3, 40], heads, kv_heads, D, 16, dt, seed=heads)
    b.fill()
    b.attend()
    b.check()


@pytest.mark.parametrize("heads,kv_heads,D", [(8, 2, 64), (14, 2, 128), (16, 1, 128)])
@pytest.mark.parametrize("page,order", [(8, "head"), (16, "token"), (64, "head"), (256, "token")])
def test_ragged_f16_chunks(heads, kv_heads, D, page, order):
    new = [0, 1, 2, 5, 16, 19, 37, 65, 130, 0, 257, 3]
    old = [5, 0, 100, 0, 128, 250, 0, 0, 126, 9, 255, 2000]
    b = Batch(old, new, heads, kv_heads, D, page, "f16", order=order, seed=page)
    b.fill()
    b.attend()
    b.check()
