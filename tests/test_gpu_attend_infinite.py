"""Queries that are infinite: a score of -inf is no key that is hidden.  Every key
of these caches is above zero where the query is -inf, so that all of a row's
scores are -inf and its sum of weights is zero; the result is NaN, for a chunk and
for a tree, whole units and joined ones, beside tokens that see nothing (zeros).
And attention repeats itself bit for bit."""
import math

import pytest

from tests.test_gpu_kv import Batch
from tests.test_gpu_tree import Trees

pytestmark = pytest.mark.gpu


def positive(b, at):
    """Keys of more than zero at one place of the head."""
    b.nk[:, :, at] = 0.5 + b.nk[:, :, at].abs()
    for i, (k, v) in enumerate(b.cached):
        k[:, :, at] = 0.5 + k[:, :, at].abs()
        b.put(i, 0, k, v)
    b.fill()


CASES = [
    ([0, 1, 130, 400], [1, 1, 1, 1], 8, 2, 64),           # single tokens, one tile and more
    ([0, 77, 300], [70, 140, 9], 4, 2, 128),              # units of up to 128 rows and of 256
    ([0, 500], [300, 260], 2, 2, 64),                     # several units, tiles one after the other
    ([9000], [3], 8, 1, 128), ([5000], [700], 4, 1, 64),  # pieces that are joined
]


@pytest.mark.parametrize("old,new,heads,kv_heads,D", CASES)
@pytest.mark.parametrize("dt", ["bf16", "f16"])
@pytest.mark.parametrize("kind", ["chunk", "chain", "tree"])
def test_scores_that_are_all_minus_infinity(old, new, heads, kv_heads, D, dt, kind):
    import torch
    b = Batch(old, new, heads, kv_heads, D, 16, dt) if kind == "chunk" else Trees(old, new, heads, kv_heads, D, 16, dt, kind=kind)
    positive(b, 5)
    b.attend()
    want = b.out.clone()
    assert not bool(b.out.isnan().any())
    bad = [(i, i % heads) for i in range(0, b.N, 7)] + [(b.N - 1, heads - 1)]
    for i, h in bad:
        b.q[i, h, 5] = -math.inf
    b.attend()
    assert (b.status == 0).all()
    for i, h in bad:
        assert bool(b.out[i, h].isnan().all()), (i, h)
        b.out[i, h] = want[i, h]
    assert torch.equal(b.out, want)


@pytest.mark.parametrize("dt", ["bf16", "f16"])
@pytest.mark.parametrize("old,new", [([0, 0, 5], [40, 300, 33]), ([0], [1024])])
def test_tokens_that_see_nothing_beside_them(dt, old, new):
    """A token without a key gets zeros whatever its query is; one with keys and an infinite query NaN."""
    import torch
    b = Trees(old, new, 4, 2, 64, 16, dt, words=32)
    g = torch.Generator(device="cuda")
    g.manual_seed(1)
    bits = [torch.rand((n, n), generator=g, device="cuda") < 0.1 for n in new]
    for m in bits:
        m[::3] = False
        m[::3] |= ~torch.ones_like(m).tril()[::3]  # (bits of later tokens do not count)
        m[1::3, 0] = True
    b.see_bits(bits)
    positive(b, 5)
    b.q[:, :, 5] = -math.inf
    b.attend()
    a = 0
    for o, n, m in zip(old, new, b.seen):
        none = ~m.any(1) if o == 0 else torch.zeros(n, dtype=torch.bool, device="cuda")
        assert bool((b.out[a:a + n][none] == 0).all()) and bool((b.lse[a:a + n][none] == -math.inf).all())
        assert bool(b.out[a:a + n][~none].isnan().all())
        assert o or (0 < int(none.sum()) < n)
        a += n


@pytest.mark.parametrize("old,new,heads,kv_heads,D", CASES)
@pytest.mark.parametrize("kind", ["chunk", "tree"])
def test_repeats(old, new, heads, kv_heads, D, kind):
    import torch
    b = Batch(old, new, heads, kv_heads, D, 16) if kind == "chunk" else Trees(old, new, heads, kv_heads, D, 16)
    b.fill()
    b.attend()
    out, lse = b.out.clone(), b.lse.clone()
    for _ in range(4):
        b.out.fill_(3)
        b.lse.fill_(3)
        b.attend()
        assert torch.equal(out, b.out) and torch.equal(lse, b.lse)
