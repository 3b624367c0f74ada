"""grid_sample where a cut ends exactly where a bound on it lies, and where masks
differ from block to block."""
import numpy as np
import pytest

from tests.test_gpu_sample import Case

pytestmark = pytest.mark.gpu


def as_type(x, dt):
    import torch
    return torch.from_numpy(x).bfloat16().float().numpy() if dt == "bf16" else x


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("top_p", [1.0, 0.9])
@pytest.mark.parametrize("k,spread", [(100, False), (200, False), (300, True), (700, True), (2000, True)])
def test_a_top_k_of_all_that_stand_out(dt, top_p, k, spread):
    """top_k ids far above the others, each in a line of its own thread (of one of the row's blocks, or of all eight), and noise
    under which any other id would be drawn if it were not cut."""
    V = 32_000
    c = Case(4, V, dt, seed=k, mask=False, greedy=0, cut="none")
    lines, each = (8 if dt == "bf16" else 4), ((V + 7) // 8 + 31) & ~31
    j = np.arange(k)
    out = (j % 8) * each + lines * (j // 8) if spread else lines * j
    c.logits[:] = as_type(c.g.uniform(-6, -4, (4, V)).astype(np.float32), dt)
    c.logits[:, out] = as_type(c.g.uniform(9, 10, (4, k)).astype(np.float32), dt)
    c.T[:] = 1
    c.k, c.p = np.full(4, k, np.int32), np.full(4, top_p, np.float32)
    rest = np.ones(V, bool)
    rest[out] = False
    c.noise[:, rest] = 1e-12
    c.check()


def test_a_tail_of_less_than_a_unit():
    """A nucleus that, with the roundings of the sums, ends among hundreds of thousands of ids of less than 2^-41 each."""
    V = 393_216
    each = V // 8
    c = Case(2, V, "f32", seed=1, greedy=0, cut="none")
    tail, ulp = 2.0 ** -41.5, 2.0 ** -23
    c.logits[:] = np.log(tail)
    c.logits[:, each::each] = np.log(0.75 * ulp - (each - 1) * tail)  # each block after the first: three quarters of a unit of Z
    c.logits[:, 0] = 0
    c.bits[:] = True
    c.bits[:, 1:each] = False
    c.T[:] = 1
    c.p = np.full(2, 1 - 2.0 ** -24, np.float32)
    c.noise[:] = 1
    c.check()
    c = Case(2, V, "f32", seed=1, greedy=0, cut="none")
    c.logits[:] = np.log(tail)
    c.logits[:, 0] = 0
    c.bits = None
    c.T[:] = 1
    c.p = np.full(2, 1 - 2.0 ** -24, np.float32)
    c.check()


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("V", [20_000, 151_937])
@pytest.mark.parametrize("cut", ["none", "k", "p", "min", "mixed"])
def test_masks_of_some_blocks_sparse_and_some_dense(dt, V, cut):
    """Blocks that take admitted ids one by one beside others that take whole lines, with few different logits (ties across every
    cut) and with many."""
    c = Case(16, V, dt, seed=V + 1, cut=cut)
    each = ((V + 7) // 8 + 31) & ~31
    share = c.g.choice([0.0, 0.004, 0.05, 0.12, 0.13, 0.5, 1.0], (16, 8))
    c.bits = c.g.random((16, V)) < np.repeat(share, each, 1)[:, :V]
    c.bits[3] = False
    c.bits[3, c.g.integers(0, V, 5)] = True
    c.logits[8:] = np.round(c.logits[8:] / 2) * 2 + np.float32(0)
    c.check()


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("top_p", [1.0, 0.9])
@pytest.mark.parametrize("V", [700, 20_000])
def test_a_top_k_of_more_ids_than_have_a_logit(dt, top_p, V):
    """More ids admitted than top_k, and fewer of them above -inf: all of those are kept; around that number, the k-th is the last."""
    c = Case(8, V, dt, seed=V, mask=True, greedy=0, cut="none")
    c.bits[:] = c.g.random((8, V)) < 0.97
    c.logits[:, c.g.permutation(V)[:V // 3]] = -np.inf
    c.logits[:, c.g.permutation(V)[:9]] = np.nan
    have = (c.bits & (c.logits > -np.inf)).sum(1)
    c.k = (have + np.array([-2, -1, 0, 1, 2, 60, 100, 150])).astype(np.int32)
    assert (c.k > 256).all() and (c.k < c.bits.sum(1)).all()
    c.p = np.full(8, top_p, np.float32)
    c.check()
