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


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("V", [300, 2048, 2049, 8200, 32_000])
def test_rows_of_many_shapes(dt, V):
    """Plateaus, outliers, steps, crowds and next to nothing, at random places or side by side; top_k around the sizes of what
    stands out, noise under which what is cut would be drawn."""
    for seed in range(4):
        c = Case(20, V, dt, seed=V + seed, cut="mixed", greedy=0.05, mask=seed % 2 == 0)
        each = ((V + 7) // 8 + 31) & ~31
        for b, l in enumerate(c.logits):
            g = np.random.default_rng([seed, V, b])
            m = int(min(V, g.choice([1, 3, 20, 60, 100, 128, 129, 256, 300, 512, 513, 700, 1000, 2000, V])))
            out = g.permutation(V)[:m] if b % 2 else np.arange(m) * (max(1, V // m) if b % 4 else 1)
            kind = b % 7
            if kind == 0:
                l[:] = g.uniform(-6, -4, V)
                l[out] = g.uniform(9, 10, m)
            elif kind == 1:
                l[:] = -3
                l[out] = g.choice([2.0, 2.5, 7.0], m)
            elif kind == 2:
                l[:] = np.round(l)
            elif kind == 3:
                l[:] *= 1e-3
                l[out] += 1
            elif kind == 4:
                l[:] = -np.abs(l) - g.choice([0, 100, 1e4])
            elif kind == 5:
                l[:] = g.choice([1e-38, 1e-30, -1e-38, 0.0], V)
                l[out] = g.choice([0.0, 1e-36, 1.0])
            if g.random() < 0.3:
                l[g.integers(0, V, V // 3)] = -np.inf
            if g.random() < 0.1:
                l[g.integers(0, V, 3)] = np.nan
            c.k[b] = g.choice([0, 0, m - 1, m, m + 1, 2 * m, 50, 256, 257, 300])
            c.p[b] = g.choice([1, 1, 0.9, 0.99, 0.5, 0.999999, 0.3])
            c.min_p[b] = g.choice([0, 0, 0, 0.1, 1e-4, 0.9])
            c.T[b] = g.choice([1, 1, 0.7, 1.5, 0.1, 10])
            if c.bits is not None and g.random() < 0.6:
                c.bits[b] = g.random(V) < np.repeat(g.choice([0, 0.003, 0.05, 0.12, 0.13, 1], 8), each)[:V]
            if g.random() < 0.5:
                order = np.argsort(-np.where(np.isnan(l), -np.inf, l), kind="stable")
                c.noise[b, order[min(V - 1, max(0, int(c.k[b]))):]] = 1e-20
        c.logits = as_type(c.logits, dt)
        c.check()
