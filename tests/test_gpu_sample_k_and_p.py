"""grid_sample with top-k and a top-p so near one that it takes all that top-k
left: the roundings of top-p's sums must not let an id past top-k in.  Plateaus of
equal logits round alike, so that their bins are off as far as bins can be."""
import numpy as np
import pytest

from tests.test_gpu_sample import Case

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("V", [32_000, 151_936, 393_216])
@pytest.mark.parametrize("share", [0.02, 0.3, 0.66])
def test_top_p_does_not_undo_top_k(dt, V, share):
    """One logit of zero, a plateau of top_k - 1 ids at some distance, the rest lower: the plateau ends at the k-th id.  Noise
    under which any id past top_k would be drawn if it were kept."""
    import torch
    n = int(V * share)
    depths = np.linspace(0.25, 0.32, 24, dtype=np.float32)
    if dt == "bf16":
        depths = np.array([0.25, 0.28515625, 0.3125, 0.5, 0.75, 1.0, 2.0, 3.5], np.float32)
    c = Case(len(depths), V, dt, seed=V + n, mask=False, greedy=0, cut="none")
    B = c.B
    c.logits[:] = c.g.uniform(-9, -4.5, (B, V)).astype(np.float32)
    if dt == "bf16":
        c.logits = torch.from_numpy(c.logits).bfloat16().float().numpy()
    c.noise[:] = 1
    for b, d in enumerate(depths):
        at = c.g.permutation(V)[:n + 1]
        c.logits[b, at[1:]] = -d
        c.logits[b, at[0]] = 0
        rest = np.ones(V, bool)
        rest[at] = False
        c.noise[b, rest] = 1e-12
    c.T[:] = 1
    c.k = np.full(B, n + 1, np.int32)
    c.p = np.full(B, 0.999999, np.float32)
    c.p[1::3], c.p[2::3] = 1 - 2.0 ** -20, 1 - 2.0 ** -24
    c.device()
    tokens, _, status = c.run()
    assert (status == 0).all()
    assert (c.logits[np.arange(B), tokens] > -4).all(), [(float(depths[b]), int(tokens[b])) for b in range(B) if c.logits[b, tokens[b]] < -4]


@pytest.mark.parametrize("V", [40_000, 151_936])
def test_any_top_k_is_a_limit(V):
    """Rows of few different logits, top_k anywhere in them, with and without a mask: the token's place in the order is below
    top_k whatever top_p is."""
    for seed in range(3):
        c = Case(24, V, "f32" if seed else "bf16", seed=seed, mask=seed == 2, greedy=0, cut="none")
        c.logits = np.round(c.logits * 2) / 2 + np.float32(0)
        c.k = c.g.integers(1, V, 24).astype(np.int32)
        c.k[:8] = [257, 300, 513, 1000, 5000, 20_000, V - 1, V // 2]
        c.p = c.g.choice([0.999999, 0.99999, 1 - 2.0 ** -24, 0.9], 24).astype(np.float32)
        for b in range(24):
            l = c.logits[b] if c.bits is None else np.where(c.bits[b], c.logits[b], -np.inf)
            order = np.lexsort((np.arange(V), -l))
            c.noise[b, order[c.k[b]:]] = 1e-20
        c.device()
        tokens, _, status = c.run()
        for b in range(24):
            l = c.logits[b] if c.bits is None else np.where(c.bits[b], c.logits[b], -np.inf)
            t = int(tokens[b])
            place = int((l > l[t]).sum() + (l[:t] == l[t]).sum())
            assert status[b] == 0 and place < c.k[b], (seed, b, place, c.k[b], c.p[b])
