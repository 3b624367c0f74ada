"""grid_draft_verify at temperatures from 1e-30 up, against the definition in 64 bits: probabilities, acceptance and draws,
the sign of the log-probabilities, and masked sampling (K = 0) over whole vocabularies."""
import numpy as np
import pytest

from tests.test_gpu_draft import Step

pytestmark = pytest.mark.gpu

# 1/T in 32 bits, its product with log2 e and the product with a difference of logits are off by 2^-24 each, the
# difference too: a log-probability lp by 2^-22 |lp|, which the bounds of Step.check (2^-21 |lp| and a constant) hold.
LOW = [1e-1, 1e-2, 1e-3, 1e-4, 1e-5, 1e-6, 1e-7, 1e-9, 1e-12, 1e-20, 1e-30]


def check(s):
    with np.errstate(all="ignore"):
        s.check()
    lp = s.got()[3]
    assert (lp <= 0).all(), lp.max()


@pytest.mark.parametrize("T", LOW)
@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("B,K,V,probs", [(64, 2, 64, True), (32, 3, 5000, True), (24, 1, 777, False), (40, 0, 300, False)])
def test_low_temperatures(T, dt, B, K, V, probs):
    s = Step(B, K, V, dt, probs, seed=K + V, sharp=6.0)
    s.temp[:] = T
    s.device()
    s.run()
    check(s)


@pytest.mark.parametrize("dt", ["f32", "bf16"])
def test_a_clear_winner_is_certain_at_low_temperatures(dt):
    """One logit well above 64 others: p = 1, whatever the size of l / T; drafted with q = 1 and u below 1 it is accepted."""
    g = np.random.default_rng(5)
    s = Step(len(LOW) * 20, 1, 64, dt, probs=False, mask=False, seed=5, sharp=6.0)
    s.temp[:] = np.repeat(np.float32(LOW), 20)
    best = g.integers(0, 64, s.B)
    top = s.logits.max(2) + np.float32(16) * np.maximum(s.temp, np.float32(1e-2))[:, None]
    s.logits[np.arange(s.B), :, best] = (np.ceil(top * 4) / 4 + 1).astype(np.float32)  # (a quarter: the same in bf16)
    s.draft[:, 0], s.draft_len[:] = best, 1
    s.u[:] = 0.999
    s.device()
    s.run()
    tokens, accepted, status, lp = s.got()
    assert (accepted == 1).all() and (tokens == best[:, None]).all() and (status == 0).all()
    assert (lp <= 0).all() and (lp >= -64 * np.exp(-16.0) - 2.0 ** -20).all()


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("V", [32_003, 151_936])
def test_masked_sampling_over_whole_vocabularies(dt, V):
    s = Step(9, 0, V, dt, probs=False, seed=V, sharp=3.0)
    s.temp[:] = np.float32([1, 0, 0.5, 1e-1, 1e-3, 1e-6, 1e-7, 1.5, 100.0])
    s.device()
    s.run()
    check(s)


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("V", [90, 6000])
def test_admitted_ids_at_the_lowest_finite_logit(dt, V):
    """A mask of another processor's making (the type's lowest value) over every admitted id: they are equally likely,
    greedy rows take the first, and the row is not empty; beside other ids they have no weight."""
    import torch
    low = torch.finfo(torch.float32 if dt == "f32" else torch.bfloat16).min
    s = Step(48, 2, V, dt, probs=False, seed=21)
    s.temp[:] = np.tile(np.float32([0, 0.3, 1, 1.4, 1.5, 1e-6]), 8)
    s.draft_len[:] = 2
    s.bits[:, :, 7] = True
    s.logits[:24] = np.where(s.bits[:24], np.float32(low), s.logits[:24])
    s.logits[24:, :, :V // 2] = low
    first = np.where(s.bits, s.logits, -np.inf).argmax(2)
    s.draft[::2] = first[::2, :2]  # (greedy ones accepted)
    s.device()
    s.run()
    check(s)
    tokens, accepted, status, _ = s.got()
    assert (status == 0).all() and (tokens[:, 0] >= 0).all() and (accepted[::6] == 2).all()


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("V,K", [(100, 2), (5000, 1), (33_000, 0)])
@pytest.mark.parametrize("T", [np.inf, np.finfo(np.float32).max, 1e30, 1e20])
def test_the_largest_temperatures(T, dt, V, K):
    """At an infinite temperature all admitted ids but those of logit -inf (or NaN) are equally likely; below it logits at
    both ends of the type's range still differ by l / T.  Masks of nothing end their row."""
    import torch
    top = torch.finfo(torch.float32 if dt == "f32" else torch.bfloat16).max
    s = Step(36, K, V, dt, probs=False, seed=V)
    s.draft_len[:] = K
    g = np.random.default_rng(V)
    odd = g.choice(np.array([np.nan, -np.inf, np.inf, top, -top, 0], np.float32), s.logits.shape)
    s.logits[:12] = np.where(g.random(s.logits[:12].shape) < 0.3, odd[:12], s.logits[:12])
    s.bits[12:16, K] = False
    s.logits[16:20, K] = np.where(np.arange(V) % 2, np.float32(np.nan), np.float32(-np.inf))
    s.temp[:] = T
    s.device()
    s.run()
    if np.isinf(T):
        s.temp = np.full(36, 1e300)
    check(s)
    status = s.got()[2]
    assert K or (status[12:20] == 4).all()
