"""grid_sample against its definition in 64 bits: cuts of every kind alone and
together, vocabularies around the blocks' ends, both types, unaligned and strided
rows, ties across the cuts, equal logits, infinities and NaN, noise of every
kind, extreme temperatures, and the distribution of what is drawn."""
import math

import numpy as np
import pytest

from tests.harness import pack_bits

pytestmark = pytest.mark.gpu

OK, EMPTY, COMPLETE = 0, 4, 6
# Decisions this close (relatively) may fall either way: a weight is off by 2^-22 of itself for each unit of its exponent's
# rounding (24 bits of up to some 30) and of the exponential, a score by the reciprocal's 2^-23 more.
NEAR = 1e-5


def expected(logits, bits, T, k, p, least, noise, big):
    """(the ids that may be drawn, log-probability of each) of one row in 64 bits."""
    l = logits.astype(np.float64)
    l = np.minimum(np.where(np.isnan(l), -np.inf, l), big)
    if bits is not None:
        l = np.where(bits, l, -np.inf)
    if not (l > -np.inf).any():
        return None
    greedy = not T > 0
    with np.errstate(over="ignore", invalid="ignore"):
        x = (l - l.max()) / (1.0 if greedy else np.float64(T)) if greedy or not math.isinf(T) else np.where(l > -np.inf, 0.0, -np.inf)
    w = np.exp(x)
    logp = x - math.log(w.sum())
    order = np.lexsort((np.arange(len(l)), -l))
    n = int((l > -np.inf).sum())
    may = [n]
    if k > 0:
        may = [min(n, k)]
    if p < 1:
        cum = np.cumsum(w[order[:may[0]]])
        target = p * cum[-1]
        lo, hi = (int((cum < target * (1 + s)).sum()) + 1 for s in (-NEAR, NEAR))
        may = list(range(max(1, lo), min(may[0], hi) + 1))
    if least > 0:
        a, z = (int((w[order] >= least * (1 + s)).sum()) for s in (NEAR, -NEAR))
        may = [max(1, min(m, y)) for m in may for y in range(a, z + 1)]
    if greedy:
        may = [1]
    out = {}
    with np.errstate(divide="ignore", invalid="ignore", over="ignore"):
        e = noise.astype(np.float64)
        score = np.where((e >= 2.0 ** -126) & (w > 2.0 ** -126), w / e, 0.0)  # (smaller weights are flushed to zero)
    lo, hi = min(may), max(may)
    if hi - lo > 50:
        may = [lo, (lo + hi) // 2, hi]
        near_ids = order[lo:hi]
    else:
        near_ids = []
    for m in set(may):
        ids = order[:m]
        s = score[ids]
        best = s.max() if m > 1 else 0.0
        if best <= 0:
            out[int(order[0])] = logp[order[0]]
            continue
        for i in ids[s >= best * (1 - NEAR)]:
            out[int(i)] = logp[i]
    for i in near_ids:
        out.setdefault(int(i), logp[i])
    return out


class Case:
    def __init__(self, B, V, dt="f32", seed=0, sharp=3.0, mask=True, cut="mixed", greedy=0.1, pad=0, off=0, temps=None):
        import torch
        g = self.g = np.random.default_rng(seed)
        self.B, self.V, self.dt = B, V, dt
        l = (g.standard_normal((B, V)) * sharp).astype(np.float32)
        if dt == "bf16":
            l = torch.from_numpy(l).bfloat16().float().numpy()
        self.logits = l
        share = g.choice([1.0, 0.6, min(1.0, 20.0 / V)], (B, 1))
        self.bits = (g.random((B, V)) < share) if mask else None
        self.T = (0.5 + g.random(B)).astype(np.float32) if temps is None else np.asarray(g.choice(temps, B), np.float32)
        self.T[g.random(B) < greedy] = 0
        pick = lambda v, t: g.choice(v, B).astype(t)  # noqa: E731
        self.k = pick([0, 1, 2, 20, 50, 1000, V, V - 1, -3], np.int32) if cut in ("k", "mixed") else None
        self.p = pick([1.0, 0.9, 0.95, 0.5, 0.1, 0.999, 0.0, 2.0], np.float32) if cut in ("p", "mixed") else None
        self.min_p = pick([0.0, 0.0, 0.02, 0.1, 0.5, 1.0, -1.0], np.float32) if cut in ("min", "mixed") else None
        self.noise = g.standard_exponential((B, V)).astype(np.float32) + np.float32(1e-12)
        self.pad, self.off = pad, off

    def device(self):
        import torch
        tdt = torch.float32 if self.dt == "f32" else torch.bfloat16
        put = lambda x: None if x is None else torch.from_numpy(np.ascontiguousarray(x)).cuda()  # noqa: E731
        stride = self.V + self.pad
        flat = torch.full((self.off + self.B * stride + 8,), 1e30, device="cuda", dtype=tdt)
        lg = torch.as_strided(flat, (self.B, self.V), (stride, 1), self.off)
        lg.copy_(torch.from_numpy(self.logits))
        i32 = dict(dtype=torch.int32, device="cuda")
        self.t = dict(logits=lg, noise=put(self.noise), tokens=torch.full((self.B,), -9, **i32), status=torch.full((self.B,), -9, **i32),
                      logprob=torch.full((self.B,), 9.0, device="cuda"), temperature=put(self.T), top_k=put(self.k),
                      top_p=put(self.p), min_p=put(self.min_p),
                      mask=None if self.bits is None else put(pack_bits(self.bits.astype(np.uint8)).view(np.int32).reshape(self.B, -1)))
        return self.t

    def run(self, **kw):
        from paper_2607_11951_gb300 import grid as G
        t = dict(self.t)
        t.update(kw)
        G.grid_sample(**t)
        return self.t["tokens"].cpu().numpy(), self.t["logprob"].cpu().numpy(), self.t["status"].cpu().numpy()

    def check(self, eos=-1):
        if not hasattr(self, "t"):
            self.device()
        tokens, logprob, status = self.run(eos=eos)
        big = np.finfo(np.float32).max if self.dt == "f32" else 3.3895313892515355e38
        at = lambda x, b, none: none if x is None else x[b]  # noqa: E731
        for b in range(self.B):
            want = expected(self.logits[b], None if self.bits is None else self.bits[b], float(self.T[b]), int(at(self.k, b, 0)),
                            float(at(self.p, b, 1.0)), float(at(self.min_p, b, 0.0)), self.noise[b], big)
            if want is None:
                assert (tokens[b], logprob[b], status[b]) == (-1, 0.0, EMPTY), b
                continue
            assert int(tokens[b]) in want, (b, tokens[b], list(want)[:5], self.T[b], at(self.k, b, 0), at(self.p, b, 1), at(self.min_p, b, 0))
            assert status[b] == (COMPLETE if tokens[b] == eos else OK)
            lp = want[int(tokens[b])]
            # (the exponent is off by 2^-22 of itself, the sum by its terms' and by 2^-24 for each of some 300 of a thread's)
            assert abs(logprob[b] - lp) <= 2.0 ** -21 * abs(lp) + 2.0 ** -14, (b, logprob[b], lp)


@pytest.mark.parametrize("V", [1, 2, 31, 32, 33, 500, 512, 4096, 4097, 8193, 16_385, 32_000, 33_333, 151_936, 151_937])
@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("cut", ["none", "k", "p", "min", "mixed"])
def test_cuts(V, dt, cut):
    Case(12, V, dt, seed=V, cut=cut).check()


@pytest.mark.parametrize("dt", ["f32", "bf16"])
def test_many_rows(dt):
    Case(300, 5000, dt, seed=1).check()
    Case(257, 700, dt, seed=2, mask=False).check()


@pytest.mark.parametrize("dt,off,pad", [("f32", 1, 0), ("f32", 3, 5), ("bf16", 1, 0), ("bf16", 5, 3), ("bf16", 7, 1)])
def test_rows_off_the_lines(dt, off, pad):
    Case(9, 10_001, dt, seed=off, off=off, pad=pad).check()


def test_the_largest_vocabulary_and_refusals():
    import torch
    from paper_2607_11951_gb300 import grid as G
    Case(2, 393_216, "f32", seed=4).check()
    c = Case(2, 40, "f32")
    t = c.device()
    with pytest.raises(G.GridError):
        G.grid_sample(torch.zeros((1, 393_217), device="cuda"), torch.ones((1, 393_217), device="cuda"), t["tokens"][:1], t["status"][:1])
    for bad in (dict(logits=t["logits"].half()), dict(noise=t["noise"].double()), dict(noise=t["noise"][:, 1:]), dict(tokens=t["tokens"].long()),
                dict(mask=t["mask"][:, :1]), dict(top_k=t["top_p"]), dict(top_p=t["top_p"][:1]), dict(logits=t["logits"].T)):
        with pytest.raises(AssertionError):
            c.run(**bad)


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("V", [700, 40_000, 151_937])
def test_ties_and_equal_logits(dt, V):
    """Few different logits, so that every cut falls among equal ones: the lower ids are kept."""
    c = Case(16, V, dt, seed=7, mask=True)
    c.logits = np.round(c.logits / 2) * 2 + np.float32(0)
    c.check()
    c = Case(8, V, dt, seed=8, mask=True, greedy=0)
    c.logits[:] = np.float32(1.5)
    c.k = np.array([1, 2, 3, 50, 1000, V // 2, 0, 0], np.int32)
    c.p = np.array([1, 1, 1, 1, 1, 1, 0.5, 0.9], np.float32)
    c.min_p = None
    c.check()


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("V", [600, 50_000])
def test_crowded_bins(dt, V):
    """Most logits within a small part of the range: outliers, masked values of -1e30, and steps of one unit in the last place."""
    c = Case(14, V, dt, seed=9, mask=False, greedy=0)
    c.logits[:] = 1.0 + c.g.standard_normal((14, V)).astype(np.float32) * np.float32(1e-4)
    c.logits[3:, 5] = 9.0
    c.logits[5:, 7:40] = -1e30
    c.logits[7:, 41] = np.finfo(np.float32).min
    c.logits[9:] = np.float32(1.0) + c.g.integers(0, 9, (5, V)).astype(np.float32) * np.float32(2.0 ** -23)
    c.logits[11:, ::3] = -1e9
    if dt == "bf16":
        import torch
        c.logits = torch.from_numpy(c.logits).bfloat16().float().numpy()
        c.logits[np.isinf(c.logits)] = -3.0e38
    c.check()


@pytest.mark.parametrize("temps", [[0.05, 0.1, 0.01], [20.0, 100.0, 1e6], [1e-30, 1e-6], [math.inf], [math.nan, -1.0, 0.0]])
@pytest.mark.parametrize("dt", ["f32", "bf16"])
def test_extreme_temperatures(temps, dt):
    Case(16, 9000, dt, seed=3, temps=temps, greedy=0).check()


@pytest.mark.parametrize("dt", ["f32", "bf16"])
def test_infinities_and_nan(dt):
    c = Case(10, 3000, dt, seed=5, greedy=0.2)
    c.logits[:, ::7] = -np.inf
    c.logits[:, 1::11] = np.nan
    c.logits[0] = np.nan
    c.logits[1] = -np.inf
    c.logits[2, [5, 900]] = np.inf
    c.logits[3] = np.inf
    c.bits[4] = False
    c.bits[5] = False
    c.bits[5, 1234] = True
    c.logits[5, 1234] = 1.0
    c.logits[6, 3] = -0.0
    c.logits[6, 4:] = np.where(c.logits[6, 4:] > 0, 0.0, c.logits[6, 4:])
    c.check()


def test_masked_places_may_hold_anything():
    c = Case(8, 5000, seed=6)
    c.check()
    want = c.run()
    for fill in (math.nan, math.inf, 1e38):
        c.logits = np.where(c.bits, c.logits, np.float32(fill))
        c.device()
        for x, y in zip(c.run(), want):
            assert (x == y).all()


def test_noise_of_every_kind():
    """Zero, subnormal, negative, infinite and NaN noise leaves ids out; where none is left the first id is drawn."""
    c = Case(9, 2000, seed=11, greedy=0, cut="none", mask=False)
    c.noise[0] = 0
    c.noise[1] = np.nan
    c.noise[2] = -1
    c.noise[3] = 1e-40
    c.noise[4] = np.inf
    c.noise[5:, ::2] = np.nan
    c.noise[6:, 1::4] = 0
    c.noise[7, 3] = np.float32(2.0 ** -126)
    want = [expected(c.logits[b], None, float(c.T[b]), 0, 1.0, 0.0, np.where(c.noise[b] >= 2.0 ** -126, c.noise[b], np.inf), 3e38)
            for b in range(9)]
    c.device()
    tokens, _, status = c.run()
    assert all(int(tokens[b]) in want[b] for b in range(9)) and (status == 0).all()
    assert all(tokens[b] == c.logits[b].argmax() for b in range(5))


def test_settings_that_are_no_numbers_count_as_not_given():
    import torch
    c = Case(6, 3000, seed=12, greedy=0, cut="none")
    c.device()
    want = c.run()
    nan = torch.full((6,), math.nan, device="cuda")
    for kw in (dict(top_p=nan), dict(min_p=nan), dict(top_p=nan, min_p=nan)):
        for x, y in zip(c.run(**kw), want):
            assert (x == y).all()


def test_eos_no_logprob_and_repeats():
    import torch
    c = Case(40, 20_000, seed=13)
    c.check()
    tokens, logprob, _ = c.run()
    for _ in range(3):
        again = c.run()
        assert (again[0] == tokens).all() and (again[1] == logprob).all()
    c.check(eos=int(tokens[0]))
    assert c.run(logprob=None)[0].tolist() == tokens.tolist()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    from paper_2607_11951_gb300 import grid as G
    c.t["tokens"].fill_(-9)
    G.grid_sample(**c.t, stream=side)
    torch.cuda.current_stream().wait_stream(side)
    assert c.t["tokens"].tolist() == tokens.tolist()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        G.grid_sample(**c.t)
    for _ in range(2):
        c.t["tokens"].fill_(-9)
        graph.replay()
        assert c.t["tokens"].tolist() == tokens.tolist()


def test_the_same_rows_in_other_batches():
    """A row's token and probability do not depend on the rows beside it."""
    c = Case(33, 7000, seed=14)
    c.device()
    tokens, logprob, _ = c.run()
    part = {k: (v[5:9] if hasattr(v, "shape") else v) for k, v in c.t.items()}
    from paper_2607_11951_gb300 import grid as G
    G.grid_sample(**part)
    assert part["tokens"].tolist() == tokens[5:9].tolist() and part["logprob"].tolist() == logprob[5:9].tolist()


def test_distribution():
    """20,000 draws from one small distribution, cut by top-p: shares as its probabilities (chi-square at 7 degrees of freedom)."""
    import torch
    B, V = 20_000, 40
    g = torch.Generator(device="cuda")
    g.manual_seed(0)
    l = torch.full((V,), -3.0)
    l[[3, 9, 17, 22, 30, 31, 38, 39]] = torch.tensor([2.0, 1.0, 0.5, 1.5, 0.0, 1.0, 0.7, 0.2])
    noise = torch.empty((B, V), device="cuda").exponential_(generator=g)
    tokens, status = (torch.zeros(B, dtype=torch.int32, device="cuda") for _ in range(2))
    from paper_2607_11951_gb300 import grid as G
    p = l.double().softmax(0)
    top_p = torch.full((B,), float(p[l > -3].sum()) - 1e-4, device="cuda")  # all eight
    G.grid_sample(l.cuda().expand(B, V).contiguous(), noise, tokens, status, top_p=top_p)
    got = torch.bincount(tokens.long().cpu(), minlength=V).double()
    want = torch.where(l > -3, p, 0.0)
    want = want / want.sum() * B
    assert float(got[l == -3].sum()) == 0
    chi = ((got - want) ** 2 / want.clamp(min=1e-9))[l > -3].sum()
    assert float(chi) < 24.3, chi  # (one in a thousand)


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("B,V,cut", [(400, 5000, "mixed"), (700, 600, "p"), (2049, 40, "mixed"), (1000, 4097, "none")])
def test_batches_of_more_rows_than_fit_at_once(dt, B, V, cut):
    """Rows of every kind in any order: each is drawn once, whichever goes first."""
    Case(B, V, dt, seed=B, cut=cut, greedy=0.3).check()


@pytest.mark.parametrize("V", [3000, 151_937])
def test_bf16_cuts_at_values(V):
    """Nuclei that end above zero, below it, at it (of either sign) and among equal values."""
    c = Case(12, V, "bf16", seed=V, cut="p", greedy=0, mask=False)
    c.T[:] = 1.0
    c.p[:] = [0.5, 0.9, 0.99, 0.999, 0.9999, 0.3, 0.9, 0.9, 0.9, 0.9, 0.5, 0.5]
    c.logits[6] = np.round(c.logits[6])
    c.logits[7] = np.abs(np.round(c.logits[7]))
    c.logits[8] = -np.abs(c.logits[8])
    c.logits[9] = np.where(np.arange(V) % 2, -0.0, 0.0)
    c.logits[10] = np.where(np.arange(V) % 3, np.abs(c.logits[10]), -0.0)
    c.logits[11, ::2] = 3.0
    c.check()
