"""grid_draft_verify against the definition in 64 bits, and the masked sampling
of single tokens (K = 0): vocabularies and row offsets around the pieces' and
lines' ends, masks of no id, one id and every id, infinities and NaN, ties,
greedy rows, ends by EOS, strides, and the distribution of the tokens."""
import math

import numpy as np
import pytest

from tests.harness import pack_bits

pytestmark = pytest.mark.gpu

OK, EMPTY, COMPLETE = 0, 4, 6
NEAR = 1e-5  # decisions this close (relatively) may fall either way in 32 bits


class Step:
    def __init__(self, B, K, V, dt="f32", probs=True, mask=True, greedy=0.0, seed=0, sharp=2.0, pad=0):
        import torch
        g = np.random.default_rng(seed)
        self.B, self.K, self.V, self.eos = B, K, V, -1
        self.logits = (g.standard_normal((B, K + 1, V + pad)) * sharp).astype(np.float32)
        if dt == "bf16":
            self.logits = torch.from_numpy(self.logits).bfloat16().float().numpy()
        self.dt = dt
        share = g.choice([1.0, 0.5, 3.0 / V], (B, K + 1, 1))
        self.bits = (g.random((B, K + 1, V)) < share) if mask else None
        self.temp = (0.5 + g.random(B)).astype(np.float32)
        self.temp[g.random(B) < greedy] = 0.0
        x = self.logits[:, :K, :V] / np.where(self.temp > 0, self.temp, 1)[:, None, None]
        x = x + g.standard_normal(x.shape) * 0.7
        if mask:
            x = np.where(self.bits[:, :K], x, -1e30)
        q = np.exp(x - x.max(2, keepdims=True)) if K else x
        self.probs = (q / q.sum(2, keepdims=True)).astype(np.float32) if probs and K else None
        e = -np.log1p(-g.random((B, K, V)))
        self.draft = np.where((self.temp > 0)[:, None], (q / e).argmax(2), x.argmax(2)).astype(np.int32) if K else \
            np.zeros((B, 0), np.int32)
        self.draft_len = g.integers(0, K + 1, B).astype(np.int32)
        self.draft_len[g.random(B) < 0.7] = K
        self.u = g.random((B, K)).astype(np.float32)
        self.noise = (-np.log1p(-g.random((B, V)))).astype(np.float32) + np.float32(1e-12)

    def device(self, off=0, stride=None):
        """Device tensors; the logits start `off` elements in, rows `stride` apart."""
        import torch
        B, K, V = self.B, self.K, self.V
        tdt = torch.float32 if self.dt == "f32" else torch.bfloat16
        stride = stride or self.logits.shape[2]
        flat = torch.full((off + B * (K + 1) * stride + 8,), 1e30, device="cuda", dtype=tdt)
        self.t = {}
        lg = torch.as_strided(flat, (B, K + 1, V), ((K + 1) * stride, stride, 1), off)
        lg.copy_(torch.from_numpy(self.logits[:, :, :V]))
        put = lambda x: None if x is None else torch.from_numpy(x).cuda()
        self.t = dict(logits=lg, draft=put(self.draft), u=put(self.u), noise=put(self.noise),
                      tokens=torch.full((B, K + 1), -7, dtype=torch.int32, device="cuda"),
                      accepted=torch.full((B,), -7, dtype=torch.int32, device="cuda"),
                      status=torch.full((B,), -7, dtype=torch.int32, device="cuda"),
                      mask=None if self.bits is None else put(pack_bits(self.bits.reshape(-1, V).astype(np.uint8))
                                                              .view(np.int32).reshape(B, K + 1, -1)),
                      probs=put(self.probs), draft_len=put(self.draft_len), temperature=put(self.temp),
                      logprob=torch.full((B, K + 1), 7.0, device="cuda"), eos=self.eos)
        return self.t

    def run(self, drafts=None, **kw):
        from paper_2607_11951_gb300 import grid as G
        drafts = drafts or G.Drafts(self.B, self.K, self.V)
        t = dict(self.t)
        t.update(kw)
        G.grid_draft_verify(drafts, **t)
        self.drafts = drafts
        return self

    def got(self):
        return [self.t[k].cpu().numpy() for k in ("tokens", "accepted", "status", "logprob")]

    def row(self, b):
        """(tokens, status, log-probabilities, smallest relative margin of a decision) of row b in 64 bits."""
        T = float(self.temp[b])
        out, lp, margin = [], [], math.inf
        nd = int(self.draft_len[b])
        for k in range(nd + 1):
            l = self.logits[b, k, :self.V].astype(np.float64)
            l = np.minimum(np.where(np.isnan(l), -np.inf, l), np.finfo(np.float32).max)
            ok = l > -np.inf
            if self.bits is not None:
                ok = ok & self.bits[b, k]
            if not ok.any():
                return out, EMPTY, lp, margin
            l = np.where(ok, l, -np.inf)
            x = (l - l.max()) / (T if T > 0 else 1.0)
            z = np.exp(x).sum()
            p = np.exp(x) / z
            best = int(np.argmax(l))
            if k < nd:
                d = int(self.draft[b, k])
                if 0 <= d < self.V and ok[d]:
                    if T > 0:
                        q = float(self.probs[b, k, d]) if self.probs is not None else 1.0
                        uq = float(self.u[b, k]) * q
                        margin = min(margin, abs(uq - p[d]) / p[d])
                        take = uq < p[d]
                    else:
                        take = d == best
                    if take:
                        out.append(d)
                        lp.append(x[d] - math.log(z))
                        if d == self.eos:
                            return out, COMPLETE, lp, margin
                        continue
            if T > 0:
                w = p
                if k < nd:
                    if self.probs is not None:
                        w = np.maximum(p - self.probs[b, k].astype(np.float64), 0)
                    else:
                        w = p.copy()
                        if 0 <= self.draft[b, k] < self.V:
                            w[self.draft[b, k]] = 0
                e = self.noise[b].astype(np.float64)
                with np.errstate(all="ignore"):
                    s = np.where(ok & (e > 0), w / e, 0)
                    if not (s > 0).any():
                        s = np.where(ok & (e > 0), p / e, 0)
                if (s > 0).any():
                    top = np.partition(s, -2)[-2:] if self.V > 1 else np.array([0, s[0]])
                    # a weight that is a small difference is known less well than p itself
                    i = int(np.argmax(s))
                    margin = min(margin, (top[1] - top[0]) / top[1] * min(1.0, w[i] / p[i]))
                    best = i
            out.append(best)
            lp.append(x[best] - math.log(z))
            return out, COMPLETE if best == self.eos else OK, lp, margin
        raise AssertionError

    def check(self, most_near=0.02):
        tokens, accepted, status, logprob = self.got()
        close = 0
        for b in range(self.B):
            out, st, lp, margin = self.row(b)
            if margin < NEAR:
                close += 1
                continue
            drawn = st == OK or (st == COMPLETE and not self.ended_by_draft(out, b))
            assert tokens[b].tolist() == out + [-1] * (self.K + 1 - len(out)), (b, margin)
            assert accepted[b] == len(out) - (1 if drawn else 0) and status[b] == st, (b, accepted[b], status[b])
            # sums of up to V / 256 + 64 terms a thread, exponents of up to some 60 in size
            near = (self.V / 256 + 64) * 2.0 ** -24 + 64 * 2.0 ** -22 + 2.0 ** -21 * np.abs(lp)
            assert (np.abs(logprob[b, :len(lp)] - lp) <= near).all(), (b, logprob[b], lp)
            assert (logprob[b, len(lp):] == 0).all()
        assert close <= most_near * self.B + 1
        return self

    def ended_by_draft(self, out, b):
        n = len(out)
        return n <= self.draft_len[b] and out[-1] == self.eos and out == self.draft[b, :n].tolist() and \
            self.row_accepts(b, n)

    def row_accepts(self, b, n):
        keep = self.eos
        self.eos = -1
        try:
            return len(self.row(b)[0]) > n
        finally:
            self.eos = keep


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("probs", [True, False])
@pytest.mark.parametrize("B,K,V", [(1, 0, 1), (3, 2, 2), (5, 1, 31), (40, 4, 512), (7, 8, 2047), (6, 3, 2049), (3, 2, 4100),
                                   (33, 5, 32_001), (2, 1, 151_937), (300, 0, 777), (4, 64, 300)])
def test_verify_against_the_definition(dt, probs, B, K, V):
    s = Step(B, K, V, dt, probs, greedy=0.25, seed=V + K)
    s.device()
    s.run().check()
    # the same bits again, on the same handle
    first = s.got()
    s.run(s.drafts)
    for a, b in zip(first, s.got()):
        assert (a == b).all()


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("off", range(0, 9))
def test_rows_at_every_offset(dt, off):
    s = Step(9, 2, 2500 + off, dt, seed=off, greedy=0.3)
    for stride in (2509, 2512):
        s.device(off, stride)
        s.run().check()


def test_positions_first_and_a_larger_handle():
    """Masks and logits as [K + 1][B][...], a handle made for more, rows that take other lengths."""
    import torch
    from paper_2607_11951_gb300 import grid as G
    s = Step(11, 3, 1000, "bf16", seed=4)
    t = s.device()
    turn = lambda x: x.transpose(0, 1).contiguous().transpose(0, 1)
    t["logits"], t["mask"], t["probs"] = turn(t["logits"]), turn(t["mask"]), turn(t["probs"])
    wide = torch.full((11, 1100), math.nan, device="cuda")
    wide[:, 7:1007] = t["noise"]
    t["noise"] = wide[:, 7:1007]
    s.run(G.Drafts(64, 9, 5000)).check()
    s.draft_len = np.array([-3, 0, 1, 2, 3, 4, 100, 3, 3, 3, 3], np.int32)
    t["draft_len"] = torch.from_numpy(s.draft_len).cuda()
    s.run(s.drafts)
    s.draft_len = s.draft_len.clip(0, 3)
    s.check()


def test_absent_arguments():
    """No mask, temperature, lengths, probabilities or logprob."""
    s = Step(20, 2, 700, mask=False, probs=False, seed=2)
    s.temp[:] = 1
    s.draft_len[:] = 2
    s.device()
    s.run(temperature=None, draft_len=None).check()
    tokens = s.got()[0]
    s.t["tokens"].fill_(-7)
    s.run(temperature=None, draft_len=None, logprob=None)
    assert (s.got()[0] == tokens).all()


@pytest.mark.parametrize("dt", ["f32", "bf16"])
def test_infinities_and_nan(dt):
    """NaN and infinities at refused ids change nothing; at admitted ids NaN counts as -inf, +inf as the largest value."""
    s = Step(24, 2, 1500, dt, seed=9, greedy=0.3)
    s.bits[:, :, 5] = True
    clean = s.device()
    s.run().check()
    want = s.got()
    g = np.random.default_rng(1)
    bad = g.choice(np.array([np.nan, np.inf, -np.inf, np.finfo(np.float32).min], np.float32), s.logits.shape)
    s.logits = np.where(s.bits, s.logits, bad)
    s.device()
    s.run()
    for a, b in zip(want, s.got()):
        assert (a == b).all()
    some = g.random(s.logits.shape)
    s.logits = np.where(s.bits & (some < 0.2), np.float32(np.nan), s.logits)
    s.logits = np.where(s.bits & (some > 0.8), np.float32(-np.inf), s.logits)
    s.logits[::3, 1, 5] = np.inf
    s.device()
    s.run().check()
    del clean


def test_empty_masks():
    """A position that admits nothing ends the row where it is reached; one that is not reached does not."""
    s = Step(30, 3, 900, "f32", probs=False, seed=3)
    s.temp[:] = 0.0
    s.draft_len[:] = 3
    for b in range(30):
        for k in range(4):
            s.bits[b, k, 100 + b] = True
            s.logits[b, k, 100 + b] = 50.0
    s.draft[:] = (100 + np.arange(30))[:, None]  # every drafted id is the largest
    for b in range(30):
        k = b % 5
        if k < 4:
            s.bits[b, k] = False
    s.draft[20:, 0] = 3  # refused at once: later positions are not reached
    s.device()
    s.run().check()
    status = s.got()[2]
    assert (status[:20:5] == EMPTY).all() and (status[4:20:5] == OK).all() and status[21] == OK and status[20] == EMPTY
    s.bits[:, 0] = True
    s.logits[:, 0] = -np.inf
    s.device()
    s.run().check()
    assert (s.got()[2] == EMPTY).all()


@pytest.mark.parametrize("dt", ["f32", "bf16"])
def test_ties_go_to_the_lowest_id(dt):
    s = Step(40, 3, 3000, dt, probs=False, seed=6)
    s.logits = np.round(s.logits)
    s.temp[:20] = 0.0
    s.noise[:] = 0.5
    for b in range(40):
        for k in range(3):
            l = np.where(s.bits[b, k], s.logits[b, k], -np.inf)
            if b % 2 and s.bits[b, k].any():
                s.draft[b, k] = np.argmax(l)
    s.device()
    s.run()
    tokens = s.got()[0]
    for b in range(40):
        out, _, _, _ = s.row(b)
        assert tokens[b, :len(out)].tolist() == out, b


def test_drafted_ids_out_of_range_or_mask_are_refused():
    s = Step(8, 2, 600, seed=8, probs=False)
    s.draft_len[:] = 2
    s.bits[:, :, 9] = True
    s.draft[:, 0] = [-1, 600, 1 << 30, -(1 << 31), 9, 9, 9, 9]
    s.draft[:, 1] = 9
    s.bits[5, 0, 9] = False
    s.device()
    s.run().check()
    assert (s.got()[1][[0, 1, 2, 3, 5]] == 0).all()


def test_eos_ends_a_row():
    s = Step(60, 3, 400, seed=12, probs=False, mask=False, greedy=1.0)
    s.draft = s.logits[:, :3].argmax(2).astype(np.int32)
    s.draft_len[:] = 3
    s.eos = int(s.draft[0, 1])
    s.draft[1], s.logits[1] = s.draft[0], s.logits[0]
    s.draft_len[1] = 1  # (the same id, drawn)
    s.device()
    s.run().check()
    tokens, accepted, status, _ = s.got()
    assert accepted[0] == 2 and accepted[1] == 1 and (status[:2] == COMPLETE).all()
    assert tokens[0].tolist() == tokens[1].tolist() == s.draft[0, :2].tolist() + [-1, -1]


def test_noise_that_is_not_positive():
    s = Step(6, 0, 300, seed=13)
    s.bits[:, :, 50:60] = True
    s.noise[:, ::2] = 0.0
    s.noise[1, 1::2] = np.nan
    s.noise[2, 1::2] = -1.0
    s.noise[3, 1::2] = np.inf
    s.device()
    s.run().check(most_near=1.0)
    tokens = s.got()[0]
    for b in (1, 2, 3):
        assert tokens[b, 0] == np.argmax(np.where(s.bits[b, 0], s.logits[b, 0], -np.inf))


@pytest.mark.parametrize("V", [300, 5000])
def test_negative_noise_after_a_refusal(V):
    """Weights below zero over noise below zero are no scores."""
    s = Step(24, 2, V, seed=16, mask=False)
    s.temp[:] = 1
    s.u[:] = 0.99999
    s.noise[:, ::3] = -s.noise[:, ::3]
    s.device()
    s.run().check(most_near=0.1)
    assert (s.got()[1] < 2).any()


def test_a_drafter_equal_to_the_target_is_always_accepted():
    s = Step(50, 4, 800, seed=14, mask=False)
    s.temp[:] = 1
    s.draft_len[:] = 4
    x = s.logits[:, :4].astype(np.float64)
    q = np.exp(x - x.max(2, keepdims=True))
    s.probs = (q / q.sum(2, keepdims=True)).astype(np.float32)
    s.u = np.minimum(s.u, 0.9999)
    s.device()
    s.run()
    assert (s.got()[1] == 4).all()


def test_tokens_are_distributed_as_the_target():
    """Over 60,000 rows of one position, drafted from another distribution, the first token's counts are within five
    standard deviations of the masked target's for every id."""
    import torch
    from paper_2607_11951_gb300 import grid as G
    B, V = 60_000, 40
    g = torch.Generator(device="cuda")
    g.manual_seed(3)
    one = torch.randn((1, 1, V), generator=g, device="cuda")
    bits = torch.rand((1, 1, V), generator=g, device="cuda") < 0.7
    mask = torch.from_numpy(pack_bits(bits.cpu().numpy()[0].astype(np.uint8)).view(np.int32)).cuda().view(1, 1, -1)
    p = torch.softmax(one.masked_fill(~bits, -math.inf), 2)[0, 0]
    q = torch.softmax(one + torch.randn((1, 1, V), generator=g, device="cuda"), 2)
    noise = lambda *shape: torch.empty(shape, device="cuda").exponential_(generator=g)
    for probs, drawn in ((q, q[0, 0]), (None, None)):
        draft = (drawn / noise(B, V)).argmax(1).int() if probs is not None else \
            torch.randint(0, V, (B,), generator=g, device="cuda", dtype=torch.int32)
        logits = one.expand(B, 2, V).contiguous()
        tokens = torch.empty((B, 2), dtype=torch.int32, device="cuda")
        acc, st = (torch.empty(B, dtype=torch.int32, device="cuda") for _ in range(2))
        G.grid_draft_verify(G.Drafts(B, 1, V), logits, draft[:, None].contiguous(),
                            torch.rand((B, 1), generator=g, device="cuda"), noise(B, V), tokens, acc, st,
                            mask=mask.expand(B, 2, -1), probs=None if probs is None else probs.expand(B, 1, V))
        count = torch.bincount(tokens[:, 0].long(), minlength=V).double()
        off = (count - B * p.double()).abs() / (B * p.double() * (1 - p.double()) + 1e-9).sqrt()
        assert float(off[bits[0, 0]].max()) < 5 and float(count[~bits[0, 0]].sum()) == 0


def test_refusals():
    import torch
    from paper_2607_11951_gb300 import grid as G
    s = Step(4, 2, 100)
    s.device()
    with pytest.raises(G.GridError) as e:
        s.run(G.Drafts(3, 2, 100))
    assert e.value.code == -8
    with pytest.raises(G.GridError):
        s.run(G.Drafts(4, 1, 100))
    with pytest.raises(G.GridError):
        s.run(G.Drafts(4, 2, 99))
    for bad in (dict(draft=s.t["draft"].long()), dict(u=s.t["u"][:, :1]), dict(noise=s.t["noise"].double()),
                dict(mask=s.t["mask"][:, :, :-1]), dict(probs=s.t["probs"][:, :1]), dict(tokens=s.t["tokens"][:, :2])):
        with pytest.raises(AssertionError):
            s.run(G.Drafts(4, 2, 100), **bad)
    with pytest.raises(KeyError):
        s.run(G.Drafts(4, 2, 100), logits=s.t["logits"].half())
