"""A chunk of tokens through the paged cache: grid_kv_append and grid_kv_attend
against the formulas in 64 bits, at the lengths, head layouts, pages, strides
and bad rows where they can go wrong.  What no row owns is NaN in these pools."""
import math

import pytest

pytestmark = pytest.mark.gpu

UNIT = {"bf16": 2.0 ** -8, "f16": 2.0 ** -11}  # the most that one rounding changes a value, relatively
TINY = 2.0 ** -24                              # f16 below its normal range


def dtype(name):
    import torch
    return {"bf16": torch.bfloat16, "f16": torch.float16}[name]


class Batch:
    """Rows of `old` cached and `new` tokens in pools whose every other value is NaN."""

    def __init__(self, old, new, heads, kv_heads, D, page, dt="bf16", order="token", seed=0, spare=3, scale=1.5,
                 pad_tokens=0, first_page=0):
        import torch
        from paper_2607_11951_gb300 import grid as G
        g = torch.Generator(device="cuda")
        g.manual_seed(seed)
        self.rand = lambda *s: torch.randn(s, generator=g, device="cuda")
        self.G, self.old, self.new, self.dt = G, old, new, dt
        self.H, self.Hk, self.D, self.page, self.B = heads, kv_heads, D, page, len(old)
        self.N = sum(new)
        need = [-(-(o + n) // page) for o, n in zip(old, new)]
        n_pages = sum(need) + spare + first_page
        ids = (torch.randperm(sum(need) + spare, generator=g, device="cuda") + first_page).tolist()
        self.table = torch.full((self.B, max(1, max(need)) + 1), 1 << 30, dtype=torch.int32)
        for b, n in enumerate(need):
            self.table[b, :n] = torch.tensor([ids.pop() for _ in range(n)], dtype=torch.int32)
        self.table = self.table.cuda()
        shape = (n_pages, page, kv_heads, D) if order == "token" else (n_pages, kv_heads, page, D)
        pools = [torch.empty(shape, dtype=dtype(dt), device="cuda") for _ in range(2)]
        for p in pools:
            p[first_page:] = math.nan
        self.k, self.v = [p if order == "token" else p.transpose(1, 2) for p in pools]
        self.lens = torch.tensor(old, dtype=torch.int32).cuda()
        starts = [sum(new[:b]) for b in range(self.B + 1)]
        self.start = torch.tensor(starts, dtype=torch.int32).cuda()
        self.status = torch.full((self.B,), -1, dtype=torch.int32, device="cuda")
        self.kv = G.PagedKV(self.k, self.v, heads)
        # what was cached before, and all of it once the chunk is in
        self.cached = [(self.rand(o, kv_heads, D).to(self.k.dtype), self.rand(o, kv_heads, D).to(self.k.dtype)) for o in old]
        for b, (ck, cv) in enumerate(self.cached):
            self.put(b, 0, ck, cv)
        N = self.N + pad_tokens
        qkv = self.rand(N, heads + 2 * kv_heads, D)
        qkv[:, :heads] *= scale
        self.qkv = qkv.to(self.k.dtype)
        self.q, self.nk, self.nv = self.qkv[:, :heads], self.qkv[:, heads:heads + kv_heads], self.qkv[:, heads + kv_heads:]
        self.out = torch.full((N, heads, D), 7.0, dtype=self.k.dtype, device="cuda")
        self.lse = torch.full((N, heads), 7.0, device="cuda")

    def places(self, b, a, n):
        import torch
        pos = torch.arange(a, a + n, device="cuda")
        return self.table[b].long()[pos // self.page], pos % self.page

    def put(self, b, a, k, v):
        if k.shape[0]:
            at = self.places(b, a, k.shape[0])
            self.k[at] = k
            self.v[at] = v

    def fill(self):
        """The chunk's keys and values as they are (no rotation), without the library."""
        a = 0
        for b, n in enumerate(self.new):
            self.put(b, self.old[b], self.nk[a:a + n], self.nv[a:a + n])
            a += n

    def attend(self, **kw):
        self.G.grid_kv_attend(self.kv, self.table, self.lens, self.q, self.out, self.status, lse=self.lse,
                              start=self.start, **kw)

    def check(self, scale=None, rows=None):
        """out and lse against 64 bits.  With d the most that D fp32 products and sums change a score, every
        probability is off by at most 2 d and by its own rounding, so out by that share of sum p |v| and its rounding."""
        import torch
        scale = self.D ** -0.5 if scale is None else scale
        unit, a = UNIT[self.dt], 0
        group = self.H // self.Hk
        for b, n in enumerate(self.new):
            z = a + n
            if n and (rows is None or b in rows):
                k = torch.cat([self.cached[b][0], self.nk[a:z]]).double()
                v = torch.cat([self.cached[b][1], self.nv[a:z]]).double()
                k, v = k.repeat_interleave(group, 1), v.repeat_interleave(group, 1)
                q = self.q[a:z].double()
                x = torch.einsum("thd,jhd->htj", q, k) * scale
                d = self.D * 2.0 ** -23 * scale * torch.einsum("thd,jhd->htj", q.abs(), k.abs()).max().item() + 2.0 ** -18
                hidden = torch.arange(k.shape[0], device="cuda") > self.old[b] + torch.arange(n, device="cuda")[:, None]
                x = x.masked_fill(hidden, -math.inf)
                lse = x.logsumexp(2)
                p = (x - lse[..., None]).exp()
                want = torch.einsum("htj,jhd->thd", p, v)
                near = unit * want.abs() + (unit + 2 * d) * torch.einsum("htj,jhd->thd", p, v.abs()) + TINY
                off = (self.out[a:z].double() - want).abs() - near
                assert bool((off <= 0).all()), (b, float(off.max()), torch.nonzero(off > 0)[:4].tolist())
                off = (self.lse[a:z].double() - lse.T).abs() - d - 2.0 ** -20 * (1 + lse.T.abs())
                assert bool((off <= 0).all()), (b, "lse", float(off.max()))
                assert int(self.status[b]) == 0
            a = z


LAYOUTS = [(8, 2, 64), (4, 4, 128), (7, 1, 64), (32, 8, 128), (14, 2, 128), (16, 1, 128), (3, 3, 64)]


@pytest.mark.parametrize("heads,kv_heads,D", LAYOUTS)
@pytest.mark.parametrize("dt", ["bf16", "f16"])
def test_attend_single_tokens_around_tiles(heads, kv_heads, D, dt):
    old = [0, 1, 2, 15, 16, 62, 63, 64, 126, 127, 128, 129, 254, 255, 256, 257, 400, 1000]
    b = Batch(old, [1] * len(old), heads, kv_heads, D, 16, dt, seed=heads)
    b.fill()
    b.attend()
    b.check()


@pytest.mark.parametrize("heads,kv_heads,D", LAYOUTS)
@pytest.mark.parametrize("page,order", [(8, "token"), (32, "head"), (128, "token"), (1024, "head")])
def test_attend_ragged_chunks(heads, kv_heads, D, page, order):
    new = [0, 1, 2, 5, 8, 9, 16, 18, 19, 31, 37, 64, 65, 127, 130, 0, 257, 3]
    old = [5, 0, 100, 0, 300, 127, 128, 1, 250, 33, 0, 64, 0, 700, 126, 0, 255, 2000]
    b = Batch(old, new, heads, kv_heads, D, page, order=order, seed=page)
    b.fill()
    b.attend()
    b.check()


@pytest.mark.parametrize("B,n,old,heads,kv_heads,D", [
    (1, 1, 16_001, 8, 1, 128), (1, 1, 16_001, 8, 8, 64), (2, 5, 9_000, 32, 8, 128), (1, 700, 5_000, 4, 1, 128),
    (3, 1300, 77, 2, 2, 64), (40, 1, 3_000, 32, 8, 128), (200, 1, 130, 8, 2, 64), (1, 2048, 0, 6, 2, 128)])
def test_attend_long_axes(B, n, old, heads, kv_heads, D):
    b = Batch([old - 3 * i if old > 3 * B else old for i in range(B)], [n] * B, heads, kv_heads, D, 64, seed=n)
    b.fill()
    b.attend()
    b.check()


@pytest.mark.parametrize("old,new,heads,kv_heads,D", [
    ([60] * 19, [1] * 19, 16, 8, 64),                # 152 key heads alike: a block each
    ([60] * 20, [1] * 20, 16, 8, 64),                # eight more than blocks
    ([100 * (i % 7) for i in range(19)], [i % 3 for i in range(19)], 8, 8, 128),  # rows without tokens between them
    ([0], [100], 32, 8, 64),                         # two units of 256 query rows to a key head
    ([0, 0, 130], [300, 0, 260], 14, 2, 64),         # several, of several lengths
    ([700], [1], 8, 4, 128), ([900], [1], 8, 4, 128), ([1100], [1], 8, 4, 128), ([1300], [3], 4, 4, 64),
    ([5000] + [10] * 5, [1] * 6, 4, 2, 128),         # one key head far dearer than the others
])
def test_attend_key_heads_whole_and_cut(old, new, heads, kv_heads, D):
    b = Batch(old, new, heads, kv_heads, D, 16, seed=len(old))
    b.fill()
    b.attend()
    b.check()


def test_attend_one_prompt_among_single_tokens():
    b = Batch([40 * i for i in range(60)], [1] * 30 + [900] + [1] * 29, 8, 2, 128, 16)
    b.fill()
    b.attend()
    b.check()


@pytest.mark.parametrize("scale", [1e-3, 0.7, 4.0])
def test_attend_sharp_and_flat_scores(scale):
    """Scores of hundreds (one key takes all) and scores that are nearly equal."""
    b = Batch([300, 0, 129], [70, 140, 1], 4, 2, 64, 16, "f16")
    b.fill()
    b.attend(scale=scale)
    b.check(scale)


def test_attend_growing_maximum():
    """Each tile's keys outweigh all before them, so that the running maximum moves in every tile."""
    import torch
    b = Batch([1500, 10], [3, 400], 4, 1, 128, 32, "f16", scale=0.0)
    b.qkv[:, :b.H, 0] = 8.0  # every score is 8 k_0 / sqrt(128)
    for i, n in enumerate(b.old):
        b.cached[i][0][:, :, 0] = (torch.arange(n, device="cuda") * 0.05)[:, None].half()
        b.put(i, 0, *b.cached[i])
    a = 0
    for i, n in enumerate(b.new):
        b.nk[a:a + n, :, 0] = ((torch.arange(n, device="cuda") + b.old[i]) * 0.05)[:, None].half()
        a += n
    b.fill()
    b.attend()
    b.check()


def test_attend_strided_heads_uniform_rows_and_spare_tokens():
    """q and out as slices of wider tensors, start None, then a start that ends before the tokens do."""
    import torch
    b = Batch([100, 7, 0], [4, 4, 4], 8, 2, 64, 16, pad_tokens=2)
    b.fill()
    wide = torch.full((b.N, b.H + 3, 2 * b.D), 7.0, dtype=b.k.dtype, device="cuda")
    b.G.grid_kv_attend(b.kv, b.table, b.lens, b.q[:b.N], wide[:, 1:1 + b.H, b.D:], b.status, lse=b.lse[:b.N])
    rest, b.out = b.out, wide[:, 1:1 + b.H, b.D:]
    b.check()
    assert bool((wide[:, :, :b.D] == 7).all()) and bool((wide[:, 0] == 7).all()) and bool((wide[:, 1 + b.H:] == 7).all())
    assert bool((b.lse[b.N:] == 7).all())
    b.out = rest
    b.attend()
    b.check()
    assert bool((b.out[b.N:] == 7).all()) and bool((b.lse[b.N:] == 7).all())


def test_attend_repeats_bit_for_bit_and_on_another_stream():
    import torch
    b = Batch([5000, 3, 800, 0], [2, 150, 1, 300], 8, 2, 128, 16)
    b.fill()
    b.attend()
    out, lse = b.out.clone(), b.lse.clone()
    side = torch.cuda.Stream()
    for _ in range(3):
        b.out.fill_(3.0)
        b.lse.fill_(3.0)
        side.wait_stream(torch.cuda.current_stream())
        b.attend(stream=side)
        torch.cuda.current_stream().wait_stream(side)
        assert torch.equal(b.out, out) and torch.equal(b.lse, lse)


def test_attend_bad_rows_are_left_out():
    """Bad page ids, lengths and orders end in a status and zeros; the other rows are whole."""
    import torch
    old, new = [40, 40, 40, 40, 300], [2, 2, 2, 2, 40]
    b = Batch(old, new, 4, 2, 64, 16)
    b.fill()
    table, lens = b.table.clone(), b.lens.clone()
    b.table[0, 1] = b.k.shape[0]     # outside the cache, in the middle
    b.table[1, 2] = -1               # its last page
    b.lens[2] = -1
    b.lens[3] = b.table.shape[1] * 16 - 1  # one token too many
    b.attend()
    assert b.status.tolist() == [7, 7, 7, 7, 0]
    assert bool((b.out[:8] == 0).all()) and bool((b.lse[:8] == -math.inf).all())
    b.check(rows=[4])
    b.table, b.lens = table, lens
    good = b.start.clone()
    b.start[2] = 1  # row 1 ends before it begins
    b.attend()
    assert b.status.tolist()[0] == 0 and b.status.tolist()[1] == 7 and b.status.tolist()[3:] == [0, 0]
    b.start = good
    b.start[5] = b.N + 1  # past the tokens
    b.attend()
    assert b.status.tolist() == [0, 0, 0, 0, 7]
    assert bool((b.out[8:] == 0).all())
    b.start = good.clone()
    b.start[5] = b.N
    b.attend()
    b.check()


def test_attend_no_tokens_at_all():
    import torch
    b = Batch([3, 4], [0, 0], 4, 2, 64, 16)
    b.attend()
    assert b.status.tolist() == [0, 0]


def test_pools_past_32_bits():
    """The used pages lie more than 2^31 elements into the pools."""
    page, Hk, D = 64, 8, 128
    first = (1 << 31) // (page * Hk * D)
    b = Batch([700, 0, 90], [3, 150, 1], 16, Hk, D, page, first_page=first)
    append(b)
    b.check_pools()
    b.attend()
    b.check()


# ---------------------------------------------------------------------------
def tables(b, rot, seed=1):
    """Cosines and sines of positions that the batch reaches."""
    import torch
    n = max(o + k for o, k in zip(b.old, b.new)) or 1
    freq = 500.0 ** (-torch.arange(0, rot, 2, device="cuda", dtype=torch.float64) / rot)
    angle = torch.arange(n, device="cuda", dtype=torch.float64)[:, None] * freq
    return angle.cos().float(), angle.sin().float()


def turned(x, pos, cos, sin, pairs, w, eps):
    """The formula in 64 bits, and by how much 32 bits may miss it."""
    import torch
    x = x.double()
    if w is not None:
        x = x / (x.pow(2).mean(-1, keepdim=True) + eps).sqrt() * w.double()
    y, near = x.clone(), x.abs() * 2.0 ** -19
    if cos is not None:
        half = cos.shape[1]
        i = torch.arange(half, device="cuda") * (2 if pairs else 1)
        j = i + (1 if pairs else half)
        c, s = cos[pos].double()[:, None], sin[pos].double()[:, None]
        y[..., i] = x[..., i] * c - x[..., j] * s
        y[..., j] = x[..., j] * c + x[..., i] * s
        near[..., i] = near[..., j] = (x[..., i].abs() + x[..., j].abs()) * 2.0 ** -19
    return y, near


def append(b, **kw):
    b.G.grid_kv_append(b.kv, b.table, b.lens, b.nk[:b.N], b.nv[:b.N], b.status, start=b.start, **kw)


def positions(b):
    import torch
    return torch.tensor([o + i for o, n in zip(b.old, b.new) for i in range(n)], device="cuda")


def check_pools(b, keys=None, near=None):
    """Every value of the pools: the chunk's, what was cached, and NaN where nothing belongs."""
    import torch
    unit = UNIT[b.dt]
    a = 0
    seen = torch.zeros(b.k.shape[:2], dtype=torch.bool, device="cuda")
    for r, n in enumerate(b.new):
        at = b.places(r, 0, b.old[r])
        assert torch.equal(b.k[at], b.cached[r][0]) and torch.equal(b.v[at], b.cached[r][1])
        seen[at] = True
        at = b.places(r, b.old[r], n)
        seen[at] = True
        assert torch.equal(b.v[at], b.nv[a:a + n])
        if keys is None:
            assert torch.equal(b.k[at], b.nk[a:a + n])
        else:
            off = (b.k[at].double() - keys[a:a + n]).abs() - unit * keys[a:a + n].abs() - near[a:a + n] - TINY
            assert not n or float(off.max()) <= 0
        assert int(b.status[r]) == 0
        a += n
    used = torch.unique(torch.cat([b.table[r, :-(-(o + n) // b.page)] for r, (o, n) in enumerate(zip(b.old, b.new))]).long())
    assert bool(b.k[used][~seen[used]].isnan().all()) and bool(b.v[used][~seen[used]].isnan().all())


Batch.check_pools = check_pools


@pytest.mark.parametrize("heads,kv_heads,D,rot", [(8, 2, 64, 64), (14, 2, 64, 32), (32, 8, 128, 128), (5, 5, 128, 96),
                                                   (1, 1, 128, 16), (7, 1, 64, 48)])
@pytest.mark.parametrize("pairs", [False, True])
@pytest.mark.parametrize("norm", ["both", "key", "none"])
@pytest.mark.parametrize("dt,order,page", [("bf16", "token", 16), ("f16", "head", 8)])
def test_append_rotates_norms_and_stores(heads, kv_heads, D, rot, pairs, norm, dt, order, page):
    import torch
    b = Batch([0, 5, 15, 16, 100, 3], [1, 0, 1, 20, 7, 0], heads, kv_heads, D, page, dt, order, seed=rot)
    cos, sin = tables(b, rot)
    qw, kw = (1 + 0.3 * b.rand(D)).to(b.k.dtype), (1 + 0.3 * b.rand(D)).to(b.k.dtype)
    qw, kw = qw if norm == "both" else None, kw if norm != "none" else None
    q_out = torch.full_like(b.out, 7.0)
    append(b, q=b.q, q_out=q_out, cos=cos, sin=sin, pairs=pairs, q_norm=qw, k_norm=kw, eps=1e-5)
    pos = positions(b)
    k, near = turned(b.nk, pos, cos, sin, pairs, kw, 1e-5)
    b.check_pools(k, near)
    q, near = turned(b.q, pos, cos, sin, pairs, qw, 1e-5)
    off = (q_out.double() - q).abs() - UNIT[dt] * q.abs() - near - TINY
    assert float(off.max()) <= 0
    # in place, the same bits; keys and values alone, the same too
    pools = b.k.clone(), b.v.clone()
    mine = b.q.clone()
    append(b, q=mine, q_out=mine, cos=cos, sin=sin, pairs=pairs, q_norm=qw, k_norm=kw, eps=1e-5)
    assert torch.equal(mine, q_out)
    append(b, cos=cos, sin=sin, pairs=pairs, k_norm=kw, eps=1e-5)
    for p, was in zip((b.k, b.v), pools):
        assert torch.equal(p.view(torch.int16), was.view(torch.int16))


@pytest.mark.parametrize("B,n", [(1, 1), (3, 1), (1000, 1), (70, 3), (1, 777)])
def test_append_uniform_rows_and_plain_copies(B, n):
    import torch
    b = Batch([(7 * i) % 50 for i in range(B)], [n] * B, 4, 2, 64, 16)
    b.G.grid_kv_append(b.kv, b.table, b.lens, b.nk, b.nv, b.status)
    b.check_pools()
    append(b)
    b.check_pools()


def test_append_many_ragged_rows():
    b = Batch([i % 37 for i in range(1500)], [(i * i) % 4 for i in range(1500)], 2, 1, 64, 8)
    append(b)
    b.check_pools()


def test_append_zero_vectors_and_large_values():
    """A head of zeros stays zeros under the norm; values near the type's limit do not overflow its mean."""
    import torch
    b = Batch([3], [4], 2, 1, 64, 8, "bf16")
    b.nk[0] = 0
    b.nk[1] = 1e18
    w = torch.ones(64, dtype=b.k.dtype, device="cuda")
    append(b, k_norm=w, eps=1e-6)
    k, near = turned(b.nk, None, None, None, False, w, 1e-6)
    b.check_pools(k, near)


def test_append_bad_rows_are_left_out():
    import torch
    b = Batch([40, 40, 40, 40, 40], [2, 2, 2, 2, 20], 4, 2, 64, 16)
    cos, sin = tables(b, 64)
    lens, table, before = b.lens.clone(), b.table.clone(), (b.k.clone(), b.v.clone())
    b.table[0, 2] = b.k.shape[0]
    b.table[1, 2] = -5
    b.lens[2] = -1
    b.lens[3] = b.table.shape[1] * 16 - 1
    q_out = torch.full_like(b.out, 7.0)
    append(b, q=b.q, q_out=q_out, cos=cos[:59].contiguous(), sin=sin[:59].contiguous())  # row 4's last position is 59
    assert b.status.tolist() == [7] * 5
    assert bool((q_out[:8] == 7).all()) and bool((q_out[8:27] != 7).any()) and bool((q_out[27] == 7).all())
    b.lens, b.table = lens, table
    for r in range(4):
        at = b.places(r, 40, 2)
        assert bool(b.k[at].isnan().all()) and bool(b.v[at].isnan().all())
    at = b.places(4, 40, 20)
    assert not bool(b.v[at][:19].isnan().any()) and bool(b.v[at][19].isnan().all())
    append(b, cos=cos, sin=sin)
    k, near = turned(b.nk, positions(b), cos, sin, False, None, 0)
    b.check_pools(k, near)


def test_refusals_of_the_binding():
    import torch
    b = Batch([3, 4], [1, 1], 4, 2, 64, 16)
    G = b.G
    with pytest.raises(AssertionError):
        G.grid_kv_attend(b.kv, b.table, b.lens, b.q.float(), b.out, b.status)
    with pytest.raises(AssertionError):
        G.grid_kv_attend(b.kv, b.table.long(), b.lens, b.q, b.out, b.status)
    with pytest.raises(AssertionError):
        G.grid_kv_attend(b.kv, b.table, b.lens, b.q[:, :2], b.out, b.status)
    with pytest.raises(AssertionError):
        G.grid_kv_append(b.kv, b.table, b.lens, b.nk, b.nv, b.status, q=b.q)
    with pytest.raises(AssertionError):
        G.grid_kv_append(b.kv, b.table, b.lens, b.nk, b.nv, b.status, start=b.start[:2])
    odd = torch.zeros((3, 4, 2, 65), dtype=b.k.dtype, device="cuda")[..., :64]
    with pytest.raises(G.GridError):  # (rows of 65 elements: no multiple of 8)
        G.PagedKV(odd, odd, 4)
    with pytest.raises(G.GridError):
        G.PagedKV(b.k, b.v, 5)
    with pytest.raises(G.GridError):
        G.grid_kv_attend(b.kv, b.table, b.lens, b.q, b.out, b.status, scale=math.inf)
    with pytest.raises(G.GridError):
        G.grid_kv_attend(b.kv, b.table, b.lens, b.qkv.flatten(1)[:, 4:4 + 4 * 64].view(2, 4, 64), b.out, b.status)


CHUNK = [dict(d_table=None), dict(d_len=None), dict(B=0), dict(B=-1), dict(n_tokens=-1), dict(max_pages=0), dict(table_stride=2),
         dict(d_start=None, n_tokens=1), dict(max_pages=1 << 30, table_stride=1 << 31)]


@pytest.mark.parametrize("what,bad,code", [("chunk", c, -1) for c in CHUNK] + [
    ("chunk", dict(B=65_536), -8), ("heads", dict(d=None), -1), ("heads", dict(d=(1 << 20) + 8), -1),
    ("heads", dict(token_stride=260), -1), ("heads", dict(head_stride=-64), -1), ("rot", dict(d_cos=None), -1),
    ("rot", dict(d_sin=(1 << 20) + 4), -1), ("rot", dict(rot=8), -1), ("rot", dict(rot=24), -1), ("rot", dict(rot=80), -1),
    ("rot", dict(n_pos=0), -1), ("norm", dict(d_q=(1 << 20) + 2), -1), ("norm", dict(eps=-1.0), -1),
    ("norm", dict(eps=math.nan), -1), ("query", dict(scale=0.0), -1), ("query", dict(scale=-1.0), -1),
    ("query", dict(scale=math.nan), -1), ("query", dict(d_lse=(1 << 20) + 2), -1), ("status", {}, -1)])
def test_calls_that_are_refused(what, bad, code):
    """Refused on the host, before anything is launched (the addresses here are never read)."""
    import ctypes
    from paper_2607_11951_gb300 import grid as G
    from tests import structs as S
    b = Batch([3, 4], [1, 1], 4, 2, 64, 16)
    at = 1 << 20
    parts = dict(chunk=S.KvChunk(at, 3, at, at, 3, 2, 2, 0), heads=S.Heads(at, 256, 64), rot=S.Rotation(at, at, 9, 64, 0, 0),
                 norm=S.HeadNorm(at, at, 1e-6, 0))
    parts["query"] = S.KvQuery(S.Heads(at, 256, 64), S.Heads(at, 256, 64), None, 0.125, 0)
    for k, v in bad.items():
        setattr(parts[what], k, v)
    if what == "heads":
        parts["query"].q = parts["heads"]
    p = {k: ctypes.byref(v) for k, v in parts.items()}
    status = None if what == "status" else at
    L, good = G.lib(), ctypes.byref(S.Heads(at, 256, 64))
    if what != "query":
        for where in range(4) if what == "heads" else [0]:
            args = [good] * 4
            args[where] = p["heads"]
            assert L.grid_kv_append(b.kv.h, p["chunk"], *args, p["rot"], p["norm"], status, None) == code
            assert G.last_error().startswith("grid_kv_append:")
    if what in ("chunk", "heads", "query", "status"):
        assert L.grid_kv_attend(b.kv.h, p["chunk"], p["query"], status, None) == code
        assert G.last_error().startswith("grid_kv_attend:")
    if what == "status":
        assert L.grid_kv_append(b.kv.h, p["chunk"], good, good, good, None, None, None, at, None) == -1  # q without q_out


def test_too_many_tiles_in_one_call():
    import ctypes
    from paper_2607_11951_gb300 import grid as G
    from tests import structs as S
    b = Batch([3, 4], [1, 1], 4, 2, 64, 16)
    at = 1 << 20
    chunk = S.KvChunk(at, 1 << 26, at, at, 1 << 26, 2, 1 << 28, 0)
    query = S.KvQuery(S.Heads(at, 256, 64), S.Heads(at, 256, 64), None, 0.125, 0)
    assert G.lib().grid_kv_attend(b.kv.h, ctypes.byref(chunk), ctypes.byref(query), at, None) == -8


def test_pages_of_other_rows_and_stale_tables_are_not_read():
    """Entries of the table past a row's tokens may hold anything; two rows may share a page of a common prefix."""
    import torch
    b = Batch([64, 64, 64], [5, 1, 150], 8, 2, 128, 64)
    b.fill()
    b.table[1, 0] = b.table[0, 0]  # rows 0 and 1 begin with the same 64 tokens
    b.cached[1] = b.cached[0]
    b.table[:, 4:] = torch.tensor([[-1], [1 << 30], [-(1 << 31)]], dtype=torch.int32, device="cuda")
    b.attend()
    b.check()
