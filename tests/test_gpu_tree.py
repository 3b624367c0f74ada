"""Trees of drafted tokens: grid_tree_plan and grid_tree_accept against plain
Python, grid_kv_append with depths and grid_kv_attend with visibility bits
against the formulas in 64 bits, grid_kv_compact bit for bit; shapes from one
token to many tiles, forests, arbitrary bits, bits that leave a token nothing to
see, bad trees, other streams and captured graphs."""
import math
import random

import pytest

from tests.test_gpu_kv import LAYOUTS, TINY, UNIT, Batch, append, tables, turned

pytestmark = pytest.mark.gpu

OK, COMPLETE, PAGES, TREE = 0, 6, 7, 8


def ints(x):
    import torch
    return torch.tensor(x, dtype=torch.int32).cuda()


def tree(n, rng, kind="tree"):
    """Parents of n tokens."""
    if kind == "chain":
        return [i - 1 for i in range(n)]
    if kind == "star":
        return [-1] + [0] * (n - 1) if n else []
    if kind == "forest":
        return [rng.randint(-1, i - 1) if rng.random() < 0.7 else -1 for i in range(n)]
    return [max(-1, i - 1 - int(rng.expovariate(0.4))) if i and rng.random() < 0.7 else rng.randint(0, i - 1) if i else -1
            for i in range(n)]


def lines(parent):
    """Per token its ancestors and itself."""
    out = []
    for i, p in enumerate(parent):
        out.append((out[p] if p >= 0 else []) + [i])
    return out


def packed(trees, words):
    """Bits of the rows' tokens as grid_tree_plan's words."""
    rows = []
    for t in trees:
        for line in lines(t):
            w = [0] * words
            for j in line:
                w[j >> 5] |= 1 << (j & 31)
            rows.append([x - (1 << 32) if x >> 31 else x for x in w])
    return ints(rows).view(-1, words)


class Trees(Batch):
    def __init__(self, old, new, *a, kind="tree", words=None, **kw):
        super().__init__(old, new, *a, **kw)
        rng = random.Random(sum(new) + len(old))
        self.trees = [tree(n, rng, kind) for n in new]
        self.words = words or max(1, -(-max(new) // 32))
        self.parent = ints([p for t in self.trees for p in t])
        self.sees = packed(self.trees, self.words)
        self.see_trees()

    def see_trees(self):
        import torch
        self.seen = []  # per row [n, n]
        for t in self.trees:
            m = torch.zeros((len(t), len(t)), dtype=torch.bool)
            for i, line in enumerate(lines(t)):
                m[i, line] = True
            self.seen.append(m.cuda())

    def see_bits(self, bits):
        """Arbitrary bits [n, n] per row; those of later tokens do not count."""
        import torch
        rows, self.seen = [], []
        for m in bits:
            full = torch.zeros((m.shape[0], 32 * self.words), dtype=torch.int64, device="cuda")
            full[:, :m.shape[1]] = m
            w = (full.view(m.shape[0], self.words, 32) << torch.arange(32, device="cuda")).sum(-1)
            rows.append(torch.where(w >= 1 << 31, w - (1 << 32), w).int())
            self.seen.append(m & torch.ones_like(m).tril())
        self.sees = torch.cat(rows).contiguous()

    def attend(self, **kw):
        super().attend(sees=self.sees, **kw)

    def check(self, scale=None, rows=None):
        """As Batch.check, with the tokens' own keys."""
        import torch
        scale = self.D ** -0.5 if scale is None else scale
        unit, a = UNIT[self.dt], 0
        group = self.H // self.Hk
        for b, n in enumerate(self.new):
            z = a + n
            if n and (rows is None or b in rows):
                k = torch.cat([self.cached[b][0], self.nk[a:z]]).double().repeat_interleave(group, 1)
                v = torch.cat([self.cached[b][1], self.nv[a:z]]).double().repeat_interleave(group, 1)
                q = self.q[a:z].double()
                x = torch.einsum("thd,jhd->htj", q, k) * scale
                d = self.D * 2.0 ** -23 * scale * torch.einsum("thd,jhd->htj", q.abs(), k.abs()).max().item() + 2.0 ** -18
                seen = torch.cat([torch.ones((n, self.old[b]), dtype=torch.bool, device="cuda"), self.seen[b]], 1)
                x = x.masked_fill(~seen, -math.inf)
                none = ~seen.any(1)
                lse = x.logsumexp(2)
                p = torch.where(none[None, :, None], 0.0, (x - lse[..., None]).exp())
                want = torch.einsum("htj,jhd->thd", p, v)
                near = unit * want.abs() + (unit + 2 * d) * torch.einsum("htj,jhd->thd", p, v.abs()) + TINY
                near[none] = 0
                off = (self.out[a:z].double() - want).abs() - near
                assert bool((off <= 0).all()), (b, float(off.max()), torch.nonzero(off > 0)[:4].tolist())
                got = self.lse[a:z]
                assert bool((got[none] == -math.inf).all())
                off = ((got.double() - lse.T).abs() - d - 2.0 ** -20 * (1 + lse.T.abs()))[~none]
                assert bool((off <= 0).all()), (b, "lse", float(off.max()))
                assert int(self.status[b]) == 0
            a = z


# ---------------------------------------------------------------------------
@pytest.mark.parametrize("new,words", [([1], 1), ([8], 1), ([32, 0, 31, 33, 1], 2), ([128] * 5, 4), ([3, 64, 65, 96, 100], 5),
                                       ([1024, 0, 1, 999], 32), ([i % 7 for i in range(300)], 1)])
@pytest.mark.parametrize("kind", ["tree", "chain", "star", "forest"])
def test_plan(new, words, kind):
    import torch
    from paper_2607_11951_gb300 import grid as G
    rng = random.Random(words)
    trees = [tree(n, rng, kind) for n in new]
    N = sum(new)
    parent, start = ints([p for t in trees for p in t]), ints([sum(new[:b]) for b in range(len(new) + 1)])
    depth, sees = torch.full((N,), -9, device="cuda").int(), torch.full((N, words), -9, device="cuda").int()
    status = torch.full((len(new),), -9, device="cuda").int()
    G.grid_tree_plan(parent, depth, sees, status, start=start)
    assert status.tolist() == [OK] * len(new)
    assert depth.tolist() == [len(line) - 1 for t in trees for line in lines(t)]
    assert torch.equal(sees, packed(trees, words))


def test_plan_uniform_rows_bad_trees_and_spare_tokens():
    import torch
    from paper_2607_11951_gb300 import grid as G
    parent = ints([-1, 0, 0, -1, 1, 0, -1, 2, 0, -1, -2, 0, -1, 0, 1])  # rows 1 (its own child), 2 (a later parent), 3 are bad
    depth, sees = torch.full((15,), -9, device="cuda").int(), torch.full((15, 1), -9, device="cuda").int()
    status = torch.full((5,), -9, device="cuda").int()
    G.grid_tree_plan(parent, depth, sees, status)
    assert status.tolist() == [OK, TREE, TREE, TREE, OK]
    assert depth.tolist() == [0, 1, 1] + [0] * 9 + [0, 1, 2]
    assert sees[:, 0].tolist() == [1, 3, 5] + [1, 2, 4] * 3 + [1, 3, 7]
    # a row of more tokens than its words hold and one out of order are left alone, as tokens of no row
    parent = torch.arange(-1, 49, device="cuda").int()
    depth, sees = torch.full((50,), -9, device="cuda").int(), torch.full((50, 1), -9, device="cuda").int()
    status = torch.full((4,), -9, device="cuda").int()
    G.grid_tree_plan(parent[:50], depth, sees, status, start=ints([0, 3, 40, 38, 47]))
    assert status.tolist() == [OK, TREE, TREE, TREE]  # (37 tokens; backwards; parents 37 .. of a row of 9)
    assert depth[:3].tolist() == [0, 1, 2] and depth[3:38].tolist() == [-9] * 35 and depth[47:].tolist() == [-9] * 3
    assert sees[38:47, 0].tolist() == [1 << i for i in range(9)]
    G.grid_tree_plan(parent[:0], depth[:0], sees[:0], status)
    assert status.tolist() == [OK] * 4


def walk(parent, tokens, sampled, most, eos):
    node, path, out = 0 if parent else -1, [], []
    while node >= 0 and len(path) < most:
        t = sampled[node]
        path.append(node)
        out.append(t)
        if t < 0 or (eos >= 0 and t == eos):
            break
        node = next((j for j in range(node + 1, len(parent)) if parent[j] == node and tokens[j] == t), -1)
    return path, out


@pytest.mark.parametrize("new,most", [([1], 1), ([8], 4), ([0, 3, 33, 64, 128, 0, 1], 9), ([129, 200, 700, 1], 40),
                                      ([(7 * i) % 65 for i in range(257)], 6)])
@pytest.mark.parametrize("kind", ["tree", "chain", "forest"])
def test_accept(new, most, kind):
    import torch
    from paper_2607_11951_gb300 import grid as G
    rng = random.Random(len(new) + most)
    trees = [tree(n, rng, kind) for n in new]
    # few different tokens, so that paths are long, siblings alike, and a child's token is often an uncle's
    tokens = [[rng.randrange(3) for _ in t] for t in trees]
    sampled = [[rng.choice([-1, 0, 0, 1, 1, 2, 2, 3]) for _ in t] for t in trees]
    B, flat = len(new), lambda x: ints([y for r in x for y in r])
    start = ints([sum(new[:b]) for b in range(B + 1)])
    for eos in (-1, 3, 1):
        path, out = (torch.full((B, most), -9, device="cuda").int() for _ in range(2))
        count, status = (torch.full((B,), -9, device="cuda").int() for _ in range(2))
        G.grid_tree_accept(flat(trees), flat(tokens), flat(sampled), path, count, out, status, start=start, eos=eos)
        for b in range(B):
            p, o = walk(trees[b], tokens[b], sampled[b], most, eos)
            assert path[b].tolist() == p + [-1] * (most - len(p)) and out[b].tolist() == o + [-1] * (most - len(o))
            assert int(count[b]) == len(p) and int(status[b]) == (COMPLETE if o and eos >= 0 and o[-1] == eos else OK)


def test_accept_rows_out_of_order():
    import torch
    from paper_2607_11951_gb300 import grid as G
    parent, tokens = ints([-1, 0, 1, -1, 0]), ints([5, 6, 7, 8, 9])
    path, out = (torch.full((3, 4), -9, device="cuda").int() for _ in range(2))
    count, status = (torch.full((3,), -9, device="cuda").int() for _ in range(2))
    G.grid_tree_accept(parent, tokens, ints([6, 7, 1, 9, 2]), path, count, out, status, start=ints([0, 3, 2, 6]))
    assert count.tolist() == [3, 0, 0] and status.tolist() == [OK, TREE, TREE]
    assert path.tolist() == [[0, 1, 2, -1], [-1] * 4, [-1] * 4] and out.tolist() == [[6, 7, 1, -1], [-1] * 4, [-1] * 4]


# ---------------------------------------------------------------------------
@pytest.mark.parametrize("heads,kv_heads,D", LAYOUTS)
@pytest.mark.parametrize("dt", ["bf16", "f16"])
def test_attend_small_trees_around_tiles(heads, kv_heads, D, dt):
    old = [0, 1, 15, 62, 63, 64, 119, 120, 121, 126, 127, 128, 129, 254, 256, 400, 1000]
    b = Trees(old, [8] * len(old), heads, kv_heads, D, 16, dt, seed=heads)
    b.fill()
    b.attend()
    b.check()


@pytest.mark.parametrize("heads,kv_heads,D", LAYOUTS)
@pytest.mark.parametrize("page,order,kind", [(8, "token", "tree"), (32, "head", "forest"), (128, "token", "star"), (64, "head", "chain")])
def test_attend_ragged_trees(heads, kv_heads, D, page, order, kind):
    new = [0, 1, 2, 5, 9, 16, 31, 32, 33, 64, 65, 127, 130, 0, 257, 3]
    old = [5, 0, 100, 0, 300, 127, 1, 250, 33, 0, 64, 0, 700, 126, 255, 2000]
    b = Trees(old, new, heads, kv_heads, D, page, order=order, seed=page, kind=kind, words=10)
    b.fill()
    b.attend()
    b.check()


@pytest.mark.parametrize("B,n,old,heads,kv_heads,D", [
    (1, 1, 16_001, 8, 1, 128), (2, 32, 9_000, 32, 8, 128), (1, 700, 5_000, 4, 1, 128), (3, 1000, 77, 2, 2, 64),
    (1, 1024, 0, 6, 2, 128), (40, 16, 3_000, 16, 8, 128), (1, 128, 3_000, 16, 1, 64), (200, 2, 130, 8, 2, 64)])
def test_attend_long_axes(B, n, old, heads, kv_heads, D):
    b = Trees([old - 3 * i if old > 3 * B else old for i in range(B)], [n] * B, heads, kv_heads, D, 64, seed=n)
    b.fill()
    b.attend()
    b.check()


@pytest.mark.parametrize("heads,kv_heads,D,dt", [(4, 2, 64, "bf16"), (7, 1, 128, "f16"), (3, 3, 64, "f16"), (16, 1, 128, "bf16")])
@pytest.mark.parametrize("share", [0.0, 0.03, 0.5, 1.0])
def test_attend_any_bits(heads, kv_heads, D, dt, share):
    """Bits that are no tree's: tokens that see nothing at all (where nothing is cached), or all before them."""
    import torch
    new = [1, 40, 0, 129, 300, 17, 130]
    b = Trees([0, 0, 9, 0, 0, 200, 127], new, heads, kv_heads, D, 16, dt, seed=3, words=11)
    g = torch.Generator(device="cuda")
    g.manual_seed(int(100 * share))
    b.see_bits([torch.rand((n, n), generator=g, device="cuda") < share for n in new])
    b.fill()
    b.attend()
    b.check()


def test_attend_a_chain_is_a_chunk_bit_for_bit():
    """A chain's bits, and no bits, hide the same keys."""
    import torch
    b = Trees([300, 0, 77, 1000], [70, 140, 1, 9], 8, 2, 128, 16, kind="chain")
    b.fill()
    b.attend()
    out, lse = b.out.clone(), b.lse.clone()
    Batch.attend(b)
    assert torch.equal(out, b.out) and torch.equal(lse, b.lse)


def test_attend_bits_past_the_row_and_of_later_tokens_do_not_count():
    import torch
    b = Trees([30, 0], [20, 50], 4, 2, 64, 16, words=3)
    b.fill()
    b.attend()
    out = b.out.clone()
    late = torch.full((70, 96), True, device="cuda")
    for a, n in ((0, 20), (20, 50)):
        late[a:a + n, :n] = ~torch.ones((n, n), dtype=torch.bool, device="cuda").tril()
    w = (late.view(70, 3, 32).long() << torch.arange(32, device="cuda")).sum(-1)
    b.sees |= torch.where(w >= 1 << 31, w - (1 << 32), w).int()
    b.attend()
    assert torch.equal(out, b.out)


def test_attend_rows_that_fail():
    import torch
    b = Trees([40, 40, 40, 0], [2, 33, 32, 4], 4, 2, 64, 16, words=2)
    b.fill()
    b.sees = b.sees[:, :1].contiguous()  # 32 tokens at most
    b.table[0, 1] = -1
    b.attend()
    assert b.status.tolist() == [PAGES, TREE, OK, OK]
    assert bool((b.out[:35] == 0).all()) and bool((b.lse[:35] == -math.inf).all())
    b.check(rows=[2, 3])


def test_attend_a_query_that_is_no_number():
    b = Trees([30, 0], [20, 50], 4, 2, 64, 16)
    b.fill()
    b.qkv[3, 1, 5] = math.nan
    b.attend()
    assert bool(b.out[3, 1].isnan().all()) and bool(b.lse[3, 1].isnan())
    b.out[3, 1], b.lse[3, 1] = 0, 0
    assert not bool(b.out.isnan().any()) and not bool(b.lse.isnan().any())


# ---------------------------------------------------------------------------
@pytest.mark.parametrize("heads,kv_heads,D,rot", [(8, 2, 64, 64), (14, 2, 64, 32), (32, 8, 128, 128), (5, 5, 128, 96)])
@pytest.mark.parametrize("pairs", [False, True])
@pytest.mark.parametrize("norm", [True, False])
@pytest.mark.parametrize("dt,order,page", [("bf16", "token", 16), ("f16", "head", 8)])
def test_append_turns_by_depth(heads, kv_heads, D, rot, pairs, norm, dt, order, page):
    import torch
    b = Trees([0, 5, 15, 16, 100, 3], [1, 0, 9, 20, 64, 0], heads, kv_heads, D, page, dt, order, seed=rot)
    cos, sin = tables(b, rot)
    qw, kw = [(1 + 0.3 * b.rand(D)).to(b.k.dtype) if norm else None for _ in range(2)]
    depth = [len(line) - 1 for t in b.trees for line in lines(t)]
    q_out = torch.full_like(b.out, 7.0)
    append(b, q=b.q, q_out=q_out, cos=cos, sin=sin, pairs=pairs, q_norm=qw, k_norm=kw, eps=1e-5, depth=ints(depth))
    pos = torch.tensor([o for o, n in zip(b.old, b.new) for _ in range(n)], device="cuda") + torch.tensor(depth, device="cuda")
    k, near = turned(b.nk, pos, cos, sin, pairs, kw, 1e-5)
    b.check_pools(k, near)
    q, near = turned(b.q, pos, cos, sin, pairs, qw, 1e-5)
    assert float(((q_out.double() - q).abs() - UNIT[dt] * q.abs() - near - TINY).max()) <= 0
    # (the depths of a chain are no news)
    pools = b.k.clone(), q_out.clone()
    chain = ints([i for n in b.new for i in range(n)])
    append(b, q=b.q, q_out=q_out, cos=cos, sin=sin, pairs=pairs, q_norm=qw, k_norm=kw, eps=1e-5, depth=chain)
    b.k, mine = b.k, (b.k.clone(), q_out.clone())
    append(b, q=b.q, q_out=q_out, cos=cos, sin=sin, pairs=pairs, q_norm=qw, k_norm=kw, eps=1e-5)
    assert torch.equal(mine[0].view(torch.int16), b.k.view(torch.int16)) and torch.equal(mine[1], q_out) and len(pools) == 2


def test_append_depths_outside_the_table():
    import torch
    b = Trees([10, 10, 10], [3, 3, 3], 4, 2, 64, 16)
    cos, sin = [x[:12].contiguous() for x in tables(b, 64)]  # positions up to 11
    append(b, cos=cos, sin=sin, depth=ints([0, 1, 1, 0, 1, 2, 0, -1, 1 << 30]))
    assert b.status.tolist() == [OK, PAGES, PAGES]
    at = [b.places(r, 10, 3) for r in range(3)]
    assert [b.v[x].isnan().all(-1).all(-1).tolist() for x in at] == [[False] * 3, [False, False, True], [False, True, True]]
    append(b, depth=ints([-5] * 9))  # (nothing is turned: depths are not read)
    assert b.status.tolist() == [OK] * 3
    b.check_pools()


# ---------------------------------------------------------------------------
@pytest.mark.parametrize("heads,D,page,order,dt", [(2, 64, 16, "token", "bf16"), (8, 128, 64, "head", "f16"), (1, 64, 8, "head", "bf16"),
                                                   (40, 128, 32, "token", "bf16"), (3, 128, 1024, "head", "f16")])
@pytest.mark.parametrize("most", [1, 7, 33, 100])
def test_compact(heads, D, page, order, dt, most):
    import torch
    rng = random.Random(most)
    new = [0, 1, 8, 64, 128, 33, 100, 5]
    b = Trees([0, 5, 63, 130, 1000, 7, 16, 0], new, heads, heads, D, page, dt, order)
    b.fill()
    paths = [sorted(rng.sample(range(n), rng.randint(0, min(n, most)))) for n in new]
    paths[3] = list(range(min(64, most)))  # nothing to move
    want = b.k.clone(), b.v.clone()
    for r, p in enumerate(paths):
        src = [b.places(r, b.old[r] + i, 1) for i in p]
        dst = b.places(r, b.old[r], len(p))
        for pool, new_pool in zip((b.k, b.v), want):
            if p:
                new_pool[dst] = torch.cat([pool[x] for x in src])
    path = ints([p + [-7] * (most - len(p)) for p in paths])
    b.G.grid_kv_compact(b.kv, b.table, b.lens, path, ints([len(p) for p in paths]), b.status, b.N, start=b.start)
    assert b.status.tolist() == [OK] * 8
    for pool, new_pool in zip((b.k, b.v), want):
        assert torch.equal(pool.view(torch.int16), new_pool.view(torch.int16))


def test_compact_rows_that_fail_are_left_as_they_were():
    import torch
    b = Trees([30] * 9, [8] * 9, 2, 2, 64, 16)
    b.fill()
    path = ints([[1, 3, 5], [0, 8, 9], [2, 2, 3], [3, 1, 2], [-1, 0, 1], [0, 2, 4], [0, 2, 4], [0, 2, 4], [0, 3, 9]])
    count = ints([3, 3, 3, 3, 3, 4, -1, 3, 2])
    b.table[7, 2] = 1 << 20
    was = b.k.clone(), b.v.clone()
    b.G.grid_kv_compact(b.kv, b.table, b.lens, path, count, b.status, b.N)
    assert b.status.tolist() == [OK, TREE, TREE, TREE, TREE, TREE, TREE, PAGES, OK]
    for pool, old in zip((b.k, b.v), was):
        for r, p in ((0, [1, 3, 5]), (8, [0, 3])):
            old[b.places(r, 30, len(p))] = torch.cat([old[b.places(r, 30 + i, 1)] for i in p])
        assert torch.equal(pool.view(torch.int16), old.view(torch.int16))
    b.lens[0] = -1
    b.G.grid_kv_compact(b.kv, b.table, b.lens, path, count, b.status, b.N)
    assert b.status.tolist()[0] == PAGES


# ---------------------------------------------------------------------------
def test_a_step_on_another_stream_and_captured():
    """Plan, append, attend, accept and compact as one graph, replayed on other inputs; two batches' graphs in turn."""
    import torch
    from paper_2607_11951_gb300 import grid as G

    class Step:
        def __init__(self, old, new, seed):
            b = self.b = Trees(old, new, 8, 2, 64, 16, seed=seed)
            self.depth, self.sees = torch.zeros(b.N, device="cuda").int(), torch.zeros_like(b.sees)
            self.tokens, self.sampled = (ints([random.Random(seed + x).randrange(2) for _ in range(b.N)]) for x in range(2))
            self.path, self.taken = (torch.zeros((b.B, 5), device="cuda").int() for _ in range(2))
            self.count = torch.zeros(b.B, device="cuda").int()
            self.cos, self.sin = tables(b, 64)
            self.q_out = torch.zeros_like(b.out)

        def run(self, stream=None):
            b = self.b
            G.grid_tree_plan(b.parent, self.depth, self.sees, b.status, start=b.start, stream=stream)
            G.grid_kv_append(b.kv, b.table, b.lens, b.nk, b.nv, b.status, start=b.start, q=b.q, q_out=self.q_out, cos=self.cos,
                             sin=self.sin, depth=self.depth, stream=stream)
            G.grid_kv_attend(b.kv, b.table, b.lens, self.q_out, b.out, b.status, lse=b.lse, start=b.start, sees=self.sees, stream=stream)
            G.grid_tree_accept(b.parent, self.tokens, self.sampled, self.path, self.count, self.taken, b.status, start=b.start,
                               stream=stream)
            G.grid_kv_compact(b.kv, b.table, b.lens, self.path, self.count, b.status, b.N, start=b.start, stream=stream)
            return [x.clone() for x in (self.depth, self.sees, self.q_out, b.out, b.lse, self.path, self.count, self.taken, b.status)] + \
                [x.clone().view(torch.int16) for x in (b.k, b.v)]

    same = lambda x, y: all(torch.equal(p, q) for p, q in zip(x, y))  # noqa: E731
    steps = [Step([100, 0, 33], [20, 7, 40], 1), Step([5, 400], [64, 3], 2)]
    want = [s.run() for s in steps]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = [s.run() for s in steps]
    torch.cuda.current_stream().wait_stream(side)
    assert all(same(x, y) for x, y in zip(want, got))
    graphs, outs = [torch.cuda.CUDAGraph() for _ in steps], []
    for s, gr in zip(steps, graphs):
        with torch.cuda.graph(gr):
            outs.append(s.run())
    for _ in range(2):
        for gr in graphs:
            gr.replay()
    assert all(same(x, y) for x, y in zip(want, outs))
    # other inputs in the same tensors
    s = steps[0]
    s.b.qkv.copy_(torch.randn_like(s.b.qkv.float()).to(s.b.qkv.dtype))
    s.sampled.fill_(1)
    s.tokens.fill_(1)
    graphs[0].replay()
    assert same(s.run(), outs[0])


def test_refusals_of_the_binding():
    import torch
    b = Trees([3, 4], [2, 3], 4, 2, 64, 16)
    G, i32 = b.G, dict(dtype=torch.int32, device="cuda")
    depth, sees, st = torch.zeros(5, **i32), torch.zeros((5, 1), **i32), torch.zeros(2, **i32)
    path, count = torch.zeros((2, 3), **i32), torch.zeros(2, **i32)
    for call in (lambda: G.grid_kv_attend(b.kv, b.table, b.lens, b.q, b.out, b.status, start=b.start, sees=sees[:4]),
                 lambda: G.grid_kv_attend(b.kv, b.table, b.lens, b.q, b.out, b.status, start=b.start, sees=sees[:, :0]),
                 lambda: G.grid_kv_attend(b.kv, b.table, b.lens, b.q, b.out, b.status, start=b.start, sees=sees.long()),
                 lambda: G.grid_kv_attend(b.kv, b.table, b.lens, b.q, b.out, b.status, start=b.start, sees=sees.cpu()),
                 lambda: append(b, depth=depth[:4]), lambda: append(b, depth=depth.float()), lambda: append(b, depth=depth.cpu()),
                 lambda: G.grid_tree_plan(b.parent.cpu(), depth, sees, st, start=b.start),
                 lambda: G.grid_tree_plan(b.parent, depth[:4], sees, st, start=b.start),
                 lambda: G.grid_tree_plan(b.parent, depth, sees[:4], st, start=b.start),
                 lambda: G.grid_tree_plan(b.parent, depth, sees, st, start=b.start[:2]),
                 lambda: G.grid_tree_accept(b.parent, depth, depth[:3], path, count, path.clone(), st, start=b.start),
                 lambda: G.grid_tree_accept(b.parent, depth, depth, path, count, path.T.contiguous(), st, start=b.start),
                 lambda: G.grid_tree_accept(b.parent, depth, depth, path[:1], count, path[:1], st, start=b.start),
                 lambda: G.grid_kv_compact(b.kv, b.table, b.lens, path[:1], count, b.status, 5, start=b.start),
                 lambda: G.grid_kv_compact(b.kv, b.table, b.lens, path, count.float(), b.status, 5, start=b.start)):
        with pytest.raises(AssertionError):
            call()
    with pytest.raises(G.GridError):
        G.grid_tree_plan(b.parent, depth, sees[:, :0].contiguous(), st, start=b.start)
    with pytest.raises(G.GridError):  # (five tokens of two rows alike)
        G.grid_tree_plan(b.parent, depth, sees, st)
