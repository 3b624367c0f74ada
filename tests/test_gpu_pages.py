"""grid_pages_update against the rules in plain Python over random states, and
grid_kv_copy bit for bit: forks, pages held in part, pins, short pools, rows that
begin and end, tables of other widths, bad rows, other streams and graphs."""
import random

import pytest

pytestmark = pytest.mark.gpu

OK, PAGES = 0, 7


def ints(x):
    import torch
    return torch.tensor(x, dtype=torch.int32).cuda()


def update(n_pages, page, table, held, parent, keep, want, pinned, width_out):
    """The rules, row by row."""
    A, B = len(held), len(want)
    rows = []
    for b in range(B):
        p = parent[b]
        ok = -1 <= p < A
        have = held[p] if ok and p >= 0 else 0
        k = keep[b] if ok and p >= 0 else 0
        pages = -(-k // page)
        ok = ok and 0 <= k <= have and want[b] >= k and pages <= min(len(table[0]), width_out)
        ids = table[p][:pages] if ok and p >= 0 else []
        ok = ok and all(0 <= x < n_pages for x in ids)
        rows.append((k, ids) if ok else None)
    whole = {x for r in rows if r for x in r[1][:r[0] // page]}
    first = {}
    for b, r in enumerate(rows):
        if r and r[0] % page:
            first.setdefault(r[1][-1], b)
    stays = {b for x, b in first.items() if x not in whole and not pinned[x]}
    taken = whole | {rows[b][1][-1] for b in stays}
    free = [x for x in range(n_pages) if x not in taken and not pinned[x]]
    used, out, held_out, copies, status = 0, [], [], [], []
    for b, r in enumerate(rows):
        if r is None:
            out.append([]), held_out.append(0), copies.append((-1, -1, 0)), status.append(PAGES)
            continue
        k, ids = r
        full, room = k // page, -(-want[b] // page)
        mine = ids if b in stays or k % page == 0 else ids[:full]
        fits = room <= width_out
        need = room - len(mine) if fits else 0
        if fits and need:
            fits = used + need <= len(free)
        fresh = free[used:used + need] if fits else []
        used += need
        out.append(mine + fresh)
        held_out.append(want[b] if fits else k if len(mine) == len(ids) else full * page)
        copied = fits and len(mine) < len(ids)
        copies.append((ids[-1], fresh[0], k % page) if copied else (-1, -1, 0))
        status.append(OK if fits else PAGES)
    refs = [0] * n_pages
    for r in out:
        for x in r:
            refs[x] += 1
    return [r + [-1] * (width_out - len(r)) for r in out], held_out, [list(x) for x in zip(*copies)], refs, status


class State:
    """A pool, a table of A rows, and what B new rows ask for."""

    def __init__(self, A, B, page, longest, seed=0, spare=1.0, bad=0.0, shared=0.3, pins=0.1, width_out=None):
        import torch
        rng = self.rng = random.Random(seed)
        held = [rng.choice([0, rng.randint(0, longest), rng.randint(0, longest)]) for _ in range(A)]
        need = [-(-h // page) for h in held]
        total = sum(need)
        self.want = []
        self.parent = [rng.choice([-1, rng.randrange(A), rng.randrange(A), b % A, b % A]) for b in range(B)]
        self.keep = [0 if p < 0 else rng.choice([held[p], rng.randint(0, held[p]), held[p] // page * page]) for p in self.parent]
        self.want = [k + rng.choice([0, 1, page, rng.randint(0, 3 * page)]) for k in self.keep]
        fresh = sum(-(-w // page) - k // page for w, k in zip(self.want, self.keep))
        self.n_pages = n = max(1, total + int(fresh * spare))
        ids = list(range(n))
        rng.shuffle(ids)
        self.width = max([1] + need) + rng.randint(0, 3)
        self.width_out = width_out or max([1] + [-(-w // page) for w in self.want])
        self.table = []
        for r in need:
            row = [ids.pop() for _ in range(r)]
            if self.table and rng.random() < shared:  # (a prefix of another row)
                other = rng.choice(self.table)
                m = rng.randint(0, min(r, sum(x >= 0 for x in other)))
                row[:m] = other[:m]
            self.table.append(row + [-1] * (self.width - r))
        self.pinned = [int(rng.random() < pins) for _ in range(n)]
        self.held, self.page = held, page
        for b in range(B):  # what is not valid
            if rng.random() < bad:
                kind = rng.randrange(5)
                if kind == 0:
                    self.parent[b] = rng.choice([A, -2, 1 << 30])
                elif kind == 1:
                    self.keep[b] = -1
                elif kind == 2 and self.parent[b] >= 0:
                    self.keep[b] = held[self.parent[b]] + 1
                    self.want[b] += 2
                elif kind == 3:
                    self.want[b] = self.keep[b] - 1
        for a in range(A):
            if rng.random() < bad / 2 and need[a]:
                self.table[a][rng.randrange(need[a])] = rng.choice([-1, n, 1 << 30])
        self.B = B
        i32 = dict(dtype=torch.int32, device="cuda")
        self.out = dict(table_out=torch.full((B, self.width_out), -9, **i32), held_out=torch.full((B,), -9, **i32),
                        copies=torch.full((3, B), -9, **i32), refs=torch.full((n,), -9, **i32), status=torch.full((B,), -9, **i32))
        self.t = dict(table=ints(self.table), held=ints(held), want=ints(self.want))
        self.more = dict(parent=ints(self.parent), keep=ints(self.keep), pinned=ints(self.pinned))

    def expect(self):
        return update(self.n_pages, self.page, self.table, self.held, self.parent, self.keep, self.want, self.pinned, self.width_out)

    def run(self, handle=None, stream=None):
        from paper_2607_11951_gb300 import grid as G
        self.handle = handle or G.Pages(self.n_pages, self.page)
        G.grid_pages_update(self.handle, **self.t, **self.out, **self.more, stream=stream)
        return [self.out[k] for k in ("table_out", "held_out", "copies", "refs", "status")]

    def check(self):
        for name, got, want in zip(("table", "held", "copies", "refs", "status"), [x.tolist() for x in self.run()], self.expect()):
            assert got == want, name


@pytest.mark.parametrize("A,B,page,longest", [(1, 1, 16, 40), (1, 4, 16, 400), (4, 1, 8, 100), (7, 9, 8, 30), (30, 33, 16, 60),
                                              (100, 80, 64, 2000), (256, 256, 16, 700), (3, 2000, 8, 40), (1100, 1030, 32, 90)])
@pytest.mark.parametrize("spare,bad", [(1.0, 0.0), (0.4, 0.0), (0.0, 0.0), (0.7, 0.3)])
def test_update(A, B, page, longest, spare, bad):
    for seed in range(3):
        State(A, B, page, longest, seed, spare, bad).check()


def test_update_a_large_pool():
    State(200, 256, 16, 12_000, 5, 0.9).check()


def test_update_a_table_that_is_too_short():
    for seed in range(4):
        State(40, 50, 8, 60, seed, 1.0, width_out=5).check()


def test_update_of_rows_that_go_on_as_they_are():
    """No parents, no keep, no pins: every row continues itself with all it holds."""
    s = State(20, 20, 16, 100, 3, 1.0, shared=0.0, pins=0.0)
    s.parent, s.keep = list(range(20)), list(s.held)
    s.want = [h + 5 for h in s.held]
    s.t["want"] = ints(s.want)
    s.more = {}
    s.width_out = s.width
    s.out["table_out"] = s.t["table"].clone().fill_(-9)
    s.check()
    assert s.out["copies"][0].tolist() == [-1] * 20
    # then one step after the other, old and new table in turn
    for _ in range(3):
        s.table, s.held = s.out["table_out"].tolist(), s.out["held_out"].tolist()
        s.t = dict(table=s.out["table_out"].clone(), held=s.out["held_out"].clone(), want=ints([min(16 * s.width, h + 1) for h in s.held]))
        s.keep, s.want = list(s.held), s.t["want"].tolist()
        s.check()


def test_update_wide_rows_strided_tables_graph_and_stream():
    import torch
    s = State(60, 70, 16, 300, 9, 0.8)
    want = s.expect()
    wide = torch.full((60, s.width + 5), 1 << 30, dtype=torch.int32, device="cuda")
    wide[:, :s.width] = s.t["table"]
    s.t["table"] = wide[:, :s.width]
    out = torch.full((70, s.width_out + 3), -5, dtype=torch.int32, device="cuda")
    s.out["table_out"] = out[:, :s.width_out]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = s.run(stream=side)
    torch.cuda.current_stream().wait_stream(side)
    assert [x.tolist() for x in got] == list(want) and bool((out[:, s.width_out:] == -5).all())
    for x in s.out.values():
        x.fill_(-9)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        s.run(s.handle)
    for _ in range(3):
        graph.replay()
    assert [x.tolist() for x in got] == list(want)


# ---------------------------------------------------------------------------
@pytest.mark.parametrize("Hk,D,page,order,dt", [(2, 64, 16, "token", "bf16"), (8, 128, 64, "head", "f16"), (1, 64, 8, "head", "bf16"),
                                                (40, 128, 1024, "token", "bf16"), (3, 128, 32, "head", "f16")])
@pytest.mark.parametrize("n", [1, 5, 300])
def test_copy(Hk, D, page, order, dt, n):
    import torch
    from paper_2607_11951_gb300 import grid as G
    rng = random.Random(n)
    n_pages = 2 * n + 3 if n * page < 10_000 else 40
    shape = (n_pages, page, Hk, D) if order == "token" else (n_pages, Hk, page, D)
    g = torch.Generator(device="cuda")
    g.manual_seed(n)
    t = torch.bfloat16 if dt == "bf16" else torch.float16
    bits = [torch.randint(-(1 << 15), 1 << 15, shape, generator=g, device="cuda", dtype=torch.int16) for _ in range(2)]
    pools = [p.view(t) if order == "token" else p.view(t).transpose(1, 2) for p in bits]
    ids = list(range(n_pages))
    rng.shuffle(ids)
    to, from_ = ids[:n_pages // 2], ids[n_pages // 2:]
    rows = []
    for i in range(n):
        if i >= len(to) or rng.random() < 0.3:
            rows.append((-1, rng.choice([-1, 0, 1 << 30]), rng.choice([0, -3, 1 << 30])))
        else:
            rows.append((rng.choice(from_), to[i], rng.choice([0, 1, page - 1, page, rng.randint(0, page)])))
    if n > 4:
        rows[1], rows[2], rows[3] = (n_pages, to[1], 1), (from_[0], -1, 1), (from_[0], to[3], page + 1)
    want = [p.clone() for p in pools]
    bad = []
    for i, (a, b, k) in enumerate(rows):
        bad.append(PAGES if a >= 0 and not (a < n_pages and 0 <= b < n_pages and 0 <= k <= page) else OK)
        if a >= 0 and bad[-1] == OK:
            for p, w in zip(pools, want):
                w[b, :k] = p[a, :k]
    kv = G.PagedKV(*pools, Hk)
    status = torch.full((n,), -9, dtype=torch.int32, device="cuda")
    G.grid_kv_copy(kv, ints([list(x) for x in zip(*rows)]), status)
    assert status.tolist() == bad
    for p, w in zip(pools, want):
        assert torch.equal(p.view(torch.int16), w.view(torch.int16))


def test_copy_past_32_bits_and_keys_and_values_of_other_strides():
    import torch
    from paper_2607_11951_gb300 import grid as G
    page, Hk, D = 64, 8, 128
    n = (1 << 31) // (page * Hk * D) + 4
    k = torch.zeros((n, page, Hk, D), dtype=torch.bfloat16, device="cuda")
    v = torch.zeros((n, Hk, page, D), dtype=torch.bfloat16, device="cuda").transpose(1, 2)
    for p in (k, v):
        p[0] = torch.randn((page, Hk, D), device="cuda").bfloat16()
        p[n - 2] = torch.randn((page, Hk, D), device="cuda").bfloat16()
    status = torch.zeros(2, dtype=torch.int32, device="cuda")
    G.grid_kv_copy(G.PagedKV(k, v, Hk), ints([[0, n - 2], [n - 1, 1], [64, 63]]), status)
    for p in (k, v):
        assert torch.equal(p[n - 1], p[0]) and torch.equal(p[1, :63], p[n - 2, :63]) and bool((p[1, 63] == 0).all())
    assert status.tolist() == [OK, OK]


def test_forks_read_what_their_parent_wrote():
    """A row parts in three in the middle of a page; each goes on for itself and attends to all of its tokens."""
    import torch
    from paper_2607_11951_gb300 import grid as G
    g = torch.Generator(device="cuda")
    g.manual_seed(0)
    rand = lambda *s: torch.randn(s, generator=g, device="cuda").bfloat16()  # noqa: E731
    Hk, H, D, page, n_pages = 2, 4, 64, 16, 20
    kv = G.PagedKV(rand(n_pages, page, Hk, D), rand(n_pages, page, Hk, D), H)
    pages = G.Pages(n_pages, page)
    i32 = dict(dtype=torch.int32, device="cuda")
    new = lambda B: dict(table_out=torch.zeros((B, 8), **i32), held_out=torch.zeros(B, **i32), copies=torch.zeros((3, B), **i32),  # noqa: E731
                         refs=torch.zeros(n_pages, **i32), status=torch.zeros(B, **i32))
    table, held = torch.full((1, 8), -1, **i32), ints([0])
    said = [[]]  # per row the keys and values that it was given
    for parent, n in (([-1], 37), ([0, 0, 0], 5), ([2, 0, 0, 1], 20), ([1, -1, 3], 1)):
        B = len(parent)
        o = new(B)
        keep = [len(said[p]) if p >= 0 else 0 for p in parent]
        G.grid_pages_update(pages, table, held, ints([k + n for k in keep]), **o, parent=ints(parent))
        assert o["status"].tolist() == [OK] * B
        G.grid_kv_copy(kv, o["copies"], torch.zeros(B, **i32))
        table, held = o["table_out"], o["held_out"]
        k, v, q = rand(B * n, Hk, D), rand(B * n, Hk, D), rand(B * n, H, D)
        said = [(list(said[p]) if p >= 0 else []) + [(k[b * n + i], v[b * n + i]) for i in range(n)] for b, p in enumerate(parent)]
        st, out = torch.zeros(B, **i32), torch.zeros_like(q)
        G.grid_kv_append(kv, table, ints(keep), k, v, st)
        G.grid_kv_attend(kv, table, ints(keep), q, out, st)
        assert st.tolist() == [OK] * B
        for b in range(B):
            ks, vs = (torch.stack([x[y] for x in said[b]]).double().repeat_interleave(H // Hk, 1) for y in (0, 1))
            last = (b + 1) * n - 1
            x = torch.einsum("hd,jhd->hj", q[last].double(), ks) / 8
            want = torch.einsum("hj,jhd->hd", x.softmax(1), vs)
            # (bf16 probabilities and result: half a step each, of up to sum p |v|; scores off by 64 products' 2^-24 of up to 64 x 16)
            near = (2.0 ** -7 + 2.0 ** -12) * torch.einsum("hj,jhd->hd", x.softmax(1), vs.abs())
            assert bool(((out[last].double() - want).abs() <= near).all())


def test_refusals_of_the_binding():
    import torch
    from paper_2607_11951_gb300 import grid as G
    s = State(3, 4, 16, 60, 1)
    h = G.Pages(s.n_pages, 16)
    args = {**s.t, **s.out, **s.more}
    G.grid_pages_update(h, **args)
    for bad in (dict(table=s.t["table"].long()), dict(table=s.t["table"].cpu()), dict(held=s.t["held"][:2]), dict(want=s.t["want"].float()),
                dict(table_out=s.out["table_out"][:3]), dict(held_out=s.out["held_out"][:3]), dict(copies=s.out["copies"].T.contiguous()),
                dict(refs=s.out["refs"][:-1]), dict(status=s.out["status"].cpu()), dict(parent=s.more["parent"][:2]),
                dict(keep=s.more["keep"].long()), dict(pinned=s.more["pinned"][:-1]),
                dict(table_out=torch.zeros((7, 4), dtype=torch.int32, device="cuda").T)):
        with pytest.raises(AssertionError):
            G.grid_pages_update(h, **{**args, **bad})
    with pytest.raises(AssertionError):  # (the new table in the old one's place)
        G.grid_pages_update(h, **{**args, "table": s.out["table_out"], "held": s.out["held_out"], "parent": None, "keep": None})
    with pytest.raises(G.GridError):  # (more rows than there are to go on)
        G.grid_pages_update(h, **{**args, "parent": None})
    with pytest.raises(G.GridError):
        G.Pages(10, 24)
    kv = G.PagedKV(*[torch.zeros((4, 16, 1, 64), dtype=torch.bfloat16, device="cuda") for _ in range(2)], 1)
    with pytest.raises(AssertionError):
        G.grid_kv_copy(kv, s.out["copies"].T.contiguous(), s.out["status"])
    with pytest.raises(AssertionError):
        G.grid_kv_copy(kv, s.out["copies"], s.out["status"].cpu())
