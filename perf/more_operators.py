"""Measured cases: a tree of drafted tokens, sampling, and the pages of a cache.

A drafter that proposes several continuations at once hands the model a tree of
tokens instead of a chain, a sampler draws from a truncated distribution, and
rows that fork, grow and end share the pages of one cache.  A step of such a
loop calls, in this order:

  grow    ``grid_tree_plan`` and ``grid_kv_append``: depths and visibility of
          the tree's tokens, then their keys and values into the paged cache,
          rotated by their depth in the tree
  tree    ``grid_kv_attend`` with the tree's visibility
  sample  ``grid_sample``: one token a row from the masked distribution at a
          temperature, cut by top-k, top-p and min-p, from given random numbers
  keep    ``grid_tree_accept`` and ``grid_kv_compact``: the tree's path that the
          sampled tokens take, and its keys and values moved next to the cache
  fork    ``grid_pages_update`` and ``grid_kv_copy``: rows continue other rows
          (or themselves), share their full pages, give back what they no
          longer need, and get pages for their next tokens

``own`` is false: ``run`` computes the operators from elementary torch
operations, rounded once at the end.  ``own`` is true: ``run`` makes the calls
of the public binding (``paper_2607_11951_gb300.grid``).

Formulas.
  plan    token i of a row's tree has a parent p < i, or -1: depth_i is its
          number of ancestors, bit j of sees_i is set for its ancestors and itself
  append  place len + i, angle of position len + depth_i; norm and rotation:
          x_d <- x_d w_d / sqrt(mean(x^2) + eps), (x_m, x_m+R/2) turned by (c, s)
  attend  out = sum_j p_j v_j, p = softmax_j(scale q.k_j) over the cached j and
          the chunk's j whose bit is set; lse = log sum_j exp(scale q.k_j)
  sample  ids ordered by logit, the largest first, then by id; p = softmax(l / T)
          over the admitted; kept are the first n: n1 = top_k, n2 the least n
          whose sum reaches top_p times the sum of the first n1, n3 the number
          with p >= min_p p_max, n = max(1, min(n1, n2, n3)); the token is
          argmax p_i / e_i over the kept (T <= 0: the first id)
  accept  from token 0 on: the child whose token was sampled at its parent
  compact kv[len + j] <- kv[len + path_j]
  update  new row b keeps `keep` tokens of old row parent_b (-1: of none) and gets
          pages for `want`: whole pages are shared; a page kept in part stays with the
          lowest row where nobody else holds it, and is copied to a fresh one
          otherwise; fresh pages are the lowest-numbered free ones, in the rows'
          order, up to the first row whose pages are not there
"""
import math
import random

import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
EPS = 1e-6  # of the norms
SPARE = 7   # pages of the pool that no row owns


# ---------------------------------------------------------------------------
# cases
def listed():
    return [
        # one interactive request over the expression grammar's vocabulary: launch latency
        dict(name="sample_expr_b1", kind="sample", B=1, V=512, dtype="f32", cut="mixed", mask=True, greedy=False),
        # the benchmark's batch and vocabulary, every request with its own settings
        dict(name="sample_sql_b32_f32", kind="sample", B=32, V=151_936, dtype="f32", cut="mixed", mask=True, greedy=False),
        # the nodes of many small trees, or the largest batch: rows off the sector boundaries, wide nuclei, some rows greedy
        dict(name="sample_nodes_b256_bf16", kind="sample", B=256, V=151_937, dtype="bf16", cut="top_p", mask=True, greedy=True),
        # one interactive request's tree in a small model
        dict(name="grow_tree_b1", kind="grow", B=1, n=8, ctx=400, heads=8, kv_heads=2, D=64, page=16, dtype="bf16",
             order="token", norm=False, depth=4),
        # a serving batch's trees, queries and keys normed per head
        dict(name="grow_trees_b32", kind="grow", B=32, n=64, ctx=2000, heads=32, kv_heads=8, D=128, page=64, dtype="bf16",
             order="head", norm=True, depth=6),
        # the interactive request's attention
        dict(name="tree_b1", kind="tree", B=1, n=8, ctx=400, heads=8, kv_heads=2, D=64, page=16, dtype="bf16",
             order="token", depth=4),
        # an odd batch of ragged trees, seven query heads to a key head
        dict(name="tree_b27", kind="tree", B=27, n=61, ctx=2000, heads=14, kv_heads=2, D=64, page=32, dtype="f16",
             order="head", depth=8),
        # the benchmark's batch with long generations
        dict(name="tree_b32_long", kind="tree", B=32, n=32, ctx=16_000, heads=32, kv_heads=8, D=128, page=64, dtype="bf16",
             order="token", depth=6),
        # the interactive request's accepted path
        dict(name="keep_path_b1", kind="keep", B=1, n=8, ctx=400, kv_heads=2, D=64, page=16, dtype="bf16", order="token",
             depth=4),
        # the largest batch of trees
        dict(name="keep_paths_b256", kind="keep", B=256, n=64, ctx=2000, kv_heads=8, D=128, page=16, dtype="bf16",
             order="head", depth=8),
        # a prompt's four samples part ways: a few pages of a small model
        dict(name="fork_b4", kind="fork", A=1, B=4, n=4, ctx=400, kv_heads=2, D=64, page=16, dtype="bf16", order="token",
             each=4, short=False),
        # beams of a large batch: every other row goes on twice, the rest end
        dict(name="fork_b256", kind="fork", A=256, B=256, n=8, ctx=2000, kv_heads=8, D=128, page=64, dtype="bf16",
             order="head", each=2, short=False),
    ]


def _spread(rng, lo, hi):
    """An integer spread evenly over the logarithm of [lo, hi]."""
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["sample", "sample", "grow", "tree", "tree", "keep", "fork"])
    most = [max(x) for x in zip(*[_cost(c) for c in listed() if c["kind"] == kind])]
    while True:
        c = _draw(rng, kind)
        if all(x <= y for x, y in zip(_cost(c), most)):
            return c


def _cost(c):
    """Bytes and operations of a pass, values of the pool, and the scores that
    the plain attention holds at once (all rows padded to the longest)."""
    w = work(c)
    if c["kind"] == "sample":
        return w["bytes"], w["flops"], 0, 0
    if c["kind"] == "fork":
        held = _forked(c)[0]
        return w["bytes"], w["flops"], (sum(held) + c["B"] * (c["n"] + 2 * c["page"])) * c["kv_heads"] * c["D"], 0
    new, old = _lengths(c)
    return (w["bytes"], w["flops"], (sum(new) + sum(old)) * c["kv_heads"] * c["D"],
            c["B"] * c["heads"] * c["n"] * (c["ctx"] + c["n"]) if c["kind"] == "tree" else 0)


def _draw(rng, kind):
    if kind == "sample":
        return dict(kind=kind, B=_spread(rng, 1, 256), V=_spread(rng, 500, 151_937), dtype=rng.choice(["f32", "bf16"]),
                    cut=rng.choice(["none", "top_k", "top_p", "min_p", "mixed"]), mask=rng.random() < 0.7,
                    greedy=rng.random() < 0.3)
    c = dict(kind=kind, B=_spread(rng, 1, 256), ctx=rng.choice([0, _spread(rng, 50, 2000), _spread(rng, 50, 16_000)]),
             kv_heads=rng.choice([1, 2, 3, 4, 8]), D=rng.choice([64, 128]), page=rng.choice([16, 32, 64, 128]),
             dtype=rng.choice(["bf16", "f16"]), order=rng.choice(["token", "head"]))
    if kind == "fork":
        c.update(A=_spread(rng, 1, 256), n=_spread(rng, 1, 16), each=rng.choice([1, 2, 3, 5]), short=rng.random() < 0.2)
        return c
    c.update(n=_spread(rng, 2, 128), depth=rng.randint(1, 12))
    if kind != "keep":
        c.update(heads=c["kv_heads"] * rng.choice([1, 2, 3, 4, 7, 8, 16]))
    if kind == "grow":
        c.update(norm=rng.random() < 0.5)
    return c


def _lengths(c):
    """Per row the tree's tokens (0 to n of them in a batch) and the cached ones before them, from ctx / 16 to ctx."""
    B, n, ctx = c["B"], c["n"], c["ctx"]
    new = [n] if B == 1 else [(n + i * (n // 2 + 1)) % (n + 1) for i in range(B)]
    old = [int(ctx * 16.0 ** (-i / (B - 1))) for i in range(B)] if B > 1 else [ctx]
    return new, old


def _paths(c):
    """Per row how many tokens of its tree are kept, and how many of those lie elsewhere: a row of the batch keeps one to
    `depth` + 1 of its tokens, and leaves the first chain half way."""
    new = _lengths(c)[0]
    kept = [min(n, 1 + (3 * i) % (c["depth"] + 1)) if n else 0 for i, n in enumerate(new)]
    # the chain holds tokens 0 .. depth; the rest of the tree hangs on it
    return kept, [k - 1 - (k - 1) // 2 if n > 2 * (c["depth"] + 1) else 0 for k, n in zip(kept, new)]


def _forked(c):
    """Tokens that the old rows hold; per new row its parent, what it keeps of it and what it wants.  Every row that goes
    on does so `each` times (rejected drafts leave it 0 to 4 tokens shorter), some new rows begin anew or are empty."""
    A, B, ctx = c["A"], c["B"], c["ctx"]
    held = [int(ctx * 16.0 ** (-i / (A - 1))) + c["n"] for i in range(A)] if A > 1 else [ctx + c["n"]]
    parent = [(b // c["each"] * c["each"]) % A if B == 1 or b % 17 != 16 else -1 for b in range(B)]
    keep = [max(0, held[p] - p % 5) if p >= 0 else 0 for p in parent]
    want = [k + c["n"] if p >= 0 or b % 2 else 0 for b, (k, p) in enumerate(zip(keep, parent))]
    return held, parent, keep, want


def work(case):
    c = case
    if c["kind"] == "sample":
        B, V = c["B"], c["V"]
        size = 4 if c["dtype"] == "f32" else 2
        # logits and masks; the noise of what is kept, which may be a few ids (all of them where nothing is cut)
        b = B * (V * size + ((V + 31) // 32 * 4 if c["mask"] else 0) + (V * 4 if c["cut"] == "none" else 0) + 32)
        return {"bytes": b, "flops": B * V * 4}
    Hk, D = c["kv_heads"], c["D"]
    if c["kind"] == "fork":
        held, parent, keep, want = _forked(c)
        page = c["page"]
        seen, copied = set(), 0
        for p, k in zip(parent, keep):
            copied += k % page if p in seen else 0
            seen.add(p)
        used = sum(-(-h // page) for h in held)
        width = max(-(-x // page) for x in held + want) or 1
        return {"bytes": 2 * copied * Hk * D * 4 + 4 * (used + c["B"] * width + _pool(c) + 4 * c["B"] + 4 * c["A"]), "flops": 0}
    new, old = _lengths(c)
    N, W = sum(new), (max(new) + 31) // 32
    if c["kind"] == "keep":
        kept, moved = _paths(c)
        return {"bytes": 2 * sum(moved) * Hk * D * 4 + 3 * 4 * N + 4 * c["B"] * (2 * (c["depth"] + 1) + 4), "flops": 0}
    H = c["heads"]
    if c["kind"] == "grow":
        return {"bytes": 2 * N * (H + 2 * Hk) * D * 2 + N * (4 + 4 + 4 * W) + (max(o + c["depth"] for o in old) - min(old)) * D * 4
                + 12 * c["B"], "flops": N * (H + Hk) * (3 * D + (4 * D if c["norm"] else 0))}
    pairs = sum(n * (o + min(n, c["depth"])) for o, n in zip(old, new))
    kv = sum(o + n for o, n in zip(old, new) if n)
    return {"bytes": 2 * kv * Hk * D * 2 + 2 * N * H * D * 2 + N * H * 4 + N * W * 4 + 12 * c["B"], "flops": pairs * H * (4 * D + 4)}


# ---------------------------------------------------------------------------
# inputs
def _randn(g, shape, dtype, scale=1.0):
    return (torch.randn(shape, generator=g, device="cuda", dtype=torch.float32) * scale).to(dtype)


def _ints(x):
    return torch.tensor(x, dtype=torch.int32).cuda()


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return {"sample": _prepare_sample, "fork": _prepare_fork}.get(case["kind"], _prepare_tree)(dict(case), g, random.Random(seed))


def _prepare_sample(c, g, rng):
    B, V, dt, cut = c["B"], c["V"], DTYPES[c["dtype"]], c["cut"]
    rand = lambda *shape: torch.rand(shape, generator=g, device="cuda")  # noqa: E731
    s = dict(case=c, logits=_randn(g, (B, V), dt, 3.0), mask=None)
    if c["mask"]:  # masks of a grammar: some rows admit a handful of tokens, others most of the vocabulary
        W = (V + 31) // 32
        bits = rand(B, W * 32) < torch.where(rand(B, 1) < 0.3, 20.0 / V, rand(B, 1))
        bits[:, V:] = False
        s["mask"] = _pack(bits)
    s["temperature"] = 0.5 + rand(B)
    if c["greedy"]:
        s["temperature"][rand(B) < 0.3] = 0.0
    # what requests ask for; a batch of `mixed` has rows with any of them, and with none
    pick = lambda *values: torch.tensor([rng.choice(values) for _ in range(B)], device="cuda")  # noqa: E731
    s["top_k"] = pick(0, 20, 50, 50, 1000).int() if cut in ("top_k", "mixed") else None
    s["top_p"] = pick(1.0, 0.9, 0.95, 0.8, 0.5).float() if cut in ("top_p", "mixed") else None
    s["min_p"] = pick(0.0, 0.0, 0.02, 0.05, 0.1).float() if cut in ("min_p", "mixed") else None
    s["noise"] = torch.empty((B, V), device="cuda").exponential_(generator=g)
    s["tokens"], s["status"] = (torch.empty((B,), dtype=torch.int32, device="cuda") for _ in range(2))
    s["logprob"] = torch.empty((B,), dtype=torch.float32, device="cuda")
    return s


def _pools(s, c, g, n_pages):
    """The cache: pages in the order [page, token, head] or [page, head, token]."""
    shape = (n_pages, c["page"], c["kv_heads"], c["D"]) if c["order"] == "token" else (n_pages, c["kv_heads"], c["page"], c["D"])
    pools = [_randn(g, shape, DTYPES[c["dtype"]]) for _ in range(2)]
    s["k_pages"], s["v_pages"] = pools if c["order"] == "token" else [p.transpose(1, 2) for p in pools]
    if own:  # the handle that a serving program makes once for its cache
        from paper_2607_11951_gb300 import grid as G
        s["kv"] = G.PagedKV(s["k_pages"], s["v_pages"], c.get("heads", c["kv_heads"]))


def _table(rows, width, ids):
    """A table of `width` pages a row, the first rows[b] of them taken from `ids`."""
    table = torch.full((len(rows), width), -1, dtype=torch.int32)
    at = 0
    for b, p in enumerate(rows):
        table[b, :p] = torch.tensor(ids[at:at + p], dtype=torch.int32)
        at += p
    return table.cuda()


def _tree(n, depth, rng):
    """Parents of a drafter's tree: the likeliest chain first (tokens 0 .. depth), then what branches off, here and there."""
    parent, at = [], []
    for i in range(n):
        p = i - 1 if i <= depth else rng.choice([j for j in range(i) if at[j] < depth])
        parent.append(p)
        at.append(at[p] + 1 if p >= 0 else 0)
    return parent


def _prepare_tree(c, g, rng):
    dt, B, D, Hk, page = DTYPES[c["dtype"]], c["B"], c["D"], c["kv_heads"], c["page"]
    new, old = _lengths(c)
    kept, moved = _paths(c)
    rows = list(zip(new, old, kept, moved))
    rng.shuffle(rows)
    new, old, kept, moved = [[x[i] for x in rows] for i in range(4)]
    N = sum(new)
    pages = [-(-(o + k) // page) for o, k in zip(old, new)]
    ids = list(range(sum(pages) + SPARE))
    rng.shuffle(ids)
    starts = [0]
    for n in new:
        starts.append(starts[-1] + n)
    s = dict(case=c, lens=_ints(old), start=_ints(starts), table=_table(pages, max(1, max(pages)), ids), T=max(new),
             S=max(1, max(o + k for o, k in zip(old, new))), W=(max(new) + 31) // 32)
    _pools(s, c, g, len(ids))
    s["status"] = torch.full((B,), -1, dtype=torch.int32, device="cuda")
    trees = [_tree(n, c["depth"], rng) for n in new]
    s["parent"] = _ints([p for t in trees for p in t])
    if c["kind"] == "keep":
        # the target takes the first chain for a while, then goes over to a branch where there is one
        tokens, sampled = [], []
        for t, k, m in zip(trees, kept, moved):
            tok = [rng.randrange(151_936) for _ in t]
            out = [rng.randrange(151_936) for _ in t]
            node, path = 0, []
            while t and len(path) < k:
                path.append(node)
                nodes = [j for j in range(node + 1, len(t)) if t[j] == node]
                far = [j for j in nodes if j > c["depth"]]
                nodes = far if far and len(path) > k - 1 - m else nodes
                if not nodes:
                    break
                node = nodes[0] if len(path) <= k - 1 - m else rng.choice(nodes)
            for a, b in zip(path, path[1:]):
                out[a] = tok[b]
            tokens += tok
            sampled += out
        s["tokens"], s["sampled"] = _ints(tokens), _ints(sampled)
        s["path"], s["out"] = (torch.empty((B, c["depth"] + 1), dtype=torch.int32, device="cuda") for _ in range(2))
        s["count"], s["moved"] = (torch.empty((B,), dtype=torch.int32, device="cuda") for _ in range(2))
        return s
    H = c["heads"]
    s["depth"] = torch.empty((N,), dtype=torch.int32, device="cuda")
    s["sees"] = torch.empty((N, s["W"]), dtype=torch.int32, device="cuda")
    if c["kind"] == "grow":
        # one projection's output holds a token's queries, keys and values
        qkv = _randn(g, (N, H + 2 * Hk, D), dt)
        s["q"], s["k"], s["v"] = qkv[:, :H], qkv[:, H:H + Hk], qkv[:, H + Hk:]
        freq = 10000.0 ** (-torch.arange(0, D, 2, device="cuda", dtype=torch.float64) / D)
        angle = torch.arange(s["S"], device="cuda", dtype=torch.float64)[:, None] * freq
        s["cos"], s["sin"] = angle.cos().float(), angle.sin().float()
        s["q_norm"] = s["k_norm"] = None
        if c["norm"]:
            s["q_norm"], s["k_norm"] = ((1 + 0.2 * _randn(g, (D,), torch.float32)).to(dt) for _ in range(2))
        s["q_out"] = torch.empty((N, H, D), dtype=dt, device="cuda")
    else:
        bits = torch.zeros((N, s["W"] * 32), dtype=torch.bool)
        for a, t in zip(starts, trees):
            for i, p in enumerate(t):
                if p >= 0:
                    bits[a + i] = bits[a + p]
                bits[a + i, i] = True
        s["sees"] = _pack(bits.cuda())
        s["q"] = _randn(g, (N, H, D), dt, 1.5)  # (scores of a few units: some keys matter more than others)
        s["out"] = torch.empty((N, H, D), dtype=dt, device="cuda")
        s["lse"] = torch.empty((N, H), dtype=torch.float32, device="cuda")
        s["scale"] = 1 / math.sqrt(D)
    return s


def _pool(c):
    """Pages of a forked cache: what the rows hold before and after (a third of what the new rows need, for `short`)."""
    held, parent, keep, want = _forked(c)
    page = c["page"]
    more = sum(-(-w // page) - k // page for w, k in zip(want, keep))
    return sum(-(-h // page) for h in held) + (more // 3 if c["short"] else more) + SPARE


def _prepare_fork(c, g, rng):
    A, B, page = c["A"], c["B"], c["page"]
    held, parent, keep, want = _forked(c)
    at = list(range(A))  # where the old rows go
    rng.shuffle(at)
    rows = list(zip(parent, keep, want))
    rng.shuffle(rows)
    old = [0] * A
    for a, x in zip(at, held):
        old[a] = x
    pages = [-(-h // page) for h in old]
    ids = list(range(_pool(c)))
    rng.shuffle(ids)
    # pages that a prefix store holds beside the rows: the first of some of them, and one that no row has
    width = max(1, max(-(-x // page) for x in held + want))
    s = dict(case=c, table=_table(pages, width, ids), held=_ints(old))
    pinned = torch.zeros(len(ids), dtype=torch.int32)
    pinned[ids[-1]] = 1
    for a in range(0, A, 8):
        if pages[a] > 1:
            pinned[int(s["table"][a, 0])] = 1
    s["pinned"] = pinned.cuda()
    s["parent"] = _ints([at[p] if p >= 0 else -1 for p, _, _ in rows])
    s["keep"], s["want"] = _ints([k for _, k, _ in rows]), _ints([w for _, _, w in rows])
    _pools(s, c, g, len(ids))
    i32 = dict(dtype=torch.int32, device="cuda")
    s["table_out"], s["held_out"] = torch.empty((B, width), **i32), torch.empty((B,), **i32)
    s["copies"], s["refs"] = torch.empty((3, B), **i32), torch.empty((len(ids),), **i32)
    s["status"], s["copied"] = torch.empty((B,), **i32), torch.empty((B,), **i32)
    if own:  # the handle that a serving program makes once for its pool
        from paper_2607_11951_gb300 import grid as G
        s["pages"] = G.Pages(len(ids), page)
    return s


def _pack(bits):
    """Truth values [..., 32 W] as int32 words [..., W], the lowest bit first."""
    x = bits.view(*bits.shape[:-1], -1, 32).to(torch.int64)
    x = (x << torch.arange(32, device=bits.device)).sum(-1)
    return torch.where(x >= 1 << 31, x - (1 << 32), x).int()


def _unpack(words, V):
    x = (words[..., None] >> torch.arange(32, device="cuda", dtype=torch.int32)) & 1
    return x.flatten(-2)[..., :V].bool()


# ---------------------------------------------------------------------------
# one pass
def run(state):
    return {"sample": _sample, "grow": _grow, "tree": _attend, "keep": _keep, "fork": _fork}[state["case"]["kind"]](state)


def _sample(s):
    if own:
        from paper_2607_11951_gb300 import grid as G
        G.grid_sample(s["logits"], s["noise"], s["tokens"], s["status"], mask=s["mask"], temperature=s["temperature"],
                      top_k=s["top_k"], top_p=s["top_p"], min_p=s["min_p"], logprob=s["logprob"])
        return {k: s[k] for k in ("tokens", "logprob", "status")}
    c = s["case"]
    V = c["V"]
    greedy = (s["temperature"] <= 0)[:, None]
    x = s["logits"].float()
    if s["mask"] is not None:
        x = torch.where(_unpack(s["mask"], V), x, -math.inf)
    x, ids = x.sort(stable=True, dim=1, descending=True)  # (equal logits stay in the order of their ids)
    empty = x[:, :1] == -math.inf
    x = (x - torch.where(empty, 0.0, x[:, :1])) / torch.where(greedy, 1.0, s["temperature"][:, None])
    w = x.exp()
    z = w.sum(1, keepdim=True)
    i = torch.arange(V, device="cuda")
    kept = (i == 0) | ~greedy
    if s["top_k"] is not None:
        kept &= (s["top_k"] <= 0)[:, None] | (i < s["top_k"][:, None])
    if s["top_p"] is not None:
        upto = torch.where(kept, w, 0.0).double().cumsum(1)  # (64 bits: sums next to the border)
        kept &= (s["top_p"] >= 1)[:, None] | (i == 0) | (upto - w < s["top_p"].double()[:, None] * upto[:, -1:])
    if s["min_p"] is not None:
        kept &= (i == 0) | (w >= s["min_p"][:, None])
    score = torch.where(kept, w, 0.0) / s["noise"].gather(1, ids)
    top = score.amax(1, keepdim=True)
    token = torch.where((score == top) & kept, ids, V).amin(1, keepdim=True)
    chosen = torch.where(ids == token, x, -math.inf).amax(1, keepdim=True)
    s["tokens"].copy_(torch.where(empty, -1, token)[:, 0])
    s["logprob"].copy_(torch.where(empty, 0.0, chosen - z.log())[:, 0])
    s["status"].copy_(torch.where(empty, 4, 0)[:, 0])
    return {k: s[k] for k in ("tokens", "logprob", "status")}


def _rows(s):
    """Row and index in the row of every token of the chunk."""
    i = torch.arange(s["parent"].shape[0], device="cuda")
    row = torch.searchsorted(s["start"], i.int(), right=True) - 1
    return row, i - s["start"].long()[row]


def _grow(s):
    c = s["case"]
    if own:
        from paper_2607_11951_gb300 import grid as G
        G.grid_tree_plan(s["parent"], s["depth"], s["sees"], s["status"], start=s["start"])
        G.grid_kv_append(s["kv"], s["table"], s["lens"], s["k"], s["v"], s["status"], start=s["start"], q=s["q"],
                         q_out=s["q_out"], cos=s["cos"], sin=s["sin"], q_norm=s["q_norm"], k_norm=s["k_norm"], eps=EPS,
                         depth=s["depth"])
        return {"depth": s["depth"], "sees": s["sees"], "q": s["q_out"], "k": s["k_pages"], "v": s["v_pages"],
                "status": s["status"]}
    row, i = _rows(s)
    first = s["start"].long()[row]
    bits = i[:, None] == torch.arange(32 * s["W"], device="cuda")
    depth, up = torch.zeros_like(i), s["parent"].long()
    for _ in range(c["depth"]):
        depth += up >= 0
        bits |= up[:, None] == torch.arange(32 * s["W"], device="cuda")
        up = torch.where(up >= 0, s["parent"].long()[first + up.clamp(min=0)], -1)
    s["depth"].copy_(depth)
    s["sees"].copy_(_pack(bits))
    place, angle = s["lens"].long()[row] + i, s["lens"].long()[row] + depth
    page = s["table"].long()[row, place // c["page"]]
    turned = [_rotate(_normed(x.float(), w), s["cos"][angle][:, None], s["sin"][angle][:, None])
              for x, w in ((s["q"], s["q_norm"]), (s["k"], s["k_norm"]))]
    s["q_out"].copy_(turned[0])
    s["k_pages"][page, place % c["page"]] = turned[1].to(s["k"].dtype)
    s["v_pages"][page, place % c["page"]] = s["v"]
    return {"depth": s["depth"], "sees": s["sees"], "q": s["q_out"], "k": s["k_pages"], "v": s["v_pages"],
            "status": torch.zeros_like(s["status"])}


def _normed(x, w):
    return x if w is None else x * torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS) * w.float()


def _rotate(x, cos, sin):
    half = cos.shape[-1]
    a, b = x[..., :half], x[..., half:]
    return torch.cat([a * cos - b * sin, b * cos + a * sin], -1)


def _attend(s):
    c = s["case"]
    if own:
        from paper_2607_11951_gb300 import grid as G
        G.grid_kv_attend(s["kv"], s["table"], s["lens"], s["q"], s["out"], s["status"], lse=s["lse"], start=s["start"],
                         scale=s["scale"], sees=s["sees"])
        return {"out": s["out"], "lse": s["lse"], "status": s["status"]}
    B, H, Hk, D, T, S = c["B"], c["heads"], c["kv_heads"], c["D"], s["T"], s["S"]
    first, n = s["start"][:-1].long(), (s["start"][1:] - s["start"][:-1]).long()
    t = torch.arange(T, device="cuda")
    there = t < n[:, None]  # [B, T]: the padded trees' own tokens
    at = torch.where(there, first[:, None] + t, 0)
    q = s["q"].float()[at].view(B, T, Hk, H // Hk, D).permute(0, 2, 3, 1, 4).reshape(B, Hk, H // Hk * T, D)
    j = torch.arange(S, device="cuda")
    old = s["lens"].long()[:, None]
    used = j < old + n[:, None]  # [B, S]: the row's own keys
    page = torch.where(used, s["table"].long()[:, j // c["page"]], 0)
    k, v = (p[page, j % c["page"]].float().masked_fill_(~used[:, :, None, None], 0.0).transpose(1, 2)
            for p in (s["k_pages"], s["v_pages"]))  # [B, Hk, S, D]
    # a cached key is seen by all, a key of the tree where its bit is set
    bits = _unpack(s["sees"][at], 32 * s["W"])  # [B, T, 32 W]
    tree = ((j - old).clamp(0, 32 * s["W"] - 1))[:, None].expand(B, T, S)
    seen = (j < old)[:, None] | (used[:, None] & bits.gather(2, tree))
    x = (q @ k.transpose(2, 3)).mul_(s["scale"]).view(B, Hk, H // Hk, T, S)
    x.masked_fill_(~seen[:, None, None], -math.inf)
    m = x.amax(-1, keepdim=True)
    p = x.sub_(m).exp_()
    z = p.sum(-1, keepdim=True)
    out = (p.view(B, Hk, H // Hk * T, S) @ v).view(B, Hk, H // Hk, T, D) / z
    s["out"].copy_(out.permute(0, 3, 1, 2, 4).reshape(B, T, H, D)[there])
    s["lse"].copy_((m + z.log()).squeeze(-1).permute(0, 3, 1, 2).reshape(B, T, H)[there])
    return {"out": s["out"], "lse": s["lse"], "status": torch.zeros_like(s["status"])}


def _keep(s):
    c = s["case"]
    if own:
        from paper_2607_11951_gb300 import grid as G
        G.grid_tree_accept(s["parent"], s["tokens"], s["sampled"], s["path"], s["count"], s["out"], s["status"],
                           start=s["start"])
        G.grid_kv_compact(s["kv"], s["table"], s["lens"], s["path"], s["count"], s["moved"], s["parent"].shape[0],
                          start=s["start"])
        return {k: s[k] for k in ("path", "count", "out", "status", "moved")} | {"k": s["k_pages"], "v": s["v_pages"]}
    B, T, D = c["B"], s["T"], c["depth"] + 1
    first, n = s["start"][:-1].long(), (s["start"][1:] - s["start"][:-1]).long()
    t = torch.arange(T, device="cuda")
    at = torch.where(t < n[:, None], first[:, None] + t, 0)
    parent = torch.where(t < n[:, None], s["parent"].long()[at], -2)
    tokens, sampled = s["tokens"][at], s["sampled"][at]
    node = torch.where(n > 0, 0, -1)
    for d in range(D):
        s["path"][:, d] = node
        drawn = torch.where(node >= 0, sampled.gather(1, node.clamp(min=0)[:, None])[:, 0], -1)
        s["out"][:, d] = drawn
        child = (parent == node[:, None]) & (tokens == drawn[:, None]) & (node >= 0)[:, None]
        node = torch.where(child, t, T).amin(1)
        node = torch.where(node < T, node, -1)
    s["count"].copy_((s["path"] >= 0).sum(1))
    j = torch.arange(D, device="cuda")
    src, dst = s["lens"].long()[:, None] + s["path"].long(), s["lens"].long()[:, None] + j
    b = torch.arange(B, device="cuda")[:, None].expand(B, D)
    on = s["path"] >= 0
    b, src, dst = b[on], src[on], dst[on]
    table = s["table"].long()
    for pool in (s["k_pages"], s["v_pages"]):
        pool[table[b, dst // c["page"]], dst % c["page"]] = pool[table[b, src // c["page"]], src % c["page"]]
    return {"path": s["path"], "count": s["count"], "out": s["out"], "k": s["k_pages"], "v": s["v_pages"],
            "status": torch.zeros_like(s["status"]), "moved": torch.zeros_like(s["moved"])}


def _fork(s):
    c = s["case"]
    if own:
        from paper_2607_11951_gb300 import grid as G
        G.grid_pages_update(s["pages"], s["table"], s["held"], s["want"], s["table_out"], s["held_out"], s["copies"],
                            s["refs"], s["status"], parent=s["parent"], keep=s["keep"], pinned=s["pinned"])
        G.grid_kv_copy(s["kv"], s["copies"], s["copied"])
        return {k: s[k] for k in ("table_out", "held_out", "copies", "refs", "status", "copied")} | \
            {"k": s["k_pages"], "v": s["v_pages"]}
    page, B = c["page"], c["B"]
    n_pages, width = s["refs"].shape[0], s["table_out"].shape[1]
    i64 = dict(dtype=torch.int64, device="cuda")
    parent, keep, want = s["parent"].long(), s["keep"].long(), s["want"].long()
    old = s["table"].long()[parent.clamp(min=0)]
    full, room = keep // page, (want + page - 1) // page
    j, b = torch.arange(width, device="cuda"), torch.arange(B, device="cuda")
    shared = j < full[:, None]  # [B, width]
    refs = torch.zeros(n_pages + 1, **i64).scatter_add_(0, torch.where(shared, old, n_pages).flatten(), shared.long().flatten())
    # the page that is kept in part: its lowest row keeps it where nobody else holds it
    part = keep % page > 0
    last = torch.where(part, old.gather(1, full.clamp(max=width - 1)[:, None])[:, 0], n_pages)
    owner = torch.full((n_pages + 1,), B, **i64).scatter_reduce_(0, last, b, "amin")
    stays = part & (owner[last] == b) & (refs[last] == 0) & (torch.cat([s["pinned"], s["pinned"][:1]])[last] == 0)
    need = room - full - stays.long()
    refs[torch.where(stays, last, n_pages)] = 1
    free = (refs[:n_pages] == 0) & (s["pinned"] == 0)
    rank = free.long().cumsum(0) - 1
    order = torch.zeros(n_pages + 1, **i64).scatter_(0, torch.where(free, rank, n_pages), torch.arange(n_pages, device="cuda"))
    upto = need.cumsum(0)
    fits = (need == 0) | (upto <= free.sum())
    nth = (upto - need)[:, None] + j - (full + stays.long())[:, None]
    fresh = (j >= (full + stays.long())[:, None]) & (j < room[:, None]) & fits[:, None]
    table = torch.where(shared | ((j == full[:, None]) & stays[:, None]), old, -1)
    table = torch.where(fresh, order[nth.clamp(0, n_pages)], table)
    refs.scatter_add_(0, torch.where(fresh, table, n_pages).flatten(), fresh.long().flatten())
    copied = part & ~stays & fits
    dst = table.gather(1, full.clamp(max=width - 1)[:, None])[:, 0]
    s["table_out"].copy_(table)
    s["held_out"].copy_(torch.where(fits, want, torch.where(stays | ~part, keep, full * page)))
    s["copies"].copy_(torch.stack([torch.where(copied, last, -1), torch.where(copied, dst, -1), torch.where(copied, keep % page, 0)]))
    s["refs"].copy_(refs[:n_pages])
    s["status"].copy_(torch.where(fits, 0, 7))
    # the copies, all rows' at once
    off = torch.arange(page, device="cuda")
    from_, to = torch.where(copied, last, 0)[:, None], torch.where(copied, dst, n_pages)[:, None]
    on = copied[:, None] & (off < (keep % page)[:, None])
    for pool in (s["k_pages"], s["v_pages"]):
        wide = to.expand(B, page)[on], off.expand(B, page)[on]
        pool[wide] = pool[from_.expand(B, page)[on], wide[1]]
    return {k: s[k] for k in ("table_out", "held_out", "copies", "refs", "status")} | \
        {"copied": torch.zeros_like(s["copied"]), "k": s["k_pages"], "v": s["v_pages"]}


# ---------------------------------------------------------------------------
# the same in 64 bits, row by row from the definitions
def exact(case, seed):
    s = prepare(case, seed)
    return {"sample": _exact_sample, "grow": _exact_grow, "tree": _exact_attend, "keep": _exact_keep,
            "fork": _exact_fork}[case["kind"]](case, s)


def _exact_sample(c, s):
    logs = []
    at = lambda name, b, none: none if s[name] is None else s[name][b].item()  # noqa: E731
    for b in range(c["B"]):
        T, k, p, least = at("temperature", b, 1.0), at("top_k", b, 0), at("top_p", b, 1.0), at("min_p", b, 0.0)
        logits = s["logits"][b].double()
        if s["mask"] is not None:
            logits = logits.masked_fill(~_unpack(s["mask"][b], c["V"]), -math.inf)
        if not bool((logits > -math.inf).any()):
            logs.append(0.0)
            continue
        logp = torch.log_softmax(logits / T if T > 0 else logits, 0)
        order = torch.argsort(-logits, stable=True)
        prob = logp[order].exp()
        n = int((logits > -math.inf).sum())
        if T <= 0:
            n = 1
        if k > 0:
            n = min(n, k)
        if p < 1:
            below = torch.cumsum(prob[:n], 0) < p * prob[:n].sum()
            n = min(n, int(below.sum()) + 1)
        if least > 0:
            n = max(1, min(n, int((prob >= least * prob[0]).sum())))
        score = prob[:n] / s["noise"][b].double()[order[:n]]
        token = int(order[:n][score == score.max()].min())
        logs.append(float(logp[token]))
    return {"tokens": None, "logprob": torch.tensor(logs, dtype=torch.float64), "status": None}


def _trees(s):
    """Per row its first token and its parents."""
    start, parent = s["start"].tolist(), s["parent"].tolist()
    return [(a, parent[a:z]) for a, z in zip(start, start[1:])]


def _slot(s, c, b, pos):
    return int(s["table"][b, pos // c["page"]]) * c["page"] + pos % c["page"]


def _exact_grow(c, s):
    lens, table = s["lens"].tolist(), s["table"].tolist()
    half = c["D"] // 2
    angle, slot = [], []
    for b, (_, tree) in enumerate(_trees(s)):
        deep = []
        for i, p in enumerate(tree):
            deep.append(deep[p] + 1 if p >= 0 else 0)
            angle.append(lens[b] + deep[i])
            slot.append(table[b][(lens[b] + i) // c["page"]] * c["page"] + (lens[b] + i) % c["page"])
    angle, slot = torch.tensor(angle, device="cuda"), torch.tensor(slot, device="cuda")
    # the tables are inputs: their 32-bit values stand
    turn = torch.complex(s["cos"].double()[angle], s["sin"].double()[angle])[:, None]

    def turned(x, w):
        x = x.double()
        if w is not None:
            x = x / (x.pow(2).sum(-1, keepdim=True) / c["D"] + EPS).sqrt() * w.double()
        z = torch.complex(x[..., :half], x[..., half:]) * turn
        return torch.cat([z.real, z.imag], -1)

    def stored(pool, x):
        flat = pool.double().reshape(-1, c["kv_heads"], c["D"])
        flat[slot] = x
        return flat.view(pool.shape)

    return {"depth": None, "sees": None, "q": turned(s["q"], s["q_norm"]), "k": stored(s["k_pages"], turned(s["k"], s["k_norm"])),
            "v": stored(s["v_pages"], s["v"].double()), "status": None}


def _exact_attend(c, s):
    H, Hk, page = c["heads"], c["kv_heads"], c["page"]
    lens, table = s["lens"].tolist(), s["table"]
    if work(c)["flops"] > 4e12:  # (about 20 s at this card's 64-bit rate)
        return None
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda")
    lse = torch.zeros(s["lse"].shape, dtype=torch.float64, device="cuda")
    for b, (a, tree) in enumerate(_trees(s)):
        n = len(tree)
        if not n:
            continue
        total = lens[b] + n
        used = table[b, :-(-total // page)].long()
        k, v = (p[used].reshape(-1, Hk, c["D"])[:total].double() for p in (s["k_pages"], s["v_pages"]))
        hidden = torch.zeros((n, total), dtype=torch.bool)
        hidden[:, lens[b]:] = True
        for i in range(n):
            j = i
            while j >= 0:
                hidden[i, lens[b] + j] = False
                j = tree[j]
        hidden = hidden.cuda()
        for h in range(H):
            x = s["q"][a:a + n, h].double() @ k[:, h * Hk // H].T * s["scale"]
            x[hidden] = -math.inf
            lse[a:a + n, h] = torch.logsumexp(x, 1)
            out[a:a + n, h] = torch.exp(x - lse[a:a + n, h, None]) @ v[:, h * Hk // H]
    return {"out": out, "lse": lse, "status": None}


def _exact_keep(c, s):
    tokens, sampled, lens = s["tokens"].tolist(), s["sampled"].tolist(), s["lens"].tolist()
    pools = {"k": s["k_pages"].double(), "v": s["v_pages"].double()}
    src, dst = [], []
    for b, (a, tree) in enumerate(_trees(s)):
        node, path = 0, []
        while tree and len(path) <= c["depth"]:
            path.append(node)
            child = [j for j in range(len(tree)) if tree[j] == node and tokens[a + j] == sampled[a + node]]
            if not child:
                break
            node = child[0]
        src += [_slot(s, c, b, lens[b] + i) for i in path]
        dst += [_slot(s, c, b, lens[b] + j) for j in range(len(path))]
    src, dst = torch.tensor(src, device="cuda"), torch.tensor(dst, device="cuda")
    for name, pool in pools.items():
        pool[dst // c["page"], dst % c["page"]] = pool[src // c["page"], src % c["page"]]
    return dict.fromkeys(("path", "count", "out", "status", "moved")) | pools


def _exact_fork(c, s):
    page = c["page"]
    table, parent, keep, want = (s[x].tolist() for x in ("table", "parent", "keep", "want"))
    taken = {p for p, x in enumerate(s["pinned"].tolist()) if x}
    whole = {table[p][j] for p, k in zip(parent, keep) if p >= 0 for j in range(k // page)}
    part, given = {}, {}
    for b, (p, k) in enumerate(zip(parent, keep)):
        if p >= 0 and k % page and table[p][k // page] not in part:
            part[table[p][k // page]] = b
    stays = {b for q, b in part.items() if q not in whole and q not in taken}
    free = [q for q in range(_pool(c)) if q not in whole and q not in taken and part.get(q, -1) not in stays]
    at = 0
    for b, (p, k, w) in enumerate(zip(parent, keep, want)):
        need = -(-w // page) - k // page - (b in stays)
        if need and at + need <= len(free) and k % page and b not in stays:
            given[b] = free[at]
        at += need
    pools = {"k": s["k_pages"].double(), "v": s["v_pages"].double()}
    for b, q in given.items():
        n = keep[b] % page
        for pool in pools.values():
            pool[q, :n] = pool[table[parent[b]][keep[b] // page], :n]
    return dict.fromkeys(("table_out", "held_out", "copies", "refs", "status", "copied")) | pools
