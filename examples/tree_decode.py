"""Decoding under a grammar with trees of drafted tokens, several samples of each prompt, and pages that rows share.

Each prompt goes through the model once; then its samples part ways: they share
the prompt's whole pages, and copies are made of the one that is held in part
(grid_pages_update, grid_kv_copy).  Every step drafts a tree for each row: the
beginning of the row's cheapest legal completion (grid_reserve) as its stem, and
on the stem's tokens the ids that the model liked best after the last step.
The tree goes through the model at once (grid_tree_plan, grid_kv_append and
grid_kv_attend with its depths and visibility), one token is drawn at every node
under the grammar's mask there (grid_sample), the path that the draws take is
kept (grid_tree_accept, grid_kv_compact), and the parser follows it
(grid_advance).  Rows that end give their pages back.  The model's weights are
random (examples/draft_decode.py): the text is nonsense, but a sentence of the
grammar.  A tree of one token decodes one token at a time; greedy rows then give
the same text.

    python examples/tree_decode.py [--stem 3] [--branches 2] [--samples 2] [--temperature 0.8] [--top-p 0.9]
"""
import argparse
import os
import sys

import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
sys.path.insert(0, ROOT)

from examples.draft_decode import Model  # noqa: E402
from paper_2607_11951_gb300 import grid as G  # noqa: E402
from workloads import configs  # noqa: E402


def shape(stem, branches):
    """Parents of a tree: a root, `stem` tokens one after the other, and `branches` more children of the root and of every
    stem token but the last."""
    parent = [-1] + list(range(stem))
    for p in range(stem):
        parent += [p] * branches
    return parent


def decode(wl, stem, branches, steps, samples=1, temperature=0.0, top_p=1.0, top_k=0, seed=0, page=16):
    """Tokens decoded after each prefix of the workload, as lists: `samples` of them in a row."""
    V, A = len(wl["tokens"]), len(wl["prefixes"])
    B, tree = A * samples, shape(stem, branches)
    n = len(tree)
    i32 = dict(device="cuda", dtype=torch.int32)
    ints = lambda x: torch.tensor(x, **i32)  # noqa: E731
    zeros = lambda *s: torch.zeros(s, **i32)  # noqa: E731
    spec = G.Spec(G.Grammar(wl["grammar"], wl["role"], wl["lexicons"]), G.Vocab(wl["tokens"], wl["eos"], wl["specials"]))
    cfg = [G.Configs(spec, B) for _ in range(n)]  # the row, and after each drafted token
    status = zeros(B)
    prefix = [list(p) if p else [0] for p in wl["prefixes"]]
    longest = max(map(len, prefix))
    fed = [list(p) + [-1] * (longest - len(p)) for p in wl["prefixes"] for _ in range(samples)]
    if longest:
        G.grid_advance(spec, cfg[0], cfg[0], ints(fed), status)

    # a pool for all rows at their longest; every prompt once, all of its tokens but the last
    per_row = -(-(longest + steps * n + 1) // page)
    model = Model(V, B, per_row * page, page=page)
    n_pages = model.kv.pools[0].shape[0]
    pages, refs = G.Pages(n_pages, page), zeros(n_pages)
    table, held = torch.full((A, per_row), -1, **i32), zeros(A)

    def update(want, rows, **kw):
        nonlocal table, held
        new, now, copies, st = torch.empty((rows, per_row), **i32), zeros(rows), zeros(3, rows), zeros(rows)
        G.grid_pages_update(pages, table, held, want, new, now, copies, refs, st, **kw)
        G.grid_kv_copy(model.kv, copies, zeros(rows))
        table, held = new, now
        return st

    start = ints([0] + [len(p) - 1 for p in prefix]).cumsum(0, dtype=torch.int32)
    update(start[1:] - start[:-1], A)
    if int(start[-1]):
        model.table, model.status = table, zeros(A)
        model(ints([t for p in prefix for t in p[:-1]]), zeros(A), start)
    lens = (start[1:] - start[:-1]).repeat_interleave(samples)
    last = ints([p[-1] for p in prefix for _ in range(samples)])
    update(lens, B, parent=torch.arange(A, **i32).repeat_interleave(samples))

    model.status = status
    parent = ints(tree * B)
    depth, sees = zeros(B * n), zeros(B * n, (n + 31) // 32)
    path, out, count = zeros(B, stem + 2), zeros(B, stem + 2), zeros(B)
    masks, sampled, drawn = zeros(n, B, spec.W), zeros(B * n), zeros(B * n)
    cost, rest = zeros(B), zeros(B, 64)
    liked = torch.zeros((B, V), device="cuda")
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    node = lambda x, t: torch.full((B * n,), float(x), device="cuda").to(t)  # noqa: E731
    temp, share, most = node(temperature, torch.float32), node(top_p, torch.float32), node(top_k, torch.int32)

    rows, alive = [[] for _ in range(B)], torch.ones(B, dtype=torch.bool, device="cuda")
    for _ in range(steps):
        # the tree: the last token, the cheapest completion's first ones, and what the model liked
        tokens = torch.full((B, n), -1, **i32)
        tokens[:, 0] = last
        if stem:
            G.grid_reserve(spec.h, cfg[0].h, cost, rest, status)
            tokens[:, 1:1 + stem] = rest[:, :stem]
            best = liked.topk(branches, 1).indices.int() if branches else None
            for p in range(stem if branches else 0):
                tokens[:, 1 + stem + p * branches:1 + stem + (p + 1) * branches] = best
        G.grid_masks(spec, cfg[0], masks[0], status)
        for i in range(1, n):  # (after a token that the grammar refuses the parser stays where it is: no draw takes it)
            G.grid_advance_masks(spec, cfg[tree[i]], cfg[i], tokens[:, i].contiguous(), masks[i], status)
        # room for it; rows that ended keep nothing
        keep = torch.where(alive, lens, 0)
        st = update(torch.where(alive, lens + n, 0), B, keep=keep)
        assert not bool((st != 0).any()), "the pool has room for all rows"
        lens = keep
        # through the model
        G.grid_tree_plan(parent, depth, sees, status)
        x = model.embed[tokens.flatten().clamp(min=0)]
        q, k, v = (x @ model.w_qkv).view(B * n, -1, model.D).split([model.heads, model.kv_heads, model.kv_heads], 1)
        at = torch.empty_like(q)
        G.grid_kv_append(model.kv, table, lens, k, v, status, q=q, q_out=q, cos=model.cos, sin=model.sin, q_norm=model.q_norm,
                         k_norm=model.k_norm, depth=depth)
        G.grid_kv_attend(model.kv, table, lens, q, at, status, sees=sees)
        logits = ((at.flatten(1) @ model.w_out + x) @ model.embed.T).float()
        # a draw at every node, the path that the draws take
        noise = torch.empty((B * n, V), device="cuda").exponential_(generator=g)
        G.grid_sample(logits, noise, sampled, drawn, mask=masks.transpose(0, 1).reshape(B * n, -1), temperature=temp,
                      top_k=most, top_p=share)
        G.grid_tree_accept(parent, tokens.flatten(), sampled, path, count, out, status, eos=wl["eos"])
        G.grid_kv_compact(model.kv, table, lens, path, count, status, B * n)
        out = torch.where(alive[:, None], out, -1)
        G.grid_advance(spec, cfg[0], cfg[0], out, status)
        new = (out >= 0).sum(1, dtype=torch.int32)
        lens = lens + new  # (a row's root was cached with its first draw)
        end = (path.gather(1, (count.long() - 1).clamp(min=0)[:, None])[:, 0].clamp(min=0).long() + torch.arange(B, device="cuda") * n)
        liked = logits[end]
        last = torch.where(new > 0, out.gather(1, (new.long() - 1).clamp(min=0)[:, None])[:, 0], last)
        for b, r in enumerate(out.tolist()):
            rows[b] += [t for t in r if t >= 0]
        alive = alive & (new > 0) & (last != wl["eos"])
        out = torch.empty_like(path)
        if not bool(alive.any()):
            break
    return rows


def main():
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--stem", type=int, default=3)
    ap.add_argument("--branches", type=int, default=2)
    ap.add_argument("--samples", type=int, default=2)
    ap.add_argument("--steps", type=int, default=24)
    ap.add_argument("--temperature", type=float, default=0.8)
    ap.add_argument("--top-p", type=float, default=0.9)
    a = ap.parse_args()
    wl = configs.tiny_expr(B=4)
    rows = decode(wl, a.stem, a.branches, a.steps, a.samples, a.temperature, a.top_p)
    for i, r in enumerate(rows):
        text = lambda ids: b"".join(wl["tokens"][t] for t in ids if t != wl["eos"]).decode()  # noqa: E731
        print("%-40r -> %r%s" % (text(wl["prefixes"][i // a.samples]), text(r), "" if wl["eos"] in r else " ..."))


if __name__ == "__main__":
    main()
