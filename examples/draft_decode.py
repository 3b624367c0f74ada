"""Drafted decoding under a grammar, with a model of one attention layer.

Every step drafts K tokens for each row (the beginning of the row's cheapest
legal completion, grid_reserve), takes the row's last token and its draft
through the model as one chunk (grid_kv_append, grid_kv_attend), verifies the
draft against the model's distribution under the grammar's masks
(grid_draft_verify), and feeds what came of it to the parser (grid_advance).
The model's weights are random: the text is nonsense (it likes to repeat
itself), but a sentence of the grammar.  K = 0 decodes one token at a time; greedy rows then give the same text.

    python examples/draft_decode.py [--draft 3] [--steps 24] [--temperature 0.8]
"""
import argparse
import os
import sys

import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
sys.path.insert(0, ROOT)

from paper_2607_11951_gb300 import grid as G  # noqa: E402
from workloads import configs  # noqa: E402


class Model:
    """Token embeddings, one attention layer with normed and rotated heads, tied output."""

    def __init__(self, V, B, positions, heads=8, kv_heads=2, D=64, width=256, page=16, seed=0):
        g = torch.Generator(device="cuda")
        g.manual_seed(seed)
        bf = torch.bfloat16
        w = lambda *shape: (torch.randn(shape, generator=g, device="cuda") * shape[0] ** -0.5).to(bf)
        self.heads, self.kv_heads, self.D = heads, kv_heads, D
        self.embed = (torch.randn((V, width), generator=g, device="cuda")).to(bf)
        self.w_qkv, self.w_out = w(width, (heads + 2 * kv_heads) * D), w(heads * D, width)
        self.q_norm, self.k_norm = (torch.ones(D, device="cuda", dtype=bf) for _ in range(2))
        per_row = -(-positions // page)
        pools = [torch.empty((B * per_row, page, kv_heads, D), device="cuda", dtype=bf) for _ in range(2)]
        self.kv = G.PagedKV(*pools, heads)
        self.table = torch.randperm(B * per_row, generator=g, device="cuda").int().view(B, per_row)
        freq = 10000.0 ** (-torch.arange(0, D, 2, device="cuda") / D)
        angle = torch.arange(positions, device="cuda")[:, None] * freq
        self.cos, self.sin = angle.cos(), angle.sin()
        self.status = torch.zeros(B, device="cuda", dtype=torch.int32)

    def __call__(self, tokens, lens, start=None):
        """Logits of the packed new tokens [n]; ``lens`` tokens per row are cached already."""
        x = self.embed[tokens.clamp(min=0)]
        qkv = (x @ self.w_qkv).view(len(tokens), -1, self.D)
        q, k, v = qkv.split([self.heads, self.kv_heads, self.kv_heads], 1)
        at = torch.empty_like(q)
        G.grid_kv_append(self.kv, self.table, lens, k, v, self.status, start=start, q=q, q_out=q, cos=self.cos,
                         sin=self.sin, q_norm=self.q_norm, k_norm=self.k_norm)
        G.grid_kv_attend(self.kv, self.table, lens, q, at, self.status, start=start)
        return ((at.flatten(1) @ self.w_out + x) @ self.embed.T).float()


def decode(wl, K, steps, temperature=0.0, seed=0):
    """Tokens decoded after each prefix of the workload, as lists."""
    V, B = len(wl["tokens"]), len(wl["prefixes"])
    i32 = dict(device="cuda", dtype=torch.int32)
    spec = G.Spec(G.Grammar(wl["grammar"], wl["role"], wl["lexicons"]), G.Vocab(wl["tokens"], wl["eos"], wl["specials"]))
    cfg = [G.Configs(spec, B) for _ in range(K + 1)]  # the row, and along its draft
    status = torch.zeros(B, **i32)
    masks = torch.zeros((K + 1, B, spec.W), **i32)    # as the mask calls write them: position by position
    cost, rest = torch.zeros(B, **i32), torch.zeros((B, 64), **i32)
    drafts = G.Drafts(B, K, V)
    out = torch.empty((B, K + 1), **i32)
    accepted, temp = torch.zeros(B, **i32), torch.full((B,), float(temperature), device="cuda")
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)

    # the prompts: a ragged chunk of all tokens but the last, which opens the first step's chunk
    prefix = [list(p) if p else [0] for p in wl["prefixes"]]
    longest = max(map(len, prefix))
    fed = torch.tensor([list(p) + [-1] * (longest - len(p)) for p in wl["prefixes"]], **i32) if longest else None
    G.grid_advance(spec, cfg[0], cfg[0], fed, status)
    model = Model(V, B, longest + steps * (K + 1) + 1)
    start = torch.zeros(B + 1, **i32)
    start[1:] = torch.cumsum(torch.tensor([len(p) - 1 for p in prefix], **i32), 0)
    lens = torch.zeros(B, **i32)
    if int(start[-1]):
        model(torch.tensor([t for p in prefix for t in p[:-1]], **i32), lens, start)
    lens += start[1:] - start[:-1]
    last = torch.tensor([p[-1] for p in prefix], **i32)

    rows = [[] for _ in range(B)]
    for _ in range(steps):
        if K:
            G.grid_reserve(spec.h, cfg[0].h, cost, rest, status)
        draft = rest[:, :K].contiguous()  # (-1 past a short completion's end: refused)
        G.grid_masks(spec, cfg[0], masks[0], status)
        for k in range(K):  # (a token that the grammar refuses leaves the configuration: its mask bit is 0 before it)
            G.grid_advance_masks(spec, cfg[k], cfg[k + 1], draft[:, k].contiguous(), masks[k + 1], status)
        chunk = torch.cat([last[:, None], draft], 1)
        logits = model(chunk.flatten(), lens).view(B, K + 1, V)
        u = torch.rand((B, K), generator=g, device="cuda")
        noise = torch.empty((B, V), device="cuda").exponential_(generator=g)
        G.grid_draft_verify(drafts, logits, draft, u, noise, out, accepted, status,
                            mask=masks.transpose(0, 1), temperature=temp, eos=wl["eos"])
        G.grid_advance(spec, cfg[0], cfg[0], out, status)
        new = (out >= 0).sum(1, dtype=torch.int32)
        lens += new
        last = torch.where(new > 0, out.gather(1, (new.long() - 1).clamp(min=0)[:, None])[:, 0], last)
        for b, r in enumerate(out.tolist()):
            rows[b] += [t for t in r if t >= 0]
        if not bool((new > 0).any()):
            break
    return rows


def main():
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--draft", type=int, default=3)
    ap.add_argument("--steps", type=int, default=24)
    ap.add_argument("--temperature", type=float, default=0.8)
    a = ap.parse_args()
    wl = configs.tiny_expr(B=8)
    for p, r in zip(wl["prefixes"], decode(wl, a.draft, a.steps, a.temperature)):
        text = lambda ids: b"".join(wl["tokens"][t] for t in ids if t != wl["eos"]).decode()
        print("%-40r -> %r%s" % (text(p), text(r), "" if wl["eos"] in r else " ..."))


if __name__ == "__main__":
    main()
