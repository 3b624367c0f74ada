"""Measured cases: a chunk of tokens through a model's attention and its outcome.

A grammar-constrained decoding loop rarely hands a model one token a row: a
forced span arrives whole, a drafter proposes several tokens at once, a prompt
arrives in chunks.  Three operators take such a chunk through the model:

  append  ``grid_kv_append``: the new tokens' keys and values go into the paged
          cache, queries and keys optionally normed per head and rotated by
          their position on the way
  attend  ``grid_kv_attend``: every new token attends to its row's cached
          tokens and to the chunk's tokens up to itself
  verify  ``grid_draft_verify``: the drafted tokens are accepted or refused
          against the masked target distribution by given random numbers, and
          the token after the accepted ones is drawn

``own`` is false: ``run`` computes the operators from elementary torch
operations in 32 bits, rounded once at the end.  ``own`` is true: ``run`` makes
the calls of the public binding (``paper_2607_11951_gb300.grid``).

Formulas.  x a head's vector of D values, t its token's position, c and s the
row t of the cosine and sine tables:
  norm    x_d <- x_d w_d / sqrt(mean(x^2) + eps)
  rotate  (x_i, x_j) <- (x_i c_m - x_j s_m, x_j c_m + x_i s_m), m < R/2, with
          (i, j) = (m, m + R/2), or (2m, 2m + 1) for ``pairs``; d >= R unchanged
  attend  out = sum_j p_j v_j, p = softmax_j(scale q.k_j) over the keys j with
          position <= the query's, lse = log sum_j exp(scale q.k_j)
  verify  p_k = softmax(l_k / T) over the admitted tokens of position k; the
          drafted x_k is accepted when u_k q_k(x_k) < p_k(x_k), up to the first
          refusal at n; the next token is argmax_i w_i / e_i with
          w = max(p_n - q_n, 0) after a refusal (p_n where that is all zero)
          and w = p_n when all were accepted; T <= 0: x_k is accepted when it
          is the first largest admitted logit, which is also the next token
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
        # one interactive request's next token in a small model: launch latency is all of it
        dict(name="append_token_b1", kind="append", B=1, n=1, ctx=400, heads=8, kv_heads=2, D=64, page=16, dtype="bf16",
             order="token", rot=64, pairs=False, norm=False),
        # the decoding step of a full serving batch, queries and keys normed per head
        dict(name="append_tokens_b256", kind="append", B=256, n=1, ctx=2000, heads=32, kv_heads=8, D=128, page=16,
             dtype="bf16", order="token", rot=128, pairs=False, norm=True),
        # forced spans of 0 to 8 tokens over an odd batch, half of each head rotated in pairs
        dict(name="append_spans_b27", kind="append", B=27, n=8, ctx=200, heads=14, kv_heads=2, D=64, page=32,
             dtype="f16", order="head", rot=32, pairs=True, norm=False),
        # a batch of prompts: the longest prefixes of the SQL workloads
        dict(name="append_prompts_b32", kind="append", B=32, n=2000, ctx=0, heads=32, kv_heads=8, D=128, page=64,
             dtype="bf16", order="token", rot=128, pairs=False, norm=True),
        # the same interactive request's attention
        dict(name="attend_token_b1", kind="attend", B=1, n=1, ctx=400, heads=8, kv_heads=2, D=64, page=16, dtype="bf16",
             order="token"),
        # the decoding step of the benchmark's batch, ragged contexts
        dict(name="attend_tokens_b32", kind="attend", B=32, n=1, ctx=2000, heads=32, kv_heads=8, D=128, page=16,
             dtype="bf16", order="token"),
        # four drafted tokens and the one before them, long generations
        dict(name="attend_drafts_b32", kind="attend", B=32, n=5, ctx=16_000, heads=32, kv_heads=8, D=128, page=64,
             dtype="bf16", order="head"),
        # prompts of an odd batch: seven query heads to a key head, 64-wide heads
        dict(name="attend_prompts_b27", kind="attend", B=27, n=2000, ctx=0, heads=14, kv_heads=2, D=64, page=32,
             dtype="f16", order="token"),
        # a chunk of a long prompt: the arithmetic of the largest call
        dict(name="attend_chunk_b2", kind="attend", B=2, n=2000, ctx=16_000, heads=32, kv_heads=8, D=128, page=64,
             dtype="bf16", order="token"),
        # two drafted tokens of one request over the expression grammar's vocabulary
        dict(name="verify_expr_b1", kind="verify", B=1, K=2, V=512, dtype="f32", draft="tokens", greedy=False),
        # the benchmark's batch and vocabulary, four drafted tokens with the drafter's probabilities
        dict(name="verify_sql_b32_f32", kind="verify", B=32, K=4, V=151_936, dtype="f32", draft="probs", greedy=False),
        # the largest batch, some rows greedy, an added token: rows off the sector boundaries
        dict(name="verify_sql_b256_bf16", kind="verify", B=256, K=4, V=151_937, dtype="bf16", draft="probs",
             greedy=True),
    ]


def _spread(rng, lo, hi):
    """An integer spread evenly over the logarithm of [lo, hi]."""
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["append", "attend", "attend", "verify"])
    most = [max(x) for x in zip(*[_cost(c) for c in listed() if c["kind"] == kind])]
    while True:
        c = _draw(rng, kind)
        if all(x <= y for x, y in zip(_cost(c), most)):
            return c


def _cost(c):
    """Bytes and operations of a pass, values of the pool, and the scores that
    the plain attention holds at once (all rows padded to the longest)."""
    w = work(c)
    if c["kind"] == "verify":
        return w["bytes"], w["flops"], 0, 0
    new, old = _lengths(c)
    return (w["bytes"], w["flops"], (sum(new) + sum(old)) * c["kv_heads"] * c["D"],
            c["B"] * c["heads"] * c["n"] * (c["ctx"] + c["n"]) if c["kind"] == "attend" else 0)


def _draw(rng, kind):
    if kind == "verify":
        return dict(kind=kind, B=_spread(rng, 1, 256), K=rng.randint(0, 8), V=_spread(rng, 500, 151_937),
                    dtype=rng.choice(["f32", "bf16"]), draft=rng.choice(["probs", "tokens"]), greedy=rng.random() < 0.3)
    D = rng.choice([64, 128])
    kv = rng.choice([1, 2, 3, 4, 8])
    heads = kv * rng.choice([1, 2, 3, 4, 7, 8, 16])
    n = rng.choice([1, 1, _spread(rng, 2, 32), _spread(rng, 32, 2000)])
    c = dict(kind=kind, B=_spread(rng, 1, 256), n=n, ctx=rng.choice([0, _spread(rng, 50, 2000), _spread(rng, 50, 16_000)]),
             heads=heads, kv_heads=kv, D=D, page=rng.choice([16, 32, 64, 128]), dtype=rng.choice(["bf16", "f16"]),
             order=rng.choice(["token", "head"]))
    if kind == "append":
        c.update(rot=rng.choice([D, D // 2]), pairs=rng.random() < 0.5, norm=rng.random() < 0.5)
    return c


def _lengths(c):
    """Per row the new tokens and the cached ones before them: rows of one token
    in a step, else 0, 1 and up to n tokens; contexts spread from ctx / 16 to ctx."""
    B, n, ctx = c["B"], c["n"], c["ctx"]
    if n == 1 or B == 1:
        new = [n] * B
    elif n <= 32:
        new = [(n + i * (n // 2 + 1)) % (n + 1) for i in range(B)]
    else:
        new = [max(1, n - (i * n) // (2 * B)) for i in range(B)]
    old = [int(ctx * 16.0 ** (-i / max(1, B - 1))) for i in range(B)] if B > 1 else [ctx]
    return new, old


def work(case):
    c = case
    if c["kind"] == "verify":
        B, K, V = c["B"], c["K"], c["V"]
        size = 4 if c["dtype"] == "f32" else 2
        # all positions' logits and masks, the noise, the draft's probabilities of the position that is drawn again,
        # the drafted tokens with their numbers, the outcome
        b = B * (K + 1) * (V * size + (V + 31) // 32 * 4) + B * V * 4 + (B * V * 4 if c["draft"] == "probs" and K else 0)
        return {"bytes": b + B * K * 12 + B * (K + 1) * 8 + B * 12, "flops": B * (K + 1) * V * 5 + B * V * 3}
    new, old = _lengths(c)
    N, H, Hk, D = sum(new), c["heads"], c["kv_heads"], c["D"]
    if c["kind"] == "append":
        moved = 2 * N * (H + 2 * Hk) * D * 2
        return {"bytes": moved + (max(o + k for o, k in zip(old, new)) - min(old)) * c["rot"] * 4 + 4 * c["B"] * 3,
                "flops": N * (H + Hk) * (3 * c["rot"] + (4 * D if c["norm"] else 0))}
    pairs = sum(k * o + k * (k + 1) // 2 for o, k in zip(old, new))
    kv = sum(o + k for o, k in zip(old, new) if k)
    return {"bytes": 2 * kv * Hk * D * 2 + 2 * N * H * D * 2 + N * H * 4 + 4 * c["B"] * 3, "flops": pairs * H * (4 * D + 4)}


# ---------------------------------------------------------------------------
# inputs
def _randn(g, shape, dtype, scale=1.0):
    return (torch.randn(shape, generator=g, device="cuda", dtype=torch.float32) * scale).to(dtype)


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return (_prepare_verify if case["kind"] == "verify" else _prepare_cache)(dict(case), g, random.Random(seed))


def _prepare_cache(c, g, rng):
    dt, B, D, H, Hk, page = DTYPES[c["dtype"]], c["B"], c["D"], c["heads"], c["kv_heads"], c["page"]
    new, old = _lengths(c)
    both = list(zip(new, old))
    rng.shuffle(both)
    new, old = [x[0] for x in both], [x[1] for x in both]
    N = sum(new)
    pages = [-(-(o + k) // page) for o, k in zip(old, new)]
    ids = list(range(sum(pages) + SPARE))
    rng.shuffle(ids)
    table = torch.full((B, max(1, max(pages))), -1, dtype=torch.int32)
    at = 0
    for b, p in enumerate(pages):
        table[b, :p] = torch.tensor(ids[at:at + p], dtype=torch.int32)
        at += p
    start = torch.zeros(B + 1, dtype=torch.int32)
    start[1:] = torch.cumsum(torch.tensor(new), 0)
    s = dict(case=c, lens=torch.tensor(old, dtype=torch.int32).cuda(), start=start.cuda(), table=table.cuda(),
             T=max(new), S=max(o + k for o, k in both), uniform=len(set(new)) == 1)
    # pages in the order [page, token, head] or [page, head, token]
    shape = (len(ids), page, Hk, D) if c["order"] == "token" else (len(ids), Hk, page, D)
    pools = [_randn(g, shape, dt) for _ in range(2)]
    s["k_pages"], s["v_pages"] = pools if c["order"] == "token" else [p.transpose(1, 2) for p in pools]
    s["status"] = torch.full((B,), -1, dtype=torch.int32, device="cuda")
    if c["kind"] == "append":
        # one projection's output holds a token's queries, keys and values
        qkv = _randn(g, (N, H + 2 * Hk, D), dt)
        s["q"], s["k"], s["v"] = qkv[:, :H], qkv[:, H:H + Hk], qkv[:, H + Hk:]
        freq = 10000.0 ** (-torch.arange(0, c["rot"], 2, device="cuda", dtype=torch.float64) / c["rot"])
        angle = torch.arange(s["S"], device="cuda", dtype=torch.float64)[:, None] * freq
        s["cos"], s["sin"] = angle.cos().float(), angle.sin().float()
        s["q_norm"] = s["k_norm"] = None
        if c["norm"]:
            s["q_norm"], s["k_norm"] = ((1 + 0.2 * _randn(g, (D,), torch.float32)).to(dt) for _ in range(2))
        s["q_out"] = torch.empty((N, H, D), dtype=dt, device="cuda")
    else:
        s["q"] = _randn(g, (N, H, D), dt, 1.5)  # (scores of a few units: some keys matter more than others)
        s["out"] = torch.empty((N, H, D), dtype=dt, device="cuda")
        s["lse"] = torch.empty((N, H), dtype=torch.float32, device="cuda")
        s["scale"] = 1 / math.sqrt(D)
    if own:  # the handle that a serving program makes once for its cache
        from paper_2607_11951_gb300 import grid as G
        s["kv"] = G.PagedKV(s["k_pages"], s["v_pages"], H)
    return s


def _prepare_verify(c, g, rng):
    B, K, V, dt = c["B"], c["K"], c["V"], DTYPES[c["dtype"]]
    s = dict(case=c)
    rand = lambda *shape: torch.rand(shape, generator=g, device="cuda")  # noqa: E731
    logits = _randn(g, (B, K + 1, V), dt, 3.0)
    # masks of a grammar: some positions admit a handful of tokens, others most of the vocabulary
    W = (V + 31) // 32
    share = torch.where(rand(B, K + 1, 1) < 0.3, 20.0 / V, rand(B, K + 1, 1))
    bits = rand(B, K + 1, W * 32) < share
    bits[:, :, V:] = False
    s["mask"] = _pack(bits)
    temp = 0.5 + rand(B)
    if c["greedy"]:
        temp[rand(B) < 0.5] = 0.0
    s["logits"], s["temperature"] = logits, temp
    # the drafter knows the grammar and is a worse model: its logits are the target's with noise
    low = logits[:, :K].float() / torch.where(temp > 0, temp, 1.0)[:, None, None]
    low = (low + 0.7 * _randn(g, (B, K, V), torch.float32)).masked_fill_(~bits[:, :K, :V], -math.inf)
    probs = torch.softmax(low, 2).nan_to_num_(0.0)
    noise = torch.empty_like(probs).exponential_(generator=g)
    draft = torch.where((temp > 0)[:, None], (probs / noise).argmax(2), probs.argmax(2)) if K else \
        torch.zeros((B, 0), dtype=torch.int64, device="cuda")
    # and now and then proposes what the grammar refuses
    stray = torch.randint(0, V, (B, K), generator=g, device="cuda")
    s["draft"] = torch.where(rand(B, K) < 0.05, stray, draft).int()
    s["draft_len"] = torch.where(rand(B) < 0.2, (rand(B) * (K + 1)).int(), K).int()
    s["probs"] = probs if c["draft"] == "probs" and K else None
    s["u"] = rand(B, K)
    s["noise"] = torch.empty((B, V), device="cuda").exponential_(generator=g)
    s["tokens"] = torch.empty((B, K + 1), dtype=torch.int32, device="cuda")
    s["accepted"], s["status"] = (torch.empty((B,), dtype=torch.int32, device="cuda") for _ in range(2))
    s["logprob"] = torch.empty((B, K + 1), dtype=torch.float32, device="cuda")
    if own:  # the handle that a serving program makes once for its batch
        from paper_2607_11951_gb300 import grid as G
        s["drafts"] = G.Drafts(B, K, V)
    return s


def _pack(bits):
    """Truth values [..., 32 W] as int32 words [..., W], the lowest bit first."""
    x = bits.view(*bits.shape[:-1], -1, 32).to(torch.int64)
    x = (x << torch.arange(32, device="cuda")).sum(-1)
    return torch.where(x >= 1 << 31, x - (1 << 32), x).int()


def _unpack(words, V):
    x = (words[..., None] >> torch.arange(32, device="cuda", dtype=torch.int32)) & 1
    return x.flatten(-2)[..., :V].bool()


# ---------------------------------------------------------------------------
# one pass
def run(state):
    return {"append": _append, "attend": _attend, "verify": _verify}[state["case"]["kind"]](state)


def _append(s):
    c = s["case"]
    start = None if s["uniform"] else s["start"]
    if own:
        from paper_2607_11951_gb300 import grid as G
        G.grid_kv_append(s["kv"], s["table"], s["lens"], s["k"], s["v"], s["status"], start=start, q=s["q"],
                         q_out=s["q_out"], cos=s["cos"], sin=s["sin"], pairs=c["pairs"], q_norm=s["q_norm"],
                         k_norm=s["k_norm"], eps=EPS)
        return {"q": s["q_out"], "k": s["k_pages"], "v": s["v_pages"], "status": s["status"]}
    i = torch.arange(s["q"].shape[0], device="cuda")
    row = torch.searchsorted(s["start"], i.int(), right=True) - 1
    pos = s["lens"].long()[row] + i - s["start"].long()[row]
    page = s["table"].long()[row, pos // c["page"]]
    rotated = [_rotate(_normed(x.float(), w), s["cos"][pos][:, None], s["sin"][pos][:, None], c["pairs"])
               for x, w in ((s["q"], s["q_norm"]), (s["k"], s["k_norm"]))]
    s["q_out"].copy_(rotated[0])
    s["k_pages"][page, pos % c["page"]] = rotated[1].to(s["k"].dtype)
    s["v_pages"][page, pos % c["page"]] = s["v"]
    return {"q": s["q_out"], "k": s["k_pages"], "v": s["v_pages"], "status": torch.zeros_like(s["status"])}


def _normed(x, w):
    return x if w is None else x * torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS) * w.float()


def _rotate(x, cos, sin, pairs):
    half = cos.shape[-1]
    if pairs:
        a, b = x[..., 0:2 * half:2], x[..., 1:2 * half:2]
        r = torch.stack([a * cos - b * sin, b * cos + a * sin], -1).flatten(-2)
    else:
        a, b = x[..., :half], x[..., half:2 * half]
        r = torch.cat([a * cos - b * sin, b * cos + a * sin], -1)
    return torch.cat([r, x[..., 2 * half:]], -1)


def _attend(s):
    c = s["case"]
    start = None if s["uniform"] else s["start"]
    if own:
        from paper_2607_11951_gb300 import grid as G
        G.grid_kv_attend(s["kv"], s["table"], s["lens"], s["q"], s["out"], s["status"], lse=s["lse"], start=start,
                         scale=s["scale"])
        return {"out": s["out"], "lse": s["lse"], "status": s["status"]}
    B, H, Hk, D, T, S = c["B"], c["heads"], c["kv_heads"], c["D"], s["T"], s["S"]
    first, n = s["start"][:-1].long(), (s["start"][1:] - s["start"][:-1]).long()
    t = torch.arange(T, device="cuda")
    there = t < n[:, None]  # [B, T]: the padded chunk's own tokens
    at = torch.where(there, first[:, None] + t, 0)
    q = s["q"].float()[at].view(B, T, Hk, H // Hk, D).permute(0, 2, 3, 1, 4).reshape(B, Hk, H // Hk * T, D)
    j = torch.arange(S, device="cuda")
    used = j < (s["lens"] + n)[:, None]  # [B, S]: the row's own keys
    page = torch.where(used, s["table"].long()[:, j // c["page"]], 0)
    k, v = (p[page, j % c["page"]].float().masked_fill_(~used[:, :, None, None], 0.0).transpose(1, 2)
            for p in (s["k_pages"], s["v_pages"]))  # [B, Hk, S, D]
    x = (q @ k.transpose(2, 3)).mul_(s["scale"]).view(B, Hk, H // Hk, T, S)
    x.masked_fill_(j > (s["lens"].long()[:, None] + t)[:, None, None, :, None], -math.inf)
    m = x.amax(-1, keepdim=True)
    p = x.sub_(m).exp_()
    z = p.sum(-1, keepdim=True)
    out = (p.view(B, Hk, H // Hk * T, S) @ v).view(B, Hk, H // Hk, T, D) / z
    s["out"].copy_(out.permute(0, 3, 1, 2, 4).reshape(B, T, H, D)[there])
    s["lse"].copy_((m + z.log()).squeeze(-1).permute(0, 3, 1, 2).reshape(B, T, H)[there])
    return {"out": s["out"], "lse": s["lse"], "status": torch.zeros_like(s["status"])}


def _verify(s):
    if own:
        from paper_2607_11951_gb300 import grid as G
        G.grid_draft_verify(s["drafts"], s["logits"], s["draft"], s["u"], s["noise"], s["tokens"], s["accepted"],
                            s["status"], mask=s["mask"], probs=s["probs"], draft_len=s["draft_len"],
                            temperature=s["temperature"], logprob=s["logprob"])
        return {k: s[k] for k in ("tokens", "accepted", "status", "logprob")}
    c = s["case"]
    B, K, V = c["B"], c["K"], c["V"]
    greedy = s["temperature"] <= 0
    inv = 1 / torch.where(greedy, 1.0, s["temperature"])
    x = s["logits"].float() * inv[:, None, None]
    x = torch.where(_unpack(s["mask"], V), x, -math.inf)
    m = x.amax(2, keepdim=True)
    w = (x - torch.where(m > -math.inf, m, 0.0)).exp()
    z = w.sum(2, keepdim=True)
    ids = torch.arange(V, device="cuda")
    best = torch.where(x == m, ids, V).amin(2)  # [B, K + 1]: the first largest
    draft = s["draft"].long()
    px = (w[:, :K].gather(2, draft[..., None]) / z[:, :K])[..., 0]  # (0 / 0, which accepts nothing, where no token is admitted)
    qx = s["probs"].gather(2, draft[..., None])[..., 0] if s["probs"] is not None else torch.ones_like(px)
    accept = torch.where(greedy[:, None], (draft == best[:, :K]) & (px > 0), s["u"] * qx < px)
    n_draft = s["draft_len"].long()
    accept &= torch.arange(K, device="cuda") < n_draft[:, None]
    n = accept.long().cumprod(1).sum(1)
    b = torch.arange(B, device="cuda")
    p = w[b, n] / z[b, n]
    refused = (n < n_draft)[:, None]
    if s["probs"] is not None:
        rest = (p - s["probs"][b, n.clamp(max=K - 1)]).clamp(min=0.0)
    elif K:
        rest = torch.where(ids == draft[b, n.clamp(max=K - 1)][:, None], 0.0, p)
    else:
        rest = p
    rest = torch.where(refused & (rest.amax(1, keepdim=True) > 0), rest, p)
    score = rest / s["noise"]
    token = torch.where(score == score.amax(1, keepdim=True), ids, V).amin(1)
    token = torch.where(greedy, best[b, n], token)
    empty = z[b, n, 0] == 0
    k = torch.arange(K + 1, device="cuda")
    tokens = torch.cat([draft, draft.new_zeros((B, 1))], 1)
    tokens = torch.where(k < n[:, None], tokens, torch.where((k == n[:, None]) & ~empty[:, None], token[:, None], -1))
    chosen = x.gather(2, tokens.clamp(min=0)[..., None])
    logprob = torch.where(tokens >= 0, (chosen - m - z.log())[..., 0], 0.0)
    return {"tokens": tokens.int(), "accepted": n.int(), "status": torch.where(empty, 4, 0).int(), "logprob": logprob}


# ---------------------------------------------------------------------------
# the same in 64 bits, row by row from the definitions
def exact(case, seed):
    s = prepare(case, seed)
    return {"append": _exact_append, "attend": _exact_attend, "verify": _exact_verify}[case["kind"]](case, s)


def _exact_append(c, s):
    half = c["rot"] // 2
    start, lens, table = s["start"].tolist(), s["lens"].tolist(), s["table"].tolist()
    pos = [lens[b] + i for b in range(c["B"]) for i in range(start[b + 1] - start[b])]
    slot = [table[b][(lens[b] + i) // c["page"]] * c["page"] + (lens[b] + i) % c["page"]
            for b in range(c["B"]) for i in range(start[b + 1] - start[b])]
    pos, slot = torch.tensor(pos, device="cuda"), torch.tensor(slot, device="cuda")
    first = torch.arange(half, device="cuda") * (2 if c["pairs"] else 1)
    second = first + (1 if c["pairs"] else half)
    # the tables are inputs: their 32-bit values stand
    turn = torch.complex(s["cos"].double()[pos], s["sin"].double()[pos])[:, None]

    def turned(x, w):
        x = x.double()
        if w is not None:
            x = x / (x.pow(2).sum(-1, keepdim=True) / c["D"] + EPS).sqrt() * w.double()
        z = torch.complex(x[..., first], x[..., second]) * turn
        y = x.clone()
        y[..., first], y[..., second] = z.real, z.imag
        return y

    def stored(pool, x):
        flat = pool.double().reshape(-1, c["kv_heads"], c["D"])
        flat[slot] = x
        return flat.view(pool.shape)

    return {"q": turned(s["q"], s["q_norm"]), "k": stored(s["k_pages"], turned(s["k"], s["k_norm"])),
            "v": stored(s["v_pages"], s["v"].double()), "status": None}


def _exact_attend(c, s):
    H, Hk, D, page = c["heads"], c["kv_heads"], c["D"], c["page"]
    start, lens, table = s["start"].tolist(), s["lens"].tolist(), s["table"]
    if work(c)["flops"] > 4e12:  # (about 20 s at this card's 64-bit rate)
        return None
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda")
    lse = torch.zeros(s["lse"].shape, dtype=torch.float64, device="cuda")
    for b in range(c["B"]):
        a, z = start[b], start[b + 1]
        total = lens[b] + z - a
        used = table[b, :-(-total // page)].long()
        k, v = (p[used].reshape(-1, Hk, D)[:total].double() for p in (s["k_pages"], s["v_pages"]))
        for t in range(a, z, 256):
            e = min(z, t + 256)
            hidden = torch.arange(total, device="cuda") > torch.arange(lens[b] + t - a, lens[b] + e - a, device="cuda")[:, None]
            for h in range(H):
                x = s["q"][t:e, h].double() @ k[:, h * Hk // H].T * s["scale"]
                x[hidden] = -math.inf
                lse[t:e, h] = torch.logsumexp(x, 1)
                out[t:e, h] = torch.exp(x - lse[t:e, h, None]) @ v[:, h * Hk // H]
    return {"out": out, "lse": lse, "status": None}


def _exact_verify(c, s):
    tokens, lp = [], []
    for b in range(c["B"]):
        T = float(s["temperature"][b])
        n_draft, draft, u = int(s["draft_len"][b]), s["draft"][b].tolist(), s["u"][b].tolist()
        logs = []
        for k in range(n_draft + 1):
            admitted = _unpack(s["mask"][b, k], c["V"])
            logits = s["logits"][b, k].double()
            if not bool(admitted.any()):
                token = -1
                break
            logp = torch.log_softmax((logits / T if T > 0 else logits).masked_fill(~admitted, -math.inf), 0)
            p = logp.exp()
            best = int(torch.nonzero(logp == logp.max())[0])
            last = k == n_draft
            if not last:
                q = s["probs"][b, k].double() if s["probs"] is not None else \
                    torch.zeros_like(p).index_fill_(0, s["draft"][b, k].long(), 1.0)
                x = draft[k]
                if (x == best) if T <= 0 else (u[k] * float(q[x]) < float(p[x])):
                    logs.append(float(logp[x]))
                    continue
                if float((p - q).max()) > 0:
                    p = (p - q).clamp(min=0)
            score = p / s["noise"][b].double()
            token = best if T <= 0 else int(torch.nonzero(score == score.max())[0])
            logs.append(float(logp[token]))
            break
        lp.append(logs + [0.0] * (c["K"] + 1 - len(logs)))
    return {"tokens": None, "accepted": None, "status": None,
            "logprob": torch.tensor(lp, dtype=torch.float64)}
