"""The calls on tensors refuse a tensor of the right number of values and the
wrong shape: each tensor of each call in turn, as a row, as a column, turned
round, and with an axis too many."""
import pytest

pytestmark = pytest.mark.gpu


def ints(x):
    import torch
    return torch.tensor(x, dtype=torch.int32).cuda()


def zeros(*s):
    import torch
    return torch.zeros(s, dtype=torch.int32, device="cuda")


def calls():
    """name -> (call, tensors by name, other arguments, which of them may be strided)."""
    import torch
    from paper_2607_11951_gb300 import grid as G
    B, n, H, Hk, D, page, V = 3, 4, 6, 2, 64, 16, 40
    N, half = B * n, 32
    bf = lambda *s: torch.randn(s, device="cuda").bfloat16()  # noqa: E731
    f32 = lambda *s: torch.rand(s, device="cuda") + 0.1  # noqa: E731
    kv = G.PagedKV(bf(6, page, Hk, D), bf(6, page, Hk, D), H)
    chunk = dict(table=ints([[0, 1], [2, 3], [4, 5]]), lens=ints([5, 0, 9]), status=zeros(B), start=ints([0, 4, 8, 12]))
    parent = ints([-1, 0, 0, 1] * B)
    pages = G.Pages(9, page)
    update = dict(table=ints([[0, 1], [2, -1]]), held=ints([20, 9]), want=ints([21, 22, 10]), table_out=zeros(B, 2), held_out=zeros(B),
                  copies=zeros(3, B), refs=zeros(9), status=zeros(B), parent=ints([0, 0, 1]), keep=ints([20, 18, 9]), pinned=zeros(9))
    return {
        "append": (G.grid_kv_append, dict(chunk, k=bf(N, Hk, D), v=bf(N, Hk, D), q=bf(N, H, D), q_out=bf(N, H, D), cos=f32(40, half),
                                          sin=f32(40, half), q_norm=bf(D), k_norm=bf(D), depth=ints([0, 1, 1, 2] * B)), dict(kv=kv)),
        "attend": (G.grid_kv_attend, dict(chunk, q=bf(N, H, D), out=bf(N, H, D), lse=f32(N, H), sees=zeros(N, 1)), dict(kv=kv)),
        "compact": (G.grid_kv_compact, dict(chunk, path=ints([[0, 1], [0, 2], [0, -1]]), count=ints([2, 2, 1])), dict(kv=kv, n_tokens=N)),
        "copy": (G.grid_kv_copy, dict(copies=ints([[0, -1], [1, 0], [3, 0]]), status=zeros(2)), dict(kv=kv)),
        "plan": (G.grid_tree_plan, dict(parent=parent, depth=zeros(N), sees=zeros(N, 1), status=zeros(B), start=chunk["start"]), {}),
        "accept": (G.grid_tree_accept, dict(parent=parent, tokens=zeros(N), sampled=zeros(N), path=zeros(B, 2), count=zeros(B),
                                            out=zeros(B, 2), status=zeros(B), start=chunk["start"]), {}),
        "sample": (G.grid_sample, dict(logits=f32(B, V), noise=f32(B, V), tokens=zeros(B), status=zeros(B), mask=zeros(B, 2) - 1,
                                       temperature=f32(B), top_k=zeros(B), top_p=f32(B), min_p=f32(B), logprob=f32(B)), {}),
        "update": (G.grid_pages_update, update, dict(pages=pages)),
    }


@pytest.mark.parametrize("name", ["append", "attend", "compact", "copy", "plan", "accept", "sample", "update"])
def test_every_shape_is_looked_at(name):
    import torch
    call, tensors, more = calls()[name]
    call(**tensors, **more)
    for key, t in tensors.items():
        bad = [t[None], t[..., None], t.flatten()[:-1]]
        if t.dim() == 1:
            bad += [t[:, None], t.view(2, -1) if t.numel() % 2 == 0 else t.view(1, -1)]
        else:
            bad += [t.flatten(), t.transpose(0, 1).contiguous()]
            bad += [t.flatten().view(1, -1), t.flatten().view(-1, 1)]
        for x in bad:
            if x.shape == t.shape:
                continue
            with pytest.raises((AssertionError,)):
                call(**{**tensors, key: x}, **more)
    torch.cuda.synchronize()
    call(**tensors, **more)
