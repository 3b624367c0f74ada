"""The drafted decoding loop of examples/draft_decode.py: everything that it
decodes is what the oracle's masks admit, and greedy rows give the same tokens
whether drafts are taken or not."""
import pytest

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("K,temperature", [(3, 0.0), (0, 0.9), (4, 0.9)])
def test_decoded_tokens_are_admitted(K, temperature):
    from examples.draft_decode import decode
    from oracle import compile_grammar
    from workloads import configs
    wl = configs.tiny_expr(B=12)
    og = compile_grammar(wl["grammar"], wl["role"], wl["lexicons"])
    rows = decode(wl, K, 6, temperature, seed=K)
    assert any(len(r) > 6 for r in rows) or K == 0
    for prefix, r in zip(wl["prefixes"], rows):
        for i, t in enumerate(r):
            cfg = og.config_from_ids(list(prefix) + r[:i], wl["tokens"], wl["eos"], wl["specials"])
            assert not cfg.complete and og.mask(cfg, wl["tokens"], wl["eos"], wl["specials"], ids=[t])[0], (prefix, r, i)


def test_greedy_rows_do_not_depend_on_the_draft():
    from examples.draft_decode import decode
    from workloads import configs
    wl = configs.tiny_expr(B=16)
    want = decode(wl, 0, 20)
    for K in (1, 3):
        got = decode(wl, K, 20)
        for a, b in zip(want, got):
            n = min(len(a), len(b))
            assert n > 0 and a[:n] == b[:n]
