"""The tree decoding loop of examples/tree_decode.py, which runs the trees,
sampling and pages together: everything that it decodes is what the oracle's
masks admit, greedy rows give the same tokens whatever tree is drafted, and
samples of one prompt do not meet in each other's pages."""
import pytest

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("stem,branches,samples,temperature,top_p", [(3, 2, 2, 0.9, 0.9), (0, 0, 3, 0.9, 1.0), (5, 7, 1, 0.7, 0.8),
                                                                     (2, 1, 2, 0.0, 1.0)])
def test_decoded_tokens_are_admitted(stem, branches, samples, temperature, top_p):
    from examples.tree_decode import decode
    from oracle import compile_grammar
    from workloads import configs
    wl = configs.tiny_expr(B=8)
    og = compile_grammar(wl["grammar"], wl["role"], wl["lexicons"])
    rows = decode(wl, stem, branches, 6, samples, temperature, top_p, seed=stem)
    assert len(rows) == 8 * samples and (any(len(r) > 6 for r in rows) or not stem)
    for i, r in enumerate(rows):
        prefix = wl["prefixes"][i // samples]
        for j, t in enumerate(r):
            cfg = og.config_from_ids(list(prefix) + r[:j], wl["tokens"], wl["eos"], wl["specials"])
            assert not cfg.complete and og.mask(cfg, wl["tokens"], wl["eos"], wl["specials"], ids=[t])[0], (prefix, r, j)


def test_greedy_rows_do_not_depend_on_the_tree_or_the_samples():
    from examples.draft_decode import decode as one_by_one
    from examples.tree_decode import decode
    from workloads import configs
    wl = configs.tiny_expr(B=12)
    want = one_by_one(wl, 0, 20)
    for stem, branches, samples in ((0, 0, 1), (3, 2, 1), (1, 4, 2), (4, 0, 3)):
        got = decode(wl, stem, branches, 20, samples)
        for i, r in enumerate(got):
            n = min(len(want[i // samples]), len(r))
            assert n > 0 and r[:n] == want[i // samples][:n], (stem, branches, i)
