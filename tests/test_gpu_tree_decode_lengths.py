"""How far the tree decoding loop of examples/tree_decode.py comes: a live row
takes a token at least in each step, one that ended takes none, and drafts that
are accepted take some rows further than the steps."""
import pytest

pytestmark = pytest.mark.gpu

STEPS = 20


@pytest.mark.parametrize("stem,branches,samples", [(0, 0, 1), (0, 0, 2), (3, 2, 1), (1, 4, 2), (4, 0, 3)])
def test_greedy_rows_go_on_until_they_end(stem, branches, samples):
    from examples.draft_decode import decode as one_by_one
    from examples.tree_decode import decode
    from workloads import configs
    wl = configs.tiny_expr(B=12)
    want = one_by_one(wl, 0, STEPS)
    assert any(len(w) == STEPS and w[-1] != wl["eos"] for w in want)
    rows = decode(wl, stem, branches, STEPS, samples)
    for i, r in enumerate(rows):
        w = want[i // samples]
        assert r[:len(w)] == w and wl["eos"] not in r[:-1], (i, r, w)
        if w[-1] == wl["eos"] or not stem:
            assert r == w, (i, r, w)
    # (a step takes the root's draw and as many of the stem's tokens as are accepted)
    assert max(map(len, rows)) <= STEPS * (1 + stem + (branches > 0))


@pytest.mark.parametrize("stem,branches", [(3, 2), (5, 7)])
def test_accepted_drafts_take_rows_further(stem, branches):
    from examples.tree_decode import decode
    from workloads import configs
    wl = configs.tiny_expr(B=12)
    rows = decode(wl, stem, branches, 8, 2, 0.9, 0.9, seed=stem)
    ended = [r[-1] == wl["eos"] for r in rows]
    assert all(len(r) >= 8 or e for r, e in zip(rows, ended))
    assert any(len(r) > 8 for r in rows)
