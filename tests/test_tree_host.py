"""What the calls for trees, sampling and pages refuse before they launch
anything, what they launch, and that a failing CUDA call leaves nothing behind:
the library on a CUDA runtime without a GPU (no pointer here is dereferenced)."""
import ctypes

import pytest

from paper_2607_11951_gb300 import grid as G
from tests import fakes
from tests import structs as S
from tests import tree_structs as T

INVALID, CUDA, TOO_LARGE = -1, -7, -8
AT = 1 << 20  # an aligned address


@pytest.fixture(scope="module")
def fake(tmp_path_factory):
    return fakes.link(tmp_path_factory.mktemp("fake"))


def refused(rt, name, code, *args):
    rt.reset()
    assert getattr(G.lib(), name)(*args) == code, (name, args)
    assert G.last_error().startswith(name + ":") and not rt.launches()


def tree(**kw):
    return ctypes.byref(T.Tree(**{**dict(d_parent=AT, d_start=AT, B=4, n_tokens=40), **kw}))


TREES = [dict(d_parent=None), dict(B=0), dict(B=-1), dict(n_tokens=-1), dict(d_start=None, n_tokens=41)]


def test_trees_that_are_refused(fake):
    with fakes.use(fake) as rt:
        for bad in TREES:
            refused(rt, "grid_tree_plan", INVALID, tree(**bad), AT, AT, 2, AT, None)
            refused(rt, "grid_tree_accept", INVALID, tree(**bad), AT, AT, -1, 4, AT, AT, AT, AT, None)
        refused(rt, "grid_tree_plan", TOO_LARGE, tree(B=65_536), AT, AT, 2, AT, None)
        refused(rt, "grid_tree_plan", TOO_LARGE, tree(), AT, AT, 33, AT, None)
        for i in (1, 2, 4):
            args = [tree(), AT, AT, 2, AT, None]
            args[i] = None
            refused(rt, "grid_tree_plan", INVALID, *args)
        refused(rt, "grid_tree_plan", INVALID, tree(), AT, AT, 0, AT, None)
        refused(rt, "grid_tree_accept", TOO_LARGE, tree(B=65_536), AT, AT, -1, 4, AT, AT, AT, AT, None)
        for i in (1, 2, 5, 6, 7, 8):
            args = [tree(), AT, AT, -1, 4, AT, AT, AT, AT, None]
            args[i] = None
            refused(rt, "grid_tree_accept", INVALID, *args)
        refused(rt, "grid_tree_accept", INVALID, tree(), AT, AT, -1, 0, AT, AT, AT, AT, None)
        for t in (tree(), tree(d_start=None), tree(n_tokens=0, d_parent=None), tree(B=65_535, n_tokens=0)):
            rt.reset()
            assert G.lib().grid_tree_plan(t, AT, AT, 2, AT, None) == 0 and len(rt.launches()) == 1
            assert rt.launches()[0][1][0] == t._obj.B
            rt.reset()
            assert G.lib().grid_tree_accept(t, AT, AT, -1, 4, AT, AT, AT, AT, None) == 0
            assert rt.launches()[0][1][0] * 4 >= t._obj.B
        assert G.lib().grid_tree_plan(tree(n_tokens=0), None, None, 2, AT, None) == 0
        assert G.lib().grid_tree_accept(tree(n_tokens=0), None, None, -1, 4, AT, AT, AT, AT, None) == 0


class Kv(ctypes.Structure):
    """A handle as far as a call that is refused looks at it: the pools, then what is behind them."""
    _fields_ = [("p", G._KvPages), ("gave_up", ctypes.c_void_p), ("log_page", ctypes.c_int), ("sms", ctypes.c_int),
                ("rest", ctypes.c_byte * 1024)]


def cache():
    kv = Kv(log_page=4, sms=152)
    kv.p = G._KvPages(AT, AT, G.GRID_DTYPE_BF16, 128, 8, 2, 16, 100, (4096, 256, 128), (4096, 256, 128))
    return kv


def test_calls_on_a_cache_that_are_refused(fake):
    chunk = lambda **kw: ctypes.byref(S.KvChunk(**{**dict(d_table=AT, table_stride=3, d_len=AT, d_start=AT, max_pages=3, B=2,  # noqa: E731
                                                          n_tokens=2), **kw}))
    heads = ctypes.byref(S.Heads(AT, 256, 128))
    query = ctypes.byref(S.KvQuery(S.Heads(AT, 256, 128), S.Heads(AT, 256, 128), None, 0.125, 0))
    kv = cache()
    h = ctypes.byref(kv)
    with fakes.use(fake) as rt:
        for bad, code in ((dict(d_table=None), INVALID), (dict(d_len=None), INVALID), (dict(B=0), INVALID), (dict(n_tokens=-1), INVALID),
                          (dict(max_pages=0), INVALID), (dict(table_stride=2), INVALID), (dict(d_start=None, n_tokens=1), INVALID),
                          (dict(B=65_536), TOO_LARGE)):
            refused(rt, "grid_kv_compact", code, h, chunk(**bad), AT, AT, 4, AT, None)
            refused(rt, "grid_kv_append_tree", code, h, chunk(**bad), heads, heads, None, None, None, None, AT, AT, None)
            refused(rt, "grid_kv_attend_tree", code, h, chunk(**bad), query, AT, 1, AT, None)
        refused(rt, "grid_kv_attend_tree", INVALID, h, chunk(), query, AT, 0, AT, None)
        refused(rt, "grid_kv_attend_tree", INVALID, h, chunk(), query, AT + 2, 1, AT, None)
        refused(rt, "grid_kv_attend_tree", INVALID, h, chunk(), query, AT, 1, None, None)
        for i, v in ((2, None), (3, None), (4, 0), (5, None)):
            args = [h, chunk(), AT, AT, 4, AT, None]
            args[i] = v
            refused(rt, "grid_kv_compact", INVALID, *args)
        for i, v, code in ((1, None, INVALID), (2, 0, INVALID), (2, 65_536, TOO_LARGE), (3, None, INVALID)):
            args = [h, AT, 3, AT, None]
            args[i] = v
            refused(rt, "grid_kv_copy", code, *args)
        rt.reset()
        assert G.lib().grid_kv_compact(h, chunk(), AT, AT, 4, AT, None) == 0
        assert G.lib().grid_kv_copy(h, AT, 3, AT, None) == 0
        assert G.lib().grid_kv_append_tree(h, chunk(), heads, heads, None, None, None, None, AT, AT, None) == 0
        assert len(rt.launches()) == 3 and all(g[0] > 0 for _, g, *_ in rt.launches())


def pages(**kw):
    return ctypes.byref(T.PagesStep(**{**dict(d_table=AT, table_stride=9, d_held=AT, d_parent=AT, d_keep=AT, d_want=AT, d_pinned=AT, A=3,
                                              width=9, B=4, width_out=8, d_table_out=AT, table_out_stride=8, d_held_out=AT,
                                              d_copies=AT, d_refs=AT, d_status=AT), **kw}))


def test_updates_that_are_refused(fake):
    with fakes.use(fake) as rt:
        for n, page, code in ((0, 16, INVALID), (-1, 16, INVALID), (10, 4, INVALID), (10, 24, INVALID), (10, 2048, INVALID)):
            out = ctypes.c_void_p()
            assert G.lib().grid_pages_create(n, page, ctypes.byref(out)) == code and not out.value
            assert G.last_error().startswith("grid_pages_create:")
        G.lib().grid_pages_free(None)
        p = G.Pages(100, 16)
        for bad in [{k: None} for k in ("d_table", "d_held", "d_want", "d_table_out", "d_held_out", "d_copies", "d_refs", "d_status")] + \
                [dict(A=0), dict(B=0), dict(width=0), dict(width_out=0), dict(table_stride=8), dict(table_out_stride=7), dict(d_parent=None)]:
            refused(rt, "grid_pages_update", INVALID, p.h, pages(**bad), None)
        for bad in (dict(A=65_536), dict(B=65_536), dict(B=60_000, width_out=60_000, table_out_stride=60_000)):
            refused(rt, "grid_pages_update", TOO_LARGE, p.h, pages(**bad), None)
        refused(rt, "grid_pages_update", INVALID, None, pages(), None)
        for s in (pages(), pages(d_parent=None, A=4), pages(d_keep=None, d_pinned=None)):
            rt.reset()
            assert G.lib().grid_pages_update(p.h, s, None) == 0 and len(rt.launches()) >= 1
        del p  # (by the library that made it)


def test_scratch_of_updates_is_freed_when_a_call_fails(fake):
    with fakes.use(fake) as rt:
        out = ctypes.c_void_p()
        rt.reset()
        assert G.lib().grid_pages_create(4, 16, ctypes.byref(out)) == 0
        calls = rt.get("calls")
        G.lib().grid_pages_free(out)
        assert rt.get("live") == 0 and calls >= 2
        for k in range(1, calls + 1):
            rt.reset(fail_at=k)
            out = ctypes.c_void_p()
            assert G.lib().grid_pages_create(4, 16, ctypes.byref(out)) == CUDA and not out.value
            assert rt.get("live") == 0, k


def sample(**kw):
    return ctypes.byref(T.SampleStep(**{**dict(d_logits=AT, logit_stride=100, d_mask=AT, mask_stride=4, d_noise=AT, noise_stride=100,
                                               d_temperature=AT, d_top_k=AT, d_top_p=AT, d_min_p=AT, dtype=G.GRID_DTYPE_F32, B=4, V=100,
                                               eos=-1, d_tokens=AT, d_logprob=AT, d_status=AT), **kw}))


@pytest.mark.parametrize("bad,code", [
    (dict(d_logits=None), INVALID), (dict(d_noise=None), INVALID), (dict(d_tokens=None), INVALID), (dict(d_status=None), INVALID),
    (dict(B=0), INVALID), (dict(V=0), INVALID), (dict(dtype=G.GRID_DTYPE_F16), INVALID), (dict(d_logits=AT + 2), INVALID),
    (dict(d_mask=AT + 2), INVALID), (dict(d_noise=AT + 1), INVALID), (dict(logit_stride=-1), INVALID), (dict(mask_stride=-4), INVALID),
    (dict(noise_stride=-1), INVALID), (dict(B=65_536), TOO_LARGE), (dict(V=393_217), TOO_LARGE)])
def test_a_draw_that_is_refused(fake, bad, code):
    with fakes.use(fake) as rt:
        refused(rt, "grid_sample", code, sample(**bad), None)
        assert G.lib().grid_sample(sample(), None) == 0 and len(rt.launches()) >= 1


@pytest.mark.parametrize("dtype", [G.GRID_DTYPE_F32, G.GRID_DTYPE_BF16])
@pytest.mark.parametrize("B,V", [(1, 1), (3, 4096), (256, 151_937), (65_535, 33), (2, 393_216)])
def test_a_draw_fits_the_device(fake, dtype, B, V):
    """Whole rows of blocks, and no more shared memory than a block may have."""
    with fakes.use(fake) as rt:
        rt.reset()
        assert G.lib().grid_sample(sample(B=B, V=V, dtype=dtype), None) == 0
        for _, g, threads, smem, limit in rt.launches():
            assert g[0] % B == 0 and g[1] == g[2] == 1 and smem <= limit <= 227 << 10 and threads <= 1024
