"""Sizes whose counts would pass 32 bits in a kernel are refused before it is
launched: the library on a CUDA runtime without a GPU."""
import ctypes

import pytest

from paper_2607_11951_gb300 import grid as G
from tests import fakes
from tests import structs as S
from tests.test_tree_host import AT, TOO_LARGE, cache, refused

# the kernels' largest steps: from page to page (eight blocks of 1,024 threads), over a chunk of pieces
STEP, CHUNK, INT_MAX = 8 * 1024, 4 * 128, (1 << 31) - 1


@pytest.fixture(scope="module")
def fake(tmp_path_factory):
    return fakes.link(tmp_path_factory.mktemp("fake"))


def test_pools_whose_indexes_would_wrap(fake):
    with fakes.use(fake) as rt:
        for n in ((1 << 30) + 1, INT_MAX - STEP + 1, INT_MAX):
            rt.reset()
            out = ctypes.c_void_p()
            assert G.lib().grid_pages_create(n, 16, ctypes.byref(out)) == TOO_LARGE and not out.value
            assert G.last_error().startswith("grid_pages_create:") and rt.get("calls") == 0
    # (the last index that a thread forms, and 32 pages to each of 256 warps)
    assert (1 << 30) + STEP + 32 * 256 <= INT_MAX


def shaped(heads, page, D):
    kv = cache()
    kv.p.n_kv_heads, kv.p.n_heads, kv.p.page_size, kv.p.head_dim = heads, heads, page, D
    kv.p.k_stride[:] = kv.p.v_stride[:] = [heads * page * D, heads * D, D]
    kv.log_page = page.bit_length() - 1
    return kv


@pytest.mark.parametrize("heads,page,D,ok", [(65_536, 1024, 128, True), (65_537, 1024, 128, False), (1 << 17, 1024, 128, False),
                                             (1 << 18, 1024, 64, False), (1 << 17, 1024, 64, True), (1 << 22, 64, 128, False)])
def test_copies_of_pages_whose_pieces_would_wrap(fake, heads, page, D, ok):
    pieces = heads * page * D // 8
    assert (pieces + 2 * CHUNK <= INT_MAX) >= ok
    kv = shaped(heads, page, D)
    with fakes.use(fake) as rt:
        if not ok:
            refused(rt, "grid_kv_copy", TOO_LARGE, ctypes.byref(kv), AT, 3, AT, None)
        else:
            rt.reset()
            assert G.lib().grid_kv_copy(ctypes.byref(kv), AT, 3, AT, None) == 0 and len(rt.launches()) == 1


@pytest.mark.parametrize("heads,ok", [(1 << 20, True), (1 << 25, True), ((1 << 25) + 1, False), (1 << 27, False), (1 << 30, False)])
def test_paths_of_heads_whose_pieces_would_wrap(fake, heads, ok):
    kv = shaped(8, 8, 128)
    kv.p.n_kv_heads = heads
    chunk = ctypes.byref(S.KvChunk(d_table=AT, table_stride=3, d_len=AT, d_start=AT, max_pages=3, B=2, n_tokens=2))
    with fakes.use(fake) as rt:
        if not ok:
            refused(rt, "grid_kv_compact", TOO_LARGE, ctypes.byref(kv), chunk, AT, AT, 4, AT, None)
        else:
            rt.reset()
            assert G.lib().grid_kv_compact(ctypes.byref(kv), chunk, AT, AT, 4, AT, None) == 0
            (_, g, threads, *_), = rt.launches()
            assert g[0] * threads == 2 * (2 * heads * 16)
