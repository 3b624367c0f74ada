"""The binding's compiled calls without a GPU: they load, take the library's
addresses and refuse what is no tensor or the wrong number of arguments."""
import ctypes

import pytest

from paper_2607_11951_gb300 import grid as G


@pytest.fixture(scope="module")
def calls():
    import os
    if not os.path.exists(G.binding_path()):
        import paper_2607_11951_gb300 as pkg
        pkg.build()
    return G._binding()


def test_every_call_refuses_a_wrong_number_of_arguments(calls):
    for name in ("bind", "kv_append", "kv_attend", "kv_compact", "kv_copy", "tree_plan", "tree_accept", "sample", "pages_update"):
        with pytest.raises(TypeError):
            getattr(calls, name)()


def test_a_cache_that_is_none(calls):
    for name, n in (("kv_append", 17), ("kv_attend", 11), ("kv_compact", 9), ("kv_copy", 4)):
        for cache in (None, b"", bytes(8), 5):
            with pytest.raises(AssertionError):
                getattr(calls, name)(cache, *[None] * (n - 1))


def test_the_bound_calls_are_the_librarys():
    assert len(set(G._BOUND)) == len(G._BOUND)
    for name in G._BOUND:
        assert name in G.EXPORTED and ctypes.cast(getattr(G.lib(), name), ctypes.c_void_p).value


def test_arguments_keep_their_places():
    """What a caller gave by position before trees came means the same."""
    import inspect

    from paper_2607_11951_gb300 import grid as G
    names = lambda f: list(inspect.signature(f).parameters)  # noqa: E731
    assert names(G.grid_kv_append)[:17] == ["kv", "table", "lens", "k", "v", "status", "start", "q", "q_out", "cos", "sin", "pairs",
                                            "q_norm", "k_norm", "eps", "stream", "depth"]
    assert names(G.grid_kv_attend)[:11] == ["kv", "table", "lens", "q", "out", "status", "lse", "start", "scale", "stream", "sees"]
