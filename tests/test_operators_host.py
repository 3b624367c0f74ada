"""What the paged cache's and the verification's calls refuse before they launch
anything, and that a failing CUDA call leaves nothing allocated: the library on
a CUDA runtime without a GPU (no pointer here is dereferenced)."""
import ctypes

import pytest

from paper_2607_11951_gb300 import grid as G
from tests import fakes
from tests import structs as S

INVALID, CUDA, TOO_LARGE = -1, -7, -8
AT = 1 << 20  # an aligned address


@pytest.fixture(scope="module")
def fake(tmp_path_factory):
    return fakes.link(tmp_path_factory.mktemp("fake"))


def last():
    return G.last_error()


def pages(**kw):
    p = G._KvPages(AT, AT, G.GRID_DTYPE_BF16, 128, 8, 2, 16, 100, (4096, 256, 128), (4096, 256, 128))
    for k, v in kw.items():
        setattr(p, k, (ctypes.c_int64 * 3)(*v) if isinstance(v, tuple) else v)
    return p


@pytest.mark.parametrize("bad", [
    dict(d_k=None), dict(d_v=None), dict(d_k=AT + 8), dict(d_v=AT + 2), dict(dtype=G.GRID_DTYPE_F32), dict(dtype=9),
    dict(head_dim=96), dict(head_dim=256), dict(head_dim=0), dict(n_heads=0), dict(n_heads=7), dict(n_kv_heads=0),
    dict(page_size=0), dict(page_size=4), dict(page_size=24), dict(page_size=2048), dict(n_pages=0),
    dict(k_stride=(4096, 256, 0)), dict(v_stride=(4096, -256, 128)), dict(k_stride=(4096, 260, 128)),
    dict(v_stride=(4100, 256, 128))])
def test_a_cache_that_is_refused(bad):
    out = ctypes.c_void_p()
    assert G.lib().grid_kv_create(ctypes.byref(pages(**bad)), ctypes.byref(out)) == INVALID and not out.value
    assert last().startswith("grid_kv_create:")


def test_free_functions_accept_null():
    G.lib().grid_kv_free(None)
    G.lib().grid_drafts_free(None)


@pytest.mark.parametrize("B,K,V,code", [(0, 1, 9, INVALID), (1, -1, 9, INVALID), (1, 65, 9, INVALID), (1, 1, 0, INVALID),
                                        (-3, 1, 9, INVALID), (65_536, 0, 9, TOO_LARGE)])
def test_draft_scratch_that_is_refused(B, K, V, code):
    out = ctypes.c_void_p()
    assert G.lib().grid_drafts_create(B, K, V, ctypes.byref(out)) == code and not out.value
    assert last().startswith("grid_drafts_create:")


def test_draft_scratch_is_freed_when_a_call_fails(fake):
    with fakes.use(fake) as rt:
        out = ctypes.c_void_p()
        rt.reset()
        assert G.lib().grid_drafts_create(4, 2, 100, ctypes.byref(out)) == 0
        calls, live = rt.get("calls"), rt.get("live")
        assert live > 0
        G.lib().grid_drafts_free(out)
        assert rt.get("live") == 0
        for k in range(1, calls + 1):
            rt.reset(fail_at=k)
            out = ctypes.c_void_p()
            assert G.lib().grid_drafts_create(4, 2, 100, ctypes.byref(out)) == CUDA and not out.value
            assert rt.get("live") == 0, k


def step(**kw):
    two = ctypes.c_int64 * 2
    s = S.DraftStep(d_logits=AT, logit_stride=two(300, 100), d_mask=AT, mask_stride=two(12, 4), d_probs=AT,
                     prob_stride=two(200, 100), d_draft=AT, d_draft_len=AT, d_u=AT, d_noise=AT, noise_stride=100,
                     d_temperature=AT, dtype=G.GRID_DTYPE_F32, B=4, K=2, V=100, eos=-1, d_tokens=AT, d_accepted=AT,
                     d_logprob=AT, d_status=AT)
    for k, v in kw.items():
        setattr(s, k, two(*v) if isinstance(v, tuple) else v)
    return s


@pytest.mark.parametrize("bad,code", [
    (dict(d_logits=None), INVALID), (dict(d_noise=None), INVALID), (dict(d_draft=None), INVALID), (dict(d_u=None), INVALID),
    (dict(d_tokens=None), INVALID), (dict(d_accepted=None), INVALID), (dict(d_status=None), INVALID), (dict(B=0), INVALID),
    (dict(K=-1), INVALID), (dict(V=0), INVALID), (dict(dtype=G.GRID_DTYPE_F16), INVALID), (dict(B=5), TOO_LARGE),
    (dict(K=3), TOO_LARGE), (dict(V=101), TOO_LARGE), (dict(d_logits=AT + 2), INVALID), (dict(d_mask=AT + 2), INVALID),
    (dict(d_probs=AT + 1), INVALID), (dict(d_noise=AT + 2), INVALID), (dict(logit_stride=(300, -1)), INVALID),
    (dict(mask_stride=(-12, 4)), INVALID), (dict(prob_stride=(200, -100)), INVALID), (dict(noise_stride=-1), INVALID)])
def test_a_verification_that_is_refused(fake, bad, code):
    with fakes.use(fake) as rt:
        d = G.Drafts(4, 2, 100)
        rt.reset()
        assert G.lib().grid_draft_verify(d.h, ctypes.byref(step(**bad)), None) == code
        assert last().startswith("grid_draft_verify:") and not rt.launches()
        assert G.lib().grid_draft_verify(d.h, ctypes.byref(step()), None) == 0 and len(rt.launches()) >= 1
        assert G.lib().grid_draft_verify(d.h, ctypes.byref(step(d_mask=None, d_probs=None, d_draft_len=None, d_logprob=None,
                                                                d_temperature=None)), None) == 0
        assert G.lib().grid_draft_verify(d.h, ctypes.byref(step(K=0, d_draft=None, d_u=None)), None) == 0


@pytest.mark.parametrize("B,K,V", [(1, 0, 1), (1, 8, 151_937), (256, 4, 151_936), (65_535, 0, 33), (3, 64, 5_000)])
def test_launches_cover_every_position(fake, B, K, V):
    """At least one block per position and per row, and no more than the scratch has room for."""
    with fakes.use(fake) as rt:
        d = G.Drafts(B, K, V)
        rt.reset()
        assert G.lib().grid_draft_verify(d.h, ctypes.byref(step(B=B, K=K, V=V, noise_stride=V)), None) == 0
        (_, g0, *_), *draw = rt.launches()
        rows = B * (K + 1)
        assert g0[0] % rows == 0 and rows <= g0[0] <= rows + 8 * 152 and g0[1] == g0[2] == 1
        assert len(draw) == (V > 4096)
        for _, g1, *_ in draw:
            assert g1[0] % B == 0 and B <= g1[0] <= B + 24 * 152


def test_packed_arguments_have_the_layout_of_the_structures():
    """What the binding packs is, byte for byte, the structure with these values."""
    for packed, structure in ((G._HEADS, S.Heads), (G._CHUNK, S.KvChunk), (G._ROTATION, S.Rotation), (G._NORM, S.HeadNorm),
                              (G._QUERY, S.KvQuery), (G._STEP, S.DraftStep)):
        assert packed.size == ctypes.sizeof(structure)
        values = list(range(1, len(packed.unpack(bytes(packed.size))) + 1))

        def fill(st, left):
            for name, kind in st._fields_:
                if issubclass(kind, ctypes.Structure):
                    setattr(st, name, fill(kind(), left))
                elif issubclass(kind, ctypes.Array):
                    setattr(st, name, kind(left.pop(0), left.pop(0)))
                else:
                    setattr(st, name, left.pop(0))
            return st

        want = fill(structure(), list(values))
        assert bytes(want) == packed.pack(*values)
