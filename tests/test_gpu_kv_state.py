"""What an attend keeps in its handle from call to call."""
import ctypes

import pytest

from tests.test_gpu_kv import Batch

pytestmark = pytest.mark.gpu


def word_of(kv):
    """The handle's word on the device that says that a wait ran out, as a tensor."""
    import torch
    from paper_2607_11951_gb300 import grid as G
    at = ctypes.c_void_p.from_address(kv.h.value + ctypes.sizeof(G._KvPages)).value

    class Word:
        __cuda_array_interface__ = dict(shape=(1,), typestr="<i4", data=(at, False), version=3, strides=None)

    return torch.as_tensor(Word(), device="cuda")


@pytest.mark.parametrize("old,new,D", [([40], [1], 64), ([5000, 3], [2, 150], 128), ([7] * 400, [1] * 400, 64), ([3, 4], [0, 0], 128)])
def test_a_wait_that_ran_out_is_reported_in_every_row_from_then_on(old, new, D):
    """The word is set by hand: no wait can be made to run out without stopping the GPU."""
    b = Batch(old, new, 4, 2, D, 16)
    b.fill()
    word = word_of(b.kv)
    assert word.tolist() == [0]
    b.attend()
    b.check()
    word[0] = 1
    b.lens[0] = -1  # (a row that is not in order reports it too)
    for _ in range(2):
        b.status[:] = -1
        b.attend()
        assert b.status.tolist() == [5] * len(old) and word.tolist() == [1]
    word[0] = 0
    b.lens[0] = old[0]
    b.attend()
    b.check()


@pytest.mark.parametrize("old,new,D", [([0], [1], 64), ([40], [1], 128), ([200], [3], 128), ([5000, 3], [2, 150], 64), ([7] * 400, [1] * 400, 64)])
def test_nothing_is_attended_to_after_a_wait_ran_out(old, new, D):
    b = Batch(old, new, 4, 2, D, 16)
    b.fill()
    word_of(b.kv)[0] = 1
    b.attend()
    assert b.status.tolist() == [5] * len(old) and bool((b.out == 7).all()) and bool((b.lse == 7).all())
