"""Other Python threads run while a compiled call is in the library: each call is
given an entry point that waits (two seconds at most) for what another thread does.
Nothing is launched."""
import ctypes
import subprocess
import threading
import time

import pytest

from tests.test_gpu_binding_shapes import calls

pytestmark = pytest.mark.gpu

SOURCE = r"""
#include <time.h>
volatile int entered, released;
int entry(void) {
  entered = 1;
  const struct timespec ms = {0, 1000000};
  for (int i = 0; i < 2000 && !released; ++i) nanosleep(&ms, 0);
  return released ? 0 : -1;
}
"""


@pytest.fixture(scope="module")
def entry(tmp_path_factory):
    d = tmp_path_factory.mktemp("entry")
    (d / "entry.c").write_text(SOURCE)
    subprocess.run(["gcc", "-O1", "-fPIC", "-shared", str(d / "entry.c"), "-o", str(d / "entry.so")], check=True)
    return ctypes.CDLL(str(d / "entry.so"))


@pytest.mark.parametrize("name", ["append", "append_chunk", "attend", "attend_chunk", "compact", "copy", "plan", "accept", "sample", "update"])
def test_others_run_during_a_call(entry, name):
    from paper_2607_11951_gb300 import grid as G
    call, tensors, more = calls()[name.split("_")[0]]
    if name.endswith("_chunk"):
        tensors = {k: t for k, t in tensors.items() if k not in ("depth", "sees")}
    entered, released = (ctypes.c_int.in_dll(entry, x) for x in ("entered", "released"))
    entered.value = released.value = 0
    over = threading.Event()

    def other():
        while not entered.value and not over.is_set():
            time.sleep(0.001)
        released.value = 1

    module, address = G._binding(), lambda f: ctypes.cast(f, ctypes.c_void_p).value
    thread = threading.Thread(target=other)
    module.bind(*[address(entry.entry)] * len(G._BOUND))
    try:
        thread.start()
        call(**tensors, **more)  # (an error where the wait ran out)
    finally:
        over.set()
        thread.join()
        module.bind(*(address(getattr(G.lib(), n)) for n in G._BOUND))
    assert entered.value == 1
    call(**tensors, **more)
