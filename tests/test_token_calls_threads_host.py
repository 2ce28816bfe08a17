"""Other Python threads run while a call on new tokens is in the library: a launch can block for as long as the GPU's queue
is full, and what empties the queue may be a host function that needs the interpreter.  The library is stood in for
by a C function that returns well only if another Python thread lets it go.  No GPU needed."""
import ctypes
import subprocess
import threading
import time
import types

import pytest
import torch

import paper_2406_11430_b200 as l2
from paper_2406_11430_b200 import binding

STAND_IN = r"""
#include <unistd.h>
volatile int entered, go;
int stand_in(void) {
  entered = 1;
  for (int i = 0; i < 2000 && !go; ++i) usleep(1000);
  return go ? 0 : -1;
}
"""
NAMES = ("l2kv_rotary_write", "l2kv_tree_commit", "l2kv_prompt_attention", "l2kv_tree_attention", "l2kv_prompt_attention_workspace_bytes")


@pytest.fixture(scope="module")
def stand_in(tmp_path_factory):
    at = tmp_path_factory.mktemp("stand_in")
    (at / "stand_in.c").write_text(STAND_IN)
    subprocess.run(["gcc", "-O1", "-shared", "-fPIC", "-o", str(at / "stand_in.so"), str(at / "stand_in.c")], check=True)
    return ctypes.CDLL(str(at / "stand_in.so"))


@pytest.fixture
def bound(stand_in):
    """The four calls lead to the stand-in, and back to the library afterwards."""
    native = binding._token_calls()
    real = [ctypes.cast(getattr(l2.lib(), name), ctypes.c_void_p).value for name in NAMES]
    address = ctypes.cast(stand_in.stand_in, ctypes.c_void_p).value
    entered, go = (ctypes.c_int.in_dll(stand_in, name) for name in ("entered", "go"))
    entered.value = go.value = 0
    native.bind(address, address, address, address, real[4])
    yield entered, go
    native.bind(*real)


def _call(which, rows=None):
    i32 = lambda *s: torch.zeros(s, dtype=torch.int32)  # noqa: E731
    K = torch.zeros((2, 1, 2, 9, 64) if rows is None else (2, 18, 64), dtype=torch.bfloat16)
    tok = torch.zeros((1, 3, 2, 64), dtype=torch.bfloat16)
    ws, kw = torch.zeros(256, dtype=torch.uint8), dict(rows=rows)
    if which == "rotary":
        l2.rotary_write(tok, tok, tok, i32(3), i32(3), None, tok, K, K, None, None, i32(2, 1), i32(2, 1), ws, **kw)
    elif which == "commit":
        l2.tree_commit(K, K, None, None, i32(2, 1), i32(2, 1), i32(2, 4), i32(2), i32(2, 1), ws, **kw)
    elif which == "prompt":
        l2.prompt_attention(tok, i32(3), K, K, i32(2, 1), 9, tok, workspace=ws, **kw)
    else:
        l2.tree_attention(tok, i32(3), torch.zeros((3, 1), dtype=torch.int64), K, K, i32(2, 1), 9, tok, workspace=ws, **kw)


def _meanwhile(entered, do):
    def wait():
        while not entered.value:
            time.sleep(1e-3)
        do()
    thread = threading.Thread(target=wait)
    thread.start()
    return thread


@pytest.mark.parametrize("which", ["rotary", "commit", "prompt", "tree"])
def test_another_thread_runs_while_the_library_does(bound, which):
    entered, go = bound
    thread = _meanwhile(entered, lambda: setattr(go, "value", 1))
    _call(which)                                             # (the stand-in's -1 would be raised)
    thread.join()


@pytest.mark.parametrize("which", ["rotary", "commit", "prompt", "tree"])
def test_row_ranges_live_as_long_as_the_call(bound, which):
    """Another thread takes the ranges away from the rows object while the library is at work with them."""
    import weakref
    entered, go = bound
    rows = types.SimpleNamespace(B=2, L=1, t_cap=9, total_rows=18, off=torch.tensor([[0], [9]]), cap=torch.full((2, 1), 9, dtype=torch.int32))
    refs = [weakref.ref(rows.off), weakref.ref(rows.cap)]
    alive = []

    def take_away():
        rows.off = rows.cap = None
        alive.extend(r() is not None for r in refs)
        go.value = 1
    thread = _meanwhile(entered, take_away)
    _call(which, rows)
    thread.join()
    assert alive == [True, True]
    assert [r() for r in refs] == [None, None]               # and no longer
