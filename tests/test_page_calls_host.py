"""Host side of the calls on caches in pages: refusals before anything is launched, workspace sizes, and what the early
kernels among theirs promise.  No GPU needed."""
import os
import re

import pytest
import torch

import paper_2406_11430_b200 as l2

B, L, H, HQ, D, N, P, PAGES, CAP = 2, 3, 2, 8, 128, 7, 16, 11, 4
I32 = lambda *s: torch.zeros(s, dtype=torch.int32)  # noqa: E731


def _offset(t):
    """The same tensor 8 bytes behind a 16-byte boundary."""
    room = torch.zeros(t.numel() + 16, dtype=t.dtype)
    at = 8 // t.element_size()
    return room[at:at + t.numel()].view(t.shape)


def _inputs(dtype=torch.bfloat16):
    tok = lambda heads: torch.zeros((L, N, heads, D), dtype=dtype)  # noqa: E731
    pool = lambda: torch.zeros((H, PAGES * P, D), dtype=dtype)  # noqa: E731
    return dict(K=pool(), V=pool(), q=tok(HQ), k=tok(H), v=tok(H), out=tok(HQ), off=I32(B + 1), pos=I32(N), start=I32(B, L), cur=I32(B, L),
                idx=I32(H, PAGES * P), key=torch.zeros((H, PAGES * P)), ws=torch.zeros(1 << 16, dtype=torch.uint8),
                freq=torch.zeros(D // 2, dtype=torch.float64), qw=torch.zeros(D, dtype=dtype), kw=None, eps=1e-6, offset=0.0,
                table=I32(B, L, CAP), table_out=I32(B, L, CAP), page_rows=P, page_rows_out=P, n_pages=PAGES, room=None, room_out=I32(B, L),
                parent=I32(B), keep=I32(B, L), grow=I32(B), pin=None, n_free=I32(1), max_len=CAP * P, policy=0, len_out=I32(B, L), scale=0.0,
                rows=None)


def _pages(a):
    return l2.Pages(a["table"], a["page_rows"], a["n_pages"], a["room"])


def _out(a):
    return l2.Pages(a["table_out"], a["page_rows_out"], a["n_pages"], a["room_out"])


def _write(a):
    l2.norm_rotary_write(a["q"], a["k"], a["v"], a["off"], a["pos"], a["freq"], a["out"], a["K"], a["V"], a["idx"], a["key"], a["start"],
                         a["cur"], a["ws"], q_weight=a["qw"], k_weight=a["kw"], eps=a["eps"], weight_offset=a["offset"], rows=a["rows"],
                         pages=_pages(a))


def _attend(a):
    l2.paged_attention(a["q"], a["off"], a["K"], a["V"], a["cur"], a["max_len"], a["out"], _pages(a), scale=a["scale"], workspace=a["ws"])


def _update(a):
    l2.page_update(a["K"], a["V"], a["idx"], a["key"], _pages(a), a["parent"], a["keep"], a["grow"], _out(a), a["ws"], pin=a["pin"],
                   n_free_out=a["n_free"])


def _compact(a):
    l2.page_compact(a["K"], a["V"], a["idx"], a["key"], _pages(a), a["cur"], a["keep"], a["max_len"], _out(a), a["len_out"], a["ws"],
                    policy=a["policy"], pin=a["pin"])


CALLS = [_write, _attend, _update, _compact]
nan, inf = float("nan"), float("inf")
SMALL = torch.zeros(255, dtype=torch.uint8)
REFUSED = [(call, change, status) for call in CALLS for change, status in [
    ({}, -1),                                                # host memory: checked like any other, never launched on
    (dict(page_rows=8, n_pages=PAGES * 2, page_rows_out=8), -2), (dict(K=_offset), -3), (dict(V=None), -1)]] + [
    (_write, dict(freq=torch.zeros(12, dtype=torch.float64)), -2), (_write, dict(eps=-1e-6), -1), (_write, dict(eps=nan), -1),
    (_write, dict(eps=inf), -1), (_write, dict(offset=nan), -1), (_write, dict(qw=_offset), -3), (_write, dict(cur="start"), -1),
    (_write, dict(ws=SMALL), -4), (_write, dict(pos=None), -1), (_write, dict(q=_offset), -3),
    (_attend, dict(max_len=CAP * P + 1), -5), (_attend, dict(max_len=-1), -1), (_attend, dict(scale=nan), -1), (_attend, dict(ws=SMALL), -4),
    (_attend, dict(out=_offset), -3),
    (_update, dict(ws=torch.zeros(1024, dtype=torch.uint8)), -4), (_update, dict(table_out="table"), -1), (_update, dict(room_out="keep"), -1),
    (_update, dict(table_out=I32(B, L, CAP + 1)), -1), (_update, dict(table_out=I32(1, L, CAP).expand(B, L, CAP)), -1),
    (_compact, dict(ws=torch.zeros(1024, dtype=torch.uint8)), -4), (_compact, dict(table_out="table"), -1), (_compact, dict(policy=2), -1),
    (_compact, dict(policy=3), -1), (_compact, dict(max_len=CAP * P + 1), -5), (_compact, dict(max_len=-1), -1), (_compact, dict(key=None), -1),
    (_compact, dict(len_out="keep"), -1), (_compact, dict(room_out="keep"), -1),
]


@pytest.mark.parametrize("call,change,status", REFUSED)
def test_refused_by_the_library(call, change, status):
    a = _inputs()
    for k, v in change.items():
        a[k] = a[v] if isinstance(v, str) else v(a[k]) if callable(v) else v
    with pytest.raises(l2.L2KVError) as e:
        call(a)
    assert e.value.status == status


i64 = lambda *s: torch.zeros(s, dtype=torch.int64)  # noqa: E731
MISFITS = [(call, change) for call in CALLS for change in [
    dict(table=i64(B, L, CAP)), dict(table=I32(B, L * CAP)), dict(table=I32(B, L, 2 * CAP)[:, :, ::2]), dict(n_pages=PAGES + 1), dict(n_pages=2 ** 40),
    dict(K=torch.zeros((H, PAGES * P, D), dtype=torch.float16)), dict(K=torch.zeros((1, B, H, P, D), dtype=torch.bfloat16)),
    dict(V=torch.zeros((H, PAGES * P, D // 2), dtype=torch.bfloat16)), dict(ws=torch.zeros(64)), dict(table=7), dict(room=I32(B, L + 1)),
    dict(room=torch.zeros((B, L)))]] + [
    (_write, dict(qw=torch.zeros(D // 2, dtype=torch.bfloat16))), (_write, dict(kw=torch.zeros(D))), (_write, dict(idx=I32(H, PAGES))),
    (_write, dict(start=I32(B))), (_write, dict(off=I32(B))), (_write, dict(k=torch.zeros((L, N + 1, H, D), dtype=torch.bfloat16))),
    (_write, dict(rows=l2.Rows([[0] * L] * B, [[4] * L] * B, PAGES * P, "cpu"))), (_write, dict(eps="x")),
    (_attend, dict(cur=I32(B, L, H))), (_attend, dict(out=torch.zeros((L, N, HQ, D)))), (_attend, dict(max_len=2 ** 40)),
    (_update, dict(parent=I32(B + 1))), (_update, dict(keep=I32(B))), (_update, dict(grow=i64(B))), (_update, dict(pin=I32(PAGES))),
    (_update, dict(pin=torch.zeros(PAGES + 1, dtype=torch.uint8))), (_update, dict(n_free=I32(2))), (_update, dict(table_out=I32(B, L + 1, CAP))),
    (_update, dict(room_out=I32(B))), (_update, dict(idx=I32(PAGES * P))), (_update, dict(key=torch.zeros(PAGES * P))),
    (_compact, dict(keep=I32(B))), (_compact, dict(len_out=I32(L))), (_compact, dict(cur=i64(B, L))), (_compact, dict(table_out=I32(B + 1, L, CAP), room_out=None)),
    (_compact, dict(max_len=2 ** 31)), (_compact, dict(pin=torch.zeros(PAGES)))]


@pytest.mark.parametrize("call,change", MISFITS)
def test_tensors_that_do_not_fit_together(call, change):
    a = _inputs()
    a.update(change)
    with pytest.raises((ValueError, TypeError)):
        call(a)


def test_a_call_without_pages():
    a = _inputs()
    with pytest.raises(ValueError):
        l2.paged_attention(a["q"], a["off"], a["K"], a["V"], a["cur"], 4, a["out"], None)
    for pages in (object(), 3):
        with pytest.raises(AttributeError):
            l2.page_workspace_bytes(a["K"], pages)


@pytest.mark.parametrize("page_rows", [0, -16, 24, 2048, 2 ** 30 + 1, 2 ** 31 - 1])
def test_page_sizes_that_are_none(page_rows):
    """Of an empty pool, so that nothing else is wrong with them."""
    a = _inputs()
    a.update(page_rows=page_rows, page_rows_out=page_rows, n_pages=0, table=I32(B, L, 0), table_out=I32(B, L, 0), idx=None, max_len=0)
    for k in ("K", "V"):
        a[k] = a[k][:, :0]
    for call in CALLS:
        a["key"] = torch.zeros((H, 0)) if call is _compact else None
        with pytest.raises(l2.L2KVError) as e:
            call(a)
        assert e.value.status == -2


def test_tables_live_as_long_as_the_call(tmp_path):
    """Another thread runs while the library is at work, and takes the tables away from the objects that held them."""
    import ctypes
    import subprocess
    import threading
    import time
    import weakref
    from paper_2406_11430_b200 import binding
    (tmp_path / "s.c").write_text("#include <unistd.h>\nvolatile int entered, go;\nint stand_in(void) { entered = 1; "
                                  "for (int i = 0; i < 2000 && !go; ++i) usleep(1000); return go ? 0 : -1; }")
    subprocess.run(["gcc", "-O1", "-shared", "-fPIC", "-o", str(tmp_path / "s.so"), str(tmp_path / "s.c")], check=True)
    lib = ctypes.CDLL(str(tmp_path / "s.so"))
    entered, go = (ctypes.c_int.in_dll(lib, name) for name in ("entered", "go"))
    names = ("l2kv_norm_rotary_write", "l2kv_paged_attention", "l2kv_paged_attention_workspace_bytes", "l2kv_page_update", "l2kv_page_compact",
             "l2kv_page_workspace_bytes")
    real = [ctypes.cast(getattr(l2.lib(), name), ctypes.c_void_p).value for name in names]
    at, native = ctypes.cast(lib.stand_in, ctypes.c_void_p).value, binding._token_calls()
    native.bind_pages(at, at, real[2], at, at, real[5])
    try:
        for call in CALLS:
            entered.value = go.value = 0
            a, alive = _inputs(), []
            pages, out = l2.Pages(I32(B, L, CAP), P, PAGES, I32(B, L)), l2.Pages(I32(B, L, CAP), P, PAGES, I32(B, L))
            held = [pages] + ([out] if call in (_update, _compact) else [])
            refs = [weakref.ref(x) for p in held for x in (p.table, p.room)]

            def take_away():
                while not entered.value:
                    time.sleep(1e-3)
                for p in held:
                    p.table = p.room = None
                alive.extend(r() is not None for r in refs)
                go.value = 1
            thread = threading.Thread(target=take_away)
            thread.start()
            if call is _write:
                l2.norm_rotary_write(a["q"], a["k"], a["v"], a["off"], a["pos"], a["freq"], a["out"], a["K"], a["V"], a["idx"], a["key"], a["start"],
                                     a["cur"], a["ws"], pages=pages)
            elif call is _attend:
                l2.paged_attention(a["q"], a["off"], a["K"], a["V"], a["cur"], a["max_len"], a["out"], pages)
            elif call is _update:
                l2.page_update(a["K"], a["V"], None, None, pages, a["parent"], a["keep"], a["grow"], out, a["ws"])
            else:
                l2.page_compact(a["K"], a["V"], None, a["key"], pages, a["cur"], a["keep"], a["max_len"], out, a["len_out"], a["ws"])
            thread.join()
            assert alive == [True] * len(refs) and [r() for r in refs] == [None] * len(refs)
    finally:
        native.bind_pages(*real)


def test_nothing_to_do():
    """No sequences, or no tokens: no error and no launch."""
    a = _inputs()
    a.update(table=I32(0, L, CAP), off=I32(1), start=I32(0, L), cur=I32(0, L), table_out=I32(0, L, CAP), room_out=I32(0, L), parent=I32(0),
             keep=I32(0, L), grow=I32(0), len_out=I32(0, L))
    for call in CALLS:
        call(a)


def test_workspace_sizes():
    a = _inputs()
    small = l2.page_workspace_bytes(a["K"], _pages(a))
    assert small >= 256 + 8 * PAGES + 8 * B * L
    assert l2.page_workspace_bytes(a["K"], _pages(a), 64) >= small + B * L * H * (64 // 8 + 4)          # a bit per row, a number per chunk
    assert l2.page_workspace_bytes(a["K"], _pages(a), 0, 1000) >= 256 + 8 * 1000 * L
    with pytest.raises(l2.L2KVError):
        l2.page_workspace_bytes(a["K"], _pages(a), CAP * P + 1)
    # no more sequences and layers than a claim on a page can name
    many = l2.Pages(I32(1, 1, 1).expand(1 << 19, 4, 1), P, PAGES)
    out = l2.Pages(I32(1 << 19, 4, 1), P, PAGES)
    with pytest.raises(l2.L2KVError) as e:
        l2.page_update(a["K"], a["V"], None, None, many, I32(1 << 19), I32(1 << 19, 4), I32(1 << 19), out, a["ws"])
    assert e.value.status == -5


def test_pools_beyond_32_bits_are_refused():
    K = torch.zeros((1, 1, 64), dtype=torch.bfloat16).expand(1, 2 ** 31, 64)
    pages = l2.Pages(I32(1, 1, 1), 16, 2 ** 27)
    with pytest.raises((l2.L2KVError, ValueError)):
        l2.page_workspace_bytes(K, pages)


def _kernels(name):
    """Signature and body of every kernel of a source file."""
    path = os.path.join(os.path.dirname(l2.__file__), "csrc", name)
    with open(path) as f:
        code = re.sub(r"//[^\n]*|/\*.*?\*/", "", f.read(), flags=re.S)
    return [part.split("{", 1) for part in code.split("__global__")[1:]]


@pytest.mark.parametrize("name,count", [("pages.cu", 7), ("few_tokens.cu", 2)])
def test_the_early_kernels_wait_and_promise_nothing(name, count):
    """All of them are set up while the kernel before them runs: they wait before they read what that one writes, and no
    __restrict__ parameter lets the compiler read earlier."""
    kernels = _kernels(name)
    assert len(kernels) == count
    for signature, body in kernels:
        assert "__restrict__" not in signature
        assert "wait_for_previous();" in body
