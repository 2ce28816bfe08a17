"""Attention over fp32 caches in pages whose rows are cut into parts and joined: lengths around the parts' ends, parts without a row,
tiles of several sequences, heads that differ in length, the same bits every time.  The bound is check_attention's: the
join adds a power of two's rounding and a product per part, which the 2^-20 in it allows for."""
import numpy as np
import pytest
import torch

from page_util import Paged
from test_gpu_paged_attention import call, check
from token_util import DEV, causal, check_attention

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def l2():
    import paper_2406_11430_b200 as lib
    lib.lib()
    return lib


@pytest.mark.parametrize("D,P", [(64, 16), (64, 128), (128, 16), (128, 64), (128, 1024)])
@pytest.mark.parametrize("G", [1, 8])
def test_lengths_around_the_ends_of_parts(l2, D, P, G):
    for x in (0, 1, 31, 62, 63, 64, 65, 126, 127, 128, 191, 400, 1023, 2049):
        check(l2, Paged(l2, [1], [[x]], 1, 2, G, D, P, "fp32", seed=x))


@pytest.mark.parametrize("workspace", ["full", "status", None])
def test_tiles_of_several_sequences(l2, workspace):
    check(l2, Paged(l2, [3, 0, 1, 40, 2], [[700, 20], [0, 5], [0, 1900], [64, 63], [333, 0]], 2, 2, 4, 128, 16, "fp32", seed=1), workspace=workspace)


def test_heads_that_differ_in_length(l2):
    """Heads with more parts than others, and with none."""
    ctx = np.array([[[0, 900, 63]], [[1500, 2, 64]]])
    check(l2, Paged(l2, [2, 1], ctx, 1, 3, 2, 64, 32, "fp32", seed=2, per_head=True, pad=3, strided=True), scale=0.2)


def test_more_tiles_than_blocks_at_once(l2):
    """No parts: as many tiles as that fill the SMs."""
    n = [1] * 40
    check(l2, Paged(l2, n, np.random.RandomState(3).randint(0, 300, (40, 1)), 1, 16, 1, 64, 64, "fp32", seed=3))


def test_a_bound_beyond_the_lengths(l2):
    """More parts than there are rows for: max_len says nothing of the lengths."""
    c = Paged(l2, [1, 1], [[40], [700]], 1, 2, 2, 128, 16, "fp32", seed=4, entries=900)
    assert c.max_len > 14000
    check(l2, c)


def test_the_same_bits_every_time(l2):
    c = Paged(l2, [2, 1], [[1700], [90]], 1, 2, 4, 128, 16, "fp32", seed=5)
    out, lse = call(l2, c)
    for _ in range(10):
        o, z = call(l2, c)
        assert torch.equal(o, out) and torch.equal(z, lse)


def test_captured_over_changing_lengths(l2):
    c = Paged(l2, [1, 2], [[900], [300]], 1, 2, 2, 64, 16, "fp32", seed=6)
    ws = torch.zeros(l2.paged_attention_workspace_bytes(c.K, c.q, c.max_len, c.pages), dtype=torch.uint8, device=DEV)
    cur, out, lse = c.lens(c.cur).clone(), c.empty_out(), torch.zeros((1, c.N, c.Hq), device=DEV)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        l2.paged_attention(c.q, c.tok_off, c.K, c.V, cur, c.max_len, out, c.pages, lse_out=lse, workspace=ws)
    full = c.cur.copy()
    for less in (0, 17, 250, 299):
        c.cur = full - less
        cur.copy_(c.lens(c.cur))
        graph.replay()
        torch.cuda.synchronize()
        check_attention(c, out, lse, causal(c))
    assert l2.read_device_status(ws) == 0


def test_one_workspace_for_calls_with_and_without_parts(l2):
    cases = [Paged(l2, [1], [[x]], 1, h, 2, 64, 16, "fp32", seed=x) for x, h in ((1500, 1), (20, 2), (700, 8), (64, 1))]
    ws = torch.zeros(max(l2.paged_attention_workspace_bytes(c.K, c.q, c.max_len, c.pages) for c in cases), dtype=torch.uint8, device=DEV)
    for c in cases + cases[::-1]:
        out, lse = c.empty_out(), torch.full((1, c.N, c.Hq), 7.0, device=DEV)
        l2.paged_attention(c.q, c.tok_off, c.K, c.V, c.lens(c.cur), c.max_len, out, c.pages, lse_out=lse, workspace=ws)
        torch.cuda.synchronize()
        check_attention(c, out, lse, causal(c))
    assert l2.read_device_status(ws) == 0


def test_a_page_that_is_none_in_one_part(l2):
    """Its rows are zeros, seen like others: the same as a page of zeros, and told."""
    c = Paged(l2, [1], [[600]], 1, 2, 2, 128, 16, "fp32", seed=7)
    t = c.pages.table.clone()
    page = int(t[0, 0, 9])
    c.K[:, page * 16:page * 16 + 16] = 0
    c.V[:, page * 16:page * 16 + 16] = 0
    want = call(l2, c)
    t[0, 0, 9] = 2 ** 31 - 1
    got = call(l2, c, pages=l2.Pages(t, 16, c.n_pages), status=-5)
    assert torch.equal(want[0], got[0]) and torch.equal(want[1], got[1])
