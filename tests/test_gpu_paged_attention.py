"""Attention of packed new tokens over caches in pages, against the definition in 64 bits: head layouts, page and tile
sizes, lengths from nothing to long, single tokens among chunks, tables of any strides, pages that the pool does not have,
shared pages, lengths per head, padding, streams and graphs."""
import numpy as np
import pytest
import torch

from page_util import Paged
from token_util import DEV, causal, check_attention, i32

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def l2():
    import paper_2406_11430_b200 as lib
    lib.lib()
    return lib


def call(l2, c, scale=0.0, workspace="full", max_len=None, stream=None, pages=None, cur=None, status=0, q=None):
    out, z = c.empty_out(), torch.full((c.L, c.N, c.Hq), 7.0, device=DEV)
    q, pages, max_len = c.q if q is None else q, c.pages if pages is None else pages, c.max_len if max_len is None else max_len
    ws = None
    if workspace:
        need = l2.paged_attention_workspace_bytes(c.K, q, max_len, pages) if workspace == "full" else 256
        ws = torch.full((need,), 255, dtype=torch.uint8, device=DEV)      # only the status block is zeroed
        ws[:256] = 0
    cur = c.lens(c.cur) if cur is None else cur
    if stream is not None:
        stream.wait_stream(torch.cuda.current_stream())
    l2.paged_attention(q, c.tok_off, c.K, c.V, cur, max_len, out, pages, lse_out=z, scale=scale, workspace=ws, per_head=c.per_head,
                       stream=stream)
    torch.cuda.synchronize()
    if ws is not None:
        assert l2.read_device_status(ws) == status
    return out, z


def check(l2, c, **kw):
    out, lse = call(l2, c, **kw)
    check_attention(c, out, lse, causal(c), kw.get("scale") or None)
    used = int(c.off[-1])
    assert (out[:, used:] == 7).all() and (lse[:, used:] == 7).all()          # padding: left alone


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("P", [16, 32, 64, 128, 1024])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("G", [1, 2, 4, 8])
def test_head_layouts_and_page_sizes(l2, G, D, P, dtype):
    check(l2, Paged(l2, [5, 0, 33, 1], [[130], [70], [0], [0]], 1, 2, G, D, P, dtype, seed=G))


@pytest.mark.parametrize("P", [16, 64, 256])
@pytest.mark.parametrize("n,ctx", [
    ([1], [[0]]), ([1], [[15]]), ([1], [[16]]), ([1], [[63]]), ([1], [[64]]), ([1], [[255]]), ([2], [[126]]), ([128], [[0]]), ([129], [[0]]),
    ([31], [[97]]), ([33], [[95]]), ([64], [[64]]), ([65], [[300]]), ([255], [[1]]), ([257], [[385]]), ([300, 1, 64, 17], [[0], [513], [128], [1000]])])
def test_lengths_around_pages_and_tiles(l2, n, ctx, P):
    check(l2, Paged(l2, n, ctx, 1, 2, 4, 128, P, seed=len(n) + n[0]))


@pytest.mark.parametrize("P", [16, 32, 128])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("workspace", ["full", "status", None])
def test_long_caches_few_tokens(l2, workspace, D, P):
    """Caches whose tables are read in several pieces of 32 entries, cut between SMs or not."""
    check(l2, Paged(l2, [3, 1, 40], [[9000], [4097], [2500]], 1, 2, 4, D, P, seed=5), workspace=workspace)


@pytest.mark.parametrize("L", [1, 2])
@pytest.mark.parametrize("G", [1, 4, 8])
def test_single_tokens_of_many_sequences(l2, G, L):
    r = np.random.RandomState(G)
    check(l2, Paged(l2, [1] * 40, r.randint(0, 1500, (40, L)), L, 2, G, 128, 16, seed=G))


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("G", [1, 2, 4, 8])
@pytest.mark.parametrize("D", [64, 128])
def test_few_tokens_in_uneven_numbers(l2, D, G, dtype):
    """No more tokens than sequences, but several of one sequence: more than one item for some, none for others."""
    check(l2, Paged(l2, [0, 5, 0, 0, 1, 0, 0, 12, 0, 2] + [0] * 12, [[i * 37 % 200] for i in range(22)], 1, 2, G, D, 32, dtype, seed=G, pad=2))
    check(l2, Paged(l2, [17] + [0] * 17, [[2500]] + [[0]] * 17, 1, 2, G, D, 16, dtype, seed=G))


@pytest.mark.parametrize("workspace", ["full", "status"])
@pytest.mark.parametrize("P", [16, 32, 64, 512])
@pytest.mark.parametrize("D", [64, 128])
def test_single_tokens_over_lengths_around_blocks(l2, D, P, workspace):
    """From a cache of the token alone to long ones, around blocks of 32 and 64 rows, pages, and shares of the work."""
    ctx = [0, 1, 14, 15, 16, 30, 31, 32, 62, 63, 64, 127, 128, 500, 511, 512, 513, 1000, 5000, 9001]
    check(l2, Paged(l2, [1] * 20, [[x] for x in ctx], 1, 3, 4, D, P, seed=D), workspace=workspace)
    for x in (0, 40, 600, 3000):
        check(l2, Paged(l2, [1], [[x]], 1, 1, 1, D, P, seed=x), workspace=workspace)


def test_single_tokens_of_hundreds_of_sequences(l2):
    """More sequences than threads work out the shares."""
    r = np.random.RandomState(6)
    check(l2, Paged(l2, [int(x) for x in r.choice([0, 1, 1, 1], 700)], r.randint(0, 90, (700, 1)), 1, 1, 4, 64, 16, seed=6))


@pytest.mark.parametrize("P", [16, 64])
def test_chunks_and_single_tokens_mixed(l2, P):
    r = np.random.RandomState(3)
    n = [int(x) for x in r.choice([0, 1, 1, 1, 7, 90, 200, 513], 30)]
    check(l2, Paged(l2, n, r.randint(0, 900, (30, 1)), 1, 2, 4, 128, P, seed=3))


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_lengths_per_head_layers_padding_and_scale(l2, dtype):
    ctx = np.random.RandomState(8).randint(0, 300, (4, 2, 3))
    check(l2, Paged(l2, [6, 1, 0, 70], ctx, 2, 3, 2, 64, 32, dtype, seed=9, per_head=True, pad=11, strided=True), scale=0.3)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_tokens_that_see_nothing(l2, dtype):
    """Fewer rows than new tokens: the first tokens see none and give zeros and -inf."""
    for more in (0, 100):                                    # (empty sequences: few tokens per sequence)
        see_nothing(l2, Paged(l2, [5, 1, 80] + [0] * more, [[0]] * (3 + more), 1, 2, 4, 128, 16, dtype, seed=2), dtype, more)


def see_nothing(l2, c, dtype, more):
    out, lse = call(l2, c, cur=i32([[2], [0], [33]] + [[0]] * more))
    for b, (n, cur) in enumerate(zip(c.n, (2, 0, 33))):
        for s in range(n):
            seen, i = max(0, cur - n + s + 1), int(c.off[b]) + s
            if seen == 0:
                assert not out[0, i].any() and torch.isneginf(lse[0, i]).all()
                continue
            for j in range(c.Hq):
                K, V = (c.unit(x, b, 0, j // c.G)[:seen].double() for x in (c.K, c.V))
                w = torch.softmax(K @ c.q[0, i, j].double() * c.D ** -0.5, 0)
                # a rounding of the weights and one of the result (bf16), or fp32 sums of 128 products and 33 rows
                half = 2.0 ** -8 if dtype == "bf16" else 400 * 2.0 ** -24
                assert ((out[0, i, j].double() - w @ V).abs() <= 2.1 * half * (w @ V.abs()) + 1e-6).all()


def test_a_table_is_read_below_the_length_only(l2):
    """Entries behind a sequence's last page can hold anything."""
    c = Paged(l2, [3, 1, 70], [[100], [16], [0]], 1, 2, 4, 128, 16, seed=4, entries=40)
    t = c.pages.table.clone()
    for b in range(c.B):
        t[b, 0, -(-int(c.cur[b, 0, 0]) // 16):] = torch.tensor([2 ** 31 - 1, -2 ** 31, -1, 10 ** 6] * 40, device=DEV)[:t.shape[2] - -(-int(c.cur[b, 0, 0]) // 16)].int()
    out, lse = call(l2, c, pages=l2.Pages(t, 16, c.n_pages))
    check_attention(c, out, lse, causal(c))


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("P", [16, 64])
def test_pages_that_the_pool_does_not_have(l2, P, dtype):
    """They are told, and read as rows of zeros."""
    no_such_pages(l2, Paged(l2, [2, 90], [[300], [40]], 1, 2, 4, 128, P, dtype, seed=6), P)
    no_such_pages(l2, Paged(l2, [1, 1], [[300], [140]], 1, 2, 4, 128, P, dtype, seed=6), P)


def no_such_pages(l2, c, P):
    t = c.pages.table.clone()
    bad = [(0, 0, c.n_pages), (0, 2, -1), (1, 1, 2 ** 31 - 1), (1, 0, -2 ** 31)]
    for b, j, page in bad:
        for x in (c.K, c.V):
            x[:, int(c.table[b, 0, j]) * P:][:, :P] = 0
        t[b, 0, j] = page
    out, lse = call(l2, c, pages=l2.Pages(t, P, c.n_pages), status=-5)
    assert torch.isfinite(out).all()
    want, want_lse = call(l2, c)
    assert torch.equal(out, want) and torch.equal(lse, want_lse)


def test_tables_of_any_strides(l2):
    c = Paged(l2, [3, 1, 40], [[300, 200], [17, 0], [64, 64]], 2, 2, 4, 128, 16, seed=7)
    want, want_lse = call(l2, c)
    by_layer = c.pages.table.transpose(0, 1).contiguous().transpose(0, 1)     # [L, B, entries] in memory
    wide = torch.full((c.B, 2, 2 * c.table.shape[2] + 1), -7, dtype=torch.int32, device=DEV)[:, :, 1:1 + c.table.shape[2]]
    wide.copy_(c.pages.table)
    for t in (by_layer, wide):
        out, lse = call(l2, c, pages=l2.Pages(t, 16, c.n_pages))
        assert torch.equal(out, want) and torch.equal(lse, want_lse)
    # one layer of the tables at a time
    for l in range(2):
        out, lse = c.empty_out()[l:l + 1], torch.zeros((1, c.N, c.Hq), device=DEV)
        l2.paged_attention(c.q[l:l + 1], c.tok_off, c.K, c.V, c.lens(c.cur)[:, l:l + 1].contiguous(), c.max_len, out,
                           l2.Pages(c.pages.table[:, l:l + 1], 16, c.n_pages), lse_out=lse)
        torch.cuda.synchronize()
        check = want[l:l + 1]
        assert (out.float() - check.float()).abs().max() <= 2 ** -6 * check.float().abs().max()
    # one prompt for all sequences: a table of stride zero
    one = l2.Pages(c.pages.table[:1].expand(3, -1, -1), 16, c.n_pages)
    cur = i32([[200, 150]] * 3)
    out, lse = call(l2, c, pages=one, cur=cur)
    each = torch.zeros_like(c.pages.table)
    each[:] = c.pages.table[0]
    same, same_lse = call(l2, c, pages=l2.Pages(each, 16, c.n_pages), cur=cur)
    assert torch.equal(out, same) and torch.equal(lse, same_lse)


@pytest.mark.parametrize("captured", [False, True])
def test_other_stream_and_graph(l2, captured):
    c = Paged(l2, [1, 33, 1], [[1300], [200], [1]], 1, 2, 4, 128, 16, seed=12)
    want, want_lse = call(l2, c)
    side = torch.cuda.Stream()
    if not captured:
        out, lse = call(l2, c, stream=side)
        assert torch.equal(out, want) and torch.equal(lse, want_lse)
        return
    out, lse, cur = c.empty_out(), torch.zeros((1, c.N, c.Hq), device=DEV), c.lens(c.cur)
    ws = torch.zeros(l2.paged_attention_workspace_bytes(c.K, c.q, c.max_len, c.pages), dtype=torch.uint8, device=DEV)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        l2.paged_attention(c.q, c.tok_off, c.K, c.V, cur, c.max_len, out, c.pages, lse_out=lse, workspace=ws)
    for _ in range(3):
        out.fill_(7)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want) and torch.equal(lse, want_lse)
    # other tables under the same graph: the pages change places, and with them the rows
    swap = torch.randperm(c.n_pages, device=DEV)
    for x in (c.K, c.V):
        y = x.view(2, c.n_pages, 16, -1).clone()
        x.view(2, c.n_pages, 16, -1)[:, swap] = y
    t = c.pages.table.long()
    c.pages.table.copy_(torch.where(t >= 0, swap[t.clamp(min=0)], t).int())
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(out, want) and torch.equal(lse, want_lse) and l2.read_device_status(ws) == 0


def test_repeated_calls_on_one_workspace(l2):
    cases = [Paged(l2, n, ctx, 1, 2, 4, 128, P, seed=P + len(n)) for P in (16, 64) for n, ctx in
             (([1], [[5000]]), ([1] * 9, [[i * 211] for i in range(9)]), ([300, 2], [[2000], [3]]))]
    ws = torch.zeros(max(l2.paged_attention_workspace_bytes(c.K, c.q, c.max_len, c.pages) for c in cases), dtype=torch.uint8, device=DEV)
    first = []
    for turn in range(3):
        for i, c in enumerate(cases):
            out, lse = c.empty_out(), torch.zeros((1, c.N, c.Hq), device=DEV)
            l2.paged_attention(c.q, c.tok_off, c.K, c.V, c.lens(c.cur), c.max_len, out, c.pages, lse_out=lse, workspace=ws)
            if turn == 0:
                first.append((out, lse))
            else:
                torch.cuda.synchronize()
                assert torch.equal(out, first[i][0]) and torch.equal(lse, first[i][1])
    for c, (out, lse) in zip(cases, first):
        check_attention(c, out, lse, causal(c))
    assert l2.read_device_status(ws) == 0
