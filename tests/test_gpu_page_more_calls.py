"""Calls on caches in pages that the documentation allows: pools laid out row by row, one table for all layers, no queries, host
bounds below the tables', large pools, written by the kernel before; and the same on the bounds-checked build."""
import os
import subprocess
import sys

import numpy as np
import pytest
import torch

from page_util import Paged, updated
from test_gpu_norm_rotary_write import assert_near, normed
from token_util import DEV, causal, check_attention, i32

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def l2():
    import paper_2406_11430_b200 as lib
    lib.lib()
    return lib


def test_the_calls_pass_on_the_bounds_checked_build():
    from paper_2406_11430_b200 import build as l2build
    env = dict(os.environ, L2KV_LIBRARY=l2build.build_debug())
    r = subprocess.run([sys.executable, "-m", "pytest", "-q", "-x", "-m", "gpu"] +
                       [os.path.join(ROOT, "tests", f"test_gpu_{name}.py") for name in
                        ("page_tables", "page_run", "paged_attention", "norm_rotary_write")],
                       env=env, cwd=ROOT, capture_output=True, text=True, timeout=1500)
    assert r.returncode == 0, r.stdout[-3000:] + r.stderr[-2000:]
    assert " passed" in r.stdout


def row_by_row(c):
    """The pool as [row, head, D], seen as [head, row, D]."""
    c.K, c.V = (x.transpose(0, 1).contiguous().transpose(0, 1) for x in (c.K, c.V))
    return c


@pytest.mark.parametrize("dtype,n,ctx", [("bf16", [1, 1, 1], [[900], [5], [64]]), ("bf16", [1, 70, 3], [[900], [5], [64]]), ("fp32", [1, 70], [[90], [5]])])
def test_attention_over_a_pool_laid_out_by_rows(l2, dtype, n, ctx):
    c = row_by_row(Paged(l2, n, ctx, 1, 3, 2, 128, 16, dtype, seed=1))
    out, lse = c.empty_out(), torch.zeros((1, c.N, c.Hq), device=DEV)
    ws = torch.zeros(l2.paged_attention_workspace_bytes(c.K, c.q, c.max_len, c.pages), dtype=torch.uint8, device=DEV)
    l2.paged_attention(c.q, c.tok_off, c.K, c.V, c.lens(c.cur), c.max_len, out, c.pages, lse_out=lse, workspace=ws)
    torch.cuda.synchronize()
    check_attention(c, out, lse, causal(c))


@pytest.mark.parametrize("with_q", [True, False])
def test_write_into_a_pool_laid_out_by_rows(l2, with_q):
    """And keys alone, without queries."""
    c = row_by_row(Paged(l2, [40, 1, 0, 300], [[3], [16], [8], [30]], 1, 3, 2, 128, 16, "bf16", seed=2))
    pos, freq = torch.arange(c.N, dtype=torch.int32, device=DEV), l2.rotary_frequencies(128)[0].to(DEV)
    new, ws, q = torch.zeros((4, 1), dtype=torch.int32, device=DEV), torch.zeros(256, dtype=torch.uint8, device=DEV), c.empty_out()
    V0 = c.V.clone()
    l2.norm_rotary_write(c.q if with_q else None, c.k, c.v, c.tok_off, pos, freq, q if with_q else None, c.K, c.V, None, None, c.lens(c.ctx), new,
                         ws, pages=c.pages)
    torch.cuda.synchronize()
    assert l2.read_device_status(ws) == 0 and torch.equal(new, c.lens(c.cur))
    want, size = normed(c.k, pos, freq, 1.0, False, True, None, 0.0, 1e-6)
    same = torch.ones(c.n_pages * 16, dtype=torch.bool, device=DEV)
    for b in range(4):
        at, of = c.at(b, 0, int(c.cur[b, 0, 0]))[int(c.ctx[b, 0, 0]):], slice(int(c.off[b]), int(c.off[b + 1]))
        same[at] = False
        for h in range(3):
            assert_near(c.K[h, at], want[0, of, h], size[0, of, h], True)
            assert torch.equal(c.V[h, at], c.v[0, of, h])
    assert torch.equal(c.V[:, same].contiguous().view(torch.uint8), V0[:, same].contiguous().view(torch.uint8))
    if with_q:
        want, size = normed(c.q, pos, freq, 1.0, False, True, None, 0.0, 1e-6)
        assert_near(q, want, size, True)


def test_one_table_for_all_layers(l2):
    """A pool of layers * heads: one entry per sequence for the calls on tables, a view of a layer's heads for the others."""
    layers, H, D, P, n_pages = 3, 2, 64, 16, 40
    g = torch.Generator().manual_seed(1)
    K, V = (torch.randn((layers * H, n_pages * P, D), generator=g).to(DEV, torch.bfloat16) for _ in range(2))
    a, b = l2.Pages.empty(2, 1, 8, P, n_pages, DEV), l2.Pages.empty(3, 1, 8, P, n_pages, DEV)
    ws = torch.zeros(1 << 20, dtype=torch.uint8, device=DEV)
    l2.page_update(K, V, None, None, a, i32([-1, -1]), i32([[0], [0]]), i32([50, 20]), a2 := l2.Pages.empty(2, 1, 8, P, n_pages, DEV), ws)
    l2.page_update(K, V, None, None, a2, i32([0, 1, 0]), i32([[50], [20], [50]]), i32([1, 1, 1]), b, ws)
    torch.cuda.synchronize()
    t = b.table.cpu().numpy()
    assert t[0, 0, 3] != t[2, 0, 3] and (t[0, 0, :3] == t[2, 0, :3]).all()
    assert torch.equal(K[:, t[2, 0, 3] * P:t[2, 0, 3] * P + 2], K[:, t[0, 0, 3] * P:t[0, 0, 3] * P + 2])      # all layers' rows are copied
    q, off, cur = torch.randn((1, 3, 4, D), generator=g).to(DEV, torch.bfloat16), i32([0, 1, 2, 3]), i32([[50], [20], [50]])
    for l in range(layers):
        out = torch.empty_like(q)
        l2.paged_attention(q, off, K[l * H:(l + 1) * H], V[l * H:(l + 1) * H], cur, 128, out, b)
        torch.cuda.synchronize()
        for s in range(3):
            rows = torch.from_numpy(t[s, 0][np.arange(int(cur[s, 0])) // P].astype(np.int64) * P + np.arange(int(cur[s, 0])) % P).to(DEV)
            for j in range(4):
                k, v = K[l * H + j // 2, rows].double(), V[l * H + j // 2, rows].double()
                w = torch.softmax(k @ q[0, s, j].double() * D ** -0.5, 0)
                assert ((out[0, s, j].double() - w @ v).abs() <= 2.1 * 2.0 ** -8 * (w @ v.abs()) + 1e-4).all()


def test_a_bound_below_the_lengths_cuts_them(l2):
    """max_len is the host's word: longer lengths are brought down to it."""
    c = Paged(l2, [1, 1], [[300], [20]], 1, 2, 4, 128, 16, seed=4)
    out, cut = c.empty_out(), c.empty_out()
    l2.paged_attention(c.q, c.tok_off, c.K, c.V, c.lens(c.cur), 100, out, c.pages)
    l2.paged_attention(c.q, c.tok_off, c.K, c.V, i32([[100], [21]]), 100, cut, c.pages)
    torch.cuda.synchronize()
    assert torch.equal(out, cut)


@pytest.mark.parametrize("captured", [False, True])
def test_tables_and_lengths_written_just_before(l2, captured):
    """Every call is set up while the kernel before it runs: what that one writes last is what counts."""
    c = Paged(l2, [1, 1], [[300], [600]], 1, 2, 4, 128, 16, seed=5)
    cur, cur_d, table = c.lens(c.cur), torch.zeros_like(c.lens(c.cur)), c.pages.table.clone()
    pages = l2.Pages(torch.zeros_like(table), 16, c.n_pages)
    out, want = c.empty_out(), c.empty_out()
    ws = torch.zeros(l2.paged_attention_workspace_bytes(c.K, c.q, c.max_len, c.pages), dtype=torch.uint8, device=DEV)
    l2.paged_attention(c.q, c.tok_off, c.K, c.V, cur, c.max_len, want, c.pages, workspace=ws)
    big = torch.zeros(1 << 26, device=DEV)
    keep, grow, parent = torch.zeros_like(cur), i32([3, 20]), i32([1, 0])
    after = l2.Pages.empty(2, 1, c.table.shape[2], 16, c.n_pages, DEV)
    ws2 = torch.zeros(l2.page_workspace_bytes(c.K, c.pages), dtype=torch.uint8, device=DEV)
    swapped = cur.flip(0).contiguous()

    def step():
        pages.table.zero_(), cur_d.zero_(), keep.zero_()
        big.fill_(1.0)
        torch.add(table, 0, out=pages.table)
        torch.add(cur, 0, out=cur_d)
        l2.paged_attention(c.q, c.tok_off, c.K, c.V, cur_d, c.max_len, out, pages, workspace=ws)
        torch.add(swapped, 0, out=keep)
        l2.page_update(c.K, c.V, None, None, pages, parent, keep, grow, after, ws2)
    run = step
    if captured:
        step()
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            step()
        run = graph.replay
    expect = updated(c.table, 16, c.n_pages, [1, 0], swapped.cpu().numpy(), [3, 20])[0]
    for _ in range(5):
        out.zero_()
        run()
        torch.cuda.synchronize()
        assert torch.equal(out, want) and np.array_equal(after.table.cpu().numpy(), expect)


def test_results_do_not_depend_on_who_takes_which_part(l2):
    """Calls large enough that their last quarter is dealt out as SMs come free: the same bits every time."""
    c = Paged(l2, [1] * 40, np.random.RandomState(1).randint(2000, 9000, (40, 1)), 1, 4, 4, 128, 32, seed=3)
    ws = torch.zeros(l2.paged_attention_workspace_bytes(c.K, c.q, c.max_len, c.pages), dtype=torch.uint8, device=DEV)
    first = None
    for _ in range(20):
        out, lse = c.empty_out(), torch.zeros((1, c.N, c.Hq), device=DEV)
        l2.paged_attention(c.q, c.tok_off, c.K, c.V, c.lens(c.cur), c.max_len, out, c.pages, lse_out=lse, workspace=ws)
        torch.cuda.synchronize()
        first = first or (out, lse)
        assert torch.equal(out, first[0]) and torch.equal(lse, first[1])
    check_attention(c, *first, causal(c))
    assert l2.read_device_status(ws) == 0


def test_rows_behind_two_gigabytes(l2):
    """Elements of the pool beyond 2^31: the last pages of a pool of 2.2 GB, and of its last head."""
    H, D, P, n_pages = 4, 128, 64, 34000
    if torch.cuda.mem_get_info()[0] < 12 << 30:
        pytest.skip("not enough memory")
    K, V = (torch.zeros((H, n_pages * P, D), dtype=torch.bfloat16, device=DEV) for _ in range(2))
    g = torch.Generator().manual_seed(2)
    pages = l2.Pages(i32([[[n_pages - 1, 5, n_pages - 2]]]), P, n_pages)
    rows = torch.cat([torch.arange(P) + p * P for p in (n_pages - 1, 5, n_pages - 2)]).to(DEV)[:150]
    tok = torch.randn((1, 150, H * 3, D), generator=g).to(DEV, torch.bfloat16)
    off, pos, start, new = i32([0, 150]), i32(range(150)), i32([[0]]), i32([[0]])
    ws = torch.zeros(1 << 22, dtype=torch.uint8, device=DEV)
    q = torch.empty((1, 150, H, D), dtype=torch.bfloat16, device=DEV)
    l2.norm_rotary_write(tok[:, :, :H], tok[:, :, H:2 * H], tok[:, :, 2 * H:], off, pos, None, q, K, V, None, None, start, new, ws, norm_q=False,
                         norm_k=False, pages=pages)
    for n in (1, 150):                                       # both forms of attention
        out = torch.empty((1, n, H, D), dtype=torch.bfloat16, device=DEV)
        l2.paged_attention(q[:, 150 - n:], i32([0, n]), K, V, new, 192, out, pages)
        torch.cuda.synchronize()
        for h in range(H):
            k, v = K[h, rows].double(), V[h, rows].double()
            assert torch.equal(K[h, rows], tok[0, :, H + h]) and torch.equal(V[h, rows], tok[0, :, 2 * H + h])
            hidden = torch.ones((n, 150), dtype=torch.bool, device=DEV).triu(151 - n)
            w = (q[0, 150 - n:, h].double() @ k.T * D ** -0.5).masked_fill(hidden, -torch.inf).softmax(-1)
            assert ((out[0, :, h].double() - w @ v).abs() <= 2.1 * 2.0 ** -8 * (w @ v.abs()) + 1e-4).all()
    # a fork of it, and its compaction
    key = torch.rand((H, n_pages * P), device=DEV)
    two = l2.Pages.empty(2, 1, 3, P, n_pages, DEV)
    l2.page_update(K, V, None, key, pages, i32([0, 0]), i32([[150], [150]]), i32([1, 1]), two, ws)
    small, n = l2.Pages.empty(2, 1, 3, P, n_pages, DEV), i32([[0], [0]])
    before, key0 = (K.clone(), key.clone())
    l2.page_compact(K, V, None, key, two, i32([[150], [150]]), i32([[150], [40]]), 192, small, n, ws)
    torch.cuda.synchronize()
    t, s = two.table.cpu().numpy(), small.table.cpu().numpy()
    assert t[1, 0, 2] == 0 and s[1, 0].tolist() == [1, -1, -1] and n.flatten().tolist() == [150, 40]
    assert torch.equal(K[:, :22], before[:, (n_pages - 2) * P:(n_pages - 2) * P + 22])
    at = torch.cat([torch.arange(P) + int(p) * P for p in t[1, 0]]).to(DEV)[:150]
    for h in range(H):
        kept = key0[h, at].sort(stable=True).indices[:40].sort().values
        assert torch.equal(K[h, P:P + 40], before[h, at[kept]])
