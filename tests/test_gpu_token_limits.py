"""The calls on new tokens where addresses, workspaces and streams reach their limits: rows beyond 2^32
bytes and 2^31 elements, two calls at once, a workspace shared with decode steps, captured writes."""
import numpy as np
import pytest
import torch

from token_util import DEV, Case, causal, check_attention, i32, mask_words, random_trees

pytestmark = pytest.mark.gpu
FAR = (1 << 31) + (1 << 20)                                   # elements


@pytest.fixture(scope="module")
def l2():
    import paper_2406_11430_b200 as lib
    lib.lib()
    return lib


def far_strides(c):
    """The same cache with its heads FAR elements apart, and tokens with their layers FAR apart."""
    for name in ("K", "V"):
        x = getattr(c, name)
        room = torch.empty(FAR + x.numel(), dtype=x.dtype, device=DEV)
        far = room.as_strided(x.shape, (x.stride(0), x.stride(1), FAR, x.stride(3), 1))
        setattr(c, name, far.copy_(x))
    far = torch.empty(FAR + c.q.numel(), dtype=c.dtype, device=DEV).as_strided(c.q.shape, (FAR, *c.q.stride()[1:]))
    c.q = far.copy_(c.q)


def far_rows(l2, c):
    """The same packed cache behind FAR elements of other rows."""
    shift = FAR // c.D
    total = c.rows.total_rows + shift
    for name in ("K", "V"):
        x = getattr(c, name)
        far = torch.empty((c.H, total, c.D), dtype=x.dtype, device=DEV)
        far[:, shift:] = x
        setattr(c, name, far)
    c.row0 = c.row0 + shift
    cap = np.array([[int(c.cap(b, l)) for l in range(c.L)] for b in range(c.B)])
    c.rows, c.meta = l2.Rows(c.row0, cap, total, DEV), (c.H, total)


@pytest.mark.parametrize("packed", [False, True])
def test_offsets_beyond_32_bits(l2, packed):
    c = Case(l2, [70, 3, 200], [[300, 5], [64, 1], [0, 90]], 2, 2, 4, 128, packed=packed, seed=13)
    far_rows(l2, c) if packed else far_strides(c)
    mask = mask_words(c, random_trees(c, 1))
    ws = torch.zeros(l2.prompt_attention_workspace_bytes(c.K, c.q, c.max_len, rows=c.rows), dtype=torch.uint8, device=DEV)
    out, lse = torch.empty_strided(c.q.shape, c.q.stride(), dtype=c.dtype, device=DEV), torch.empty((2, c.N, c.Hq), device=DEV)
    args = (c.K, c.V, c.lens(c.cur), c.max_len, out)
    l2.prompt_attention(c.q, c.tok_off, *args, lse_out=lse, workspace=ws, rows=c.rows)
    torch.cuda.synchronize()
    check_attention(c, out, lse, causal(c))
    l2.tree_attention(c.q, c.tok_off, mask, *args, lse_out=lse, workspace=ws, rows=c.rows)
    torch.cuda.synchronize()
    check_attention(c, out, lse, random_trees(c, 1))
    # writes and commits of rows out there
    idx, key = torch.full(c.meta, -1, dtype=torch.int32, device=DEV), torch.zeros(c.meta, device=DEV)
    start, cur = c.lens(c.ctx), torch.zeros_like(c.lens(c.ctx))
    pos = torch.arange(c.N, dtype=torch.int32, device=DEV)
    l2.rotary_write(c.q, c.k, c.v, c.tok_off, pos, None, out, c.K, c.V, idx, key, start, cur, ws, rows=c.rows)
    torch.cuda.synchronize()
    assert torch.equal(cur, c.lens(c.cur)) and torch.equal(out, c.q)
    l2.tree_commit(c.K, c.V, idx, key, start, cur, i32([[5, 60], [2, 0], [3, 199]]), i32([2, 1, 2]), start, ws, rows=c.rows)
    torch.cuda.synchronize()
    assert l2.read_device_status(ws) == 0
    for b, path in enumerate(([5, 60], [2], [3, 199])):
        for l in range(2):
            for h in range(2):
                at, first = int(c.ctx[b, l, h]), int(c.off[b])
                K, V, I = (c.unit(x, b, l, h) for x in (c.K, c.V, idx))
                for j, p in enumerate(path):
                    assert torch.equal(K[at + j], c.k[l, first + p, h]) and torch.equal(V[at + j], c.v[l, first + p, h])
                    assert int(I[at + j]) == first + p
                rest = [j for j in range(c.n[b]) if j >= len(path)]
                assert torch.equal(K[[at + j for j in rest]], c.k[l, [first + j for j in rest], h])


def test_two_calls_at_once(l2):
    """Two streams, a workspace each, many calls in flight: every call gives the bits it gives alone."""
    cases = [Case(l2, [40, 64, 9], [[9000], [3000], [12000]], 1, 4, 4, 128, seed=3),
             Case(l2, [500, 30], [[0], [2000]], 1, 8, 2, 64, seed=4)]
    jobs, streams = [], [torch.cuda.Stream() for _ in cases]
    for c in cases:
        mask, cur = mask_words(c, random_trees(c, 3)), c.lens(c.cur)
        ws = torch.zeros(l2.prompt_attention_workspace_bytes(c.K, c.q, c.max_len), dtype=torch.uint8, device=DEV)

        def job(out, tree, stream, c=c, mask=mask, cur=cur, ws=ws):
            if tree:
                l2.tree_attention(c.q, c.tok_off, mask, c.K, c.V, cur, c.max_len, out, workspace=ws, stream=stream)
            else:
                l2.prompt_attention(c.q, c.tok_off, c.K, c.V, cur, c.max_len, out, workspace=ws, stream=stream)
        jobs.append((job, c, ws))
    alone = [[c.empty_out(), c.empty_out()] for _, c, _ in jobs]
    for (job, _, _), outs in zip(jobs, alone):
        for tree in (0, 1):
            job(outs[tree], tree, None)
    torch.cuda.synchronize()
    outs = [[c.empty_out() for _ in range(40)] for _, c, _ in jobs]
    torch.cuda.synchronize()
    for i in range(40):
        for (job, _, _), o, s in zip(jobs, outs, streams):
            job(o[i], i % 2, s)
    torch.cuda.synchronize()
    for (_, _, ws), o, a in zip(jobs, outs, alone):
        assert l2.read_device_status(ws) == 0
        for i in range(40):
            assert torch.equal(o[i], a[i % 2])


def test_a_workspace_shared_with_decode_steps(l2):
    """Calls in order on one workspace: the completion counters of decode attention survive the others' scratch."""
    c = Case(l2, [5, 30], [[9000], [4000]], 1, 2, 4, 128, seed=5)
    cur, trees = c.lens(c.cur), random_trees(c, 2)
    mask = mask_words(c, trees)
    lay = l2.Layout(c.K, q_heads=c.Hq)
    need = max(l2.workspace_bytes(lay, c.max_len), l2.prompt_attention_workspace_bytes(c.K, c.q, c.max_len))
    ws = torch.zeros(need, dtype=torch.uint8, device=DEV)
    q1 = torch.randn((c.B, 1, c.Hq, c.D), device=DEV).to(c.dtype)
    dec = [torch.empty((c.B, 1, c.Hq, c.D), device=DEV) for _ in range(4)]
    l2.decode_attention(q1, c.K, c.V, cur, c.max_len, dec[0], ws)
    for i in range(1, 4):
        out = c.empty_out()
        l2.tree_attention(c.q, c.tok_off, mask, c.K, c.V, cur, c.max_len, out, workspace=ws)
        l2.decode_attention(q1, c.K, c.V, cur, c.max_len, dec[i], ws)
        torch.cuda.synchronize()
        check_attention(c, out, None, trees)
        assert torch.equal(dec[i], dec[0])
    assert l2.read_device_status(ws) == 0


def test_captured_writes_and_commits_with_other_lengths(l2):
    """One graph of a write and a commit for a padded batch; offsets, positions, lengths and paths change between
    replays, and the lengths are updated in place by the graph itself."""
    c = Case(l2, [20, 20], [[30], [40]], 1, 2, 4, 128, seed=6, room=64)
    idx, key = torch.full(c.meta, -1, dtype=torch.int32, device=DEV), torch.zeros(c.meta, device=DEV)
    start, cur = c.lens(c.ctx), torch.zeros_like(c.lens(c.ctx))
    pos = torch.zeros(c.N, dtype=torch.int32, device=DEV)
    path, n_path = i32(np.zeros((2, 4))), i32([0, 0])
    ws = torch.zeros(256, dtype=torch.uint8, device=DEV)
    out = c.empty_out()
    freq = l2.rotary_frequencies(128)[0].to(DEV)

    def step():
        l2.rotary_write(c.q, c.k, c.v, c.tok_off, pos, freq, out, c.K, c.V, idx, key, start, cur, ws)
        l2.tree_commit(c.K, c.V, idx, key, start, cur, path, n_path, start, ws)
    c.tok_off.zero_()
    step()                                                   # nothing yet: no token, no path
    torch.cuda.synchronize()
    assert torch.equal(start, c.lens(c.ctx)) and (out == 7).all()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    have = [30, 40]
    for off, paths in (([0, 20, 40], [[0, 3, 7], [1]]), ([0, 1, 12], [[0], [0, 5, 10]]), ([3, 3, 9], [[], [4]])):
        c.tok_off.copy_(i32(off))
        pos.copy_(torch.randint(0, 5000, (c.N,), dtype=torch.int32))
        path.zero_()
        for b, p in enumerate(paths):
            path[b, :len(p)] = i32(p)
        n_path.copy_(i32([len(p) for p in paths]))
        out.fill_(7)
        graph.replay()
        torch.cuda.synchronize()
        assert (out[:, :off[0]] == 7).all() and (out[:, off[2]:] == 7).all()
        for b, p in enumerate(paths):
            for h in range(2):
                for j, s in enumerate(p):
                    assert torch.equal(c.V[b, 0, h, have[b] + j], c.v[0, off[b] + s, h])
                    assert int(idx[b, 0, h, have[b] + j]) == int(pos[off[b] + s])
            have[b] += len(p)
        assert start.flatten().tolist() == have
    assert l2.read_device_status(ws) == 0


@pytest.mark.parametrize("captured", [False, True])
def test_calls_wait_for_whatever_is_before_them(l2, captured):
    """A call may be set up while the work before it runs, but reads and writes only behind it: large copies, fills,
    other streams' kernels and the calls themselves, eager and in one graph."""
    c = Case(l2, [30, 200], [[300], [100]], 1, 2, 4, 128, seed=9, room=8192)
    meta, freq = c.meta, l2.rotary_frequencies(128)[0].to(DEV)
    idx, key = torch.zeros(meta, dtype=torch.int32, device=DEV), torch.zeros(meta, device=DEV)
    start, cur, kept = c.lens(c.ctx), c.lens(c.cur), c.lens(c.ctx)
    pos, path, n_path = torch.arange(c.N, dtype=torch.int32, device=DEV), i32([[1, 5, 8], [0, 100, 150]]), i32([3, 3])
    K, V = torch.zeros_like(c.K), torch.zeros_like(c.V)
    q, out, out2 = (c.empty_out() for _ in range(3))
    ws = torch.zeros(l2.prompt_attention_workspace_bytes(K, q, c.max_len), dtype=torch.uint8, device=DEV)
    big = torch.zeros(1 << 27, device=DEV)
    host_off, other = c.tok_off.cpu().pin_memory(), torch.cuda.Stream()
    off, lens, work = torch.zeros_like(c.tok_off), torch.zeros_like(start), torch.zeros_like(start)

    def step():
        big.fill_(1.0)                                       # half a gigabyte, so that what follows is all queued up
        K.copy_(c.K), V.copy_(c.V)
        off.copy_(host_off, non_blocking=True)
        lens.zero_()
        l2.rotary_write(c.q, c.k, c.v, off, pos, freq, q, K, V, idx, key, start, lens, ws)
        l2.prompt_attention(q, off, K, V, lens, c.max_len, out, workspace=ws)
        l2.tree_commit(K, V, idx, key, start, lens, path, n_path, kept, ws)
        here = torch.cuda.current_stream()
        other.wait_stream(here)
        with torch.cuda.stream(other):
            big.mul_(2.0)
            work.copy_(kept)
            work.add_(torch.tensor([[27], [197]], dtype=torch.int32, device=DEV) if not captured else add)
        here.wait_stream(other)
        l2.prompt_attention(q, off, K, V, work, c.max_len, out2, workspace=ws)      # the 3 kept rows as context
    add = i32([[27], [197]])
    step()
    torch.cuda.synchronize()
    want = [x.clone() for x in (out, out2, q, kept)]
    check_q = Case(l2, [30, 200], [[300], [100]], 1, 2, 4, 128, seed=9, room=8192)
    check_q.q, check_q.K, check_q.V = q, c.K.clone(), c.V.clone()
    l2.rotary_write(c.q, c.k, c.v, c.tok_off, pos, freq, torch.empty_like(q), check_q.K, check_q.V, None, None, start, cur, ws)
    torch.cuda.synchronize()
    check_attention(check_q, out, None, causal(c))
    if captured:
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            step()
        run = graph.replay
    else:
        run = step
    for _ in range(10):
        for x in (out, out2, q, K, V):
            x.zero_()
        kept.zero_(), off.zero_(), lens.zero_()
        run()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(want, (out, out2, q, kept)))
    assert l2.read_device_status(ws) == 0


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_keys_that_a_token_does_not_see_may_be_anything(l2, dtype):
    c = Case(l2, [40, 7], [[200], [30]], 1, 2, 4, 128, dtype, seed=14)
    cur = c.lens(c.cur)
    trees = [torch.tril(torch.ones((m, m), dtype=torch.bool)) for m in c.n]
    for t in trees:
        t[:, 3] = False                                      # nobody sees the fourth new row, itself included
    mask = mask_words(c, trees)

    def both():
        a, b = c.empty_out(), c.empty_out()
        l2.tree_attention(c.q, c.tok_off, mask, c.K, c.V, cur, c.max_len, a)
        l2.prompt_attention(c.q, c.tok_off, c.K, c.V, cur, c.max_len, b)
        torch.cuda.synchronize()
        return a, b
    tree, causal_out = both()
    check_attention(c, tree, None, trees)
    for bad in (float("nan"), float("inf"), -float("inf")):
        saved = c.K.clone(), c.V.clone()
        for b, m in enumerate(c.n):
            for h in range(2):
                at = int(c.ctx[b, 0, h]) + 3
                c.K[b, 0, h, at] = bad
                if dtype == "fp32":
                    c.V[b, 0, h, at] = bad
                c.K[b, 0, h, int(c.cur[b, 0, h]) - 1] = bad       # and the last token's own
        got, got_causal = both()
        for b, m in enumerate(c.n):
            first = int(c.off[b])
            assert torch.equal(got[:, first:first + m - 1], tree[:, first:first + m - 1])
            assert torch.equal(got_causal[:, first:first + 3], causal_out[:, first:first + 3])   # tokens before the bad row
        c.K, c.V = saved
