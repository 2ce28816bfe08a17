"""Calls on new tokens that a program makes and the other files do not: from two Python threads at once, hundreds of
sequences of one token, batches of nothing but padding, commits of more heads than a block has warps and of paths that
break off late."""
import threading

import numpy as np
import pytest
import torch

from test_gpu_token_rows import check_commit
from token_util import DEV, Case, causal, check_attention, i32, mask_words, random_trees

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def l2():
    import paper_2406_11430_b200 as lib
    lib.lib()
    return lib


def test_two_threads_call_at_once(l2):
    """A cache, a workspace and a stream each; every call gives the bits it gives alone."""
    jobs = []
    for seed, (n, ctx, H, G, D) in enumerate((([40, 64, 9], [[3000], [1000], [5000]], 4, 4, 128), ([90, 30], [[0], [2000]], 8, 2, 64))):
        c = Case(l2, n, ctx, 1, H, G, D, seed=seed, room=100)
        c.mask, c.stream = mask_words(c, random_trees(c, seed)), torch.cuda.Stream()
        c.ws = torch.zeros(l2.prompt_attention_workspace_bytes(c.K, c.q, c.max_len), dtype=torch.uint8, device=DEV)
        c.idx, c.key = torch.zeros(c.meta, dtype=torch.int32, device=DEV), torch.zeros(c.meta, device=DEV)
        c.pos, c.freq = torch.arange(c.N, dtype=torch.int32, device=DEV), l2.rotary_frequencies(D)[0].to(DEV)
        c.start, c.new = c.lens(c.ctx), torch.zeros_like(c.lens(c.ctx))
        c.path, c.n_path = i32([[0, 3, 8]] * len(n)), i32([3] * len(n))
        c.kept = torch.zeros_like(c.start)
        c.result = [c.empty_out() for _ in range(3)]
        jobs.append(c)

    def step(c, result):
        l2.rotary_write(c.q, c.k, c.v, c.tok_off, c.pos, c.freq, result[0], c.K, c.V, c.idx, c.key, c.start, c.new, c.ws, stream=c.stream)
        l2.prompt_attention(result[0], c.tok_off, c.K, c.V, c.new, c.max_len, result[1], workspace=c.ws, stream=c.stream)
        l2.tree_attention(result[0], c.tok_off, c.mask, c.K, c.V, c.new, c.max_len, result[2], workspace=c.ws, stream=c.stream)
        l2.tree_commit(c.K, c.V, c.idx, c.key, c.start, c.new, c.path, c.n_path, c.kept, c.ws, stream=c.stream)
    torch.cuda.synchronize()
    for c in jobs:
        step(c, c.result)
    torch.cuda.synchronize()
    want = [[x.clone() for x in (*c.result, c.K, c.V, c.idx, c.key, c.kept)] for c in jobs]
    errors = []

    def work(c, w):
        try:
            with torch.cuda.stream(c.stream):
                for _ in range(60):
                    result = [torch.zeros_like(x) for x in c.result]
                    step(c, result)
                    got = [*result, c.K, c.V, c.idx, c.key, c.kept]
                    bad = [not torch.equal(a.contiguous().view(torch.uint8), b.contiguous().view(torch.uint8)) for a, b in zip(got, w)]
                    assert not any(bad), bad
        except BaseException as e:                            # (raised in the test below)
            errors.append(e)
    threads = [threading.Thread(target=work, args=job) for job in zip(jobs, want)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    torch.cuda.synchronize()
    assert not errors, errors
    for c in jobs:
        assert l2.read_device_status(c.ws) == 0


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("longest", [200, 1500])
def test_hundreds_of_sequences_of_one_token(l2, longest, dtype):
    r = np.random.RandomState(longest)
    ctx = r.randint(0, longest, (300, 1))
    ctx[::7] = 0
    c = Case(l2, [1] * 300, ctx, 1, 2, 4, 64, dtype, packed=True, seed=3)
    ws = torch.zeros(l2.prompt_attention_workspace_bytes(c.K, c.q, c.max_len, rows=c.rows), dtype=torch.uint8, device=DEV)
    out, lse = c.empty_out(), torch.empty((1, c.N, c.Hq), device=DEV)
    l2.prompt_attention(c.q, c.tok_off, c.K, c.V, c.lens(c.cur), c.max_len, out, lse_out=lse, workspace=ws, rows=c.rows)
    torch.cuda.synchronize()
    assert l2.read_device_status(ws) == 0
    check_attention(c, out, lse, causal(c))


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("offsets", [[0, 0, 0], [9, 9, 9], [20, 20, 20], [1 << 20, 1 << 20, 1 << 20]])
def test_nothing_but_padding(l2, offsets, dtype):
    c = Case(l2, [15, 5], [[3000], [7]], 1, 2, 4, 128, dtype, seed=4)
    ws = torch.zeros(l2.prompt_attention_workspace_bytes(c.K, c.q, c.max_len), dtype=torch.uint8, device=DEV)
    off, cur, out, lse = i32(offsets), c.lens(c.cur), c.empty_out(), torch.full((1, c.N, c.Hq), 7.0, device=DEV)
    K, V = c.K.clone(), c.V.clone()
    l2.prompt_attention(c.q, off, c.K, c.V, cur, c.max_len, out, lse_out=lse, workspace=ws)
    l2.tree_attention(c.q, off, torch.full((c.N, 1), -1, dtype=torch.int64, device=DEV), c.K, c.V, cur, c.max_len, out, lse_out=lse, workspace=ws)
    new = torch.zeros_like(cur)
    l2.rotary_write(c.q, c.k, c.v, off, torch.arange(c.N, dtype=torch.int32, device=DEV), None, out, c.K, c.V, None, None, cur, new, ws)
    torch.cuda.synchronize()
    assert (out == 7).all() and (lse == 7).all() and torch.equal(new, cur) and l2.read_device_status(ws) == 0
    assert torch.equal(K.view(torch.uint8), c.K.view(torch.uint8)) and torch.equal(V.view(torch.uint8), c.V.view(torch.uint8))


@pytest.mark.parametrize("alias", ["start", "cur", "none"])
@pytest.mark.parametrize("per_head", [False, True])
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_commit_of_more_heads_than_warps(l2, dtype, per_head, alias):
    r = np.random.RandomState(4)
    ctx = r.randint(0, 50, (2, 2, 19) if per_head else (2, 2))
    c = Case(l2, [6, 70], ctx, 2, 19, 1, 64, dtype, seed=3, per_head=per_head)
    check_commit(l2, c, [[1, 3, 5] + [0] * 37, list(range(10, 50))], [3, 40], [3, 40], alias)


def test_paths_that_break_off_late(l2):
    """In the second group of 32 entries, at its first entry, and by an entry that repeats the first group's last."""
    c = Case(l2, [90, 90, 90], [[3], [0], [9]], 1, 3, 2, 128, seed=2)
    path = [[j + 1 for j in range(50)], [j + 2 for j in range(50)], [j for j in range(50)]]
    path[0][40] = 90                                         # leaves the tree
    path[1][32] = path[1][31]                                # does not increase
    path[2][49] = 48
    check_commit(l2, c, path, [50, 50, 50], [40, 32, 49], status=-5)
