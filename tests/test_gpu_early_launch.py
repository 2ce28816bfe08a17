"""What an early-launched call reads may be written by the kernel right before it: accepted paths and their lengths,
offsets, positions, cached lengths and masks, with other values in them beforehand."""
import pytest
import torch

from token_util import DEV, Case, check_attention, i32, mask_words, random_trees

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def l2():
    import paper_2406_11430_b200 as lib
    lib.lib()
    return lib


@pytest.mark.parametrize("dtype,D", [("bf16", 128), ("bf16", 64), ("fp32", 128)])
@pytest.mark.parametrize("captured", [False, True])
def test_a_path_written_just_before_its_commit(l2, captured, dtype, D):
    """A long kernel, then copies that write n_path and path, then the commit: a commit that read either of them early would
    move the rows of the path before (valid too, so that nothing else would show it)."""
    c = Case(l2, [8, 60], [[30], [100]], 1, 3, 2, D, dtype, seed=5)
    idx, key = torch.arange(2 * 3 * c.max_len, dtype=torch.int32, device=DEV).view(c.meta), torch.rand(c.meta, device=DEV)
    start, cur = c.lens(c.ctx), c.lens(c.cur)
    ws, big = torch.zeros(256, dtype=torch.uint8, device=DEV), torch.zeros(1 << 27, device=DEV)
    old, new = [[1, 2, 3, 4, 5], [7, 8, 9, 10, 11]], [[0, 3, 6, 0, 0], [2, 20, 31, 58, 59]]
    path, n_path, kept = i32(old), i32([5, 4]), i32([[0], [0]])
    new_path, new_n = i32(new), i32([3, 5])
    old_path, old_n = i32(old), i32([5, 4])
    K, V, I, S = (torch.empty_like(x) for x in (c.K, c.V, idx, key))

    def step():
        K.copy_(c.K), V.copy_(c.V), I.copy_(idx), S.copy_(key)
        path.copy_(old_path), n_path.copy_(old_n)
        big.fill_(1.0)
        # ordinary kernels (an addition each) write the path that counts
        torch.add(new_path, 0, out=path)
        torch.add(new_n, 0, out=n_path)
        l2.tree_commit(K, V, I, S, start, cur, path, n_path, kept, ws)
    step()
    run = step
    if captured:
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            step()
        run = graph.replay
    for _ in range(10):
        kept.zero_()
        run()
        torch.cuda.synchronize()
        assert kept.flatten().tolist() == [33, 105] and l2.read_device_status(ws) == 0
        for x, was in ((K, c.K), (V, c.V), (I, idx), (S, key)):
            for b, (p, m) in enumerate(zip(new, (3, 5))):
                want = was[b, 0].clone()
                at = int(c.ctx[b, 0, 0])
                want[:, at:at + m] = was[b, 0][:, [at + j for j in p[:m]]]
                assert torch.equal(x[b, 0].contiguous().view(torch.uint8), want.contiguous().view(torch.uint8))


def test_a_path_written_by_a_call_of_the_library_just_before(l2):
    """The same with an early-launched kernel ahead: rotary_write leaves its new lengths, which the commit takes as its path's
    count, its start and its tree's end."""
    c = Case(l2, [4], [[10]], 1, 2, 2, 128, seed=6, room=16)
    idx, key = torch.zeros(c.meta, dtype=torch.int32, device=DEV), torch.zeros(c.meta, device=DEV)
    pos, ws, big = torch.arange(4, dtype=torch.int32, device=DEV), torch.zeros(256, dtype=torch.uint8, device=DEV), torch.zeros(1 << 27, device=DEV)
    three, start, lens, kept = i32([[-1]]), c.lens(c.ctx), i32([[0]]), i32([[0]])
    path = i32([[0, 2, 3, 3]])
    none, three_rows, out = i32([0, 0]), i32([[3]]), c.empty_out()
    for _ in range(10):
        lens.zero_(), three.fill_(1), kept.zero_()
        big.fill_(1.0)
        # no tokens: three = 3 (a length without new rows), by the library's own kernel
        l2.rotary_write(c.q[:, :0], c.k[:, :0], c.v[:, :0], none, pos[:0], None, c.q[:, :0], c.K, c.V, None, None, three_rows, three, ws)
        l2.rotary_write(c.q, c.k, c.v, c.tok_off, pos, None, out, c.K, c.V, idx, key, start, lens, ws)
        l2.tree_commit(c.K, c.V, idx, key, start, lens, path, three.view(1), kept, ws)
        torch.cuda.synchronize()
        assert kept.item() == 13 and idx[0, 0, 0, 10:13].tolist() == [0, 2, 3]
        for h in range(2):
            assert torch.equal(c.V[0, 0, h, 10:13], c.v[0, [0, 2, 3], h])
    assert l2.read_device_status(ws) == 0


def test_masks_and_offsets_written_just_before_attention(l2):
    c = Case(l2, [20, 40], [[3000], [100]], 1, 2, 4, 128, seed=7)
    trees = random_trees(c, 3)
    right, mask = mask_words(c, trees), torch.zeros_like(mask_words(c, trees))
    cur, off = torch.zeros_like(c.lens(c.cur)), torch.zeros_like(c.tok_off)
    want_cur, big = c.lens(c.cur), torch.zeros(1 << 27, device=DEV)
    ws = torch.zeros(l2.prompt_attention_workspace_bytes(c.K, c.q, c.max_len), dtype=torch.uint8, device=DEV)
    out, lse = c.empty_out(), torch.empty((1, c.N, c.Hq), device=DEV)
    for _ in range(5):
        mask.zero_(), cur.zero_(), off.zero_()
        big.fill_(1.0)
        torch.add(c.tok_off, 0, out=off)
        torch.add(want_cur, 0, out=cur)
        torch.add(right, 0, out=mask)
        l2.tree_attention(c.q, off, mask, c.K, c.V, cur, c.max_len, out, lse_out=lse, workspace=ws)
        torch.cuda.synchronize()
        check_attention(c, out, lse, trees)
    assert l2.read_device_status(ws) == 0
