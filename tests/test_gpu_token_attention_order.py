"""Many calls of one shape back to back on one workspace: the hand-offs inside the kernel have to hold
whatever the roles' pace, and every call has to give the first one's bits."""
import numpy as np
import pytest
import torch

from token_util import DEV, Case, mask_words, random_trees

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("n,ctx", [
    ([17, 24, 12, 20, 13, 14, 23, 16], [[1024], [16000], [9000], [700], [12000], [4000], [2000], [15000]]),   # trees
    ([5], [[700]]), ([1], [[64]]), ([64, 64], [[9000], [9000]]),
    ([2000, 1, 333, 64, 700, 65], [[0], [0], [1], [100], [0], [63]])])                                     # prompts
def test_back_to_back_calls_agree(n, ctx, D):
    import paper_2406_11430_b200 as l2
    c = Case(l2, n, ctx, 1, 8, 4, D, seed=3, packed=len(n) > 5)
    trees = random_trees(c, 3)
    mask, cur = mask_words(c, trees), c.lens(c.cur)
    ws = torch.zeros(l2.prompt_attention_workspace_bytes(c.K, c.q, c.max_len, rows=c.rows), dtype=torch.uint8, device=DEV)
    outs = [c.empty_out() for _ in range(6)]
    for round in range(40):
        for i in range(3):
            l2.tree_attention(c.q, c.tok_off, mask, c.K, c.V, cur, c.max_len, outs[i], workspace=ws, rows=c.rows)
            l2.prompt_attention(c.q, c.tok_off, c.K, c.V, cur, c.max_len, outs[3 + i], workspace=ws, rows=c.rows)
        torch.cuda.synchronize()
        assert l2.read_device_status(ws) == 0
        for i in (1, 2):
            assert torch.equal(outs[0], outs[i]) and torch.equal(outs[3], outs[3 + i])
