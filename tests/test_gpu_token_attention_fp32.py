"""Prompt and tree attention over fp32 caches: packed rows, several layers, lengths per head, strided tokens, more
sequences than a group of the search, and lengths around its tiles of 32."""
import numpy as np
import pytest
import torch

from token_util import DEV, Case, causal, check_attention, mask_words, random_trees

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def l2():
    import paper_2406_11430_b200 as lib
    lib.lib()
    return lib


def _both(l2, c, seed=1, out_of=None):
    trees = random_trees(c, seed)
    for tree in (False, True):
        out = c.empty_out() if out_of is None else out_of(c)
        lse = torch.full((c.L, c.N, c.Hq), 7.0, device=DEV)
        ws = torch.zeros(256, dtype=torch.uint8, device=DEV)
        kw = dict(lse_out=lse, workspace=ws, rows=c.rows, per_head=c.per_head)
        if tree:
            l2.tree_attention(c.q, c.tok_off, mask_words(c, trees), c.K, c.V, c.lens(c.cur), c.max_len, out, **kw)
        else:
            l2.prompt_attention(c.q, c.tok_off, c.K, c.V, c.lens(c.cur), c.max_len, out, **kw)
        torch.cuda.synchronize()
        assert l2.read_device_status(ws) == 0
        check_attention(c, out, lse, trees if tree else causal(c))
        used = int(c.off[-1])
        assert (out[:, used:] == 7).all() and (lse[:, used:] == 7).all()


@pytest.mark.parametrize("packed", [False, True])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("G", [1, 2, 4, 8])
def test_layers_packed_and_strided(l2, G, D, packed):
    c = Case(l2, [5, 0, 33, 1], [[130, 7], [70, 0], [0, 300], [31, 32]], 2, 3, G, D, "fp32", packed=packed, seed=G, pad=3, strided=True)
    _both(l2, c, out_of=lambda c: torch.full((c.L, c.N, c.Hq, 2 * c.D), 7.0, device=DEV)[..., :c.D])


@pytest.mark.parametrize("packed", [False, True])
def test_lengths_per_head(l2, packed):
    ctx = np.random.RandomState(8).randint(0, 400, (3, 2, 2))
    ctx[1, 1] = [0, 900]
    _both(l2, Case(l2, [3, 21, 66], ctx, 2, 2, 4, 128, "fp32", packed=packed, seed=7, per_head=True))


@pytest.mark.parametrize("G", [1, 8])
def test_many_sequences(l2, G):
    r = np.random.RandomState(G)
    n = r.randint(0, 40, 70)
    n[30:35] = 0
    _both(l2, Case(l2, n, r.randint(0, 200, (70, 2)), 2, 2, G, 64, "fp32", packed=True, seed=9, pad=11))


@pytest.mark.parametrize("n,ctx", [([1], 0), ([1], 31), ([1], 32), ([8], 24), ([31], 1), ([32], 0), ([33], 31), ([64], 64), ([65], 2000)])
def test_lengths_around_the_tiles(l2, n, ctx):
    _both(l2, Case(l2, n, [[ctx]], 1, 2, 4, 128, "fp32", seed=n[0] + ctx))


def test_scales_and_rising_maxima(l2):
    c = Case(l2, [40], [[700]], 1, 2, 4, 128, "fp32", seed=8)
    c.K *= torch.linspace(0.1, 6.0, c.max_len, device=DEV)[:, None]
    _both(l2, c)
    c.K = c.K.flip(3).contiguous().nan_to_num(0.0)
    _both(l2, c)
