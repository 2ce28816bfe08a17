"""Prompt and tree attention where caches are shared out over the SMs: items cut at share ends and joined, for every
group size, dense and packed, several layers, lengths per head that differ widely, more sequences than one group
of the plan, and caches shorter than their new tokens; and the shares themselves against a plain restatement."""
import numpy as np
import pytest
import torch

from token_util import DEV, Case, causal, check_attention, mask_words, random_trees

pytestmark = pytest.mark.gpu
SUB, ITEM, GRID = 64, 4, 148                                  # cached rows per sub-block, an item's own cost, CTAs
SPOT = np.dtype([("at", "<i8"), ("e", "<i4"), ("p", "<i4"), ("h", "<i4"), ("off", "<i4")])


@pytest.fixture(scope="module")
def l2():
    import paper_2406_11430_b200 as lib
    lib.lib()
    return lib


def _workspace(l2, c, max_len):
    ws = torch.full((l2.prompt_attention_workspace_bytes(c.K, c.q, max_len, rows=c.rows),), 255, dtype=torch.uint8, device=DEV)
    ws[:256] = 0
    return ws


def _plan(c, ws):
    """Where the shares begin, as the call left it in its workspace: behind the completion counters."""
    head = 256 + -(-c.B * c.L * c.H * 4 // 256) * 256
    return ws[head:head + GRID * SPOT.itemsize].cpu().numpy().view(SPOT)


def _both(l2, c, seed=1, check=True):
    """Both calls with a full workspace; returns how many shares began inside an item."""
    cur, cuts, max_len = c.lens(c.cur), [], c.max_len
    trees = random_trees(c, seed)
    for tree in (False, True):
        ws, out, lse = _workspace(l2, c, max_len), c.empty_out(), torch.full((c.L, c.N, c.Hq), 7.0, device=DEV)
        kw = dict(lse_out=lse, workspace=ws, rows=c.rows, per_head=c.per_head)
        if tree:
            l2.tree_attention(c.q, c.tok_off, mask_words(c, trees), c.K, c.V, cur, max_len, out, **kw)
        else:
            l2.prompt_attention(c.q, c.tok_off, c.K, c.V, cur, max_len, out, **kw)
        torch.cuda.synchronize()
        assert l2.read_device_status(ws) == 0
        if check:
            check_attention(c, out, lse, trees if tree else causal(c))
        used = int(c.off[-1])
        assert (out[:, used:] == 7).all() and (lse[:, used:] == 7).all()
        plan = _plan(c, ws)
        check_plan(c, plan, tree)
        cuts.append(int((plan["off"] > 0).sum()))
    return cuts


def check_plan(c, plan, tree):
    """Every share begins at an item of the list, at the cost of everything before it, no later than the next one begins,
    and within the item; so each sub-block is in exactly one share."""
    QP = 2 * (128 // c.G)
    items, at = [], 0
    for b in range(c.B):
        for l in range(c.L):
            n, cur = c.n[b], int(c.cur[b, l].max())
            for p in range(-(-n // QP)):
                end = cur if tree else max(0, min(cur, cur - n + min((p + 1) * QP, n)))
                for h in range(c.H):
                    items.append((at, b * c.L + l, p, h, -(-end // SUB)))
                    at += -(-end // SUB) + ITEM
    whole = all(s["off"] == 0 for s in plan) and all(s["at"] == min(i, len(items)) for i, s in enumerate(plan)) and len(items) <= GRID
    starts = {(i if whole else it[0]): it for i, it in enumerate(items)}
    assert plan[0]["at"] == 0 and plan[0]["off"] == 0
    for i, s in enumerate(plan):
        if s["at"] == (len(items) if whole else at):          # behind everything
            assert s["off"] == 0
            continue
        _, e, p, h, subs = starts[int(s["at"])]
        assert (s["e"], s["p"], s["h"]) == (e, p, h), (i, s)
        assert 0 <= s["off"] < max(subs, 1)
        if i:
            assert (s["at"], s["off"]) >= (plan[i - 1]["at"], plan[i - 1]["off"])


@pytest.mark.parametrize("packed", [False, True])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("G", [1, 2, 4, 8])
def test_cut_items_of_every_group_size(l2, G, D, packed):
    c = Case(l2, [3, 0, 40, 1], [[9000, 5100], [70, 0], [2500, 6100], [4097, 1]], 2, 2, G, D, packed=packed, seed=G + D)
    cuts = _both(l2, c, seed=G)
    assert min(cuts) > 20, cuts


@pytest.mark.parametrize("packed", [False, True])
@pytest.mark.parametrize("G", [1, 2, 4, 8])
def test_cut_items_with_lengths_per_head_far_apart(l2, G, packed):
    """Shares are dealt out by the longest head: pieces behind a shorter one's end are empty."""
    ctx = np.zeros((3, 2, 3), int)
    ctx[0] = [[100, 9000, 0], [7000, 3, 64]]
    ctx[1] = [[0, 0, 5000], [1, 2, 3]]
    ctx[2] = [[6000, 129, 6000], [63, 8000, 4000]]
    c = Case(l2, [5, 33, 70], ctx, 2, 3, G, 128, packed=packed, seed=G, per_head=True)
    cuts = _both(l2, c, seed=2)
    assert min(cuts) > 20, cuts


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("G", [1, 8])
def test_long_prompts_of_many_cut_items(l2, G, D):
    """Items of very different lengths; with groups of eight the items' ends fall into the middle of a sub-block."""
    c = Case(l2, [1500, 333, 1], [[1000], [31], [5000]], 1, 2, G, D, seed=G)
    cuts = _both(l2, c)
    assert min(cuts) > 0, cuts


@pytest.mark.parametrize("G", [2, 8])
def test_more_entries_than_one_group_of_the_plan(l2, G):
    r = np.random.RandomState(G)
    n, ctx = r.randint(0, 30, 40), r.randint(0, 300, (40, 2))
    ctx[[3, 31, 32, 39]] = [[5000, 100], [9000, 9000], [100, 7000], [6000, 0]]
    n[[3, 31, 32, 39]] = [7, 1, 29, 12]
    c = Case(l2, n, ctx, 2, 2, G, 128, packed=True, seed=G, pad=4)
    cuts = _both(l2, c)
    assert min(cuts) > 0, cuts


@pytest.mark.parametrize("G", [4, 8])
def test_a_few_rows_and_few_tokens_with_a_capacity_as_the_longest_length(l2, G):
    """What a captured step passes: room for far more rows than there are."""
    c = Case(l2, [5, 0, 77, 1], [[700], [0], [0], [64]], 1, 8, G, 128, seed=G, room=20000 // G)
    _both(l2, c)
    single = Case(l2, [1] * 5, [[0], [63], [64], [4000], [1216]], 1, 8, G, 128, seed=G)
    _both(l2, single)


@pytest.mark.parametrize("G", [1, 4, 8])
def test_more_new_tokens_than_rows_where_others_are_cut(l2, G):
    """cur_len < n beside a long cache: the first tokens lie before the cache and see nothing."""
    c = Case(l2, [300, 40], [[0], [9000]], 1, 2, G, 128, seed=G)
    c.cur = c.cur.copy()
    c.cur[0] = 150
    cur, ws, out = c.lens(c.cur), _workspace(l2, c, c.max_len), c.empty_out()
    lse = torch.empty((1, c.N, c.Hq), device=DEV)
    l2.prompt_attention(c.q, c.tok_off, c.K, c.V, cur, c.max_len, out, lse_out=lse, workspace=ws)
    torch.cuda.synchronize()
    assert l2.read_device_status(ws) == 0
    plan = _plan(c, ws)
    check_plan(c, plan, False)
    assert (plan["off"] > 0).sum() > 20
    assert not out[:, :150].any() and torch.isneginf(lse[:, :150]).all()
    # tokens 150 .. 299 are the 150 rows' own
    d = Case(l2, [150, 40], [[0], [9000]], 1, 2, G, 128, seed=G)
    d.q, d.K, d.V = c.q[:, 150:], c.K, c.V
    check_attention(d, out[:, 150:], lse[:, 150:], causal(d))


@pytest.mark.parametrize("seed", range(24))
def test_shares_of_drawn_calls(l2, seed):
    """The shares of all kinds of calls against the plain restatement (the outputs are other tests' matter)."""
    r = np.random.RandomState(seed)
    B, L, H, G = int(r.choice([1, 2, 5, 17, 40])), int(r.choice([1, 2, 3])), int(r.choice([1, 2, 5])), int(r.choice([1, 2, 4, 8]))
    per_head = bool(r.rand() < 0.3)
    n = np.where(r.rand(B) < 0.2, 0, np.exp(r.uniform(0, np.log(400 if B > 5 else 2000), B)).astype(int))
    n[r.randint(B)] += 1
    top = 1500 if B > 5 else 9000
    ctx = np.exp(r.uniform(0, np.log(top), (B, L, H) if per_head else (B, L))).astype(int) - 1
    ctx[0, 0] = 1300
    c = Case(l2, n, ctx, L, H, G, 64, packed=bool(r.rand() < 0.5), seed=seed, per_head=per_head)
    _both(l2, c, seed=seed, check=seed % 4 == 0)
