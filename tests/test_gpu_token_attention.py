"""Prompt and tree attention over packed tokens against the definition in 64 bits: head layouts and
sizes, lengths around the kernels' tiles, sequences without tokens or without a cache, dense, packed and
strided tensors, padding, lengths per head, streams and graphs."""
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


def call(l2, c, trees, mask=None, scale=0.0, workspace="full", max_len=None, stream=None, lse=True, q=None):
    out = c.empty_out()
    z = torch.full((c.L, c.N, c.Hq), 7.0, device=DEV) if lse else None
    q = c.q if q is None else q
    max_len = c.max_len if max_len is None else max_len
    ws = None
    if workspace:
        need = l2.prompt_attention_workspace_bytes(c.K, q, max_len, rows=c.rows) if workspace == "full" else 256
        ws = torch.full((need,), 255, dtype=torch.uint8, device=DEV)      # only the status block is zeroed
        ws[:256] = 0
    kw = dict(lse_out=z, scale=scale, workspace=ws, rows=c.rows, per_head=c.per_head, stream=stream)
    cur = c.lens(c.cur)
    if stream is not None:
        stream.wait_stream(torch.cuda.current_stream())
    if trees is None:
        l2.prompt_attention(q, c.tok_off, c.K, c.V, cur, max_len, out, **kw)
    else:
        l2.tree_attention(q, c.tok_off, mask if mask is not None else mask_words(c, trees), c.K, c.V, cur, max_len, out, **kw)
    torch.cuda.synchronize()
    if ws is not None:
        assert l2.read_device_status(ws) == 0
    return out, z


def check_both(l2, c, seed=1, **kw):
    out, lse = call(l2, c, None, **kw)
    scale = kw.get("scale") or None
    check_attention(c, out, lse, causal(c), scale)
    used = int(c.off[-1])
    assert (out[:, used:] == 7).all() and (lse is None or (lse[:, used:] == 7).all())   # padding: left alone
    trees = random_trees(c, seed)
    out, lse = call(l2, c, trees, **kw)
    check_attention(c, out, lse, trees, scale)
    assert (out[:, used:] == 7).all()


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("G", [1, 2, 4, 8])
def test_head_layouts(l2, G, D, dtype):
    check_both(l2, Case(l2, [5, 0, 33, 1], [[130], [70], [0], [0]], 1, 2, G, D, dtype, seed=G))


@pytest.mark.parametrize("packed", [False, True])
@pytest.mark.parametrize("n,ctx", [
    ([1], [[0]]), ([1], [[127]]), ([1], [[128]]), ([2], [[126]]), ([128], [[0]]), ([129], [[0]]), ([31], [[97]]), ([32], [[96]]),
    ([33], [[95]]), ([63], [[1]]), ([64], [[64]]), ([65], [[300]]), ([255], [[1]]), ([256], [[0]]), ([257], [[385]]),
    ([300, 1, 64, 17], [[0], [513], [128], [1000]])])
def test_lengths_around_the_tiles(l2, n, ctx, packed):
    check_both(l2, Case(l2, n, ctx, 1, 2, 4, 128, packed=packed, seed=len(n) + n[0]))


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("workspace", ["full", "status", None])
def test_long_caches_few_tokens(l2, workspace, D):
    c = Case(l2, [3, 1, 40], [[9000], [4097], [2500]], 1, 2, 4, D, seed=5)
    check_both(l2, c, workspace=workspace)


def test_many_ragged_sequences(l2):
    r = np.random.RandomState(3)
    n = r.randint(0, 90, 70)
    check_both(l2, Case(l2, n, r.randint(0, 700, (70, 2)), 2, 2, 2, 128, packed=True, seed=9, pad=11))


def test_prompts_of_more_than_one_wave_of_tiles(l2):
    c = Case(l2, [1500, 700, 2100], [[0], [40], [0]], 1, 8, 4, 128, seed=2)
    out, lse = call(l2, c, None)
    check_attention(c, out, lse, causal(c))


def test_layers_strides_and_padding(l2):
    c = Case(l2, [40, 7], [[200, 31], [0, 129]], 2, 2, 4, 128, seed=4, pad=5, strided=True)
    check_both(l2, c)
    wide = torch.zeros((2, c.N, c.Hq, 2 * c.D), dtype=c.dtype, device=DEV)     # rows 2 D apart
    wide[..., :c.D] = c.q
    check_both(l2, c, q=wide[..., :c.D])


def test_a_cache_that_is_a_view(l2):
    """Token-major storage, and rows that are wider than a head."""
    c = Case(l2, [9, 50], [[100], [3]], 1, 2, 2, 128, seed=6)
    for name in ("K", "V"):
        x = getattr(c, name)
        room = torch.full((c.B, 1, c.max_len, c.H, 192), float("nan"), dtype=c.dtype, device=DEV)
        room[..., :128] = x.transpose(2, 3)
        setattr(c, name, room[..., :128].transpose(2, 3))
    check_both(l2, c)


@pytest.mark.parametrize("packed", [False, True])
def test_lengths_per_head(l2, packed):
    ctx = np.random.RandomState(8).randint(0, 400, (3, 2, 2))
    c = Case(l2, [3, 21, 66], ctx, 2, 2, 4, 128, packed=packed, seed=7, per_head=True)
    check_both(l2, c)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_more_tokens_than_cached_rows(l2, dtype):
    """cur_len < n: the first tokens lie before the cache and see nothing."""
    c = Case(l2, [50, 4], [[0], [0]], 1, 2, 2, 64, dtype, seed=1)
    lens = torch.tensor([[20], [0]], dtype=torch.int32, device=DEV)
    out, lse = c.empty_out(), torch.empty((1, c.N, c.Hq), device=DEV)
    l2.prompt_attention(c.q, c.tok_off, c.K, c.V, lens, c.max_len, out, lse_out=lse)
    torch.cuda.synchronize()
    assert not out[:, :30].any() and torch.isneginf(lse[:, :30]).all()
    assert not out[:, 50:].any() and torch.isneginf(lse[:, 50:]).all()
    # tokens 30 .. 49 are the 20 rows' own
    d = Case(l2, [20], [[0]], 1, 2, 2, 64, dtype, seed=1)
    d.q, d.K, d.V = c.q[:, 30:50], c.K[:1], c.V[:1]
    check_attention(d, out[:, 30:50], lse[:, 30:50], causal(d))


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_no_cached_rows_at_all_and_lengths_out_of_range(l2, dtype):
    c = Case(l2, [6, 3], [[0], [0]], 1, 2, 4, 128, dtype, seed=1)
    out, lse = c.empty_out(), torch.empty((1, c.N, c.Hq), device=DEV)
    for lens in ([[0], [0]], [[-5], [-1]]):
        out.fill_(7)
        l2.prompt_attention(c.q, c.tok_off, c.K, c.V, torch.tensor(lens, dtype=torch.int32, device=DEV), c.max_len, out,
                            lse_out=lse)
        torch.cuda.synchronize()
        assert not out.any() and torch.isneginf(lse).all()
    # device lengths above max_len are clamped to it
    big = torch.tensor([[1 << 30], [1 << 30]], dtype=torch.int32, device=DEV)
    l2.prompt_attention(c.q, c.tok_off, c.K, c.V, big, 3, out, lse_out=lse)
    torch.cuda.synchronize()
    assert torch.isneginf(lse[:, :3]).all() and torch.isfinite(out[:, 3:]).all()
    # offsets outside [0, n_tokens] are brought into it, and what is then no sequence's is left alone
    out.fill_(7)
    l2.prompt_attention(c.q, torch.tensor([-4, 2, 1 << 20], dtype=torch.int32, device=DEV), c.K, c.V, c.lens(c.cur),
                        c.max_len, out)
    torch.cuda.synchronize()
    l2.prompt_attention(c.q, torch.tensor([5, 5, 3], dtype=torch.int32, device=DEV), c.K, c.V, c.lens(c.cur), c.max_len,
                        c.empty_out())
    torch.cuda.synchronize()


def test_masks_shorter_than_the_tree_and_empty_ones(l2):
    c = Case(l2, [100, 70], [[30], [0]], 1, 2, 4, 128, seed=3)
    trees = random_trees(c, 2)
    for t in trees:
        t[:, 64:] = False                                    # one word: nothing beyond bit 63 is visible
    out, lse = call(l2, c, trees, mask=mask_words(c, trees, 1))
    check_attention(c, out, lse, trees)
    out, lse = call(l2, c, trees, mask=torch.zeros((c.N, 2), dtype=torch.int64, device=DEV))
    none = [torch.zeros_like(t) for t in trees]
    check_attention(c, out, lse, none)
    full = [torch.ones_like(t) for t in trees]
    out, lse = call(l2, c, full, mask=torch.full((c.N, 3), -1, dtype=torch.int64, device=DEV))
    check_attention(c, out, lse, full)


def test_scales_and_large_scores(l2):
    c = Case(l2, [70, 3], [[300], [64]], 1, 2, 4, 128, seed=8)
    check_both(l2, c, scale=0.25)
    check_both(l2, c, scale=1e-6)
    # maxima that keep rising: every block brings larger scores than all before it
    c = Case(l2, [40], [[700]], 1, 2, 4, 128, seed=8)
    c.K *= torch.linspace(0.1, 6.0, c.max_len, device=DEV, dtype=torch.bfloat16)[:, None]
    check_both(l2, c)
    c.K = c.K.flip(3).contiguous()                           # ... and falling (the rows with NaN come first)
    c.K = c.K.nan_to_num(0.0)
    check_both(l2, c)


def test_infinite_scores_of_rows_that_are_not_seen(l2):
    """Keys that no token may see hold infinities; so do the values behind the last visible row."""
    c = Case(l2, [4], [[250]], 1, 2, 4, 128, seed=8)
    out, lse = call(l2, c, None)
    c.K[:, :, :, 254:] = torch.inf
    c.V[:, :, :, 254:] = -torch.inf
    again, lse2 = call(l2, c, None)
    assert torch.equal(out, again) and torch.equal(lse, lse2)


def test_streams_without_lse_and_repeated(l2):
    c = Case(l2, [33, 200], [[400], [5000]], 1, 2, 4, 128, seed=11)
    s = torch.cuda.Stream()
    a, _ = call(l2, c, None, lse=False)
    b, _ = call(l2, c, None, lse=False, stream=s)
    assert torch.equal(a, b)                                  # the same bits, whatever the stream
    trees = random_trees(c, 4)
    a, _ = call(l2, c, trees)
    b, _ = call(l2, c, trees, stream=s)
    assert torch.equal(a, b)


def test_captured_and_replayed_with_other_lengths(l2):
    """One graph for a padded batch: lengths and offsets change between replays, on one workspace."""
    c = Case(l2, [64, 64], [[3000], [3000]], 1, 2, 4, 128, seed=12)
    trees = random_trees(c, 5)
    mask, cur = mask_words(c, trees), c.lens(c.cur)
    ws = torch.zeros(l2.prompt_attention_workspace_bytes(c.K, c.q, c.max_len), dtype=torch.uint8, device=DEV)
    out, lse = c.empty_out(), torch.empty((1, c.N, c.Hq), device=DEV)
    l2.tree_attention(c.q, c.tok_off, mask, c.K, c.V, cur, c.max_len, out, lse_out=lse, workspace=ws)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        l2.tree_attention(c.q, c.tok_off, mask, c.K, c.V, cur, c.max_len, out, lse_out=lse, workspace=ws)
    for n, ctx in (([64, 64], [[3000], [3000]]), ([5, 20], [[100], [2900]]), ([0, 1], [[0], [0]])):
        d = Case(l2, n, ctx, 1, 2, 4, 128, seed=12)
        d.K, d.V = c.K.clone(), c.V.clone()
        d.q, d.max_len = c.q, c.max_len
        c.tok_off.copy_(d.tok_off)
        cur.copy_(d.lens(d.cur))
        d.N = c.N
        trees = random_trees(d, 6)
        mask.copy_(mask_words(d, trees, mask.shape[1]))
        out.fill_(7)
        graph.replay()
        torch.cuda.synchronize()
        check_attention(d, out, lse, trees)
        assert (out[:, sum(n):] == 7).all()
    assert l2.read_device_status(ws) == 0


def test_a_gave_up_mark_stops_the_call(l2):
    c = Case(l2, [3], [[20]], 1, 2, 4, 128, seed=1)
    ws = torch.zeros(l2.prompt_attention_workspace_bytes(c.K, c.q, c.max_len), dtype=torch.uint8, device=DEV)
    l2.selftest_wait_timeout(ws)
    out = c.empty_out()
    l2.prompt_attention(c.q, c.tok_off, c.K, c.V, c.lens(c.cur), c.max_len, out, workspace=ws)
    assert l2.read_device_status(ws) == -8
    assert (out == 7).all()


def test_a_query_that_is_a_broadcast_view_is_refused(l2):
    c = Case(l2, [3], [[20]], 1, 2, 4, 128, seed=1)
    q = c.q[:, :, :1].expand(-1, -1, c.Hq, -1)
    with pytest.raises(l2.L2KVError) as e:
        l2.prompt_attention(q, c.tok_off, c.K, c.V, c.lens(c.cur), c.max_len, c.empty_out())
    assert e.value.status == -1
    K = c.K[:, :, :1].expand(-1, -1, 2, -1, -1)
    with pytest.raises(l2.L2KVError) as e:
        l2.prompt_attention(c.q, c.tok_off, K, K, c.lens(c.cur), c.max_len, c.empty_out())
    assert e.value.status == -2
