"""Rotary positions with the cache write, and the commit of a tree's accepted path."""
import numpy as np
import pytest
import torch

from token_util import DEV, Case, check_attention, causal, i32, mask_words

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def l2():
    import paper_2406_11430_b200 as lib
    lib.lib()
    return lib


def rotated(x, pos, freq, scale, interleaved):
    """x [L, N, heads, D] in 64 bits, by rotation matrices of complex numbers."""
    r = freq.numel()
    turn = torch.polar(torch.full((pos.numel(), r), scale, dtype=torch.float64, device=DEV),
                       pos.double()[:, None] * freq.double())[:, None]
    y = x.double().clone()
    a, b = (slice(0, 2 * r, 2), slice(1, 2 * r, 2)) if interleaved else (slice(0, r), slice(r, 2 * r))
    z = torch.complex(y[..., a], y[..., b]) * turn
    size = torch.complex(y[..., a].abs(), y[..., b].abs()).abs() * abs(scale)
    y[..., a], y[..., b] = z.real, z.imag
    spread = y.abs()
    spread[..., a] = spread[..., b] = size
    return y, spread


def assert_rotated(got, want, spread):
    """Cosine, sine, two products and a sum in fp32 (at most 4 roundings of 2^-24 of the pair's size), one
    rounding to the stored type (2^-8 of the value for bf16)."""
    half = 2.0 ** -8 if got.dtype == torch.bfloat16 else 2.0 ** -24
    bound = 4 * 2.0 ** -24 * 1.5 * spread + half * 1.01 * want.abs() + 1e-30
    assert ((got.double() - want).abs() <= bound).all()


def make(l2, c, start):
    c.K0, c.V0 = c.K.clone(), c.V.clone()
    c.idx = torch.full(c.meta, -1, dtype=torch.int32, device=DEV)
    c.key = torch.full(c.meta, -1.0, device=DEV)
    c.start, c.new = c.lens(start), torch.full_like(c.lens(start), 99)
    c.ws = torch.zeros(256, dtype=torch.uint8, device=DEV)
    c.q_out = c.empty_out()


def write(l2, c, pos, freq, **kw):
    l2.rotary_write(c.q, c.k, c.v, c.tok_off, pos, freq, c.q_out, c.K, c.V, c.idx, c.key, c.start, c.new, c.ws,
                    rows=c.rows, per_head=c.per_head, **kw)
    torch.cuda.synchronize()


def check_write(l2, c, pos, freq, scale, interleaved):
    used = int(c.off[-1])
    freq = torch.zeros(0, dtype=torch.float64, device=DEV) if freq is None else freq
    want_q, spread_q = rotated(c.q, pos, freq, scale, interleaved)
    want_k, spread_k = rotated(c.k, pos, freq, scale, interleaved)
    assert_rotated(c.q_out[:, :used], want_q[:, :used], spread_q[:, :used])
    assert (c.q_out[:, used:] == 7).all()
    rot = 2 * freq.numel()
    assert torch.equal(c.q_out[:, :used, :, rot:], c.q[:, :used, :, rot:])       # the rest is copied
    # the keys of the stored rows, by the library's own norm pass
    key = torch.full(c.meta, -1.0, device=DEV)
    t_cap = c.max_len
    full = torch.tensor([t_cap if c.rows is None else int(c.cur[b].max()) + 3 for b in range(c.B)], dtype=torch.int32, device=DEV)
    l2.key_norms(c.K, full, t_cap, key, rows=c.rows)
    for b in range(c.B):
        of = slice(int(c.off[b]), int(c.off[b + 1]))
        for l in range(c.L):
            for h in range(c.H):
                s, e = int(c.ctx[b, l, h]), int(c.cur[b, l, h])
                K, V, idx, K0, V0 = (c.unit(x, b, l, h) for x in (c.K, c.V, c.idx, c.K0, c.V0))
                assert_rotated(K[s:e], want_k[l, of, h], spread_k[l, of, h])
                assert torch.equal(V[s:e], c.v[l, of, h])
                assert torch.equal(idx[s:e], pos[of])
                got = c.unit(c.key, b, l, h)
                assert torch.equal(got[s:e], c.unit(key, b, l, h)[s:e])
                outside = torch.ones(K.shape[0], dtype=torch.bool, device=DEV)
                outside[s:e] = False
                for x, y in ((K, K0), (V, V0)):                 # every other row as it was, bit for bit
                    assert torch.equal(x[outside].contiguous().view(torch.uint8), y[outside].contiguous().view(torch.uint8))
                assert (idx[outside] == -1).all() and (got[outside] == -1).all()
    assert torch.equal(c.new, c.lens(c.cur))
    assert l2.read_device_status(c.ws) == 0


@pytest.mark.parametrize("packed", [False, True])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("dtype,D,rot", [("bf16", 128, 128), ("bf16", 128, 16), ("bf16", 128, 96), ("bf16", 64, 64),
                                         ("bf16", 64, 48), ("fp32", 128, 128), ("fp32", 128, 48), ("fp32", 64, 32)])
def test_rotary_write(l2, dtype, D, rot, interleaved, packed):
    c = Case(l2, [1, 37, 0, 5], [[0, 3], [100, 0], [7, 7], [64, 1]], 2, 2, 4, D, dtype, packed=packed, seed=rot, pad=3,
             strided=True)
    make(l2, c, c.ctx)
    pos = torch.randint(0, 131072, (c.N,), dtype=torch.int32, device=DEV)
    freq, _ = l2.rotary_frequencies(rot, 500000.0, l2.ROTARY_LLAMA3, factor=8.0)
    write(l2, c, pos, freq.to(DEV), interleaved=interleaved, attn_scale=1.1)
    check_write(l2, c, pos, freq.to(DEV), 1.1, interleaved)


@pytest.mark.parametrize("H,G", [(1, 1), (3, 1), (8, 8), (2, 3)])
def test_rotary_write_heads(l2, H, G):
    c = Case(l2, [9, 1], [[5], [2]], 1, H, G, 128, seed=H)
    make(l2, c, c.ctx)
    pos = torch.arange(c.N, dtype=torch.int32, device=DEV)
    freq, _ = l2.rotary_frequencies(128)
    write(l2, c, pos, freq.to(DEV))
    check_write(l2, c, pos, freq.to(DEV), 1.0, False)


def test_no_rotation_in_place_and_backwards(l2):
    c = Case(l2, [40, 3], [[0], [9]], 1, 2, 2, 128, seed=1)
    make(l2, c, c.ctx)
    pos = torch.randint(0, 1 << 30, (c.N,), dtype=torch.int32, device=DEV)       # angles of very far positions
    write(l2, c, pos, None)
    check_write(l2, c, pos, None, 1.0, False)
    assert torch.equal(c.q_out, c.q)
    freq = l2.rotary_frequencies(128)[0].to(DEV)
    make(l2, c, c.ctx)
    q = c.q.clone()
    c.q_out = c.q                                                              # in place
    write(l2, c, pos, freq)
    want, spread = rotated(q, pos, freq, 1.0, False)
    assert_rotated(c.q, want, spread)
    write(l2, c, pos, -freq)                                                   # and back again
    assert ((c.q.double() - q.double()).abs() <= (2 * 2.0 ** -8 + 1e-5) * 1.01 * spread).all()


def test_queries_may_be_missing_and_so_may_index_and_keys(l2):
    c = Case(l2, [4, 70], [[10], [0]], 1, 2, 4, 64, seed=3)
    make(l2, c, c.ctx)
    pos = torch.arange(c.N, dtype=torch.int32, device=DEV)
    freq = l2.rotary_frequencies(64)[0].to(DEV)
    write(l2, c, pos, freq)
    K, V = c.K.clone(), c.V.clone()
    c.K.copy_(c.K0), c.V.copy_(c.V0)
    l2.rotary_write(None, c.k, c.v, c.tok_off, pos, freq, None, c.K, c.V, None, None, c.start, c.new, c.ws)
    torch.cuda.synchronize()
    assert torch.equal(K.view(torch.uint8), c.K.view(torch.uint8)) and torch.equal(V.view(torch.uint8), c.V.view(torch.uint8))


@pytest.mark.parametrize("packed", [False, True])
def test_rotary_write_with_lengths_per_head(l2, packed):
    ctx = np.random.RandomState(2).randint(0, 50, (2, 2, 3))
    c = Case(l2, [6, 20], ctx, 2, 3, 2, 128, packed=packed, seed=3, per_head=True)
    make(l2, c, c.ctx)
    pos = torch.arange(c.N, dtype=torch.int32, device=DEV)
    freq = l2.rotary_frequencies(128)[0].to(DEV)
    write(l2, c, pos, freq)
    check_write(l2, c, pos, freq, 1.0, False)


@pytest.mark.parametrize("packed", [False, True])
def test_rows_without_room_are_dropped_and_reported(l2, packed):
    c = Case(l2, [6, 4], [[20], [5]], 1, 2, 2, 128, packed=packed, seed=3)
    make(l2, c, c.ctx)
    late = c.ctx.copy()
    late[0] = c.cap(0, 0) - 2                                                  # two of the six rows fit
    late[1] = -3                                                               # taken as 0
    c.start = c.lens(late)
    pos = torch.arange(c.N, dtype=torch.int32, device=DEV)
    freq = l2.rotary_frequencies(128)[0].to(DEV)
    write(l2, c, pos, freq)
    assert l2.read_device_status(c.ws) == -7
    assert c.new.flatten().tolist() == [c.cap(0, 0), 4]
    for h in range(2):
        at = c.cap(0, 0) - 2
        assert torch.equal(c.unit(c.V, 0, 0, h)[at:at + 2], c.v[0, :2, h])
        assert torch.equal(c.unit(c.V, 1, 0, h)[:4], c.v[0, 6:, h])
        assert torch.equal(c.unit(c.V, 1, 0, h)[4:].contiguous().view(torch.uint8), c.unit(c.V0, 1, 0, h)[4:].contiguous().view(torch.uint8))
    want, spread = rotated(c.q, pos, freq, 1.0, False)
    assert_rotated(c.q_out, want, spread)


def test_no_tokens_at_all_still_set_the_lengths(l2):
    c = Case(l2, [0, 0], [[4], [9]], 1, 2, 2, 128, seed=3)
    make(l2, c, c.ctx)
    write(l2, c, torch.zeros(0, dtype=torch.int32, device=DEV), None)
    assert torch.equal(c.new, c.start)


def test_many_sequences(l2):
    r = np.random.RandomState(5)
    c = Case(l2, r.randint(0, 4, 100), r.randint(0, 9, (100, 1)), 1, 2, 2, 64, packed=True, seed=3)
    make(l2, c, c.ctx)
    pos = torch.randint(0, 5000, (c.N,), dtype=torch.int32, device=DEV)
    freq = l2.rotary_frequencies(64)[0].to(DEV)
    write(l2, c, pos, freq)
    check_write(l2, c, pos, freq, 1.0, False)


# ---- commit --------------------------------------------------------------------------------------

def check_commit(l2, c, path, n_path, kept, alias="start", status=0):
    """kept[b][l][h]: entries that are kept."""
    c.idx = torch.randint(0, 1 << 20, c.meta, dtype=torch.int32, device=DEV)
    c.key = torch.rand(c.meta, device=DEV)
    before = [x.clone() for x in (c.K, c.V, c.idx, c.key)]
    ws = torch.zeros(256, dtype=torch.uint8, device=DEV)
    start, cur = c.lens(c.ctx), c.lens(c.cur)
    out = {"start": start, "cur": cur, "none": torch.full_like(start, 99)}[alias]
    l2.tree_commit(c.K, c.V, c.idx, c.key, start, cur, i32(path), i32(n_path), out, ws, rows=c.rows, per_head=c.per_head)
    torch.cuda.synchronize()
    assert l2.read_device_status(ws) == status
    kept = np.broadcast_to(np.asarray(kept).reshape(c.B, *([1, 1] if np.ndim(kept) == 1 else np.shape(kept)[1:])), c.ctx.shape)
    assert torch.equal(out, c.lens(c.ctx + kept))
    for x, old in zip((c.K, c.V, c.idx, c.key), before):
        for b in range(c.B):
            for l in range(c.L):
                for h in range(c.H):
                    want, s = c.unit(old, b, l, h).clone(), int(c.ctx[b, l, h])
                    for j in range(kept[b, l, h]):
                        want[s + j] = c.unit(old, b, l, h)[s + path[b][j]]
                    got = c.unit(x, b, l, h)
                    assert torch.equal(got.contiguous().view(torch.uint8), want.contiguous().view(torch.uint8))


@pytest.mark.parametrize("packed", [False, True])
@pytest.mark.parametrize("dtype,D", [("bf16", 128), ("bf16", 64), ("fp32", 128), ("fp32", 64)])
@pytest.mark.parametrize("alias", ["start", "cur", "none"])
def test_tree_commit(l2, dtype, D, packed, alias):
    c = Case(l2, [8, 1, 60, 3], [[0, 9], [5, 5], [100, 2], [7, 0]], 2, 3, 2, D, dtype, packed=packed, seed=2)
    path = [[0, 3, 4, 7, -1], [0, -1, -1, -1, -1], [1, 2, 30, 58, 59], [9, 9, 9, 9, 9]]
    check_commit(l2, c, path, [4, 1, 5, 0], [4, 1, 5, 0], alias)


def test_tree_commit_of_long_paths(l2):
    """More entries than a pass of the kernel moves, overlapping sources and targets."""
    c = Case(l2, [400, 300], [[11], [0]], 1, 8, 1, 128, seed=2)
    path = [list(range(1, 400)) + [0], list(range(300)) + [0] * 100]
    check_commit(l2, c, path, [399, 300], [399, 300])


def test_paths_that_leave_the_tree_are_cut_and_reported(l2):
    c = Case(l2, [8, 8, 8, 8], [[3], [3], [3], [3]], 1, 2, 2, 128, seed=2)
    path = [[0, 2, 8, 9], [1, 1, 2, 3], [-1, 0, 1, 2], [0, 5, 7, 1 << 30]]
    check_commit(l2, c, path, [4, 4, 4, 99], [2, 1, 0, 3], status=-5)


def test_commit_lengths_per_head(l2):
    ctx = np.random.RandomState(2).randint(0, 50, (2, 2, 3))
    c = Case(l2, [6, 20], ctx, 2, 3, 2, 128, seed=3, per_head=True)
    check_commit(l2, c, [[1, 3, 5], [4, 18, 19]], [3, 2], [3, 2])


def test_commit_without_index_or_keys_and_without_entries(l2):
    c = Case(l2, [6], [[4]], 1, 2, 2, 128, seed=3)
    want = c.K.clone()
    want[0, 0, :, 4:6] = c.K[0, 0, :, [5, 9]]
    ws = torch.zeros(256, dtype=torch.uint8, device=DEV)
    start = c.lens(c.ctx)
    l2.tree_commit(c.K, c.V, None, None, start, c.lens(c.cur), i32([[1, 5]]), i32([2]), start, ws)
    torch.cuda.synchronize()
    assert torch.equal(c.K.view(torch.uint8), want.view(torch.uint8)) and start.item() == 6
    l2.tree_commit(c.K, c.V, None, None, start, c.lens(c.cur), torch.zeros((1, 0), dtype=torch.int32, device=DEV), i32([2]), start, ws)
    torch.cuda.synchronize()
    assert start.item() == 6 and l2.read_device_status(ws) == 0


# ---- together ------------------------------------------------------------------------------------

@pytest.mark.parametrize("D", [64, 128])
def test_prompt_compress_draft_commit(l2, D):
    """Prompts are written, attended to and compressed with the keys of the write; two speculative steps
    follow on the compressed cache: drafts written behind it, tree attention, the accepted path committed;
    a decode step over the result closes the loop."""
    B, L, H, G, n, keep, nodes, cap = 3, 2, 2, 4, [700, 31, 260], [350, 31, 100], [12, 1, 20], 800
    c = Case(l2, n, np.zeros((B, L), int), L, H, G, D, seed=21)
    K, V = (torch.zeros((B, L, H, cap, D), dtype=c.dtype, device=DEV) for _ in range(2))
    idx, key = torch.zeros((B, L, H, cap), dtype=torch.int32, device=DEV), torch.zeros((B, L, H, cap), device=DEV)
    ws = torch.zeros(max(256, l2.workspace_bytes(l2.Layout(K, q_heads=H * G), cap)), dtype=torch.uint8, device=DEV)
    zero, cur = torch.zeros((B, L), dtype=torch.int32, device=DEV), torch.zeros((B, L), dtype=torch.int32, device=DEV)
    freq, scale = l2.rotary_frequencies(D, 10000.0, l2.ROTARY_YARN, factor=4.0, high=32.0, original_len=4096)
    pos = torch.cat([torch.arange(m) for m in n]).to(DEV, torch.int32)
    q = torch.empty_like(c.q)
    l2.rotary_write(c.q, c.k, c.v, c.tok_off, pos, freq.to(DEV), q, K, V, idx, key, zero, cur, ws, attn_scale=scale)
    c.q, c.K, c.V, c.max_len = q, K, V, cap
    out, lse = c.empty_out(), torch.empty((L, c.N, c.Hq), device=DEV)
    l2.prompt_attention(q, c.tok_off, K, V, cur, cap, out, lse_out=lse, workspace=torch.zeros(
        l2.prompt_attention_workspace_bytes(K, q, cap), dtype=torch.uint8, device=DEV))
    torch.cuda.synchronize()
    assert check_attention(c, out, lse, causal(c)) > 0
    # compression with the keys of the write is compression with the keys it forms itself
    got = []
    for given in (key, None):
        Kc, Vc, ic, kc = torch.zeros_like(K), torch.zeros_like(V), torch.zeros_like(idx), torch.zeros_like(key)
        kept = torch.zeros((B, L), dtype=torch.int32, device=DEV)
        l2.select_compact(K, V, i32(n), i32(keep), cap, (0,), Kc, Vc, ic, kc, kept, ws, sumsq_in=given)
        got.append((Kc, Vc, ic, kc, kept))
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(*got))
    Kc, Vc, ic, kc, start = got[0]
    for step in range(2):
        ctx = start.cpu().numpy()
        d = Case(l2, nodes, ctx, L, H, G, D, seed=30 + step)
        parents = [[(j - 1) // 2 for j in range(m)] for m in nodes]           # binary trees
        trees, depth = [], []
        for p in parents:
            a, dep = torch.eye(len(p), dtype=torch.bool), [0] * len(p)
            for j in range(1, len(p)):
                a[j] |= a[p[j]]
                dep[j] = dep[p[j]] + 1
            trees.append(a)
            depth.append(torch.tensor(dep))
        pos = torch.cat([m + 3 * step + x for m, x in zip(n, depth)]).to(DEV, torch.int32)
        q = torch.empty_like(d.q)
        l2.rotary_write(d.q, d.k, d.v, d.tok_off, pos, freq.to(DEV), q, Kc, Vc, ic, kc, start, cur, ws, attn_scale=scale)
        d.q, d.K, d.V, d.max_len = q, Kc, Vc, cap
        out, lse = d.empty_out(), torch.empty((L, d.N, d.Hq), device=DEV)
        l2.tree_attention(q, d.tok_off, mask_words(d, trees), Kc, Vc, cur, cap, out, lse_out=lse)
        torch.cuda.synchronize()
        check_attention(d, out, lse, trees)
        path = [[0, 2, 5], [0, -1, -1], [0, 1, 4]]
        rows = [[[Kc[b, l, :, ctx[b, l] + j].clone() for j in path[b] if j >= 0] for l in range(L)] for b in range(B)]
        l2.tree_commit(Kc, Vc, ic, kc, start, cur, i32(path), i32([3, 1, 3]), start, ws)
        torch.cuda.synchronize()
        assert np.array_equal(start.cpu().numpy(), ctx + np.array([[3], [1], [3]]))
        for b in range(B):
            for l in range(L):
                for j, row in enumerate(rows[b][l]):
                    assert torch.equal(Kc[b, l, :, ctx[b, l] + j], row)
    fresh = torch.zeros_like(kc)
    l2.key_norms(Kc, start.amax(1).to(torch.int32).contiguous(), cap, fresh)
    for b in range(B):
        for l in range(L):
            m = int(start[b, l])
            assert torch.equal(fresh[b, l, :, :m], kc[b, l, :, :m])            # every key still fits its row
    one = torch.randn((B, L, H * G, D), device=DEV).to(c.dtype)
    dec = torch.empty((B, L, H * G, D), device=DEV)
    l2.decode_attention(one, Kc, Vc, start, cap, dec, ws)
    e = Case(l2, [1] * B, start.cpu().numpy() - 1, L, H, G, D, seed=1)
    e.q, e.K, e.V, e.max_len = one.transpose(0, 1).contiguous(), Kc, Vc, cap
    out = e.empty_out()
    l2.prompt_attention(e.q, e.tok_off, Kc, Vc, start, cap, out)
    torch.cuda.synchronize()
    check_attention(e, out, None, causal(e))
    assert ((out.transpose(0, 1).float() - dec).abs() <= 2e-2 * dec.abs() + 2e-2).all()
    assert l2.read_device_status(ws) == 0
