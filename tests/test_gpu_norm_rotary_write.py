"""Norms of queries and keys with the rotary write, into dense and packed caches and into pages, against the formula in
64 bits: every other row is left as it was, bit for bit."""
import numpy as np
import pytest
import torch

from page_util import Paged
from token_util import DEV, Case, i32

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def l2():
    import paper_2406_11430_b200 as lib
    lib.lib()
    return lib


def normed(x, pos, freq, scale, interleaved, norm, weight, offset, eps):
    """x [L, N, heads, D] in 64 bits, and the size of the pair that each element comes from."""
    y = x.double().clone()
    if norm:
        y = y / (y.square().mean(-1, keepdim=True) + eps).sqrt()
        if weight is not None:
            y = y * (weight.double() + offset)
    r = freq.numel()
    turn = torch.polar(torch.full((pos.numel(), r), scale, dtype=torch.float64, device=DEV), pos.double()[:, None] * freq)[:, None]
    a, b = (slice(0, 2 * r, 2), slice(1, 2 * r, 2)) if interleaved else (slice(0, r), slice(r, 2 * r))
    size = y.abs()
    size[..., a] = size[..., b] = torch.complex(y[..., a], y[..., b]).abs() * abs(scale)
    z = torch.complex(y[..., a], y[..., b]) * turn
    y[..., a], y[..., b] = z.real, z.imag
    return y, size


def assert_near(got, want, size, norm):
    """Roundings of 2^-24 of the pair's size: cosine or sine, its weight and offset, two products and a sum: 6.  With a norm, besides, the
    factor's: D / 2 of the sum of squares (half of it behind the root), mean, eps, root, reciprocal and product: D / 2 + 5.
    One rounding to the stored type, 2^-8 of the value for bf16."""
    half = 2.0 ** -8 if got.dtype == torch.bfloat16 else 2.0 ** -24
    steps = 6 + (got.shape[-1] / 2 + 5 if norm else 0)
    assert torch.isfinite(got).all()
    assert ((got.double() - want).abs() <= steps * 2.0 ** -24 * 1.5 * size + half * 1.01 * want.abs() + 1e-30).all()


def bits(x):
    return x.contiguous().view(torch.uint8)


def run(l2, c, rot, interleaved=False, norm_q=True, norm_k=True, weights=True, offset=0.0, eps=1e-6, scale=1.0, no_meta=False, start=None,
        room=None):
    paged = isinstance(c, Paged)
    g = torch.Generator().manual_seed(rot)
    qw, kw = ((torch.randn(c.D, generator=g) * 0.4 + 1).to(DEV, c.dtype) if weights else None for _ in range(2))
    pos = torch.randint(0, 131072, (c.N,), generator=g, dtype=torch.int32).to(DEV)
    freq = l2.rotary_frequencies(rot, 500000.0)[0].to(DEV) if rot else None
    K0, V0 = c.K.clone(), c.V.clone()
    idx, key = torch.full(c.meta, -1, dtype=torch.int32, device=DEV), torch.full(c.meta, -1.0, device=DEV)
    start = c.lens(c.ctx) if start is None else start
    new, ws, q_out = torch.full_like(start, 99), torch.zeros(256, dtype=torch.uint8, device=DEV), c.empty_out()
    pages = l2.Pages(c.pages.table, c.P, c.n_pages, room) if paged else None
    l2.norm_rotary_write(c.q, c.k, c.v, c.tok_off, pos, freq, q_out, c.K, c.V, None if no_meta else idx, None if no_meta else key, start,
                         new, ws, q_weight=qw, k_weight=kw, norm_q=norm_q, norm_k=norm_k, eps=eps, weight_offset=offset,
                         interleaved=interleaved, attn_scale=scale, rows=c.rows, per_head=c.per_head, pages=pages)
    torch.cuda.synchronize()
    f = torch.zeros(0, dtype=torch.float64, device=DEV) if freq is None else freq
    want_q = normed(c.q, pos, f, scale, interleaved, norm_q, qw, offset, eps)
    want_k = normed(c.k, pos, f, scale, interleaved, norm_k, kw, offset, eps)
    return dict(pos=pos, K0=K0, V0=V0, idx=idx, key=key, new=new, ws=ws, q_out=q_out, q=want_q, k=want_k, norm_q=norm_q, norm_k=norm_k,
                no_meta=no_meta)


def stored_keys(l2, c):
    """The ordering keys of all rows as they are stored, by the library's own norm pass."""
    key, R = torch.full(c.meta, -1.0, device=DEV), c.meta[-1]
    if isinstance(c, Paged):
        l2.key_norms(c.K, i32([R]), R, key, rows=l2.Rows([[0]], [[R]], R, DEV))
    else:
        full = i32([c.max_len if c.rows is None else int(c.cur[b].max()) + 3 for b in range(c.B)])
        l2.key_norms(c.K, full, c.max_len, key, rows=c.rows)
    return key


def check(l2, c, w):
    used = int(c.off[-1])
    assert_near(w["q_out"][:, :used], w["q"][0][:, :used], w["q"][1][:, :used], w["norm_q"])
    assert (w["q_out"][:, used:] == 7).all()
    paged, keys = isinstance(c, Paged), stored_keys(l2, c)
    touched = torch.zeros(c.meta, dtype=torch.bool, device=DEV)
    for b in range(c.B):
        of = slice(int(c.off[b]), int(c.off[b + 1]))
        for l in range(c.L):
            for h in range(c.H):
                s, e = int(c.ctx[b, l, h]), int(c.cur[b, l, h])
                at = (h, c.at(b, l, e)[s:]) if paged else (b, l, h, slice(s, e)) if c.rows is None else \
                    (h, slice(int(c.row0[b, l]) + s, int(c.row0[b, l]) + e))
                K, V = c.K[at], c.V[at]
                assert_near(K, w["k"][0][l, of, h], w["k"][1][l, of, h], w["norm_k"])
                assert torch.equal(V, c.v[l, of, h])
                touched[at] = True
                if not w["no_meta"]:
                    assert torch.equal(w["idx"][at], w["pos"][of])
                    assert torch.equal(w["key"][at], keys[at])
    for x, y in ((c.K, w["K0"]), (c.V, w["V0"])):
        assert torch.equal(bits(x[~touched]), bits(y[~touched]))
    outside = ~touched if not w["no_meta"] else torch.ones_like(touched)
    assert (w["idx"][outside] == -1).all() and (w["key"][outside] == -1).all()
    assert torch.equal(w["new"], c.lens(c.cur))
    assert l2.read_device_status(w["ws"]) == 0


FORMS = ["dense", "packed", 16, 128]


def make(l2, form, n, ctx, L, H, G, D, dtype, **kw):
    if isinstance(form, int):
        return Paged(l2, n, ctx, L, H, G, D, form, dtype, **kw)
    return Case(l2, n, ctx, L, H, G, D, dtype, packed=form == "packed", **kw)


@pytest.mark.parametrize("form", FORMS)
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("dtype,D,rot", [("bf16", 128, 128), ("bf16", 128, 16), ("bf16", 128, 0), ("bf16", 64, 64), ("bf16", 64, 48),
                                         ("fp32", 128, 128), ("fp32", 128, 48), ("fp32", 64, 32)])
def test_norm_and_rotation(l2, dtype, D, rot, interleaved, form):
    c = make(l2, form, [1, 37, 0, 5], [[0, 3], [100, 0], [7, 7], [64, 1]], 2, 2, 4, D, dtype, seed=rot, pad=3, strided=True)
    check(l2, c, run(l2, c, rot, interleaved, scale=1.1, offset=0.5))


@pytest.mark.parametrize("norm_q,norm_k,weights,offset", [(True, False, True, 0.0), (False, True, True, 1.0), (False, False, False, 0.0),
                                                          (True, True, False, 1.0)])
def test_what_is_normed(l2, norm_q, norm_k, weights, offset):
    """Queries only, keys only, neither; without weights the factor is one, whatever is added to them."""
    c = make(l2, 32, [9, 1, 300], [[5], [2], [31]], 1, 3, 2, 128, "bf16", seed=3)
    check(l2, c, run(l2, c, 128, norm_q=norm_q, norm_k=norm_k, weights=weights, offset=offset))


def test_without_norms_it_is_the_rotary_write(l2):
    """The same bits as l2kv_rotary_write."""
    c = make(l2, "dense", [9, 1, 30], [[5], [2], [31]], 1, 3, 2, 128, "bf16", seed=3)
    w = run(l2, c, 128, norm_q=False, norm_k=False, no_meta=True)
    K, V, q = w["K0"].clone(), w["V0"].clone(), c.empty_out()
    l2.rotary_write(c.q, c.k, c.v, c.tok_off, w["pos"], l2.rotary_frequencies(128, 500000.0)[0].to(DEV), q, K, V, None, None, c.lens(c.ctx),
                    w["new"].clone(), w["ws"])
    torch.cuda.synchronize()
    assert torch.equal(q, w["q_out"]) and torch.equal(bits(K), bits(c.K)) and torch.equal(bits(V), bits(c.V))


@pytest.mark.parametrize("form", [16, "packed"])
@pytest.mark.parametrize("H,G", [(1, 1), (3, 1), (8, 8), (2, 4)])
def test_head_counts(l2, H, G, form):
    c = make(l2, form, [9, 1], [[5], [2]], 1, H, G, 128, "bf16", seed=H)
    check(l2, c, run(l2, c, 128, no_meta=True))


@pytest.mark.parametrize("dtype,D", [("bf16", 128), ("bf16", 64), ("fp32", 128)])
@pytest.mark.parametrize("form", [16, 64, "dense"])
def test_many_tokens(l2, form, dtype, D):
    """Enough tokens for a warp per token, and lengths per head."""
    r = np.random.RandomState(1)
    c = make(l2, form, [int(x) for x in r.randint(0, 300, 9)] + [1], r.randint(0, 60, (10, 1, 2)), 1, 2, 4, D, dtype, seed=4, per_head=True)
    check(l2, c, run(l2, c, D))


@pytest.mark.parametrize("size", [1e-18, 1e-3, 1e15])
def test_small_and_large_rows(l2, size):
    """eps decides where rows are tiny; squares of 1e15 fit fp32."""
    c = make(l2, 16, [40], [[3]], 1, 2, 4, 128, "fp32", seed=5)
    c.q, c.k = c.q * size, c.k * size
    check(l2, c, run(l2, c, 64, no_meta=True))


def test_rows_of_zeros(l2):
    c = make(l2, 16, [40], [[3]], 1, 2, 4, 128, "bf16", seed=5)
    c.q, c.k = c.q * 0, c.k * 0
    check(l2, c, run(l2, c, 128))


def test_room_and_pages_that_are_none(l2):
    """Rows at or beyond the room, or in a page that the pool does not have, are not written; their queries are."""
    c = make(l2, 16, [10, 4, 3], [[12], [30], [0]], 1, 2, 4, 128, "bf16", seed=6)
    K0 = c.K.clone()
    w = run(l2, c, 128, room=i32([[20], [1], [16]]))
    assert l2.read_device_status(w["ws"]) == -7 and w["new"].flatten().tolist() == [20, 1, 3]
    assert_near(w["q_out"], *w["q"], True)
    written = {0: range(12, 20), 1: range(0), 2: range(3)}
    same = torch.ones(c.n_pages * 16, dtype=torch.bool, device=DEV)
    for b, rows in written.items():
        if len(rows):
            at = c.at(b, 0, rows[-1] + 1)[rows[0]:]
            same[at] = False
            first = int(c.off[b]) + rows[0] - int(c.ctx[b, 0, 0])
            for h in range(2):
                assert_near(c.K[h, at], *(x[0, first:first + len(rows), h] for x in w["k"]), True)
    assert torch.equal(bits(c.K[:, same]), bits(K0[:, same]))
    for page in (-1, c.n_pages, 2 ** 31 - 1, -2 ** 31):
        c.K.copy_(K0)
        t = c.pages.table.clone()
        t[0, 0, 1] = page                                    # rows 16 to 21 of the first sequence
        was, c.pages = c.pages, l2.Pages(t, 16, c.n_pages)
        w = run(l2, c, 128)
        c.pages = was
        assert l2.read_device_status(w["ws"]) == -5
        same = torch.ones(c.n_pages * 16, dtype=torch.bool, device=DEV)
        for b, (s, e) in enumerate(((12, 16), (30, 34), (0, 3))):
            same[c.at(b, 0, e)[s:]] = False
        assert torch.equal(bits(c.K[:, same]), bits(K0[:, same]))
        assert (~torch.isnan(c.K[:, ~same])).all()


def test_captured(l2):
    c = make(l2, 16, [1, 1, 1], [[5], [16], [31]], 1, 2, 4, 128, "bf16", seed=8)
    w = run(l2, c, 128, weights=False)
    want, q = c.K.clone(), w["q_out"].clone()
    freq, start, new, ws = l2.rotary_frequencies(128, 500000.0)[0].to(DEV), c.lens(c.ctx), torch.zeros_like(w["new"]), w["ws"]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        l2.norm_rotary_write(c.q, c.k, c.v, c.tok_off, w["pos"], freq, w["q_out"], c.K, c.V, None, None, start, new, ws, pages=c.pages)
    for _ in range(2):
        c.K.copy_(w["K0"]), w["q_out"].zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(bits(c.K), bits(want)) and torch.equal(w["q_out"], q) and torch.equal(new, c.lens(c.cur))
