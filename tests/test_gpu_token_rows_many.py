"""rotary_write with as many tokens as make it give each a warp of its own (from 1184 tokens times layers on), and just
fewer: every type, pairing and layout, calls in place, rows without room, lengths per head, and the rows that a
prompt's attention and compression start from."""
import numpy as np
import pytest
import torch

from test_gpu_token_rows import assert_rotated, check_write, make, rotated, write
from token_util import DEV, Case

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def l2():
    import paper_2406_11430_b200 as lib
    lib.lib()
    return lib


def _case(l2, tokens, L=1, H=2, G=4, D=128, dtype="bf16", packed=False, seed=0, pad=0, per_head=False, strided=True):
    """Ragged sequences, one of them empty, one of a single token; `tokens` counts the padding too."""
    n = [tokens - pad - 412, 0, 1, 37, 374]
    ctx = np.random.RandomState(seed).randint(0, 60, (5, L, H) if per_head else (5, L))
    return Case(l2, n, ctx, L, H, G, D, dtype, packed=packed, seed=seed, pad=pad, per_head=per_head, strided=strided)


def _positions(c, far=131072):
    return torch.randint(0, far, (c.N,), dtype=torch.int32, device=DEV, generator=torch.Generator(DEV).manual_seed(c.N))


@pytest.mark.parametrize("tokens,L,pad", [(1183, 1, 0), (1184, 1, 3), (593, 2, 1), (2501, 1, 5)])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("dtype,D,rot", [("bf16", 128, 128), ("bf16", 128, 96), ("bf16", 64, 64), ("bf16", 64, 16),
                                         ("fp32", 128, 128), ("fp32", 128, 48), ("fp32", 64, 64), ("fp32", 64, 32)])
def test_types_pairings_and_partial_rotation(l2, dtype, D, rot, interleaved, tokens, L, pad):
    c = _case(l2, tokens, L, D=D, dtype=dtype, packed=(rot + tokens) % 3 == 0, seed=rot, pad=pad)
    make(l2, c, c.ctx)
    pos, freq = _positions(c), l2.rotary_frequencies(rot, 500000.0, l2.ROTARY_LLAMA3, factor=8.0)[0].to(DEV)
    write(l2, c, pos, freq, interleaved=interleaved, attn_scale=1.1)
    check_write(l2, c, pos, freq, 1.1, interleaved)


@pytest.mark.parametrize("packed", [False, True])
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("H,G", [(1, 1), (3, 1), (8, 8), (2, 3), (9, 1)])
def test_head_counts(l2, H, G, dtype, packed):
    """Fewer and more rows of a kind than a warp has in flight, and numbers that leave a remainder."""
    c = _case(l2, 1301, H=H, G=G, dtype=dtype, packed=packed, seed=H)
    make(l2, c, c.ctx)
    pos, freq = _positions(c), l2.rotary_frequencies(128)[0].to(DEV)
    write(l2, c, pos, freq)
    check_write(l2, c, pos, freq, 1.0, False)


@pytest.mark.parametrize("packed", [False, True])
@pytest.mark.parametrize("interleaved", [False, True])
def test_lengths_per_head(l2, packed, interleaved):
    c = _case(l2, 701, 2, H=3, G=2, packed=packed, seed=3, per_head=True)
    make(l2, c, c.ctx)
    pos, freq = _positions(c), l2.rotary_frequencies(128)[0].to(DEV)
    write(l2, c, pos, freq, interleaved=interleaved)
    check_write(l2, c, pos, freq, 1.0, interleaved)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("interleaved", [False, True])
def test_in_place_and_without_rotation(l2, dtype, interleaved):
    c = _case(l2, 1250, dtype=dtype, seed=4, strided=False)
    make(l2, c, c.ctx)
    pos = _positions(c, 1 << 30)
    write(l2, c, pos, None)
    check_write(l2, c, pos, None, 1.0, False)
    assert torch.equal(c.q_out, c.q)
    make(l2, c, c.ctx)
    freq, q = l2.rotary_frequencies(128)[0].to(DEV), c.q.clone()
    c.q_out = c.q
    write(l2, c, pos, freq, interleaved=interleaved)
    want, spread = rotated(q, pos, freq, 1.0, interleaved)
    assert_rotated(c.q, want, spread)
    k = c.k.clone()
    want, spread = rotated(k, pos, freq, 1.0, interleaved)
    for b in range(c.B):
        of, s, e = slice(int(c.off[b]), int(c.off[b + 1])), int(c.ctx[b, 0, 0]), int(c.cur[b, 0, 0])
        for h in range(c.H):
            assert_rotated(c.unit(c.K, b, 0, h)[s:e], want[0, of, h], spread[0, of, h])


@pytest.mark.parametrize("packed", [False, True])
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_rows_without_room_are_dropped_and_reported(l2, dtype, packed):
    c = _case(l2, 1400, dtype=dtype, packed=packed, seed=5)
    make(l2, c, c.ctx)
    late = c.ctx.copy()
    fit = 200
    late[0] = c.cap(0, 0) - fit                              # the first sequence's later rows do not fit
    c.start = c.lens(late)
    pos, freq = _positions(c), l2.rotary_frequencies(128)[0].to(DEV)
    write(l2, c, pos, freq)
    assert l2.read_device_status(c.ws) == -7
    assert c.new.flatten().tolist() == [c.cap(0, 0)] + [int(c.cur[b, 0, 0]) for b in range(1, 5)]
    want, spread = rotated(c.k, pos, freq, 1.0, False)
    for b in range(c.B):
        m = fit if b == 0 else c.n[b]
        s, first = int(late[b, 0, 0]), int(c.off[b])
        for h in range(c.H):
            K, V, idx, K0, V0 = (c.unit(x, b, 0, h) for x in (c.K, c.V, c.idx, c.K0, c.V0))
            assert_rotated(K[s:s + m], want[0, first:first + m, h], spread[0, first:first + m, h])
            assert torch.equal(V[s:s + m], c.v[0, first:first + m, h]) and torch.equal(idx[s:s + m], pos[first:first + m])
            outside = torch.ones(K.shape[0], dtype=torch.bool, device=DEV)
            outside[s:s + m] = False
            for x, y in ((K, K0), (V, V0)):
                assert torch.equal(x[outside].contiguous().view(torch.uint8), y[outside].contiguous().view(torch.uint8))
            assert (idx[outside] == -1).all()
    want, spread = rotated(c.q, pos, freq, 1.0, False)       # every query is rotated all the same
    assert_rotated(c.q_out, want, spread)


def test_the_rows_are_those_of_the_calls_with_fewer_tokens(l2):
    """Token by token the same bits, whichever way a call takes: the long call's against calls of one sequence's pieces."""
    c = _case(l2, 1600, H=2, G=4, seed=6)
    make(l2, c, c.ctx)
    pos, freq = _positions(c), l2.rotary_frequencies(128)[0].to(DEV)
    write(l2, c, pos, freq)
    K, V, key, q = c.K.clone(), c.V.clone(), c.key.clone(), c.q_out.clone()
    c.K.copy_(c.K0), c.V.copy_(c.V0), c.key.fill_(-1), c.q_out.fill_(7)
    used = c.N
    for at in range(0, used, 400):                           # 400 tokens a call: a block each
        to = min(at + 400, used)
        off = c.tok_off.clamp(at, to) - at
        start = c.start + (c.tok_off[:-1].clamp(max=at).neg() + at).clamp(min=0).view(-1, 1).minimum(
            (c.tok_off[1:] - c.tok_off[:-1]).view(-1, 1))
        l2.rotary_write(c.q[:, at:to], c.k[:, at:to], c.v[:, at:to], off.contiguous(), pos[at:to], freq, c.q_out[:, at:to], c.K, c.V,
                        c.idx, c.key, start.to(torch.int32).contiguous(), c.new, c.ws)
    torch.cuda.synchronize()
    assert l2.read_device_status(c.ws) == 0
    for x, y in ((K, c.K), (V, c.V), (key, c.key), (q, c.q_out)):
        assert torch.equal(x.contiguous().view(torch.uint8), y.contiguous().view(torch.uint8))


def test_prompts_end_up_rotated_in_the_cache(l2):
    """The first step of a prefill by its own definition: queries, keys and values of two layers of three prompts."""
    n, L, H, G, D = [700, 31, 260], 2, 2, 4, 128
    c = Case(l2, n, np.zeros((3, L), int), L, H, G, D, seed=21)
    make(l2, c, c.ctx)
    freq, scale = l2.rotary_frequencies(D, 10000.0, l2.ROTARY_YARN, factor=4.0, high=32.0, original_len=4096)
    pos = torch.cat([torch.arange(m) for m in n]).to(DEV, torch.int32)
    write(l2, c, pos, freq.to(DEV), attn_scale=scale)
    check_write(l2, c, pos, freq.to(DEV), scale, False)
