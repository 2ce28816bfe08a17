"""Host side of the calls on packed new tokens: refusals before anything is launched, workspace sizes,
and the rotary frequencies against their formulas.  No GPU needed."""
import ctypes
import math

import numpy as np
import pytest
import torch

import paper_2406_11430_b200 as l2

B, L, H, HQ, T, D, N = 2, 3, 2, 8, 40, 128, 7


def _inputs(dtype=torch.bfloat16, D=D):
    i32 = lambda *s: torch.zeros(s, dtype=torch.int32)  # noqa: E731
    tok = lambda heads: torch.zeros((L, N, heads, D), dtype=dtype)  # noqa: E731
    return dict(K=torch.zeros((B, L, H, T, D), dtype=dtype), V=torch.zeros((B, L, H, T, D), dtype=dtype), q=tok(HQ),
                k=tok(H), v=tok(H), out=tok(HQ), off=i32(B + 1), pos=i32(N), start=i32(B, L), cur=i32(B, L),
                idx=i32(B, L, H, T), key=torch.zeros((B, L, H, T)), ws=torch.zeros(256, dtype=torch.uint8),
                freq=torch.zeros(D // 2, dtype=torch.float64), path=i32(B, 4), n_path=i32(B),
                mask=torch.zeros((N, 1), dtype=torch.int64), scale=0.0, max_len=T, attn_scale=1.0)


def _rotary(a):
    l2.rotary_write(a["q"], a["k"], a["v"], a["off"], a["pos"], a["freq"], a["out"], a["K"], a["V"], a["idx"], a["key"],
                    a["start"], a["cur"], a["ws"], attn_scale=a["attn_scale"])


def _prompt(a):
    l2.prompt_attention(a["q"], a["off"], a["K"], a["V"], a["cur"], a["max_len"], a["out"], scale=a["scale"],
                        workspace=a["ws"])


def _tree(a):
    l2.tree_attention(a["q"], a["off"], a["mask"], a["K"], a["V"], a["cur"], a["max_len"], a["out"], scale=a["scale"],
                      workspace=a["ws"])


def _commit(a):
    l2.tree_commit(a["K"], a["V"], a["idx"], a["key"], a["start"], a["cur"], a["path"], a["n_path"], a["start"], a["ws"])


def _offset(t):
    """The same tensor 8 bytes behind a 16-byte boundary."""
    room = torch.zeros(t.numel() + 16, dtype=t.dtype)
    at = 8 // t.element_size()
    return room[at:at + t.numel()].view(t.shape)


REFUSED = [
    (_rotary, dict(freq=torch.zeros(12, dtype=torch.float64)), -2),        # 24 dimensions: not a multiple of 16
    (_rotary, dict(freq=torch.zeros(72, dtype=torch.float64)), -2),        # more than the head has
    (_rotary, dict(attn_scale=float("nan")), -1),
    (_rotary, dict(attn_scale=float("inf")), -1),
    (_rotary, dict(cur="start"), -1),                                      # lengths in and out are one array
    (_rotary, dict(ws=torch.zeros(255, dtype=torch.uint8)), -4),
    (_rotary, dict(V=None), -1), (_rotary, dict(pos=None), -1), (_rotary, dict(q=_offset), -3),
    (_rotary, dict(k=_offset), -3), (_rotary, dict(out=_offset), -3), (_rotary, dict(K=_offset), -3),
    (_prompt, dict(max_len=T + 1), -5), (_prompt, dict(max_len=-1), -1), (_prompt, dict(scale=float("nan")), -1),
    (_prompt, dict(ws=torch.zeros(100, dtype=torch.uint8)), -4), (_prompt, dict(out=_offset), -3),
    (_prompt, dict(V=_offset), -3), (_prompt, dict(V=None), -1), (_tree, dict(max_len=T + 1), -5),
    (_tree, dict(q=_offset), -3), (_tree, dict(ws=torch.zeros(100, dtype=torch.uint8)), -4),
    (_tree, dict(mask=torch.zeros((N, 0), dtype=torch.int64)), -1),
    (_commit, dict(ws=torch.zeros(255, dtype=torch.uint8)), -4), (_commit, dict(V=None), -1),
    (_commit, dict(K=_offset), -3),
]


@pytest.mark.parametrize("call,change,status", REFUSED)
def test_refused_with_a_status(call, change, status):
    a = _inputs()
    for key, value in change.items():
        a[key] = value(a[key]) if callable(value) else a[value] if isinstance(value, str) else value
    with pytest.raises(l2.L2KVError) as e:
        call(a)
    assert e.value.status == status


@pytest.mark.parametrize("call", [_prompt, _tree])
def test_query_groups_of_three_are_refused(call):
    a = _inputs()
    a["q"] = a["out"] = torch.zeros((L, N, 6, D), dtype=torch.bfloat16)
    with pytest.raises(l2.L2KVError) as e:
        call(a)
    assert e.value.status == -2


WRONG_SHAPES = [
    (_rotary, "q", torch.float32), (_rotary, "k", torch.float32), (_prompt, "q", torch.float16),
    (_rotary, "off", (B,)), (_rotary, "pos", (N + 1,)), (_rotary, "start", (B,)), (_rotary, "cur", (B, L, H)),
    (_rotary, "k", (L, N, H + 1, D)), (_rotary, "v", (L, N + 1, H, D)), (_rotary, "out", (L, N, HQ + 1, D)),
    (_rotary, "freq", torch.float32), (_prompt, "off", (B + 2,)), (_prompt, "cur", (B, L, H)), (_prompt, "out", (L, N, HQ, 64)),
    (_prompt, "q", (L + 1, N, HQ, D)), (_tree, "mask", (N + 1, 1)), (_tree, "mask", torch.int32), (_commit, "path", (B + 1, 4)),
    (_commit, "n_path", (B + 1,)), (_commit, "start", (B,)), (_commit, "path", torch.int64),
]


@pytest.mark.parametrize("call,name,to", WRONG_SHAPES)
def test_tensors_that_do_not_fit_are_refused(call, name, to):
    a = _inputs()
    a[name] = a[name].to(to) if isinstance(to, torch.dtype) else torch.zeros(to, dtype=a[name].dtype)
    with pytest.raises(ValueError):
        call(a)


def test_tensors_on_two_devices_are_refused():
    for call, name in ((_rotary, "pos"), (_prompt, "off"), (_tree, "mask"), (_commit, "path")):
        a = _inputs()
        a[name] = a[name].to("meta")
        with pytest.raises(ValueError):
            call(a)


def test_nothing_to_do_is_not_an_error():
    a = _inputs()
    for name in ("q", "out"):
        a[name] = torch.zeros((L, 0, HQ, D), dtype=torch.bfloat16)
    a["mask"] = torch.zeros((0, 1), dtype=torch.int64)
    _prompt(a)
    _tree(a)
    a = _inputs()
    a.update(K=torch.zeros((0, L, H, T, D), dtype=torch.bfloat16), V=torch.zeros((0, L, H, T, D), dtype=torch.bfloat16),
             off=torch.zeros(1, dtype=torch.int32), start=torch.zeros((0, L), dtype=torch.int32),
             cur=torch.zeros((0, L), dtype=torch.int32), path=torch.zeros((0, 4), dtype=torch.int32),
             n_path=torch.zeros(0, dtype=torch.int32))
    _rotary(a)
    _prompt(a)
    _commit(a)


def test_unknown_flags_are_refused():
    a = _inputs()
    lay = l2.Layout(a["K"], q_heads=HQ)
    p = lambda t: ctypes.c_void_p(t.data_ptr())  # noqa: E731
    assert l2.lib().l2kv_tree_commit(p(a["K"]), p(a["V"]), None, None, lay.ref(), p(a["start"]), p(a["cur"]), p(a["path"]),
                                     4, p(a["n_path"]), p(a["start"]), 2, p(a["ws"]), 256, None) == -1
    assert l2.lib().l2kv_tree_commit(p(a["K"]), p(a["V"]), None, None, lay.ref(), p(a["start"]), p(a["cur"]), p(a["path"]),
                                     -1, p(a["n_path"]), p(a["start"]), 0, p(a["ws"]), 256, None) == -1


def test_workspace_size_is_at_least_the_status_block_and_bounded():
    for n, max_len, dt in ((1, T, torch.bfloat16), (N, 0, torch.bfloat16), (N, T, torch.float32)):
        K = torch.zeros((B, L, H, T, D), dtype=dt, device="meta")
        q = torch.zeros((L, n, HQ, D), dtype=dt, device="meta")
        assert l2.prompt_attention_workspace_bytes(K, q, max_len) >= 256
    big = torch.zeros((4, 1, 8, 131072, D), dtype=torch.bfloat16, device="meta")
    q = torch.zeros((1, 256, 32, D), dtype=torch.bfloat16, device="meta")
    assert l2.prompt_attention_workspace_bytes(big, q, 131072) < 128 << 20
    with pytest.raises(l2.L2KVError) as e:
        l2.prompt_attention_workspace_bytes(big, q, 131073)
    assert e.value.status == -5


def _plain(rot, base):
    return base ** (-2.0 * np.arange(rot // 2) / rot)


def test_frequencies_without_scaling_linear_and_ntk():
    f, s = l2.rotary_frequencies(128, 500000.0)
    np.testing.assert_allclose(f.numpy(), _plain(128, 500000.0), rtol=1e-14)
    assert s == 1.0
    f, _ = l2.rotary_frequencies(64, 10000.0, l2.ROTARY_LINEAR, factor=8.0)
    np.testing.assert_allclose(f.numpy(), _plain(64, 10000.0) / 8.0, rtol=1e-14)
    f, _ = l2.rotary_frequencies(64, 10000.0, l2.ROTARY_NTK, factor=4.0)
    np.testing.assert_allclose(f.numpy(), _plain(64, 10000.0 * 4.0 ** (64 / 62)), rtol=1e-13)
    # what the changed base is chosen for: the fastest pair stays, the slowest is `factor` times slower
    assert f[0] == 1.0 and abs(f[-1] * 4.0 / _plain(64, 10000.0)[-1] - 1) < 1e-12


def test_frequencies_that_mix_two_scales():
    f, s = l2.rotary_frequencies(128, 500000.0, l2.ROTARY_LLAMA3, factor=8.0, low=1.0, high=4.0, original_len=8192)
    plain, wave = _plain(128, 500000.0), 2 * math.pi / _plain(128, 500000.0)
    want = np.where(wave < 8192 / 4, plain, np.where(wave > 8192, plain / 8, np.nan))
    known = ~np.isnan(want)
    np.testing.assert_allclose(f.numpy()[known], want[known], rtol=1e-13)
    assert known.sum() < 64 and np.all(np.diff(f.numpy()) < 0)
    ramp = (8192 / wave[~known] - 1) / 3
    np.testing.assert_allclose(f.numpy()[~known], (1 - ramp) * plain[~known] / 8 + ramp * plain[~known], rtol=1e-12)
    assert s == 1.0
    f, s = l2.rotary_frequencies(64, 10000.0, l2.ROTARY_YARN, factor=16.0, low=1.0, high=32.0, original_len=4096)
    plain = _plain(64, 10000.0)
    turns = 4096 * plain / (2 * math.pi)                     # over the original length
    assert abs(s - (0.1 * math.log(16.0) + 1)) < 1e-15
    fast, slow = turns > 40, turns < 0.7
    assert fast.any() and slow.any()
    np.testing.assert_allclose(f.numpy()[fast], plain[fast], rtol=1e-14)
    np.testing.assert_allclose(f.numpy()[slow], plain[slow] / 16, rtol=1e-14)
    # the two sides' powers are rounded separately: the same 1e-14 as above
    assert np.all(f.numpy() <= plain * (1 + 1e-14)) and np.all(f.numpy() >= plain / 16 * (1 - 1e-14))


@pytest.mark.parametrize("bad", [dict(rot_dim=0), dict(rot_dim=7), dict(base=1.0), dict(base=float("nan")),
                                 dict(scaling=5), dict(scaling=-1), dict(scaling=1, factor=0.0),
                                 dict(scaling=3, low=4.0, high=1.0), dict(scaling=4, original_len=0),
                                 dict(scaling=2, rot_dim=2, factor=2.0)])
def test_frequencies_refuse(bad):
    with pytest.raises(l2.L2KVError) as e:
        l2.rotary_frequencies(**dict(dict(rot_dim=64), **bad))
    assert e.value.status == -1


@pytest.mark.parametrize("call", [_rotary, _prompt, _tree, _commit])
def test_host_tensors_that_fit_launch_nothing(call):
    """A call whose arguments are all in order, but in host memory: no kernel may be given such pointers."""
    with pytest.raises(l2.L2KVError) as e:
        call(_inputs())
    assert e.value.status == -1


@pytest.mark.parametrize("max_len", [1 << 31, (1 << 32) + 5, -(1 << 40)])
def test_lengths_beyond_32_bits_are_refused(max_len):
    a = _inputs()
    a["max_len"] = max_len
    for call in (_prompt, _tree):
        with pytest.raises(ValueError):
            call(a)
    with pytest.raises(ValueError):
        l2.prompt_attention_workspace_bytes(a["K"], a["q"], max_len)
