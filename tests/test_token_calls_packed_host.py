"""Host side of the calls on new tokens with packed caches: what describes the rows has to have the type, the order
and the number of entries that the kernels read it with, and every size has to fit the library's 32 bits.  No GPU needed."""
import types

import pytest
import torch

import paper_2406_11430_b200 as l2

B, L, H, HQ, D, N, TOTAL, CAP = 2, 3, 2, 8, 128, 7, 90, 15


def _rows(**change):
    rows = dict(B=B, L=L, t_cap=CAP, total_rows=TOTAL, off=torch.arange(0, TOTAL, CAP).view(B, L),
                cap=torch.full((B, L), CAP, dtype=torch.int32))
    rows.update(change)
    return types.SimpleNamespace(**rows)


def _call(which, rows, K=None, n=N, path_cap=4):
    i32 = lambda *s: torch.zeros(s, dtype=torch.int32)  # noqa: E731
    tok = lambda heads: torch.zeros((1, 1, heads, D), dtype=torch.bfloat16).expand(L, n, heads, D)  # noqa: E731
    K = torch.zeros((H, TOTAL, D), dtype=torch.bfloat16) if K is None else K
    off, start, cur, ws = i32(B + 1), i32(B, L), i32(B, L), torch.zeros(256, dtype=torch.uint8)
    if which == "rotary":
        l2.rotary_write(tok(HQ), tok(H), tok(H), off, i32(N), None, tok(HQ), K, K, i32(H, TOTAL), torch.zeros((H, TOTAL)), start, cur, ws,
                        rows=rows)
    elif which == "commit":
        l2.tree_commit(K, K, None, None, start, cur, i32(B, 4) if path_cap == 4 else i32(B, 1).expand(B, path_cap), i32(B), start, ws, rows=rows)
    elif which == "prompt":
        l2.prompt_attention(tok(HQ), off, K, K, cur, CAP, tok(HQ), workspace=ws, rows=rows)
    elif which == "tree":
        l2.tree_attention(tok(HQ), off, torch.zeros((N, 1), dtype=torch.int64), K, K, cur, CAP, tok(HQ), workspace=ws, rows=rows)
    else:
        return l2.prompt_attention_workspace_bytes(K, tok(HQ), CAP, rows=rows)


CALLS = ["rotary", "commit", "prompt", "tree", "workspace"]


@pytest.mark.parametrize("which", CALLS)
def test_rows_that_fit_get_as_far_as_the_launch(which):
    if which == "workspace":
        assert _call(which, _rows()) >= 256
        return
    with pytest.raises(l2.L2KVError) as e:                   # host tensors: nothing is launched
        _call(which, _rows())
    assert e.value.status == -1


@pytest.mark.parametrize("which", CALLS)
@pytest.mark.parametrize("change", [
    dict(off=torch.arange(0, TOTAL, CAP, dtype=torch.int32).view(B, L)),              # half of the bytes
    dict(off=torch.arange(0, TOTAL - CAP, CAP)), dict(off=torch.zeros(0, dtype=torch.int64)),
    dict(off=torch.arange(0, TOTAL, CAP).view(L, B).t()), dict(off=torch.arange(0, TOTAL, CAP).double().view(B, L)),
    dict(cap=torch.full((B, L), CAP)), dict(cap=torch.full((B * L - 1,), CAP, dtype=torch.int32)),
    dict(cap=torch.full((1, 1), CAP, dtype=torch.int32).expand(B, L)), dict(off=list(range(0, TOTAL, CAP)))])
def test_rows_of_another_type_order_or_number_are_refused(which, change):
    with pytest.raises(ValueError):
        _call(which, _rows(**change))


@pytest.mark.parametrize("which", CALLS)
@pytest.mark.parametrize("change", [dict(B=(1 << 32) + B), dict(L=(1 << 32) + L), dict(t_cap=(1 << 32) + CAP), dict(t_cap=1 << 31),
                                    dict(L=-(1 << 40))])
def test_row_counts_beyond_32_bits_are_refused(which, change):
    with pytest.raises(ValueError):
        _call(which, _rows(**change))


@pytest.mark.parametrize("which", ["rotary", "prompt", "tree", "workspace"])
def test_more_tokens_than_32_bits_count_are_refused(which):
    with pytest.raises(ValueError):
        _call(which, _rows(), n=(1 << 32) + N)


def test_longer_paths_and_more_heads_than_32_bits_count_are_refused():
    with pytest.raises(ValueError):
        _call("commit", _rows(), path_cap=(1 << 32) + 4)
    K = torch.zeros((1, TOTAL, D), dtype=torch.bfloat16).expand((1 << 32) + H, TOTAL, D)
    for which in ("commit", "prompt", "workspace"):
        with pytest.raises(ValueError):
            _call(which, _rows(), K=K)
