"""Truth values of the calls on new tokens that raise when asked: the error is the caller's to see, and nothing is called."""
import numpy as np
import pytest
import torch

import paper_2406_11430_b200 as l2


class Undecided:
    def __bool__(self):
        raise KeyError("undecided")


def _call(which, **kw):
    i32 = lambda *s: torch.zeros(s, dtype=torch.int32)  # noqa: E731
    K, tok = torch.zeros((2, 1, 2, 9, 64), dtype=torch.bfloat16), torch.zeros((1, 3, 2, 64), dtype=torch.bfloat16)
    ws = torch.zeros(256, dtype=torch.uint8)
    if which == "rotary":
        l2.rotary_write(tok, tok, tok, i32(3), i32(3), None, tok, K, K, None, None, i32(2, 1), i32(2, 1), ws, **kw)
    elif which == "commit":
        l2.tree_commit(K, K, None, None, i32(2, 1), i32(2, 1), i32(2, 4), i32(2), i32(2, 1), ws, **kw)
    elif which == "prompt":
        l2.prompt_attention(tok, i32(3), K, K, i32(2, 1), 9, tok, workspace=ws, **kw)
    else:
        l2.tree_attention(tok, i32(3), torch.zeros((3, 1), dtype=torch.int64), K, K, i32(2, 1), 9, tok, workspace=ws, **kw)


@pytest.mark.parametrize("which,name", [("rotary", "per_head"), ("rotary", "interleaved"), ("commit", "per_head"), ("prompt", "per_head"),
                                        ("tree", "per_head")])
@pytest.mark.parametrize("value,error", [(Undecided(), KeyError), (np.zeros(2), ValueError), (torch.zeros(2), RuntimeError)])
def test_a_truth_value_that_cannot_be_had_raises_its_own_error(which, name, value, error):
    with pytest.raises(error) as e:
        _call(which, **{name: value})
    assert not isinstance(e.value, l2.L2KVError)
