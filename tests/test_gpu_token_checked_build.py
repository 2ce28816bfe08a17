"""The calls on new tokens on the library built with -DL2KV_DEBUG: their own tests pass there, and row ranges that leave
the cache are recorded and skipped."""
import ctypes
import os
import subprocess
import sys

import pytest
import torch

from token_util import DEV, i32

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
NAMES = ("l2kv_rotary_write", "l2kv_tree_commit", "l2kv_prompt_attention", "l2kv_tree_attention", "l2kv_prompt_attention_workspace_bytes")


def test_the_calls_on_new_tokens_pass_on_the_bounds_checked_build():
    from paper_2406_11430_b200 import build as l2build
    env = dict(os.environ, L2KV_LIBRARY=l2build.build_debug())
    r = subprocess.run([sys.executable, "-m", "pytest", "-q", "-x", "-m", "gpu"] +
                       [os.path.join(ROOT, "tests", f"test_gpu_{name}.py") for name in
                        ("token_rows", "token_attention", "token_limits", "early_launch")],
                       env=env, cwd=ROOT, capture_output=True, text=True, timeout=1500)
    assert r.returncode == 0, r.stdout[-3000:] + r.stderr[-2000:]
    assert " passed" in r.stdout


@pytest.fixture
def checked():
    """The calls lead to the checked build, and back to the library afterwards."""
    import paper_2406_11430_b200 as l2
    from paper_2406_11430_b200 import binding, build as l2build
    native, debug = binding._token_calls(), ctypes.CDLL(l2build.build_debug())
    address = lambda lib: [ctypes.cast(getattr(lib, name), ctypes.c_void_p).value for name in NAMES]  # noqa: E731
    native.bind(*address(debug))
    yield l2
    native.bind(*address(l2.lib()))


class Beyond:
    """Two packed sequences, the second with a range that ends 6 rows behind the cache's; the storage goes on for as many
    rows as any of its rows could reach, so that nothing here leaves the memory that it owns."""
    H, D, total = 2, 128, 40

    def __init__(self, l2, dtype=torch.bfloat16):
        room = self.H * self.total + 64
        self.rows = l2.Rows([[0], [26]], [[20], [20]], self.total, DEV)
        g = torch.Generator().manual_seed(1)
        stores = [torch.randn((room, self.D), generator=g).to(DEV, dtype) for _ in range(2)]
        self.K, self.V = (x[:self.H * self.total].view(self.H, self.total, self.D) for x in stores)
        metas = [torch.full((room,), -1, dtype=torch.int32, device=DEV), torch.full((room,), -1.0, device=DEV)]
        self.idx, self.key = (x[:self.H * self.total].view(self.H, self.total) for x in metas)
        self.stores = stores + metas
        self.before = [x.clone() for x in self.stores]
        self.ws = torch.zeros(256, dtype=torch.uint8, device=DEV)

    def assert_only(self, allowed):
        """No row but those of `allowed` (per head) has changed."""
        same = torch.ones(self.stores[0].shape[0], dtype=torch.bool, device=DEV)
        for h in range(self.H):
            same[[h * self.total + t for t in allowed]] = False
        for x, y in zip(self.stores, self.before):
            assert torch.equal(x[same], y[same])


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_rows_written_behind_the_cache_are_recorded_and_skipped(checked, dtype):
    c = Beyond(checked, dtype)
    q = torch.randn((1, 8, 2, c.D), device=DEV).to(dtype)
    out, new = torch.empty_like(q), i32([[0], [0]])
    # the second sequence's rows 12 .. 16 are rows 38 .. 42 of 40
    checked.rotary_write(q, q, q, i32([0, 3, 8]), i32(range(8)), None, out, c.K, c.V, c.idx, c.key, i32([[5], [12]]), new, c.ws, rows=c.rows)
    torch.cuda.synchronize()
    assert checked.read_device_status(c.ws) == -9
    c.assert_only([5, 6, 7, 38, 39])
    for h in range(2):
        assert torch.equal(c.V[h, 38:], q[0, 3:5, h]) and torch.equal(c.V[h, 5:8], q[0, :3, h])


def test_rows_moved_from_behind_the_cache_are_recorded_and_skipped(checked):
    c = Beyond(checked)
    start = i32([[2], [10]])
    # the second sequence's entries 1, 3 and 5 are rows 37, 39 and 41 of 40
    checked.tree_commit(c.K, c.V, c.idx, c.key, start, i32([[8], [18]]), i32([[1, 2, 3], [1, 3, 5]]), i32([3, 3]), start, c.ws, rows=c.rows)
    torch.cuda.synchronize()
    assert checked.read_device_status(c.ws) == -9
    c.assert_only([2, 3, 4, 36, 37])


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_rows_read_behind_the_cache_are_recorded(checked, dtype):
    c = Beyond(checked, dtype)
    q = torch.randn((1, 2, 2, c.D), device=DEV).to(dtype)
    mask = torch.full((2, 1), -1, dtype=torch.int64, device=DEV)
    for lens, status in (([[20], [14]], 0), ([[20], [15]], -9)):
        for tree in (False, True):
            c.ws.zero_()
            out = torch.empty_like(q)
            if tree:
                checked.tree_attention(q, i32([0, 1, 2]), mask, c.K, c.V, i32(lens), 20, out, workspace=c.ws, rows=c.rows)
            else:
                checked.prompt_attention(q, i32([0, 1, 2]), c.K, c.V, i32(lens), 20, out, workspace=c.ws, rows=c.rows)
            torch.cuda.synchronize()
            assert checked.read_device_status(c.ws) == status
    c.assert_only([])
