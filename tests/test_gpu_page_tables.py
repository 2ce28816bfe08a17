"""The calls on tables of pages against a model of them in Python's integers: sequences that go on, fork, give rows back, end
and begin; the copy of pages that are shared; pools that run out; pinned pages; compaction by key norm."""
import numpy as np
import pytest
import torch

from page_util import compacted, updated
from token_util import DEV, DT, i32

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def l2():
    import paper_2406_11430_b200 as lib
    lib.lib()
    return lib


class Pool:
    """A pool with B sequences of `rows` rows [B, L]; every byte of it is known."""

    def __init__(self, l2, rows, P, H=2, D=64, dtype="bf16", cap=None, spare=20, seed=0, integer_keys=False):
        self.l2, self.P, self.rows = l2, P, np.asarray(rows)
        self.B, self.L = self.rows.shape
        r = np.random.RandomState(seed)
        pages = -(-self.rows // P)
        self.cap = cap or int(pages.max()) + 4
        self.n_pages = int(pages.sum()) + spare
        self.table = np.full((self.B, self.L, self.cap), -1, np.int64)
        self.table[np.arange(self.cap) < pages[:, :, None]] = r.permutation(self.n_pages)[:pages.sum()]
        g = torch.Generator().manual_seed(seed)
        R = self.n_pages * P
        self.K, self.V = (torch.randn((H, R, D), generator=g).to(DEV, DT[dtype]) for _ in range(2))
        self.idx = torch.randint(0, 1 << 20, (H, R), generator=g, dtype=torch.int32).to(DEV)
        self.key = (torch.randint(0, 7, (H, R), generator=g).float() if integer_keys else torch.rand((H, R), generator=g)).to(DEV)
        self.tensors = (self.K, self.V, self.idx, self.key)
        self.pages = l2.Pages(i32(self.table).reshape(self.table.shape), P, self.n_pages)

    def next(self, B=None, cap=None):
        B = self.B if B is None else B
        return self.l2.Pages(torch.full((B, self.L, cap or self.cap), 12345, dtype=torch.int32, device=DEV), self.P, self.n_pages,
                             torch.full((B, self.L), 12345, dtype=torch.int32, device=DEV))

    def workspace(self, max_len=0, B=None):
        ws = torch.full((self.l2.page_workspace_bytes(self.K, self.pages, max_len, B),), 255, dtype=torch.uint8, device=DEV)
        ws[:256] = 0
        return ws

    def update(self, parent, keep, grow, pinned=(), check=True, n_free=True, out=None):
        l2, B = self.l2, len(parent)
        out = self.next(B) if out is None else out
        free = torch.full((1,), -1, dtype=torch.int32, device=DEV)
        pin = None
        if pinned:
            pin = torch.zeros(self.n_pages, dtype=torch.uint8, device=DEV)
            pin[list(pinned)] = 1
        before = [x.clone() for x in self.tensors]
        ws = self.workspace(B=B)
        l2.page_update(*self.tensors, self.pages, i32(parent), i32(keep).reshape(B, self.L), i32(grow), out, ws, pin=pin,
                       n_free_out=free if n_free else None)
        torch.cuda.synchronize()
        table, room, n, copies, short = updated(self.table, self.P, self.n_pages, parent, keep, grow, set(pinned))
        assert np.array_equal(out.table.cpu().numpy(), table)
        assert np.array_equal(out.room.cpu().numpy(), room)
        assert not n_free or free.item() == n
        assert l2.read_device_status(ws) == (-7 if short else 0)
        for x, y in zip(self.tensors, before):
            for src, dst, rows in copies:
                y[:, dst * self.P:dst * self.P + rows] = y[:, src * self.P:src * self.P + rows]
            assert torch.equal(x, y)
        return table, room, copies, short


@pytest.mark.parametrize("P", [16, 32, 1024])
def test_sequences_go_on(l2, P):
    """From no row to several pages, with nothing shared: nothing is copied."""
    rows = [[0], [1], [P - 1], [P], [P + 1], [3 * P], [3 * P + 5]]
    for grow in (0, 1, P, 2 * P + 1):
        p = Pool(l2, rows, P, seed=grow)
        assert p.update(list(range(7)), rows, [grow] * 7)[2] == []


def test_one_sequence_of_one_row(l2):
    Pool(l2, [[1]], 16).update([0], [[1]], [1])
    Pool(l2, [[0]], 16, spare=1).update([0], [[0]], [1])
    Pool(l2, [[16]], 16, spare=1).update([-1], [[0]], [16])


@pytest.mark.parametrize("dtype,D", [("bf16", 64), ("bf16", 128), ("fp32", 64), ("fp32", 128)])
@pytest.mark.parametrize("H", [1, 3, 40])
def test_forks_copy_the_page_that_they_write(l2, H, dtype, D):
    p = Pool(l2, [[37, 20], [16, 0], [5, 31]], 16, H=H, D=D, dtype=dtype, seed=H)
    _, _, copies, _ = p.update([0, 0, 0, 2, 1, 2], [[37, 20]] * 3 + [[5, 31], [16, 0], [3, 31]], [1, 1, 0, 4, 1, 4])
    assert len(copies) == 4                                  # the second child's two, and the second child of sequence 2


def test_who_keeps_a_shared_page(l2):
    """The one with most rows in it; the first of several; a full reference before any part; nobody a pinned page."""
    p = Pool(l2, [[60]], 16, spare=30)
    assert len(p.update([0, 0], [[50], [55]], [1, 1])[2]) == 1
    assert p.update([0, 0], [[50], [55]], [1, 1])[2][0][2] == 50 % 16
    assert len(p.update([0, 0], [[40], [60]], [1, 0])[2]) == 1                   # a full page of the other's
    assert len(p.update([0, 0], [[60], [60]], [0, 1])[2]) == 1                   # the first does not grow, but keeps it
    assert len(p.update([0, 0], [[59], [60]], [0, 1])[2]) == 0
    assert len(p.update([0], [[60]], [1], pinned=[int(p.table[0, 0, 3])])[2]) == 1
    assert len(p.update([0], [[48]], [1], pinned=[int(p.table[0, 0, 2])])[2]) == 0   # full: nothing to write in it


def test_the_same_page_twice_in_one_table(l2):
    p = Pool(l2, [[40], [8]], 16)
    p.table[0, 0, 1] = p.table[0, 0, 0]
    p.table[1, 0, 0] = p.table[0, 0, 2]
    p.pages.table.copy_(i32(p.table))
    p.update([0, 1], [[40], [8]], [1, 1])
    p.table[0, 0, 2] = p.table[0, 0, 0]                      # its last page is one of its full ones
    p.pages.table.copy_(i32(p.table))
    assert len(p.update([0, 1], [[40], [8]], [1, 0])[2]) == 1


def test_ended_sequences_pages_are_handed_out_at_once(l2):
    p = Pool(l2, [[100], [90], [80]], 16, spare=0)
    assert not p.update([1, -1], [[90], [0]], [1, 150])[3]


def test_pools_that_run_out(l2):
    """Whoever the pages do not reach keeps what it has and gets no room; what asks for none always gets its own."""
    for spare in range(6):
        p = Pool(l2, [[16, 3], [16, 16], [7, 16], [40, 32]], 16, spare=spare, seed=spare)
        p.update([0, 1, 2, 3], p.rows.tolist(), [1, 17, 9, 1])
        p.update([0, 0, 2, 3, 2], [[16, 3], [16, 3], [7, 16], [39, 32], [7, 16]], [1, 5, 9, 0, 3])
    assert p.update([0, 1, 2, 3], p.rows.tolist(), [1, 17, 9, 1])[3] or spare >= 6


def test_tables_that_run_out(l2):
    p = Pool(l2, [[60], [10]], 16, cap=4)
    assert p.update([0, 1], [[60], [10]], [4, 1])[3] is False
    assert p.update([0, 1], [[60], [10]], [5, 1])[3] is True
    assert p.update([0, 1], [[64 - 4], [10]], [2 ** 31 - 1, 2 ** 31 - 1])[3] is True


def test_more_or_fewer_sequences_than_before(l2):
    p = Pool(l2, [[20, 40], [33, 0], [16, 5]], 16, spare=200)
    p.update([2], [[16, 5]], [3])
    p.update([0, 1, 2] * 11, [[20, 40], [33, 0], [16, 5]] * 11, [2] * 33)
    p.update([-1] * 4, [[0, 0]] * 4, [5] * 4)


@pytest.mark.parametrize("P", [16, 128])
@pytest.mark.parametrize("B,L", [(70, 3), (1200, 1), (40, 32)])
def test_random_steps(l2, B, L, P):
    """More (b, l) than one pass over the requests takes, more pages than one block of the scan."""
    r = np.random.RandomState(B + P)
    p = Pool(l2, r.randint(0, 30 if P == 16 else 300, (B, L)), P, H=1, spare=B * L * 3 + 9000, seed=B)
    for seed in range(2):
        parent = r.randint(-1, B, B)
        keep = np.where(parent[:, None] >= 0, np.minimum(p.rows[parent], r.randint(0, 400, (B, 1))), 0)
        p.update(parent.tolist(), keep.tolist(), r.choice([0, 1, 3, 20], B).tolist(), pinned=r.randint(0, p.n_pages, 50).tolist())


def test_strided_tables_and_no_optional_outputs(l2):
    p = Pool(l2, [[20, 40], [33, 0]], 16)
    want = updated(p.table, 16, p.n_pages, [1, 0], [[33, 0], [20, 40]], [2, 3])[0]
    room = torch.full((2, p.L, 2 * p.cap), 5, dtype=torch.int32, device=DEV)
    out = l2.Pages(room.transpose(0, 1)[:, :, :p.cap], 16, p.n_pages)
    p.pages = l2.Pages(p.pages.table.transpose(0, 1).contiguous().transpose(0, 1), 16, p.n_pages)
    l2.page_update(p.K, p.V, None, None, p.pages, i32([1, 0]), i32([[33, 0], [20, 40]]), i32([2, 3]), out, p.workspace())
    torch.cuda.synchronize()
    assert np.array_equal(out.table.cpu().numpy(), want) and (room[:, :, p.cap:] == 5).all()


def test_entries_that_are_no_pages(l2):
    """They are told, take part in nothing, and stay in the table; a parent that is no sequence counts as none."""
    p = Pool(l2, [[40], [20]], 16)
    for bad in (-1, p.n_pages, 2 ** 31 - 1, -2 ** 31):
        for j in (0, 2):
            p.pages.table[0, 0, j] = bad
            out, ws, free = p.next(), p.workspace(), i32([0])
            before = [x.clone() for x in p.tensors]
            l2.page_update(*p.tensors, p.pages, i32([0, 1]), i32([[40], [20]]), i32([10, 10]), out, ws, n_free_out=free)
            torch.cuda.synchronize()
            assert l2.read_device_status(ws) == -5
            held = {int(x) for x in p.pages.table.flatten().tolist()} & set(range(p.n_pages))
            unheld = [x for x in range(p.n_pages) if x not in held]
            want = p.pages.table.clone()
            want[0, 0, 3] = unheld[0]
            assert torch.equal(out.table, want) and free.item() == len(unheld) - 1
            for x, y in zip(p.tensors, before):
                assert torch.equal(x, y)
            p.pages.table.copy_(i32(p.table))
    out, ws = p.next(), p.workspace()
    l2.page_update(*p.tensors, p.pages, i32([2 ** 31 - 1, 2]), i32([[40], [20]]), i32([0, 0]), out, ws)
    torch.cuda.synchronize()
    assert l2.read_device_status(ws) == -5 and (out.table == -1).all() and not out.room.any()


def test_update_captured_over_changing_inputs(l2):
    p = Pool(l2, [[20, 40], [33, 0]], 16)
    out, ws, free = p.next(), p.workspace(), i32([0])
    parent, keep, grow = i32([0, 1]), i32([[20, 40], [33, 0]]), i32([1, 1])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        l2.page_update(*p.tensors, p.pages, parent, keep, grow, out, ws, n_free_out=free)
    for pa, ke, gr in (([0, 1], [[20, 40], [33, 0]], [1, 1]), ([1, 1], [[30, 0], [33, 0]], [9, 20]), ([-1, 0], [[0, 0], [20, 40]], [0, 1])):
        parent.copy_(i32(pa)), keep.copy_(i32(ke)), grow.copy_(i32(gr))
        graph.replay()
        torch.cuda.synchronize()
        table, room, n, _, _ = updated(p.table, 16, p.n_pages, pa, ke, gr)
        assert np.array_equal(out.table.cpu().numpy(), table) and np.array_equal(out.room.cpu().numpy(), room) and free.item() == n


# ---- compaction ------------------------------------------------------------------------------------

def compact(p, keep, lens=None, pinned=(), policy=0, in_place=False, max_len=None):
    l2, lens = p.l2, p.rows if lens is None else lens
    keep = np.asarray(keep).reshape(lens.shape)
    out = p.next()
    len_d = i32(lens)
    len_out = len_d if in_place else torch.full_like(len_d, 99)
    pin = None
    if len(pinned):
        pin = torch.zeros(p.n_pages, dtype=torch.uint8, device=DEV)
        pin[list(pinned)] = 1
    max_len = int(lens.max()) if max_len is None else max_len
    ws = p.workspace(max(1, max_len))
    before = [x.clone() for x in p.tensors]
    l2.page_compact(*p.tensors, p.pages, len_d, i32(keep), max_len, out, len_out, ws, policy=policy, pin=pin)
    torch.cuda.synchronize()
    table, after, moved, short = compacted(p.table, p.P, p.n_pages, lens, np.maximum(keep, 0), set(pinned))
    assert np.array_equal(out.table.cpu().numpy(), table)
    assert np.array_equal(len_out.cpu().numpy(), after) and np.array_equal(out.room.cpu().numpy(), after)
    assert l2.read_device_status(ws) == (-7 if short else 0)
    key = before[3].cpu().numpy()
    for b, l in moved:
        T, k = int(lens[b, l]), max(0, int(keep[b, l]))
        t, j = np.arange(T), np.arange(k)
        old = p.table[b, l][t // p.P] * p.P + t % p.P
        new = torch.from_numpy(table[b, l][j // p.P] * p.P + j % p.P).to(DEV)
        for h in range(key.shape[0]):
            x = key[h, old]
            kept = np.sort(np.lexsort((t, -x if policy else x))[:k])
            src = torch.from_numpy(old[kept]).to(DEV)
            for y in before:
                y[h, new] = y[h, src]
    for x, y in zip(p.tensors, before):
        assert torch.equal(x, y)
    return short


@pytest.mark.parametrize("integer_keys", [False, True])
@pytest.mark.parametrize("policy", [0, 1])
@pytest.mark.parametrize("P", [16, 64, 1024])
def test_compaction(l2, P, policy, integer_keys):
    """Lengths around chunks and pages, from nothing kept to everything; many equal keys."""
    rows = np.array([[1, 2], [17, 511], [512, 513], [1025, 3000], [0, 64]])
    keep = np.array([[0, 1], [16, 511], [100, 512], [513, 77], [0, 63]])
    p = Pool(l2, rows, P, H=3, spare=400 if P == 16 else 120, seed=P, integer_keys=integer_keys)
    assert not compact(p, keep, policy=policy)


@pytest.mark.parametrize("policy", [0, 1])
@pytest.mark.parametrize("rows", [25600, 25601, 53248, 53249, 60001])
def test_compaction_of_long_caches(l2, rows, policy):
    """Around what the selection keeps in shared memory; keys of one value, of two, and of far apart ones among others."""
    for kind in ("random", "equal", "two", "far"):
        p = Pool(l2, [[rows]], 1024, H=2, spare=80, seed=rows % 97)
        if kind == "equal":
            p.key.fill_(0.25)
        if kind == "two":
            p.key.copy_((p.key > 0.7).float() * 3 + 1e-30)
        if kind == "far":
            p.key[:, ::3] = 0
            p.key[:, 1::7] = 3e38
            p.key[:, 5::1000] = 1e-42
        for keep in (1, rows // 2, rows - 1):
            compact(p, [[keep]], policy=policy)


def test_compaction_of_many_units(l2):
    """More units than SMs."""
    r = np.random.RandomState(2)
    rows = r.randint(0, 1500, (7, 6))
    p = Pool(l2, rows, 16, H=4, spare=2200, seed=9, integer_keys=True)
    compact(p, (rows * r.rand(7, 6)).astype(int))


@pytest.mark.parametrize("dtype,D", [("bf16", 128), ("fp32", 64), ("fp32", 128)])
def test_compaction_types(l2, dtype, D):
    p = Pool(l2, [[700], [90]], 32, H=2, D=D, dtype=dtype, spare=60)
    compact(p, [[350], [90]], in_place=True)


def test_compaction_leaves_shared_pages_to_the_others(l2):
    p = Pool(l2, [[200], [200]], 16, spare=40)
    p.table[1, 0] = p.table[0, 0]
    p.pages.table.copy_(i32(p.table))
    compact(p, [[60], [200]], pinned=[3, 4])


def test_compaction_of_a_pool_that_runs_out(l2):
    for spare in (0, 3, 4, 9, 10):
        p = Pool(l2, [[100], [100], [100], [9]], 16, spare=spare, seed=spare)
        assert compact(p, [[50], [90], [0], [9]]) == (spare < 10)


def test_compaction_bounds(l2):
    """Keeps below zero keep nothing, above the length everything; lengths are cut at max_len."""
    p = Pool(l2, [[100], [100], [100]], 16, spare=40)
    compact(p, [[-5], [1000], [99]])
    p = Pool(l2, [[100], [100]], 16, spare=40)
    out, n, ws = p.next(), i32([[0], [0]]), p.workspace(64)
    l2.page_compact(*p.tensors, p.pages, i32([[100], [-3]]), i32([[70], [0]]), 64, out, n, ws)
    torch.cuda.synchronize()
    assert n.flatten().tolist() == [64, 0]


def test_compaction_of_keys_that_are_no_numbers(l2):
    """Infinite keys come last, NaN behind them; equal ones by row."""
    p = Pool(l2, [[100]], 16, H=1, spare=40)
    at = torch.from_numpy(p.table[0, 0][np.arange(100) // 16] * 16 + np.arange(100) % 16).to(DEV)
    p.key[0, at[10:40]] = float("inf")
    p.key[0, at[50]] = float("nan")
    before = p.idx.clone()
    out, n, ws = p.next(), i32([[0]]), p.workspace(100)
    l2.page_compact(*p.tensors, p.pages, i32([[100]]), i32([[80]]), 100, out, n, ws)
    torch.cuda.synchronize()
    kept = [t for t in range(100) if t != 50 and not 10 <= t < 40] + list(range(10, 21))
    j = np.arange(80)
    new = torch.from_numpy(out.table.cpu().numpy()[0, 0].astype(np.int64)[j // 16] * 16 + j % 16).to(DEV)
    assert torch.equal(p.idx[0, new], before[0, at[sorted(kept)]])


def test_compaction_with_a_page_that_is_none(l2):
    """The sequence stays whole."""
    for bad in (-1, 10 ** 6, 2 ** 31 - 1, -2 ** 31):
        p = Pool(l2, [[100], [100]], 16, spare=40)
        p.pages.table[0, 0, 3] = bad
        out, n, ws = p.next(), i32([[0], [0]]), p.workspace(100)
        K = p.K.clone()
        l2.page_compact(*p.tensors, p.pages, i32([[100], [100]]), i32([[50], [100]]), 100, out, n, ws)
        torch.cuda.synchronize()
        assert l2.read_device_status(ws) == -5 and n.flatten().tolist() == [100, 100]
        assert torch.equal(out.table, p.pages.table) and torch.equal(p.K, K)


def test_compaction_captured(l2):
    p = Pool(l2, [[600], [90]], 16, spare=80)
    out, n, ws, len_d, keep = p.next(), i32([[0], [0]]), p.workspace(600), i32(p.rows), i32([[300], [10]])
    was = [x.clone() for x in p.tensors]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        l2.page_compact(*p.tensors, p.pages, len_d, keep, 600, out, n, ws)
    got = []
    for _ in range(2):
        for x, y in zip(p.tensors, was):
            x.copy_(y)
        graph.replay()
        torch.cuda.synchronize()
        got.append([x.clone() for x in (*p.tensors, out.table, n)])
    for x, y in zip(p.tensors, was):
        x.copy_(y)
    compact(p, [[300], [10]])
    for x, y, z in zip(*got, p.tensors):
        assert torch.equal(x, y) and torch.equal(x, z)
