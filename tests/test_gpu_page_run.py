"""A server's steps over a cache in pages, one call behind the other without a wait between them: requests begin, fork, take
single tokens, give rows back, are compacted by key norm and end.  Every row of the cache is kept track of in Python, and every
step's attention is held against the definition in 64 bits over those rows."""
import numpy as np
import pytest
import torch

from page_util import compacted, updated
from token_util import DEV, i32

pytestmark = pytest.mark.gpu
H, G, D, P, L, CAP, PAGES = 2, 4, 128, 16, 2, 14, 400


@pytest.fixture(scope="module")
def l2():
    import paper_2406_11430_b200 as lib
    lib.lib()
    return lib


class Server:
    def __init__(self, l2, B):
        self.l2, self.B = l2, B
        self.g = torch.Generator().manual_seed(3)
        self.K, self.V = (torch.full((H, PAGES * P, D), float("nan"), dtype=torch.bfloat16, device=DEV) for _ in range(2))
        self.idx = torch.full((H, PAGES * P), -1, dtype=torch.int32, device=DEV)
        self.key = torch.full((H, PAGES * P), float("nan"), device=DEV)
        self.tables = [l2.Pages.empty(B, L, CAP, P, PAGES, DEV) for _ in range(2)]
        self.cur = torch.zeros((B, L), dtype=torch.int32, device=DEV)
        self.room = torch.zeros((B, L), dtype=torch.int32, device=DEV)
        self.freq = l2.rotary_frequencies(D, 10000.0)[0].to(DEV)
        self.weights = [(torch.rand(D, generator=self.g) + 0.5).to(DEV, torch.bfloat16) for _ in range(2)]
        self.ws = torch.zeros(1 << 24, dtype=torch.uint8, device=DEV)
        self.free = i32([0])
        # what should be there: tables, lengths, and per (b, l, h) the positions of the rows
        self.table, self.len = np.full((B, L, CAP), -1), np.zeros((B, L), np.int64)
        self.pos = [0] * B
        self.checks = []

    def update(self, parent, keep, grow):
        l2 = self.l2
        keep = np.broadcast_to(np.asarray(keep).reshape(self.B, -1), (self.B, L))
        a, b = self.tables
        l2.page_update(self.K, self.V, self.idx, self.key, a, i32(parent), i32(keep), i32(grow), b, self.ws, n_free_out=self.free)
        self.tables = [b, a]
        self.table, _, n, _, short = updated(self.table, P, PAGES, parent, keep, grow)
        assert not short
        self.len = np.where(np.asarray(parent)[:, None] >= 0, keep, 0)
        was = list(self.pos)
        self.pos = [was[p] if p >= 0 else 0 for p in parent]
        self.cur = i32(self.len)
        self.checks.append((b.table.clone(), self.table.copy(), self.free.clone(), n))

    def tokens(self, n, back=0):
        """n[b] new tokens, written and attended to (back: positions that rejected tokens gave back)."""
        l2, N = self.l2, sum(n)
        tok = torch.randn((L, N, (G + 2) * H, D), generator=self.g).to(DEV, torch.bfloat16)
        off = i32(np.concatenate([[0], np.cumsum(n)]))
        pos = i32(np.concatenate([self.pos[b] - back + np.arange(n[b]) for b in range(self.B)]))
        q, out, lse = (torch.empty((L, N, G * H, D), dtype=torch.bfloat16, device=DEV) for _ in range(2)), None, None
        q, out = q
        lse, new = torch.empty((L, N, G * H), device=DEV), torch.zeros_like(self.cur)
        l2.norm_rotary_write(tok[:, :, :G * H], tok[:, :, G * H:-H], tok[:, :, -H:], off, pos, self.freq, q, self.K, self.V, self.idx, self.key,
                             self.cur, new, self.ws, q_weight=self.weights[0], k_weight=self.weights[1], pages=self.tables[0])
        l2.paged_attention(q, off, self.K, self.V, new, CAP * P, out, self.tables[0], lse_out=lse, workspace=self.ws)
        self.cur = new
        self.len = self.len + np.asarray(n)[:, None]
        self.pos = [p - back + m for p, m in zip(self.pos, n)]
        # (clones in stream order; nothing is waited for)
        self.checks.append((q, out, lse, new, self.K.clone(), self.V.clone(), self.key.clone(), list(n), self.table.copy(), self.len.copy()))

    def compact(self, keep):
        l2 = self.l2
        keep = np.broadcast_to(np.asarray(keep).reshape(self.B, -1), (self.B, L))
        a, b = self.tables
        new = torch.zeros_like(self.cur)
        l2.page_compact(self.K, self.V, self.idx, self.key, a, self.cur, i32(keep), CAP * P, b, new, self.ws)
        self.tables, self.cur = [b, a], new
        self.table, self.len, _, short = compacted(self.table, P, PAGES, self.len, keep)
        assert not short
        self.checks.append((b.table.clone(), self.table.copy(), new.clone(), self.len.copy()))

    def rows(self, table, b, l, n):
        t = np.arange(n)
        return torch.from_numpy(table[b, l][t // P] * P + t % P).to(DEV)

    def check(self):
        torch.cuda.synchronize()
        assert self.l2.read_device_status(self.ws) == 0
        for c in self.checks:
            if len(c) == 4:
                assert np.array_equal(c[0].cpu().numpy(), c[1])
                assert np.array_equal(c[2].cpu().numpy().reshape(-1), np.asarray(c[3]).reshape(-1))
                continue
            q, out, lse, new, K, V, key, n, table, length = c
            assert np.array_equal(new.cpu().numpy(), length)
            first = 0
            for b in range(self.B):
                for l in range(L):
                    T = int(length[b, l])
                    at = self.rows(table, b, l, T)
                    for h in range(H):
                        k, v = K[h, at].double(), V[h, at].double()
                        assert torch.isfinite(k).all() and torch.isfinite(v).all()
                        # the keys are those of the rows that lie there: fp32 sums of D squares
                        assert ((key[h, at].double() - k.square().sum(-1)).abs() <= D * 2.0 ** -24 * k.square().sum(-1)).all()
                        for j in range(h * G, (h + 1) * G if n[b] else 0):
                            of = slice(first, first + n[b])
                            hidden = torch.ones((n[b], T), dtype=torch.bool, device=DEV).triu(T - n[b] + 1)
                            x = q[l, of, j].double()
                            z = (x @ k.T * D ** -0.5).masked_fill(hidden, -torch.inf)
                            w = z.softmax(-1)
                            # weights and result rounded to bf16; scores are fp32 sums of D products (D 2^-24 sum |q k|)
                            size = ((x.abs() @ k.abs().T) * D ** -0.5).amax(-1, keepdim=True)
                            rel = 2.0 ** -8 + 2 * size * (D + 8) * 2.0 ** -24 + (2 * T + 16) * 2.0 ** -24 + 2.0 ** -20
                            bound = (rel * (w @ v.abs()) + 2.0 ** -8 * (w @ v).abs()) * 1.01 + 1e-30
                            assert ((out[l, of, j].double() - w @ v).abs() <= bound).all()
                            assert ((lse[l, of, j].double() - z.logsumexp(-1)).abs() <= 1e-4).all()
                first += n[b]
        self.checks.clear()


@pytest.mark.parametrize("warm", [False, True])
def test_a_server_s_steps(l2, warm):
    for _ in range(2 if warm else 1):                        # (again, over a workspace that has been used)
        s = Server(l2, 5)
        s.update([-1] * 5, [0] * 5, [70, 33, 0, 16, 1])
        s.tokens([70, 33, 0, 16, 1])
        for _ in range(3):                                   # single tokens
            s.update(range(5), s.len, [1, 1, 0, 1, 1])
            s.tokens([1, 1, 0, 1, 1])
        s.update([0, 0, 0, 1, 3], s.len[[0, 0, 0, 1, 3]], [1, 1, 1, 4, 1])      # forks; sequence 4 ends
        s.tokens([1, 1, 1, 4, 1])
        s.compact(np.stack([s.len[:, 0], s.len[:, 1] // 2], 1))                # the second layer to half
        s.update(range(5), s.len, [2] * 5)
        s.tokens([2] * 5)
        s.update([4, 1, 2, 3, 0], np.maximum(s.len[[4, 1, 2, 3, 0]] - 1, 0), [1] * 5)   # a rejected token each, and changed places
        s.tokens([1] * 5, back=1)
        s.compact(np.minimum(s.len, 20))
        s.update([0, 1, 2, 3, -1], s.len * (np.arange(5) < 4)[:, None], [1, 30, 1, 1, 50])
        s.tokens([1, 30, 1, 1, 50])
        s.check()


def test_a_step_as_a_graph(l2):
    """A decode step captured once and replayed: every replay takes up the lengths and tables that the one before left."""
    B = 3
    s = Server(l2, B)
    s.update([-1] * B, [0] * B, [40, 17, 100])
    s.tokens([40, 17, 100])
    s.check()
    parent, grow = i32(range(B)), i32([1] * B)
    a, b = s.tables[0], s.tables[1]
    cur = s.cur.clone()
    tok = torch.zeros((L, B, (G + 2) * H, D), dtype=torch.bfloat16, device=DEV)
    off, pos, new = i32(range(B + 1)), i32(s.pos), torch.zeros_like(cur)
    q, out = (torch.zeros((L, B, G * H, D), dtype=torch.bfloat16, device=DEV) for _ in range(2))
    lse = torch.zeros((L, B, G * H), device=DEV)

    def step():
        l2.page_update(s.K, s.V, s.idx, s.key, a, parent, cur, grow, b, s.ws, n_free_out=s.free)
        l2.norm_rotary_write(tok[:, :, :G * H], tok[:, :, G * H:-H], tok[:, :, -H:], off, pos, s.freq, q, s.K, s.V, s.idx, s.key, cur, new,
                             s.ws, q_weight=s.weights[0], k_weight=s.weights[1], pages=b)
        l2.paged_attention(q, off, s.K, s.V, new, CAP * P, out, b, lse_out=lse, workspace=s.ws)
        a.table.copy_(b.table)
        cur.copy_(new)
        pos.add_(1)

    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for _ in range(30):
        tok.copy_(torch.randn(tok.shape, generator=s.g).to(torch.bfloat16))
        graph.replay()
        s.table = updated(s.table, P, PAGES, list(range(B)), s.len, [1] * B)[0]
        s.len = s.len + 1
        s.checks.append((q.clone(), out.clone(), lse.clone(), new.clone(), s.K.clone(), s.V.clone(), s.key.clone(), [1] * B, s.table.copy(),
                         s.len.copy()))
        s.checks.append((b.table.clone(), s.table.copy(), s.free.clone(), PAGES - sum(-(-int(x) // P) for x in s.len.reshape(-1))))
    s.check()


def test_two_servers_at_once(l2):
    """Two streams, a cache and a workspace each."""
    servers, streams = [Server(l2, 4) for _ in range(2)], [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    for turn in range(8):
        for s, stream in zip(servers, streams):
            with torch.cuda.stream(stream):
                if turn == 0:
                    s.update([-1] * 4, [0] * 4, [50, 20, 90, 1])
                    s.tokens([50, 20, 90, 1])
                else:
                    s.update([0, 1, 2, 0] if turn == 3 else range(4), s.len[[0, 1, 2, 0]] if turn == 3 else s.len, [1] * 4)
                    s.tokens([1] * 4)
                    if turn == 5:
                        s.compact(s.len // 2)
    for s in servers:
        s.check()
