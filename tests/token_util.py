"""Inputs and 64-bit references of the calls on packed new tokens."""
import numpy as np
import torch

DEV = "cuda:0"
DT = {"bf16": torch.bfloat16, "fp32": torch.float32}


def i32(x, device=DEV):
    return torch.tensor(np.asarray(x, dtype=np.int32), dtype=torch.int32, device=device)


class Case:
    """Caches with `ctx[b][l]` (or [b][l][h]) rows before the n[b] new tokens; NaN wherever no row is valid."""

    def __init__(self, l2, n, ctx, L, H, G, D, dtype="bf16", packed=False, seed=0, room=3, pad=0, strided=False,
                 per_head=False):
        self.l2, self.n, self.L, self.H, self.G, self.D, self.B = l2, list(n), L, H, G, D, len(n)
        self.dtype, self.per_head, self.Hq = DT[dtype], per_head, H * G
        g = torch.Generator().manual_seed(seed)
        rand = lambda *s: torch.randn(s, generator=g)  # noqa: E731
        ctx = np.asarray(ctx)
        self.ctx = ctx if ctx.ndim == 3 else np.repeat(ctx.reshape(self.B, L, 1), H, 2)
        self.cur = self.ctx + np.asarray(self.n).reshape(-1, 1, 1)
        self.N = sum(self.n) + pad
        self.off = np.concatenate([[0], np.cumsum(self.n)])
        self.tok_off = i32(self.off)
        cap = self.cur.max(-1) + room
        self.max_len, self.rows = int(cap.max()), None
        if packed:
            starts = np.concatenate([[0], np.cumsum(cap.reshape(-1))])
            total = int(starts[-1])
            self.rows = l2.Rows(starts[:-1].reshape(self.B, L), cap, total, DEV)
            K, V = (torch.full((total, H, D), float("nan")) for _ in range(2))
            self.row0 = starts[:-1].reshape(self.B, L)
            K, V = K.transpose(0, 1), V.transpose(0, 1)       # as a projection leaves them
            self.meta = (H, total)
        else:
            shape = (self.B, L, H, self.max_len, D)
            K, V = torch.full(shape, float("nan")), torch.full(shape, float("nan"))
            self.meta = shape[:4]
        scale = (0.5 * rand(D)).exp()
        for b in range(self.B):
            for l in range(L):
                for h in range(H):
                    m = int(self.cur[b, l, h])
                    self.unit(K, b, l, h)[:m] = rand(m, D) * scale
                    self.unit(V, b, l, h)[:m] = rand(m, D)
        keep = lambda t: t.transpose(0, 1).contiguous().to(DEV, self.dtype).transpose(0, 1) if packed else t.to(DEV, self.dtype)  # noqa: E731
        self.K, self.V = keep(K), keep(V)
        tok = rand(L, self.N, self.Hq + 2 * H, D).to(DEV, self.dtype)
        self.q, self.k, self.v = tok[:, :, :self.Hq], tok[:, :, self.Hq:-H], tok[:, :, -H:]
        if not strided:
            self.q, self.k, self.v = (t.contiguous() for t in (self.q, self.k, self.v))
        self.lens = lambda a: i32(a if per_head else a[:, :, 0])

    def unit(self, x, b, l, h):
        """The rows (or per-row entries) of one (b, l, h)."""
        if self.rows is None:
            return x[b, l, h]
        o = int(self.row0[b, l])
        return x[h, o:o + int(self.cap(b, l))]

    def cap(self, b, l):
        return self.cur[b, l].max() + 3 if self.rows is not None else self.max_len

    def empty_out(self, fill=7.0):
        return torch.full((self.L, self.N, self.Hq, self.D), fill, dtype=self.dtype, device=DEV)


def causal(case):
    return [torch.tril(torch.ones((m, m), dtype=torch.bool)) for m in case.n]


def random_trees(case, seed):
    """Ancestors and self; several roots, and one token that sees nothing of the tail."""
    r = np.random.RandomState(seed)
    trees = []
    for m in case.n:
        a = np.zeros((m, m), bool)
        for j in range(m):
            parent = r.randint(-1, j) if j else -1
            if parent >= 0:
                a[j] = a[parent]
            a[j, j] = True
        if m > 2:
            a[m // 2] = False
        trees.append(torch.from_numpy(a))
    return trees


def mask_words(case, trees, words=None):
    words = words or max(1, -(-max(case.n + [1]) // 64))
    w = np.zeros((case.N, words), np.uint64)
    for b, t in enumerate(trees):
        a = t.numpy()
        for j in range(min(a.shape[1], 64 * words)):
            w[case.off[b]:case.off[b + 1], j // 64] |= a[:, j].astype(np.uint64) << np.uint64(j % 64)
    return torch.from_numpy(w.view(np.int64)).to(DEV)


def check_attention(case, out, lse, trees, scale=None):
    """out and lse against the definition in 64 bits.  Error bound, element-wise, from how the result is
    formed: every weight is rounded to bf16 (at most 2^-8 of it; fp32 caches: none), a score is an fp32
    sum of D products in any order (at most D 2^-24 sum|q k| off, and its weight by as much; the scale's
    product and the exponential's argument add a few 2^-24 of the score), the sums over T rows
    lose at most T 2^-24 in each of numerator and denominator, and the result is rounded once (2^-8 of it)."""
    D, G = case.D, case.G
    scale = D ** -0.5 if scale is None else scale
    bf16 = case.dtype == torch.bfloat16
    half = 2.0 ** -8 if bf16 else 2.0 ** -24
    worst = 0.0
    for b in range(case.B):
        m, of = case.n[b], slice(int(case.off[b]), int(case.off[b + 1]))
        if m == 0:
            continue
        for l in range(case.L):
            for h in range(case.H):
                cur = int(case.cur[b, l, h])
                K = case.unit(case.K, b, l, h)[:cur].double()
                V = case.unit(case.V, b, l, h)[:cur].double()
                sees = torch.cat([torch.ones((m, cur - m), dtype=torch.bool), trees[b]], 1).to(DEV)
                for j in range(h * G, (h + 1) * G):
                    q = case.q[l, of, j].double()
                    z = (q @ K.T * scale).masked_fill(~sees, -torch.inf)
                    size = ((q.abs() @ K.abs().T) * abs(scale)).masked_fill(~sees, 0).amax(-1)
                    top = z.amax(-1, keepdim=True).clamp(min=-1e300)
                    w = (z - top).exp()
                    total = w.sum(-1, keepdim=True)
                    w = w / total.clamp(min=1e-300)
                    want, spread = w @ V, w @ V.abs()
                    e_score = size * (D + 8) * 2.0 ** -24
                    rel = (2.0 ** -8 if bf16 else 0.0) + 2 * e_score + (2 * cur + 16) * 2.0 ** -24 + 2.0 ** -20
                    bound = rel[:, None] * spread * 1.01 + half * want.abs() * 1.01 + 1e-30
                    got = out[l, of, j].double()
                    assert torch.isfinite(got).all()
                    excess = ((got - want).abs() / bound).max().item()
                    worst = max(worst, excess)
                    assert excess <= 1.0, f"b {b} l {l} head {j}: {excess:.3f} of the bound"
                    if lse is not None:
                        ref = (top + total.log()).squeeze(-1)
                        seen = sees.any(-1)
                        g = lse[l, of, j].double()
                        assert torch.isneginf(g[~seen]).all() and not out[l, of, j][~seen].any()
                        e = e_score + (cur + 16) * 2.0 ** -24 + 4 * ref.abs() * 2.0 ** -24 + 2.0 ** -20
                        assert ((g - ref).abs() <= e)[seen].all()
    return worst
