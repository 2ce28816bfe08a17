"""Caches in pages for the tests, and the tables that the calls on them have to make, in Python's integers."""
import numpy as np
import torch

from token_util import DEV, Case, i32


class Paged(Case):
    """A Case whose rows lie in the pages of a pool, in any order; NaN wherever no row is valid."""

    def __init__(self, l2, n, ctx, L, H, G, D, P, dtype="bf16", spare=5, entries=2, seed=0, **kw):
        super().__init__(l2, n, ctx, L, H, G, D, dtype, seed=seed, **kw)
        r = np.random.RandomState(seed + 77)
        self.P = P
        pages = -(-self.cur.max(-1) // P)
        cap = int(pages.max()) + entries
        self.n_pages = int(pages.sum()) + spare
        order = r.permutation(self.n_pages)
        self.table = np.full((self.B, L, cap), -1, np.int64)
        self.table[np.arange(cap) < pages[:, :, None]] = order[:pages.sum()]
        dense = self.K, self.V
        self.K, self.V = (torch.full((H, self.n_pages * P, D), float("nan"), dtype=self.dtype, device=DEV) for _ in range(2))
        for x, d in zip((self.K, self.V), dense):
            for b in range(self.B):
                for l in range(L):
                    at = self.at(b, l, int(self.cur[b, l].max()))
                    x[:, at] = d[b, l, :, :len(at)]
        self.meta = (H, self.n_pages * P)
        self.max_len = cap * P
        self.pages = l2.Pages(i32(self.table), P, self.n_pages)

    def at(self, b, l, rows):
        """Pool rows of the first `rows` rows of (b, l)."""
        t = np.arange(rows)
        return torch.from_numpy(self.table[b, l][t // self.P] * self.P + t % self.P).to(DEV)

    def unit(self, x, b, l, h):
        if x.dim() == 5:                                     # (the dense tensors it is made from)
            return x[b, l, h]
        return x[h, self.at(b, l, int(self.cur[b, l].max()))]


def held_pages(table, rows, P):
    """(b, l) -> pages below the length, as a list."""
    return {(b, l): [int(p) for p in table[b, l][:-(-int(rows[b, l]) // P)]] for b in range(table.shape[0]) for l in range(table.shape[1])}


def updated(table, P, n_pages, parent, keep, grow, pinned=()):
    """What page_update leaves: tables, room, pages free, copies (from page, to page, rows), whether anything went short."""
    B, L, cap = len(parent), table.shape[1], table.shape[2]
    keep = [[int(keep[b][l]) if parent[b] >= 0 else 0 for l in range(L)] for b in range(B)]
    old = {(b, l): [int(p) for p in table[max(parent[b], 0), l][:-(-keep[b][l] // P)]] for b in range(B) for l in range(L)}
    claims = {}
    for (b, l), pages in old.items():
        for j, p in enumerate(pages):
            claim = (min(P, keep[b][l] - j * P), -(b * L + l))
            claims[p] = max(claims.get(p, claim), claim)
    free = [p for p in range(n_pages) if p not in claims and p not in pinned]
    out, room, copies, short, wanted, given = np.full((B, L, cap), -1, np.int64), np.zeros((B, L), np.int64), [], False, 0, 0
    for b in range(B):
        for l in range(L):
            have, k = old[b, l], keep[b][l]
            out[b, l, :len(have)] = have
            room[b, l] = k
            if grow[b] <= 0:
                continue
            more = -(-(k + int(grow[b])) // P)
            if more > cap:
                short = True
                continue
            copy = k % P != 0 and (have[-1] in pinned or claims[have[-1]] != (k % P, -(b * L + l)))
            need = more - len(have) + copy
            wanted += need
            if need and wanted > len(free):
                short = True
                continue
            mine = free[wanted - need:wanted]
            given += need
            if copy:
                copies.append((have[-1], mine[0], k % P))
            out[b, l, len(have) - copy:more] = mine
            room[b, l] = more * P
    return out, room, len(free) - given, copies, short


def compacted(table, P, n_pages, lens, keep, pinned=()):
    """What page_compact leaves: tables, lengths, which (b, l) moved, whether anything went short."""
    B, L, cap = table.shape
    held = {p for pages in held_pages(table, lens, P).values() for p in pages}
    free = [p for p in range(n_pages) if p not in held and p not in pinned]
    out, after, moved, short, wanted = np.full((B, L, cap), -1, np.int64), np.array(lens), [], False, 0
    for b in range(B):
        for l in range(L):
            n = -(-int(lens[b, l]) // P)
            out[b, l, :n] = table[b, l, :n]
            if keep[b, l] >= lens[b, l]:
                continue
            need = -(-int(keep[b, l]) // P)
            wanted += need
            if need and wanted > len(free):
                short = True
                continue
            out[b, l] = -1
            out[b, l, :need] = free[wanted - need:wanted]
            after[b, l] = keep[b, l]
            moved.append((b, l))
    return out, after, moved, short
