"""The operators of a paged cache, and what is measured of them.

  attend   causal attention of packed new tokens (single tokens, chunks, whole prompts) over the pages of their sequences
  write    norms of queries and keys per head, rotary positions, and the write of keys and values into pages
  update   the page tables of the next step: sequences that go on, fork, give rows back or end, and room for new rows
           (with the copy of a page that several sequences hold and one of them is about to write)
  compact  the rows with the lowest key norms of every head, gathered into fresh pages

`run` computes them in a plain form (elementary torch operations in 32 bits, angles in 64), or, where `own` is set,
through the library.  A paged cache is [Hkv, n_pages * P, D]: row t of sequence b in layer l is row
table[b, l, t // P] * P + t % P, and what lies along the rows (position, ordering key) is [Hkv, n_pages * P].  New tokens
are packed: token i belongs to sequence b with tok_off[b] <= i < tok_off[b + 1].  A page is free where no table names it
below its sequence's length and it is not pinned; free pages are dealt out in ascending order, to (b, l) in ascending order."""
import math
import types

import numpy as np
import torch

own = False
DEV = "cuda"
_TYPES = {"bf16": torch.bfloat16, "fp32": torch.float32}
_workspace = {}


# ---- cases ---------------------------------------------------------------------------------------

def _case(name, op, B, L, Hkv, Hq, D, P, n_lo, n_hi, ctx_lo, ctx_hi, dtype="bf16", lens=1, **more):
    """n_lo..n_hi: new tokens per sequence; ctx_lo..ctx_hi: rows cached before them; P: rows of a page; lens: seed of the lengths."""
    c = dict(op=op, B=B, L=L, Hkv=Hkv, Hq=Hq, D=D, P=P, n_lo=n_lo, n_hi=n_hi, ctx_lo=ctx_lo, ctx_hi=ctx_hi, dtype=dtype, lens=lens)
    if op == "write":
        c.update(rot=D, interleaved=False, far=0, norm_q=True, norm_k=True, offset=0.0)
    if op == "update":
        c.update(parents=B, pinned=0.0)
    if op == "compact":
        c.update(keep=0.5, highest=False)
    c.update(more)
    return dict(c, name=name) if name else c


def listed():
    return [
        # one token of one sequence, one layer of an 8-billion-parameter model: all latency
        _case("attend-one-token", "attend", 1, 1, 8, 32, 128, 16, 1, 1, 2900, 2900),
        # a decode step of a serving batch, caches of very different lengths, small pages
        _case("attend-serving-tokens", "attend", 48, 1, 8, 32, 128, 16, 1, 1, 500, 16000),
        # a decode step over long caches: 64-wide heads in groups of eight
        _case("attend-long-64", "attend", 4, 1, 4, 32, 64, 32, 1, 1, 60000, 100000),
        # decode and prefill mixed in one step: chunks of up to 256 tokens next to a few of one
        _case("attend-mixed", "attend", 24, 1, 8, 32, 128, 64, 1, 256, 0, 6000),
        # a chunk of a long prompt behind what is cached of it
        _case("attend-chunk-32k", "attend", 1, 1, 8, 32, 128, 128, 8192, 8192, 24500, 24500),
        # new tokens of a decode step, one layer
        _case("write-tokens", "write", 48, 1, 8, 32, 128, 16, 1, 1, 100, 900, far=120000),
        # prompts of different lengths, one layer
        _case("write-prompts", "write", 8, 1, 8, 32, 128, 64, 100, 2500, 0, 300, far=4000),
        # one sequence takes its next page: all latency
        _case("update-one", "update", 1, 1, 8, 32, 128, 16, 1, 1, 800, 800),
        # a beam search over all layers: hypotheses fork, and copy the page that they go on writing
        _case("update-beams", "update", 16, 32, 8, 32, 128, 16, 1, 1, 700, 700, parents=5),
        # a serving step over all layers: most sequences go on, some fork from a shared prompt, some end
        _case("update-serving", "update", 64, 32, 2, 8, 64, 16, 1, 24, 200, 4000, parents=48, pinned=0.03),
        # one layer of one sequence down to half
        _case("compact-one", "compact", 1, 1, 8, 32, 128, 16, 1, 1, 8000, 8000),
        # eight layers of long sequences, down to half
        _case("compact-long", "compact", 4, 8, 8, 32, 128, 64, 1, 1, 20000, 32000),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["attend", "attend", "write", "update", "compact"])
    D, G, Hkv, P = rng.choice([64, 128]), rng.choice([1, 2, 4, 8]), rng.choice([1, 2, 4, 8]), rng.choice([16, 32, 64, 128, 256])
    a = dict(lens=rng.randrange(1 << 20), dtype=rng.choice(["bf16", "bf16", "bf16", "fp32"]))
    heads = (Hkv, Hkv * G, D, P)
    if op == "attend":
        if a["dtype"] == "fp32":     # the path for correctness: small calls
            return _case(None, op, _log(rng, 1, 6), 1, *heads, 1, _log(rng, 1, 300), 0, _log(rng, 16, 1000), **a)
        B, L = _log(rng, 1, 48), rng.choice([1, 1, 2])
        hi = 1 if rng.random() < 0.4 else _log(rng, 1, max(2, 6000 // B))
        return _case(None, op, B, L, *heads, rng.randint(1, hi), hi, 0, _log(rng, 16, 16000), **a)
    if op == "write":
        B, L = _log(rng, 1, 48), rng.choice([1, 1, 2])
        hi = _log(rng, 1, max(1, 8192 // (B * L)))
        return _case(None, op, B, L, *heads, rng.randint(1, hi), hi, 200, _log(rng, 200, 1000), rot=rng.choice([D, D, D // 2, 16]),
                     interleaved=rng.random() < 0.5, far=_log(rng, 1, 120000), norm_q=rng.random() < 0.8, norm_k=rng.random() < 0.8,
                     offset=rng.choice([0.0, 0.0, 1.0]), **a)
    if op == "update":
        B = _log(rng, 1, 64)
        return _case(None, op, B, _log(rng, 1, 32), rng.choice([1, 2]), 8, D, P, 0, _log(rng, 1, 100), 0, _log(rng, 16, 1500),
                     parents=rng.randint(1, B), pinned=rng.choice([0.0, 0.05]), **a)
    L = _log(rng, 1, 8)
    return _case(None, op, _log(rng, 1, max(1, 16 // L)), L, *heads, 1, 1, 0, _log(rng, 16, 16000), keep=rng.uniform(0.05, 1.0),
                 highest=rng.random() < 0.2, **a)


# ---- inputs --------------------------------------------------------------------------------------

def _lengths(c):
    """New tokens [B] and rows cached before them [B, L], from the case alone."""
    r = np.random.RandomState(c["lens"])
    n = r.randint(c["n_lo"], c["n_hi"] + 1, c["B"])
    # the layers of a sequence differ where some are compressed: up to an eighth
    ctx = r.randint(c["ctx_lo"], c["ctx_hi"] + 1, (c["B"], 1)) - r.randint(0, 1 + c["ctx_lo"] // 8, (c["B"], c["L"]))
    return n.astype(np.int64), ctx.astype(np.int64)


def _keeps(c):
    """Rows that survive a compaction, [B, L]."""
    _, ctx = _lengths(c)
    keep = np.ceil(c["keep"] * ctx).astype(np.int64)
    if c["L"] > 4:
        keep[:, :2] = ctx[:, :2]     # the first two layers stay whole
    return keep


def _next_step(c):
    """Parents [B], rows kept [B, L] and new tokens [B] of the next step's sequences."""
    r = np.random.RandomState(c["lens"] + 5)
    n, ctx = _lengths(c)
    B, m = c["B"], c["parents"]
    parent = np.arange(B)
    if m < B:                        # as many go on, the others fork from them or (one in eight) stay empty
        parent = np.concatenate([r.permutation(B)[:m], r.randint(0, m, B - m)])
        parent[m:] = np.where(r.rand(B - m) < 0.125, -1, parent[parent[m:]])
    keep = np.where(parent[:, None] >= 0, ctx[np.maximum(parent, 0)], 0)
    # some give rows back: rejected drafts
    keep = np.where((r.rand(B) < 0.2)[:, None], np.maximum(keep - r.randint(0, 9, B)[:, None], 0), keep)
    return parent, keep, np.where(parent >= 0, n, 0)


def _dev(a, dtype):
    return torch.from_numpy(np.ascontiguousarray(a)).to(DEV, dtype)


def prepare(case, seed):
    c = case
    B, L, H, Hq, D, P, op = (c[k] for k in ("B", "L", "Hkv", "Hq", "D", "P", "op"))
    dt = _TYPES[c["dtype"]]
    g = torch.Generator(device=DEV).manual_seed(seed)
    r = np.random.RandomState(seed % (1 << 31))

    def rows(*shape, per_channel=True):
        """Channels of a model's keys and values differ in scale, and so do tokens."""
        x = torch.randn(shape, generator=g, device=DEV, dtype=torch.float32 if op == "write" else dt)
        if per_channel:
            x *= (0.5 * torch.randn(shape[-1:], generator=g, device=DEV)).exp().to(x.dtype)
            x *= (0.2 * torch.randn((*shape[:-1], 1), generator=g, device=DEV)).exp().to(x.dtype)
        return x.to(dt)

    n, ctx = _lengths(c)
    N = int(n.sum())
    cur = ctx + n[:, None] if op in ("attend", "write") else ctx
    pages = -(-cur // P)
    # tables: pages anywhere in the pool, with some left free
    table_cap = int(pages.max()) + (2 + -(-c["n_hi"] // P) if op == "update" else 1)
    used = int(pages.sum())
    spare = used // 16 + (16 if op == "write" else 3)
    if op == "update":
        spare += B * L * (2 + -(-c["n_hi"] // P))
    if op == "compact":
        spare += int((-(-_keeps(c) // P)).sum())
    n_pages = used + spare
    free = r.permutation(n_pages)
    pinned, free = free[:int(c.get("pinned", 0) * spare)], free[int(c.get("pinned", 0) * spare):]
    table = np.full((B, L, table_cap), -1, np.int64)
    filled = np.arange(table_cap) < pages[:, :, None]
    table[filled] = free[:used]
    s = dict(op=op, B=B, L=L, H=H, Hq=Hq, D=D, N=N, P=P, n=n.tolist(), cur_host=cur.tolist(), cur_max=int(cur.max()))
    tok_off = np.concatenate([[0], np.cumsum(n)])
    s["tok_off"] = _dev(tok_off, torch.int32)
    s["start"], s["cur"] = _dev(ctx, torch.int32), _dev(cur, torch.int32)

    def tables(t):
        return types.SimpleNamespace(table=_dev(t, torch.int32), page_rows=P, n_pages=n_pages, room=None)

    s["pages"] = tables(table)
    if op != "attend":
        s["idx"] = torch.randint(0, 1 << 20, (H, n_pages * P), generator=g, device=DEV, dtype=torch.int32)
    s["K"], s["V"] = rows(H, n_pages * P, D), rows(H, n_pages * P, D)
    if op != "attend":
        s["sumsq"] = s["K"].float().square_().sum(-1)
    if op in ("update", "compact"):
        s["next"] = tables(np.full_like(table, -1))
        s["next"].room = torch.zeros((B, L), dtype=torch.int32, device=DEV)
        s["len_out"] = torch.zeros((B, L), dtype=torch.int32, device=DEV)
        s["n_free"] = torch.zeros(1, dtype=torch.int32, device=DEV)
    if op == "attend":
        s["q"] = rows(L, N, Hq, D, per_channel=False)
        s["out"] = torch.zeros((L, N, Hq, D), dtype=dt, device=DEV)
        s["lse"] = torch.zeros((L, N, Hq), device=DEV)
    if op == "write":
        # queries, keys and values of a fused projection: views of one [L, N, heads, D] tensor
        qkv = rows(L, N, Hq + 2 * H, D)
        s["q"], s["k"], s["v"] = qkv[:, :, :Hq], qkv[:, :, Hq:Hq + H], qkv[:, :, Hq + H:]
        first = r.randint(0, c["far"] + 1, B)
        s["pos"] = _dev(np.concatenate([first[b] + np.arange(n[b]) for b in range(B)]), torch.int32)
        s["freq"] = _dev(500000.0 ** (-2 * np.arange(c["rot"] // 2) / c["rot"]), torch.float64)
        s["interleaved"], s["norm_q"], s["norm_k"], s["offset"], s["eps"] = c["interleaved"], c["norm_q"], c["norm_k"], c["offset"], 1e-6
        s["q_weight"], s["k_weight"] = ((1 - c["offset"] + 0.3 * torch.randn(D, generator=g, device=DEV)).to(dt) for _ in range(2))
        s["q_out"] = torch.zeros((L, N, Hq, D), dtype=dt, device=DEV)
        s["out_len"] = torch.zeros((B, L), dtype=torch.int32, device=DEV)
    if op == "update":
        parent, keep, grow = _next_step(c)
        s["parent"], s["keep"], s["grow"] = _dev(parent, torch.int32), _dev(keep, torch.int32), _dev(grow, torch.int32)
        pin = np.zeros(n_pages, np.uint8)
        pin[pinned] = 1
        pin[table[0, 0, :int(pages[0, 0])][: 3]] = 1       # a prompt that a program keeps for later requests
        s["pin"] = _dev(pin, torch.uint8) if c["pinned"] else None
    if op == "compact":
        s["keep"], s["highest"] = _dev(_keeps(c), torch.int32), c["highest"]
    return s


# ---- the plain forms -----------------------------------------------------------------------------

def _row_index(s, b, l, count):
    """Pool rows of the first `count` rows of (b, l)."""
    P, t = s["P"], torch.arange(count, device=DEV)
    return s["pages"].table[b, l].long()[t // P] * P + t % P


def _plain_attend(s):
    L, H, Hq, D = s["L"], s["H"], s["Hq"], s["D"]
    G, first = Hq // H, 0
    for b, n in enumerate(s["n"]):
        q = s["q"][:, first:first + n].float().view(L, n, H, G, D).permute(0, 2, 3, 1, 4)      # [L, H, G, n, D]
        for l in range(L):
            T = s["cur_host"][b][l]
            at = _row_index(s, b, l, T)
            hidden = torch.arange(T, device=DEV) > T - n + torch.arange(n, device=DEV)[:, None]
            step = max(1, min(H, (1 << 29) // (G * n * T)))
            for h in range(0, H, step):
                K, V = (x[h:h + step].index_select(1, at).float()[:, None] for x in (s["K"], s["V"]))
                z = torch.matmul(q[l, h:h + step].reshape(-1, 1, G * n, D), K.transpose(-1, -2)).mul_(D ** -0.5).view(-1, G, n, T)
                if n > 1:
                    z.masked_fill_(hidden, -math.inf)
                top = z.amax(-1, keepdim=True)
                z.sub_(top).exp_()
                total = z.sum(-1, keepdim=True)
                o = torch.matmul(z.view(-1, 1, G * n, T), V).view(-1, G, n, D) / total
                s["out"][l, first:first + n].view(n, H, G, D)[:, h:h + step].copy_(o.permute(2, 0, 1, 3))
                s["lse"][l, first:first + n].view(n, H, G)[:, h:h + step].copy_((top + total.log()).squeeze(-1).permute(2, 0, 1))
        first += n
    return s["out"], s["lse"]


def _plain_write(s):
    L, H, P = s["L"], s["H"], s["P"]
    angle = (s["pos"].double()[:, None] * s["freq"])[:, None]
    cos, sin = angle.cos().float(), angle.sin().float()
    r = cos.shape[-1]

    def row(x, norm, weight):
        x = x.float()
        if norm:
            x = x / (x.square().mean(-1, keepdim=True) + s["eps"]).sqrt() * (weight.float() + s["offset"])
        if s["interleaved"]:
            a, b = x[..., 0:2 * r:2], x[..., 1:2 * r:2]
            y = torch.stack([a * cos - b * sin, b * cos + a * sin], -1).flatten(-2)
        else:
            a, b = x[..., :r], x[..., r:2 * r]
            y = torch.cat([a * cos - b * sin, b * cos + a * sin], -1)
        return torch.cat([y, x[..., 2 * r:]], -1)

    s["q_out"].copy_(row(s["q"], s["norm_q"], s["q_weight"]))
    k = row(s["k"], s["norm_k"], s["k_weight"]).to(s["K"].dtype)
    i = torch.arange(s["N"], device=DEV, dtype=torch.int32)
    b = torch.bucketize(i, s["tok_off"][1:], right=True)
    t = s["start"][b].long() + (i.long() - s["tok_off"][b].long())[:, None]                    # [N, L]
    page = s["pages"].table[b[:, None], torch.arange(L, device=DEV), t // P].long()
    at = (page * P + t % P).T                                                                  # [L, N]
    for x, y in ((s["K"], k), (s["V"], s["v"]), (s["idx"], s["pos"][None, :, None].expand(L, -1, H)), (s["sumsq"], k.float().square().sum(-1))):
        x.transpose(0, 1)[at] = y
    s["out_len"].copy_(s["start"] + (s["tok_off"][1:] - s["tok_off"][:-1])[:, None])
    return s["q_out"], s["K"], s["V"], s["idx"], s["sumsq"], s["out_len"]


def _deal(s, taken, need):
    """Free pages in ascending order, where each (b, l) of `need` pages begins in that order, and whether it gets them."""
    n_pages = s["pages"].n_pages
    free = ~taken
    rank = free.cumsum(0) - 1
    order = torch.zeros(n_pages + 1, dtype=torch.int64, device=DEV)
    order[torch.where(free, rank, n_pages)] = torch.arange(n_pages, device=DEV)
    upto = need.view(-1).cumsum(0).view(need.shape)
    return order, upto - need, (need == 0) | (upto <= free.sum())


def _plain_update(s):
    B, L, P, table, n_pages = s["B"], s["L"], s["P"], s["pages"].table.long(), s["pages"].n_pages
    cap = table.shape[2]
    parent, grow = s["parent"].long(), s["grow"].long()[:, None]
    keep = torch.where(parent[:, None] >= 0, s["keep"].long(), 0)
    old = table[parent.clamp(min=0)]
    j = torch.arange(cap, device=DEV)
    used = (keep[:, :, None] - j * P).clamp(0, P)
    # a page stays with whoever has most rows in it, the first of several
    claim = (used << 20) + ((1 << 20) - 1 - torch.arange(B * L, device=DEV)).view(B, L, 1)
    best = torch.zeros(n_pages, dtype=torch.int64, device=DEV)
    best.scatter_reduce_(0, old[used > 0], claim[used > 0], "amax")
    if s["pin"] is not None:
        best[s["pin"] != 0] = 1 << 40
    have, more = (keep + P - 1) // P, (keep + grow + P - 1) // P
    last = (have - 1).clamp(min=0)[:, :, None]
    shared = best[old.gather(2, last).clamp(min=0)] != claim.gather(2, last)
    copy = (grow > 0) & (keep % P != 0) & shared[:, :, 0]
    fits = (grow > 0) & (more <= cap)
    need = torch.where(fits, more - have + copy, 0)
    order, before, granted = _deal(s, best > 0, need)
    granted &= fits
    begin = have - copy.long()
    fresh = granted[:, :, None] & (j >= begin[:, :, None]) & (j < more[:, :, None])
    new = order[(before[:, :, None] + j - begin[:, :, None]).clamp(0, n_pages)]
    s["next"].table.copy_(torch.where(fresh, new, torch.where(used > 0, old, -1)))
    s["next"].room.copy_(torch.where(granted, more * P, keep))
    s["n_free"].copy_((best == 0).sum() - (need * granted).sum())
    copy &= granted
    src, dst = (t.gather(2, last)[:, :, 0][copy] for t in (old, s["next"].table.long()))
    some = torch.arange(P, device=DEV) < (keep % P)[copy][:, None]
    src, dst = ((t[:, None] * P + torch.arange(P, device=DEV))[some] for t in (src, dst))
    for x in (s["K"], s["V"], s["idx"], s["sumsq"]):
        x[:, dst] = x[:, src]
    return s["next"].table, s["next"].room, s["n_free"], s["K"], s["V"], s["idx"], s["sumsq"]


def _plain_compact(s):
    B, L, P, table, n_pages = s["B"], s["L"], s["P"], s["pages"].table.long(), s["pages"].n_pages
    cur, j = s["cur"].long(), torch.arange(table.shape[2], device=DEV)
    keep = torch.minimum(s["keep"].long(), cur)
    taken = torch.zeros(n_pages, dtype=torch.bool, device=DEV)
    held = j < ((cur + P - 1) // P)[:, :, None]
    taken[table[held]] = True
    need = torch.where(keep < cur, (keep + P - 1) // P, 0)
    order, before, granted = _deal(s, taken, need)
    granted &= keep < cur
    new = order[(before[:, :, None] + j).clamp(0, n_pages)]
    s["next"].table.copy_(torch.where(granted[:, :, None], torch.where(j < need[:, :, None], new, -1), torch.where(held, table, -1)))
    s["len_out"].copy_(torch.where(granted, keep, cur))
    s["next"].room.copy_(s["len_out"])
    # of all (b, l) at once, padded to the longest: keys in order, equal ones by row, and the first of them by row
    t = torch.arange(s["cur_max"], device=DEV)
    at = table[:, :, t // P] * P + t % P
    seen = t < cur[:, :, None]
    key = s["sumsq"][:, at.clamp(min=0)]                                                       # [H, B, L, T]
    key = (-key if s["highest"] else key).masked_fill_(~seen, math.inf)
    rank = torch.empty_like(key, dtype=torch.int64)
    rank.scatter_(3, torch.sort(key, dim=3, stable=True).indices, t.expand_as(key))
    kept = (rank < keep[:, :, None]) & seen & granted[:, :, None]
    to = kept.cumsum(3) - 1
    h, b, l, of = kept.nonzero(as_tuple=True)
    to = to[h, b, l, of]
    src, dst = at[b, l, of], s["next"].table.long()[b, l, to // P] * P + to % P
    for x in (s["K"], s["V"], s["idx"], s["sumsq"]):
        x[h, dst] = x[h, src]
    return s["next"].table, s["next"].room, s["len_out"], s["K"], s["V"], s["idx"], s["sumsq"]


# ---- one pass ------------------------------------------------------------------------------------

def _room(need):
    """The one workspace that a program keeps for these calls, zeroed when it is made."""
    if "ws" not in _workspace or _workspace["ws"].numel() < need:
        _workspace["ws"] = torch.zeros(need, dtype=torch.uint8, device=DEV)
    return _workspace["ws"]


def run(state):
    s = state
    if not own:
        return {"attend": _plain_attend, "write": _plain_write, "update": _plain_update, "compact": _plain_compact}[s["op"]](s)
    import paper_2406_11430_b200 as l2
    if s["op"] == "attend":
        ws = _room(l2.paged_attention_workspace_bytes(s["K"], s["q"], s["cur_max"], s["pages"]))
        l2.paged_attention(s["q"], s["tok_off"], s["K"], s["V"], s["cur"], s["cur_max"], s["out"], s["pages"], lse_out=s["lse"], workspace=ws)
        return s["out"], s["lse"]
    if s["op"] == "write":
        l2.norm_rotary_write(s["q"], s["k"], s["v"], s["tok_off"], s["pos"], s["freq"], s["q_out"], s["K"], s["V"], s["idx"], s["sumsq"],
                             s["start"], s["out_len"], _room(256), q_weight=s["q_weight"], k_weight=s["k_weight"], norm_q=s["norm_q"],
                             norm_k=s["norm_k"], eps=s["eps"], weight_offset=s["offset"], interleaved=s["interleaved"], pages=s["pages"])
        return s["q_out"], s["K"], s["V"], s["idx"], s["sumsq"], s["out_len"]
    ws = _room(l2.page_workspace_bytes(s["K"], s["pages"], s["cur_max"]))
    if s["op"] == "update":
        l2.page_update(s["K"], s["V"], s["idx"], s["sumsq"], s["pages"], s["parent"], s["keep"], s["grow"], s["next"], ws, pin=s["pin"],
                       n_free_out=s["n_free"])
        return s["next"].table, s["next"].room, s["n_free"], s["K"], s["V"], s["idx"], s["sumsq"]
    l2.page_compact(s["K"], s["V"], s["idx"], s["sumsq"], s["pages"], s["cur"], s["keep"], s["cur_max"], s["next"], s["len_out"], ws,
                    policy=l2.KEEP_HIGHEST_NORM if s["highest"] else l2.KEEP_LOWEST_NORM)
    return s["next"].table, s["next"].room, s["len_out"], s["K"], s["V"], s["idx"], s["sumsq"]


# ---- what a pass cannot do without ---------------------------------------------------------------

def work(case):
    c = case
    B, L, H, Hq, D, P = (c[k] for k in ("B", "L", "Hkv", "Hq", "D", "P"))
    e = 2 if c["dtype"] == "bf16" else 4
    n, ctx = _lengths(c)
    N = int(n.sum())
    if c["op"] == "attend":          # query s sees everything before it and itself
        pairs = sum(int(x) * int(m) + int(m) * (int(m) + 1) // 2 for m, r in zip(n, ctx) for x in r)
        cached = int((ctx + n[:, None]).sum())
        return {"bytes": L * N * Hq * (2 * D * e + 4) + 2 * cached * H * D * e + 4 * int((-(-(ctx + n[:, None]) // P)).sum()),
                "flops": 4 * pairs * Hq * D}
    if c["op"] == "write":           # queries in and out, keys and values in and to the cache, a position and a key per row
        return {"bytes": L * N * ((2 * Hq + 4 * H) * D * e + 8 * H + 4) + 4 * N, "flops": L * N * (Hq + H) * 8 * D}
    if c["op"] == "update":          # the old tables' pages, the new tables whole, and the rows of pages that are copied
        parent, keep, grow = _next_step(c)
        pages = -(-ctx // P)
        cap = int(pages.max()) + 2 + -(-c["n_hi"] // P)
        copied = 0                   # by those that grow and do not come first in their page
        for b in range(B):
            of = [o for o in range(B) if parent[o] == parent[b] and o != b]
            for k, ks in zip(keep[b], keep[of].T):
                used = np.clip(ks - k // P * P, 0, P)
                first = ~((used > k % P) | ((used == k % P) & (np.array(of, int) < b))).any()
                copied += 0 if grow[b] == 0 or first else int(k % P)
        return {"bytes": 4 * int((-(-keep // P)).sum()) + 4 * B * L * cap + copied * 2 * H * (2 * D * e + 8), "flops": 0}
    keep = _keeps(c)                 # every key of what is compacted, and the kept rows in and out
    moved = int(np.where(keep < ctx, keep, 0).sum())
    return {"bytes": 4 * H * int(np.where(keep < ctx, ctx, 0).sum()) + 2 * moved * H * (2 * D * e + 8), "flops": 0}


# ---- the definitions in 64 bits ------------------------------------------------------------------

def exact(case, seed):
    s = prepare(case, seed)
    n, ctx = _lengths(case)
    off = np.concatenate([[0], np.cumsum(n)])
    B, L, H, G, P, D = s["B"], s["L"], s["H"], s["Hq"] // s["H"], s["P"], s["D"]
    table = s["pages"].table.cpu().numpy().astype(np.int64)

    def rows_of(b, l, upto, t=table):
        """Pool rows of the first `upto` rows of (b, l), page by page."""
        all_rows = (t[b, l][:-(-int(upto) // P)][:, None] * P + np.arange(P)).reshape(-1)[:int(upto)]
        return torch.from_numpy(all_rows).to(DEV)

    if s["op"] == "attend":
        out = torch.zeros((L, s["N"], s["Hq"], D), dtype=torch.float64, device=DEV)
        lse = torch.zeros((L, s["N"], s["Hq"]), dtype=torch.float64, device=DEV)
        for b in range(B):
            m, of = int(n[b]), slice(int(off[b]), int(off[b + 1]))
            for l in range(L):
                end = int(ctx[b, l]) + m
                sees = torch.ones((m, end), dtype=torch.bool, device=DEV).tril(end - m)
                at = rows_of(b, l, end)
                for h in range(H):
                    K, V = s["K"][h, at].double(), s["V"][h, at].double()
                    for i in range(h * G, (h + 1) * G):
                        z = (s["q"][l, of, i].double() @ K.T / math.sqrt(D)).masked_fill_(~sees, -math.inf)
                        lse[l, of, i] = torch.logsumexp(z, -1)
                        out[l, of, i] = torch.softmax(z, -1) @ V
        return out, lse
    if s["op"] == "write":
        r = case["rot"] // 2
        turn = torch.polar(torch.ones((s["N"], r), dtype=torch.float64, device=DEV), s["pos"].double().outer(s["freq"]))[:, None]

        def row(x, norm, weight):
            y = x.double().clone()
            if norm:
                y *= torch.rsqrt((y * y).sum(-1, keepdim=True) / D + s["eps"])
                y *= weight.double() + s["offset"]
            a, b = (slice(0, 2 * r, 2), slice(1, 2 * r, 2)) if s["interleaved"] else (slice(0, r), slice(r, 2 * r))
            z = torch.complex(y[..., a], y[..., b]) * turn
            y[..., a], y[..., b] = z.real, z.imag
            return y

        k = row(s["k"], s["norm_k"], s["k_weight"])
        held = k.to(s["K"].dtype).double()                 # the ordering key is that of the stored row
        K, V, key = s["K"].double(), s["V"].double(), s["sumsq"].double()
        for b in range(B):
            of = slice(int(off[b]), int(off[b + 1]))
            for l in range(L):
                at = rows_of(b, l, ctx[b, l] + n[b])[int(ctx[b, l]):]
                K[:, at], V[:, at] = k[l, of].transpose(0, 1), s["v"][l, of].double().transpose(0, 1)
                key[:, at] = held[l, of].square().sum(-1).T
        return row(s["q"], s["norm_q"], s["q_weight"]), K, V, None, key, None
    # what moves is moved bit by bit, into pages that follow from the definition in Python's integers
    K, V, key = s["K"], s["V"], s["sumsq"].double()
    if s["op"] == "update":
        parent, keep, grow = _next_step(case)
        pinned = set() if s["pin"] is None else set(s["pin"].nonzero().flatten().tolist())
        holds, moves, wants = {}, [], []
        for b in range(B):
            for l in range(L):
                for j in range(-(-int(keep[b, l]) // P)):
                    p, rank = int(table[parent[b], l, j]), (min(P, int(keep[b, l]) - j * P), -(b * L + l))
                    holds[p] = max(holds.get(p, rank), rank)
        for b in range(B):
            for l in range(L):
                k, have, more = int(keep[b, l]), -(-int(keep[b, l]) // P), -(-int(keep[b, l] + grow[b]) // P)
                if grow[b] == 0 or more > table.shape[2]:
                    continue
                last = int(table[parent[b], l, have - 1]) if k % P else -1
                copies = last >= 0 and (last in pinned or holds[last][1] != -(b * L + l))
                wants.append((more - have + copies, last if copies else -1, k % P))
        free = [p for p in range(s["pages"].n_pages) if p not in holds and p not in pinned]
        at_free = 0                                        # (there are enough)
        for count, src, part in wants:
            if src >= 0:
                moves += [(src * P + t, free[at_free] * P + t) for t in range(part)]
            at_free += count
    else:
        keep, moves = _keeps(case), []
        held = set(int(p) for b in range(B) for l in range(L) for p in table[b, l][:-(-int(ctx[b, l]) // P)])
        free = [p for p in range(s["pages"].n_pages) if p not in held]
        K, V, key = K.clone(), V.clone(), key.clone()
        at_free = 0
        for b in range(B):
            for l in range(L):
                k, T = int(keep[b, l]), int(ctx[b, l])
                if k >= T:
                    continue
                mine = free[at_free:at_free + -(-k // P)]
                at_free += len(mine)
                old = rows_of(b, l, T)
                to = (torch.tensor(mine, dtype=torch.int64, device=DEV)[:, None] * P + torch.arange(P, device=DEV)).reshape(-1)[:k]
                for h in range(H):
                    x = s["sumsq"][h, old].double().cpu().numpy()
                    best = np.sort(np.lexsort((np.arange(T), -x if s["highest"] else x))[:k])
                    src = old[torch.from_numpy(best).to(DEV)]
                    K[h, to], V[h, to], key[h, to] = s["K"][h, src], s["V"][h, src], s["sumsq"][h, src].double()
        return None, None, None, K.double(), V.double(), None, key
    if moves:
        src, dst = (torch.tensor(x, dtype=torch.int64, device=DEV) for x in zip(*moves))
        K[:, dst], V[:, dst], key[:, dst] = K[:, src], V[:, src], key[:, src]
    return None, None, None, K.double(), V.double(), None, key
