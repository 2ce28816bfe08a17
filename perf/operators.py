"""The operators that put new tokens of a model next to its compressed KV cache, and what is measured of them.

  rotary   rotary positions of the queries and keys of new tokens; keys and values written to their cache rows
           together with the row's position and ordering key
  prompt   causal attention of packed prompts of different lengths over their cached rows
  tree     attention of a tree of drafted tokens over a cache
  commit   the accepted path of a tree moved down to the end of the committed rows

`run` computes them in a plain form (elementary torch operations in 32 bits, angles in 64), or, where `own` is set,
through the library.  Sequences are packed: token i of the call belongs to sequence b with
tok_off[b] <= i < tok_off[b + 1].  Caches are [B, L, Hkv, t_cap, D] or packed [Hkv, total_rows, D]."""
import math
import types

import numpy as np
import torch

own = False
DEV = "cuda"
_TYPES = {"bf16": torch.bfloat16, "fp32": torch.float32}
_workspace = {}


# ---- cases ---------------------------------------------------------------------------------------

def _case(name, op, B, L, Hkv, Hq, D, n_lo, n_hi, ctx_lo=0, ctx_hi=0, dtype="bf16", packed=False, lens=1, rot=0,
          interleaved=False, scaling="none", far=0, path_hi=0):
    """n_lo..n_hi: new tokens per sequence; ctx_lo..ctx_hi: rows cached before them; lens: seed of both."""
    c = dict(op=op, B=B, L=L, Hkv=Hkv, Hq=Hq, D=D, n_lo=n_lo, n_hi=n_hi, ctx_lo=ctx_lo, ctx_hi=ctx_hi, dtype=dtype,
             packed=packed, lens=lens)
    if op == "rotary":
        c.update(rot=rot or D, interleaved=interleaved, scaling=scaling, far=far)
    if op == "commit":
        c.update(path_hi=path_hi)
    return dict(c, name=name) if name else c


def listed():
    return [
        # one token of one sequence, one layer of an 8-billion-parameter model: a decode step's call, all latency
        _case("rotary-one-token", "rotary", 1, 1, 8, 32, 128, 1, 1, 4000, 4000, far=120000, scaling="llama3"),
        # the prompts of a serving batch, 32 k tokens in all, one layer: memory traffic
        _case("rotary-prompts-32k", "rotary", 4, 1, 8, 32, 128, 4096, 12288, 0, 0, scaling="llama3"),
        # fp32 caches, interleaved pairs in half of a 64-wide head, odd lengths, two layers
        _case("rotary-fp32-partial", "rotary", 7, 2, 8, 8, 64, 3, 611, 0, 100, dtype="fp32", rot=32, interleaved=True,
              scaling="yarn", far=5000),
        # a few short prompts, no head groups: latency
        _case("prompt-short", "prompt", 3, 1, 32, 32, 128, 1, 77),
        # prompts of a serving batch as the projection leaves them: packed, 1 to 2048 tokens
        _case("prompt-ragged-packed", "prompt", 24, 1, 8, 32, 128, 1, 2048, packed=True),
        # one long document
        _case("prompt-16k", "prompt", 1, 1, 8, 32, 128, 16384, 16384),
        # a chunk of a longer prompt: 64-wide heads in groups of eight, rows already cached before it
        _case("prompt-chunk-64", "prompt", 2, 1, 4, 32, 64, 1100, 1500, 5000, 7000),
        # five drafted tokens of one sequence over a short cache: latency
        _case("tree-small", "tree", 1, 1, 8, 32, 128, 5, 5, 700, 700),
        # a serving batch of small trees, caches of very different lengths
        _case("tree-serving", "tree", 16, 1, 8, 32, 128, 12, 24, 1024, 16384),
        # wide trees over long caches, two layers at once
        _case("tree-32k", "tree", 4, 2, 8, 32, 128, 64, 64, 32700, 32700),
        # one sequence's accepted path: latency
        _case("commit-one", "commit", 1, 1, 8, 32, 128, 16, 16, 60, 60, path_hi=5),
        # the accepted paths of a serving batch, eight layers at once
        _case("commit-serving", "commit", 64, 8, 8, 32, 128, 24, 48, 10, 40, path_hi=9),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["rotary", "prompt", "tree", "commit"])
    D = rng.choice([64, 128])
    G = rng.choice([1, 2, 4, 8])
    Hkv = rng.choice([2, 4, 8])
    lens, packed = rng.randrange(1 << 20), rng.random() < 0.4
    if op == "rotary":
        B, L = _log(rng, 1, 32), rng.choice([1, 1, 2])
        hi = _log(rng, 1, 16384 // (B * L)) if B * L < 8192 else 1
        return _case(None, op, B, L, Hkv, Hkv * G, D, rng.randint(1, hi), hi, 0, _log(rng, 1, 300), lens=lens, packed=packed,
                     dtype=rng.choice(["bf16", "bf16", "fp32"]), rot=rng.choice([D, D, D // 2, 16]),
                     interleaved=rng.random() < 0.5, scaling=rng.choice(["none", "linear", "llama3", "yarn"]),
                     far=_log(rng, 1, 120000))
    if op == "prompt":
        B = _log(rng, 1, 24)
        hi = _log(rng, 1, 2000 if B > 8 else 4000)
        return _case(None, op, B, 1, Hkv, Hkv * G, D, rng.randint(1, hi), hi, 0, _log(rng, 1, 1500), lens=lens, packed=packed)
    if op == "tree":
        B, L = _log(rng, 1, 16), rng.choice([1, 1, 2])
        hi = _log(rng, 1, 100)
        return _case(None, op, B, L, Hkv, Hkv * G, D, rng.randint(1, hi), hi, 0, _log(rng, 16, 16000), lens=lens, packed=packed)
    hi = _log(rng, 1, 60)
    return _case(None, op, _log(rng, 1, 64), rng.choice([1, 2, 8]), Hkv, Hkv * G, D, rng.randint(1, hi), hi, 0, _log(rng, 1, 40),
                 lens=lens, packed=packed, dtype=rng.choice(["bf16", "bf16", "fp32"]), path_hi=rng.randint(1, 12))


# ---- inputs --------------------------------------------------------------------------------------

def _lengths(c):
    """New tokens [B] and rows cached before them [B, L], from the case alone."""
    r = np.random.RandomState(c["lens"])
    n = r.randint(c["n_lo"], c["n_hi"] + 1, c["B"])
    ctx = r.randint(c["ctx_lo"], c["ctx_hi"] + 1, (c["B"], c["L"]))
    return n.astype(np.int64), ctx.astype(np.int64)


def _trees(c, n):
    """Per sequence: depths and the ancestors (and self) of every drafted token; parents come before their children."""
    r = np.random.RandomState(c["lens"] + 7)
    depth, sees = [], []
    for nodes in n:
        d, a = np.zeros(nodes, np.int64), np.zeros((nodes, nodes), bool)
        for j in range(nodes):
            parent = r.randint(-1, j) if j < 4 else r.randint(j // 3, j)
            if parent >= 0:
                d[j], a[j] = d[parent] + 1, a[parent]
            a[j, j] = True
        depth.append(d)
        sees.append(a)
    return depth, sees


def frequencies(rot, scaling):
    """Radians per position of each pair, and the factor on cosine and sine, for the usual long-context scalings."""
    i = np.arange(rot // 2, dtype=np.float64)
    if scaling == "llama3":          # low frequencies divided by 8, a ramp between wavelengths 2048 and 8192
        f = 500000.0 ** (-2 * i / rot)
        wave = 2 * np.pi / f
        keep = np.clip((8192.0 / wave - 1.0) / (4.0 - 1.0), 0, 1)
        return f * keep + f / 8.0 * (1 - keep), 1.0
    f = 10000.0 ** (-2 * i / rot)
    if scaling == "linear":          # positions four times closer
        return f / 4.0, 1.0
    if scaling == "yarn":            # as llama3 over the pair's index, and a temperature
        at = lambda turns: rot * math.log(4096 / (turns * 2 * math.pi)) / (2 * math.log(10000.0))  # noqa: E731
        lo, hi = max(math.floor(at(32)), 0), min(math.ceil(at(1)), rot - 1)
        keep = 1 - np.clip((i - lo) / max(hi - lo, 1e-3), 0, 1)
        return f * keep + f / 16.0 * (1 - keep), 0.1 * math.log(16.0) + 1.0
    return f, 1.0


def _dev(a, dtype):
    return torch.from_numpy(np.ascontiguousarray(a)).to(DEV, dtype)


def prepare(case, seed):
    c = case
    B, L, H, Hq, D = c["B"], c["L"], c["Hkv"], c["Hq"], c["D"]
    dt = _TYPES[c["dtype"]]
    g = torch.Generator(device=DEV).manual_seed(seed)

    def rows(*shape, per_channel=True):
        x = torch.randn(shape, generator=g, device=DEV)
        if per_channel:              # channels of a model's keys and values differ in scale
            x = x * (0.5 * torch.randn(shape[-2:], generator=g, device=DEV)).exp()
        return x.to(dt)

    n, ctx = _lengths(c)
    N = int(n.sum())
    cur = ctx + n[:, None]
    s = dict(op=c["op"], B=B, L=L, H=H, Hq=Hq, D=D, N=N, n_max=int(n.max()), ctx_max=int(cur.max()), rows=None)
    tok_off = np.concatenate([[0], np.cumsum(n)])
    s["tok_off"] = _dev(tok_off, torch.int32)
    s["start"], s["cur"] = _dev(ctx, torch.int32), _dev(cur, torch.int32)
    cap = cur + 3                    # room that stays free behind every sequence's rows
    t_cap = int(cap.max())
    if c["packed"]:
        off = np.concatenate([[0], np.cumsum(cap.reshape(-1))])
        total = int(off[-1])
        s["rows"] = types.SimpleNamespace(B=B, L=L, total_rows=total, t_cap=t_cap, off=_dev(off[:-1].reshape(B, L), torch.int64),
                                          cap=_dev(cap, torch.int32))
        # as a projection leaves them: [row, head, D]
        s["K"], s["V"] = rows(total, H, D).transpose(0, 1), rows(total, H, D).transpose(0, 1)
        meta = (H, total)
    else:
        s["K"], s["V"] = (rows(B, L, t_cap, H, D).permute(0, 1, 3, 2, 4).contiguous() for _ in range(2))
        meta = (B, L, H, t_cap)
    if c["op"] in ("rotary", "commit"):
        s["idx"] = torch.randint(0, 1 << 20, meta, generator=g, device=DEV, dtype=torch.int32)
        s["sumsq"] = torch.rand(meta, generator=g, device=DEV)
        s["out_len"] = torch.zeros((B, L), dtype=torch.int32, device=DEV)
    if c["op"] == "rotary":
        # queries, keys and values of a fused projection: views of one [L, N, heads, D] tensor
        qkv = rows(L, N, Hq + 2 * H, D)
        s["q"], s["k"], s["v"] = qkv[:, :, :Hq], qkv[:, :, Hq:Hq + H], qkv[:, :, Hq + H:]
        first = np.random.RandomState(seed % (1 << 31)).randint(0, c["far"] + 1, B)
        s["pos"] = _dev(np.concatenate([first[b] + np.arange(n[b]) for b in range(B)]), torch.int32)
        f, s["attn_scale"] = frequencies(c["rot"], c["scaling"])
        s["freq"], s["interleaved"] = _dev(f, torch.float64), c["interleaved"]
        s["q_out"] = torch.zeros((L, N, Hq, D), dtype=dt, device=DEV)
    if c["op"] in ("prompt", "tree"):
        s["q"] = rows(L, N, Hq, D, per_channel=False)
        s["out"] = torch.zeros((L, N, Hq, D), dtype=dt, device=DEV)
        s["lse"] = torch.zeros((L, N, Hq), device=DEV)
    if c["op"] == "tree":
        words = -(-int(n.max()) // 64)
        w = np.zeros((N, words), np.uint64)
        for b, a in enumerate(_trees(c, n)[1]):
            for j in range(a.shape[1]):
                w[tok_off[b]:tok_off[b + 1], j // 64] |= a[:, j].astype(np.uint64) << np.uint64(j % 64)
        s["mask"] = _dev(w.view(np.int64), torch.int64)
    if c["op"] == "commit":
        r = np.random.RandomState((seed + 3) % (1 << 31))
        take = np.minimum(r.randint(0, c["path_hi"] + 1, B), n)
        path = np.full((B, c["path_hi"]), -1, np.int64)
        for b in range(B):
            path[b, :take[b]] = np.sort(r.permutation(n[b])[:take[b]])
        s["path"], s["n_path"] = _dev(path, torch.int32), _dev(take, torch.int32)
    return s


# ---- the plain forms -----------------------------------------------------------------------------

def _token_index(s):
    """Sequence and place within it of every new token."""
    i = torch.arange(s["N"], device=DEV, dtype=torch.int32)
    b = torch.bucketize(i, s["tok_off"][1:], right=True)
    return b, i.long() - s["tok_off"][b].long()


def _cache_rows(s, x, b, l, t):
    """Index of rows t of (b, l), all heads, in a cache-shaped tensor x: x[index] is [..., H, ...]."""
    if s["rows"] is not None:
        return x.transpose(0, 1), (s["rows"].off[b, l] + t,)
    return x.transpose(2, 3), (b, l, t)


def _rotate(s, x, cos, sin):
    r = cos.shape[-1]
    x = x.float()
    if s["interleaved"]:
        a, b = x[..., 0:2 * r:2], x[..., 1:2 * r:2]
        y = torch.stack([a * cos - b * sin, b * cos + a * sin], -1).flatten(-2)
    else:
        a, b = x[..., :r], x[..., r:2 * r]
        y = torch.cat([a * cos - b * sin, b * cos + a * sin], -1)
    return torch.cat([y, x[..., 2 * r:]], -1)


def _plain_rotary(s):
    angle = s["pos"].double()[:, None] * s["freq"]
    cos, sin = ((f(angle) * s["attn_scale"]).float()[:, None] for f in (torch.cos, torch.sin))
    s["q_out"].copy_(_rotate(s, s["q"], cos, sin))
    k = _rotate(s, s["k"], cos, sin).to(s["K"].dtype)
    b, at = _token_index(s)
    b, l = b[None], torch.arange(s["L"], device=DEV)[:, None]
    t = s["start"][b, l].long() + at
    for x, y in ((s["K"], k), (s["V"], s["v"]), (s["idx"], s["pos"][None, :, None].expand(s["L"], -1, s["H"])),
                 (s["sumsq"], k.float().square().sum(-1))):
        view, index = _cache_rows(s, x, b, l, t)
        view[index] = y
    n = s["tok_off"][1:] - s["tok_off"][:-1]
    s["out_len"].copy_(s["start"] + n[:, None])
    return s["q_out"], s["K"], s["V"], s["idx"], s["sumsq"], s["out_len"]


def _plain_attention(s):
    B, L, H, Hq, D, n_max, T = (s[k] for k in ("B", "L", "H", "Hq", "D", "n_max", "ctx_max"))
    G = Hq // H
    bl = torch.arange(B, device=DEV)[:, None, None], torch.arange(L, device=DEV)[:, None]
    t = torch.arange(T, device=DEV)
    if s["rows"] is not None:        # rows behind a sequence's own are clamped into the tensor, and masked
        at = (s["rows"].off[:, :, None] + t).clamp(max=s["rows"].total_rows - 1)
        K, V = (x[:, at].permute(1, 2, 0, 3, 4).float() for x in (s["K"], s["V"]))
    else:
        K, V = (x[:, :, :, :T].float() for x in (s["K"], s["V"]))
    n = (s["tok_off"][1:] - s["tok_off"][:-1]).long()
    at = torch.arange(n_max, device=DEV)
    i = (s["tok_off"][:-1, None] + at).clamp(max=s["N"] - 1)
    q = s["q"][:, i].permute(1, 0, 3, 2, 4).reshape(B, L, H, G * n_max, D).float()
    score = torch.matmul(q, K.transpose(-1, -2)).mul_(D ** -0.5)
    base = (s["cur"].long() - n[:, None])[:, :, None, None]
    if s["op"] == "prompt":
        sees = t <= base + at[:, None]
    else:
        col = t - base               # which drafted token's row this is
        own_row = col.clamp(0, n_max - 1)
        word = torch.gather(s["mask"][i][:, None].expand(-1, L, -1, -1), 3, (own_row // 64).expand(-1, -1, n_max, -1))
        sees = (col < 0) | ((((word >> (own_row % 64)) & 1) != 0) & (col < n_max))
    sees = sees & (t < s["cur"].long()[:, :, None, None])
    score = score.view(B, L, H, G, n_max, T).masked_fill_(~sees[:, :, None, None], -math.inf)
    top = score.amax(-1, keepdim=True)
    score.sub_(top.clamp(min=-1e30)).exp_()
    total = score.sum(-1, keepdim=True)
    V = V * (t < s["cur"][:, :, None])[:, :, None, :, None]
    out = torch.matmul(score.view(B, L, H, G * n_max, T), V).view(B, L, H, G, n_max, D) / total.clamp(min=1e-30)
    b, at = _token_index(s)
    s["out"].copy_(out.permute(0, 4, 1, 2, 3, 5).reshape(B, n_max, L, Hq, D)[b, at].transpose(0, 1))
    lse = (top + total.log()).squeeze(-1)
    s["lse"].copy_(lse.permute(0, 4, 1, 2, 3).reshape(B, n_max, L, Hq)[b, at].transpose(0, 1))
    return s["out"], s["lse"]


def _plain_commit(s):
    P = s["path"].shape[1]
    j = torch.arange(P, device=DEV)
    taken = (j < s["n_path"][:, None])[:, None].expand(-1, s["L"], -1)
    b, l, j = (x.expand(s["B"], s["L"], P)[taken] for x in (torch.arange(s["B"], device=DEV)[:, None, None],
                                                           torch.arange(s["L"], device=DEV)[:, None], j))
    first = s["start"][b, l].long()
    src, dst = first + s["path"][b, j], first + j
    for x in (s["K"], s["V"], s["idx"], s["sumsq"]):
        view, at = _cache_rows(s, x, b, l, src)
        moved = view[at]
        view, at = _cache_rows(s, x, b, l, dst)
        view[at] = moved
    s["out_len"].copy_(s["start"] + s["n_path"][:, None])
    return s["K"], s["V"], s["idx"], s["sumsq"], s["out_len"]


# ---- one pass ------------------------------------------------------------------------------------

def _room(need):
    """The one workspace that a program keeps for these calls, zeroed when it is made."""
    if "ws" not in _workspace or _workspace["ws"].numel() < need:
        _workspace["ws"] = torch.zeros(need, dtype=torch.uint8, device=DEV)
    return _workspace["ws"]


def run(state):
    s = state
    if not own:
        return {"rotary": _plain_rotary, "prompt": _plain_attention, "tree": _plain_attention, "commit": _plain_commit}[s["op"]](s)
    import paper_2406_11430_b200 as l2
    if s["op"] == "rotary":
        l2.rotary_write(s["q"], s["k"], s["v"], s["tok_off"], s["pos"], s["freq"], s["q_out"], s["K"], s["V"], s["idx"], s["sumsq"],
                        s["start"], s["out_len"], _room(256), interleaved=s["interleaved"], attn_scale=s["attn_scale"], rows=s["rows"])
        return s["q_out"], s["K"], s["V"], s["idx"], s["sumsq"], s["out_len"]
    if s["op"] == "commit":
        l2.tree_commit(s["K"], s["V"], s["idx"], s["sumsq"], s["start"], s["cur"], s["path"], s["n_path"], s["out_len"], _room(256),
                       rows=s["rows"])
        return s["K"], s["V"], s["idx"], s["sumsq"], s["out_len"]
    ws = _room(l2.prompt_attention_workspace_bytes(s["K"], s["q"], s["ctx_max"], rows=s["rows"]))
    if s["op"] == "prompt":
        l2.prompt_attention(s["q"], s["tok_off"], s["K"], s["V"], s["cur"], s["ctx_max"], s["out"], lse_out=s["lse"], workspace=ws,
                            rows=s["rows"])
    else:
        l2.tree_attention(s["q"], s["tok_off"], s["mask"], s["K"], s["V"], s["cur"], s["ctx_max"], s["out"], lse_out=s["lse"],
                          workspace=ws, rows=s["rows"])
    return s["out"], s["lse"]


# ---- what a pass cannot do without ---------------------------------------------------------------

def work(case):
    c = case
    L, H, Hq, D = c["L"], c["Hkv"], c["Hq"], c["D"]
    e = 2 if c["dtype"] == "bf16" else 4
    n, ctx = _lengths(c)
    N = int(n.sum())
    if c["op"] == "rotary":          # queries in and out, keys and values in and to the cache, a position and a key per row
        return {"bytes": L * N * ((2 * Hq + 4 * H) * D * e + 8 * H) + 4 * N, "flops": L * N * ((Hq + H) * 3 * c["rot"] + 2 * H * D)}
    if c["op"] == "commit":          # half of the longest path on average
        rows = c["B"] * L * H * c["path_hi"] / 2
        return {"bytes": rows * (4 * D * e + 16), "flops": 0}
    if c["op"] == "prompt":          # query s sees everything before it and itself
        pairs = sum(int(x) * int(m) + int(m) * (int(m) + 1) // 2 for m, r in zip(n, ctx) for x in r)
    else:
        seen = [int(a.sum()) for a in _trees(c, n)[1]]
        pairs = sum(int(x) * int(m) + a for m, r, a in zip(n, ctx, seen) for x in r)
    cached = int((ctx + n[:, None]).sum())
    return {"bytes": L * N * Hq * (2 * D * e + 4) + 2 * cached * H * D * e, "flops": 4 * pairs * Hq * D}


# ---- the definitions in 64 bits ------------------------------------------------------------------

def _unit(s, x, b, l, h):
    """Rows of one (b, l, h) of a cache-shaped tensor, as a view."""
    if s["rows"] is None:
        return x[b, l, h]
    o = int(s["rows"].off[b, l])
    return x[h, o:o + int(s["rows"].cap[b, l])]


def exact(case, seed):
    s = prepare(case, seed)
    n, ctx = _lengths(case)
    off = np.concatenate([[0], np.cumsum(n)])
    B, L, H, G = s["B"], s["L"], s["H"], s["Hq"] // s["H"]
    if s["op"] == "rotary":
        r = case["rot"] // 2
        turn = torch.polar(torch.full((s["N"], r), float(s["attn_scale"]), dtype=torch.float64, device=DEV),
                           s["pos"].double().outer(s["freq"]))[:, None]

        def rotated(x):
            y = x.double().clone()
            even, odd = (slice(0, 2 * r, 2), slice(1, 2 * r, 2)) if case["interleaved"] else (slice(0, r), slice(r, 2 * r))
            z = torch.complex(y[..., even], y[..., odd]) * turn
            y[..., even], y[..., odd] = z.real, z.imag
            return y

        k = rotated(s["k"])
        held = k.to(s["K"].dtype).double()      # the ordering key is that of the stored row
        K, V, key = s["K"].double(), s["V"].double(), s["sumsq"].double()
        for b in range(B):
            for l in range(L):
                to = slice(int(ctx[b, l]), int(ctx[b, l] + n[b]))
                of = slice(int(off[b]), int(off[b + 1]))
                for h in range(H):
                    _unit(s, K, b, l, h)[to] = k[l, of, h]
                    _unit(s, V, b, l, h)[to] = s["v"][l, of, h].double()
                    _unit(s, key, b, l, h)[to] = held[l, of, h].square().sum(-1)
        return rotated(s["q"]), K, V, None, key, None
    if s["op"] == "commit":
        return _moved(s, ctx)
    sees_of = _trees(case, n)[1] if s["op"] == "tree" else None
    out = torch.zeros((L, s["N"], s["Hq"], s["D"]), dtype=torch.float64, device=DEV)
    lse = torch.zeros((L, s["N"], s["Hq"]), dtype=torch.float64, device=DEV)
    for b in range(B):
        of = slice(int(off[b]), int(off[b + 1]))
        m = int(n[b])
        tail = torch.tril(torch.ones((m, m), dtype=torch.bool, device=DEV)) if sees_of is None else torch.from_numpy(sees_of[b]).to(DEV)
        for l in range(L):
            end = int(ctx[b, l]) + m
            hidden = ~torch.cat([torch.ones((m, end - m), dtype=torch.bool, device=DEV), tail], 1)
            for h in range(H):
                K, V = _unit(s, s["K"], b, l, h)[:end].double(), _unit(s, s["V"], b, l, h)[:end].double()
                for j in range(h * G, (h + 1) * G):
                    z = (s["q"][l, of, j].double() @ K.T / math.sqrt(s["D"])).masked_fill_(hidden, -math.inf)
                    lse[l, of, j] = torch.logsumexp(z, -1)
                    out[l, of, j] = z.sub_(lse[l, of, j][:, None]).exp_() @ V
    return out, lse


def _moved(s, ctx):
    K, V, key = s["K"].double(), s["V"].double(), s["sumsq"].double()
    path, n_path = s["path"].tolist(), s["n_path"].tolist()
    for x in (K, V, key):
        for b in range(s["B"]):
            for l in range(s["L"]):
                for h in range(s["H"]):
                    u = _unit(s, x, b, l, h)[int(ctx[b, l]):]
                    u[:n_path[b]] = u[path[b][:n_path[b]]].clone()
    return K, V, None, key, None
