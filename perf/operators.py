"""Performance cases of the token-level operators and of the page operators of the paged pool.

One pass is one call of an operator as a serving loop makes it.  Kinds:

  rope     qk_norm_rope: the queries and keys of the new tokens are normed per head and rotated to their positions
  attn     window_sink_attn: the new tokens attend to the sinks, the window and each other (a chain, or a draft tree)
  commit   token_commit: rows of new tokens (all of a chain, or an accepted path of a tree) go into the token cache
  fork     pages_free of the children of the last pass, then pages_fork of a batch of sequences
  compact  pages_compact of a pool with holes

Fields of a case
  dtype                 "bf16" or "fp32": storage type
  B                     sequences
  H, Hk, d              query heads, key heads, head dim
  shared                keys are the values too (one latent vector per token)
  window, sinks         a token sees the last `window` positions (itself included) and the first `sinks`
  L_min, L_max          committed tokens of a sequence
  n_min, n_max          new tokens of a sequence
  tree                  the new tokens form a draft tree (up to 32 nodes) instead of a chain
  page_tokens           0: a ring of sinks + window rows per sequence; else a pool of pages of that many tokens
  rot, first, pairs     rotated dims, the first of them, and whether neighbours form a pair (else: i and i + rot / 2)
  fused                 q, k and v are column ranges of one projection
  layers                layers whose planes the pages have
  children              children of each forked sequence
  used                  share of the pool's pages in use
"""
import json
import math
import random

import torch

own = False

BASE = 10000.0          # of the rotation's frequencies
EPS = 1e-6
M_CSA, M_HCA, D_KV, D_IK = 4, 128, 512, 128      # the compressed layers of the product shape


def _tok(kind, name, dtype="bf16", B=1, H=64, Hk=1, d=512, shared=True, window=128, sinks=4, L_min=0, L_max=0, n_min=1, n_max=1,
         tree=False, page_tokens=0, **more):
    c = {"kind": kind, "name": name, "dtype": dtype, "B": B, "H": H, "Hk": Hk, "d": d, "shared": shared, "window": window, "sinks": sinks,
         "L_min": L_min, "L_max": L_max, "n_min": n_min, "n_max": n_max, "tree": tree, "page_tokens": page_tokens}
    c.update(more)
    return c


def listed():
    return [
        # one user's next token in the numerics configuration's layer: the smallest call, all latency
        _tok("attn", "attn_one_token_fp32", dtype="fp32", H=16, d=128, L_min=1024, L_max=1024),
        # draft trees of a full batch over the paged pool's token-level KV: the benchmark's batch, budget and head shape
        _tok("attn", "attn_trees_b64_paged", B=64, L_min=256, L_max=2048, n_min=5, n_max=8, tree=True, page_tokens=128),
        # prompts of widely differing lengths through a window layer of the product shape
        _tok("attn", "attn_prompts_latent", B=8, L_min=0, L_max=700, n_min=97, n_max=4000),
        # the same through a drafter's grouped heads with values of their own and a longer window: the largest call
        _tok("attn", "attn_prompts_grouped", B=6, H=32, Hk=8, d=128, shared=False, window=1024, L_min=0, L_max=5000, n_min=300, n_max=8191,
             page_tokens=64),
        # one user's draft tree: queries and keys of a handful of nodes
        _tok("rope", "rope_one_tree", L_min=4096, L_max=4096, n_min=8, n_max=8, tree=True, rot=64, first=448, pairs=True, fused=False),
        # prompts of a batch, straight from the fused projection
        _tok("rope", "rope_prompts_grouped", B=16, H=32, Hk=8, d=128, shared=False, L_min=0, L_max=131072, n_min=33, n_max=2048, rot=128, first=0,
             pairs=False, fused=True),
        # accepted paths of a full batch into the pool
        _tok("commit", "commit_paths_b64_paged", B=64, L_min=256, L_max=2048, n_min=8, n_max=8, tree=True, page_tokens=128),
        # prompts of a batch into the pool: keys and values
        _tok("commit", "commit_prompts_paged", B=16, Hk=8, d=128, shared=False, window=1024, L_min=0, L_max=1000, n_min=511, n_max=4096, page_tokens=64),
        # two samples of one conversation
        {"kind": "fork", "name": "fork_one", "B": 1, "layers": 1, "page_tokens": 128, "L_min": 1000, "L_max": 1000, "children": 1},
        # parallel sampling of a batch over a stack of layers
        {"kind": "fork", "name": "fork_b16_by_4", "B": 16, "layers": 8, "page_tokens": 128, "L_min": 256, "L_max": 2048, "children": 4},
        # a small pool after some sequences have ended
        {"kind": "compact", "name": "compact_small", "B": 8, "layers": 1, "page_tokens": 128, "L_min": 256, "L_max": 2048, "used": 0.5},
        # a stack's pool, a third of it free, before it gives memory back
        {"kind": "compact", "name": "compact_stack", "B": 64, "layers": 8, "page_tokens": 128, "L_min": 256, "L_max": 2048, "used": 0.66},
    ]


def _log(rng, lo, hi):
    return min(hi, max(lo, int(math.exp(rng.uniform(math.log(lo), math.log(hi + 1))))))


def draw(rng):
    kind = rng.choice(["attn", "attn", "attn", "rope", "commit", "fork", "compact"])
    page = rng.choice([16, 32, 64, 128, 256])
    if kind in ("fork", "compact"):
        c = {"kind": kind, "layers": rng.randint(1, 8), "page_tokens": rng.choice([128, 256])}
        c["B"] = _log(rng, 1, 16) if kind == "fork" else _log(rng, 2, 64)
        c["L_max"] = _log(rng, 200, 2048)
        c["L_min"] = rng.randint(1, c["L_max"])
        c.update({"children": rng.randint(1, 4)} if kind == "fork" else {"used": round(rng.uniform(0.3, 0.9), 3)})
        return c
    dtype = "fp32" if rng.random() < 0.2 else "bf16"
    heads = [(64, 1, 512), (64, 1, 512), (32, 8, 128), (40, 8, 128), (16, 16, 64), (16, 1, 128), (20, 4, 80), (12, 2, 96), (8, 1, 256), (7, 1, 72)]
    H, Hk, d = rng.choice(heads[4:] if dtype == "fp32" else heads)
    shared = Hk == 1 and rng.random() < 0.7
    form = rng.choice(["token", "tree", "chain", "prompt", "prompt"])
    window = _log(rng, 1, 1024)
    if form == "token":
        B, n_min, n_max = _log(rng, 1, 256), 1, 1
        if B <= 8:
            window = _log(rng, 64, 32768)
    elif form == "tree":
        B = _log(rng, 1, 128)
        n_max = rng.randint(2, min(32, 1024 // B))
        n_min = rng.randint(1, n_max)
    elif form == "chain":
        B = _log(rng, 1, 128)
        n_max = _log(rng, 2, min(32, 1024 // B))
        n_min = rng.randint(0, n_max)
    else:
        B = _log(rng, 1, 16)
        n_max = _log(rng, 33, max(40, (4096 if H * d > 8192 else 8192) // B))
        window = min(window, 512) if H * d > 8192 else window
        n_min = rng.randint(0, n_max)
    if dtype == "fp32":                     # (the numerics type: short)
        B, n_max, window = min(B, 8), min(n_max, 600), min(window, 600)
        n_min = min(n_min, n_max)
    L_max = _log(rng, 1, 131072) if B <= 4 else _log(rng, 1, 4096)
    c = _tok(kind, "", dtype, B, H, Hk, d, shared, window, rng.choice([0, 0, 1, 4, 7, 64]), rng.randint(0, L_max), L_max, n_min, n_max, form == "tree",
             rng.choice([0, page]))
    del c["name"]
    if kind == "rope":
        pairs, rot = rng.random() < 0.5, rng.choice([r for r in (16, 32, 64, 128, d // 16 * 16) if r <= d])
        c.update(rot=rot, first=rng.choice([0, d - rot]), pairs=pairs, fused=rng.random() < 0.5)
    return c


# ------------------------------------------------------------------------------------------------ inputs
def _spread(lo, hi, B, by):
    """B whole numbers over [lo, hi], the same ones for every seed."""
    return [lo + int((hi - lo + 1) * ((b + 1) * by % 1.0)) for b in range(B)]


def _lengths(c):
    L = _spread(c["L_min"], c["L_max"], c["B"], 0.6180339887498949)
    return L, _spread(c["n_min"], c["n_max"], c["B"], 0.7548776662466927) if "n_min" in c else None


def _tree(r, n):
    return [-1] + [r.randrange(k) for k in range(1, n)]


def prepare(case, seed):
    r, dev = random.Random(seed * 1000003 + 17), torch.device("cuda")
    gen = torch.Generator(device=dev)
    gen.manual_seed(seed)
    L, n = _lengths(case)
    order = list(range(case["B"]))
    r.shuffle(order)
    L = [L[b] for b in order]
    if case["kind"] in ("fork", "compact"):
        return _prepare_pages(case, L, r, gen, dev)
    n = [n[b] for b in order]
    dt = torch.bfloat16 if case["dtype"] == "bf16" else torch.float32
    B, H, Hk, d, T = case["B"], case["H"], case["Hk"], case["d"], max(1, sum(n))
    row0 = [sum(n[:b]) for b in range(B)]
    i32 = dict(dtype=torch.int32, device=dev)
    s = {"case": case, "L_host": L, "n_host": n, "row0_host": row0, "T": T, "L": torch.tensor(L, **i32), "n": torch.tensor(n, **i32),
         "row0": torch.tensor(row0, dtype=torch.int64, device=dev), "parent": None}
    trees = [_tree(r, k) if k else [] for k in n] if case["tree"] else None
    if trees:
        s["parent"] = torch.tensor(sum(trees, []) or [-1], **i32)
    normal = lambda *shape: torch.randn(*shape, generator=gen, device=dev).to(dt)  # noqa: E731
    unit = lambda x: (x.float() * torch.rsqrt(x.float().square().mean(-1, keepdim=True) + EPS)).to(dt)  # noqa: E731
    kv = Hk * d * (1 if case["shared"] else 2)
    if case["kind"] == "rope" and case["fused"]:
        s["proj"] = normal(T, H * d + kv)
        s["q"], s["k"] = s["proj"][:, :H * d].view(T, H, d), s["proj"][:, H * d:H * d + Hk * d].view(T, Hk, d)
    else:
        s["q"] = normal(T, H, d) if case["kind"] != "commit" else None
        s["k"] = normal(T, Hk, d)
    if case["kind"] == "rope":
        s["wq"], s["wk"] = (1 + 0.1 * torch.randn(d, generator=gen, device=dev) for _ in range(2))
        s["inv_freq"] = BASE ** (-torch.arange(0, case["rot"], 2, dtype=torch.float32, device=dev) / case["rot"])
        return s
    # attention and commit: what they get is normed; the cache's rows
    s["v"] = None if case["shared"] else normal(T, Hk, d)
    page = case["page_tokens"]
    if page:
        need = [max(1, -(-(a + b) // page)) for a, b in zip(L, n)]
        ids = list(range(sum(need)))
        r.shuffle(ids)
        table = torch.full((B, max(need)), -1, dtype=torch.int32)
        for b in range(B):
            table[b, :need[b]] = torch.tensor(ids[:need[b]], dtype=torch.int32)
            del ids[:need[b]]
        s["table"], rows = table.to(dev), sum(need) * page
    else:
        s["table"], rows = None, B * (case["sinks"] + case["window"])
    s["ck"] = unit(normal(rows, Hk, d))
    s["cv"] = None if case["shared"] else normal(rows, Hk, d)
    if case["kind"] == "attn":
        s["q"], s["k"] = unit(s["q"]), unit(s["k"])
    else:
        s["L0"] = s["L"].clone()
        s["path"] = s["count"] = None
        s["count_host"] = n
        if trees:
            walks = []
            for t in trees:
                at, way = 0, []
                while t and at is not None:
                    way.append(at)
                    below = [k for k in range(len(t)) if t[k] == at]
                    at = r.choice(below) if below and r.random() < 0.8 else None
                walks.append(way)
            width = max(1, case["n_max"])
            s["path"] = torch.tensor([w + [-1] * (width - len(w)) for w in walks], **i32)
            s["count"] = torch.tensor([len(w) for w in walks], **i32)
            s["count_host"] = [len(w) for w in walks]
    return s


def _planes(case):
    """Rows of a page in the planes of a layer, and their widths: entries, indexer keys, 128-token entries, token-level KV."""
    p = case["page_tokens"]
    return [(p // M_CSA, D_KV), (p // M_CSA, D_IK), (p // M_HCA, D_KV), (p, D_KV)]


def _prepare_pages(case, L, r, gen, dev):
    page, B, layers = case["page_tokens"], case["B"], case["layers"]
    need = [-(-a // page) for a in L]
    if case["kind"] == "fork":
        slots, n_pages = B * (1 + case["children"]), 8 + sum(need) + sum(need) * case["children"] // 2 + B * case["children"]
    else:
        slots, n_pages = B, max(sum(need) + 1, int(sum(need) / case["used"]))
    ids = list(range(n_pages))
    r.shuffle(ids)
    table, ref = torch.full((slots, max(need)), -1, dtype=torch.int32), torch.zeros(n_pages, dtype=torch.int32)
    for b in range(B):
        mine = torch.tensor(ids[:need[b]], dtype=torch.int32)
        del ids[:need[b]]
        table[b, :need[b]] = mine
        ref[mine.long()] += 1
    i32 = dict(dtype=torch.int32, device=dev)
    s = {"case": case, "table0": table.to(dev), "ref0": ref.to(dev), "table": table.to(dev), "ref": ref.to(dev), "L_host": L,
         "planes": [torch.randn(n_pages, a * w, generator=gen, device=dev, dtype=torch.bfloat16) for _ in range(layers) for a, w in _planes(case)]}
    s["L"] = torch.tensor(L + [0] * (slots - B), **i32)
    s["moves_host"] = sum(int(p) >= sum(need) for p in ref.nonzero().flatten().tolist())
    if case["kind"] == "fork":          # the open blocks of a sequence: weights and sums of both compressed layers
        s["rows"] = [torch.randn(slots, w, generator=gen, device=dev) for _ in range(layers) for w in (4, D_KV, D_IK, D_KV)]
        src = [b for b in range(B) for _ in range(case["children"])]
        s["src_host"], s["dst_host"] = src, list(range(B, slots))
        s["src"], s["dst"] = torch.tensor(src, **i32), torch.tensor(s["dst_host"], **i32)
        s["first"], s["last"] = torch.zeros(len(src), **i32), torch.full((len(src),), max(need), **i32)
    return s


# ------------------------------------------------------------------------------------------------ the framework's calls
def _handles(s):
    """What a program keeps beside its data: the shapes, the descriptions of its buffers, its outputs and workspaces."""
    if "handles" in s:
        return s["handles"]
    from paper_2609_24698_b200 import pages, tokens
    c = s["case"]
    if c["kind"] in ("fork", "compact"):
        pool = pages.PagePool(s["table"], s["ref"], c["page_tokens"], s["planes"], [s["L"]] + s.get("rows", []))
        h = {"api": pages, "pool": pool, "ws": pages.alloc_workspace(pool), "status": torch.zeros(max(1, len(s.get("src_host", []))), dtype=torch.int32, device="cuda"),
             "n_used": torch.zeros(1, dtype=torch.int32, device="cuda")}
    else:
        shape = tokens.TokenShape(c["dtype"], c["B"], c["H"], c["Hk"], c["d"], c["window"], c["sinks"], max_L=c["L_max"] + c["n_max"], max_n=c["n_max"])
        h = {"api": tokens, "shape": shape, "batch": tokens.TokenBatch(s["row0"], s["n"], s["parent"]), "status": torch.zeros(c["B"], dtype=torch.int32, device="cuda")}
        if c["kind"] == "rope":
            h["q"], h["k"] = torch.empty(s["q"].shape, dtype=s["q"].dtype, device="cuda"), torch.empty(s["k"].shape, dtype=s["k"].dtype, device="cuda")
        else:
            h["cache"] = tokens.TokenCache(s["L"], s["ck"], s["cv"], s["table"], c["page_tokens"])
        if c["kind"] == "attn":
            h["out"], h["ws"] = torch.empty_like(s["q"]), tokens.alloc_workspace(shape, s["T"])
    s["handles"] = h
    return h


def run(state):
    kind = state["case"]["kind"]
    if own:
        return globals()["_own_" + kind](state, _handles(state))
    return globals()["_plain_" + kind](state)


def _own_rope(s, h):
    c = s["case"]
    h["api"].qk_norm_rope(h["shape"], s["L"], h["batch"], s["q"], s["k"], h["q"], h["k"], s["wq"], s["wk"], EPS, s["inv_freq"], c["first"], c["pairs"], h["status"])
    return h["q"], h["k"]


def _own_attn(s, h):
    h["api"].window_sink_attn(h["shape"], h["cache"], h["batch"], s["q"], s["k"], s["v"], h["out"], h["ws"], h["status"])
    return h["out"]


def _own_commit(s, h):
    s["L"].copy_(s["L0"])
    h["api"].token_commit(h["shape"], h["cache"], h["batch"], s["k"], s["v"], h["status"], path=s["path"], count=s["count"])
    return (s["ck"], s["L"]) if s["cv"] is None else (s["ck"], s["cv"], s["L"])


def _own_fork(s, h):
    h["api"].pages_free(h["pool"], s["dst"], s["first"], s["last"], h["status"])
    h["api"].pages_fork(h["pool"], s["src"], s["dst"], s["L"], h["ws"], h["status"])
    return {"table": s["table"], "ref": s["ref"], "planes": s["planes"], "rows": s["rows"][:4], "L": s["L"]}


def _own_compact(s, h):
    s["table"].copy_(s["table0"])
    s["ref"].copy_(s["ref0"])
    h["api"].pages_compact(h["pool"], h["n_used"], h["ws"])
    return {"table": s["table"], "ref": s["ref"], "planes": s["planes"], "used": h["n_used"]}


# ------------------------------------------------------------------------------------------------ the plain forms
def _family(s):
    """Depths and ancestors (self included) of the nodes of every sequence, padded to n_max: [B, n], [B, n, n]."""
    c = s["case"]
    B, N = c["B"], c["n_max"]
    slot = torch.arange(N, device=s["L"].device)
    live = slot < s["n"][:, None]
    up = torch.where(live, s["parent"][(s["row0"][:, None] + slot).clamp(max=s["T"] - 1)], -1)
    reach = ((up[:, :, None] == slot) | (slot[:, None] == slot)).float()
    for _ in range(5):                  # 2^5 generations
        reach = (reach @ reach > 0).float()
    return reach.sum(-1).long() - 1, reach > 0


def _positions(s):
    """The position of every new row, [T] 64-bit."""
    dev, c = s["L"].device, s["case"]
    seq = torch.repeat_interleave(torch.arange(c["B"], device=dev), s["n"].long(), output_size=sum(s["n_host"]))
    i = torch.arange(seq.numel(), device=dev) - s["row0"][seq]
    at = _family(s)[0][seq, i] if s["parent"] is not None else i
    return seq, s["L"][seq].long() + at


def _plain_rope(s):
    c = s["case"]
    _, p = _positions(s)
    angle = p.double()[:, None] * s["inv_freq"].double()
    cos, sin = torch.cos(angle).float()[:, None], torch.sin(angle).float()[:, None]
    f, e, half = c["first"], c["first"] + c["rot"], c["rot"] // 2

    def one(x, w):
        x = x[:p.numel()].float()
        y = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS) * w
        a, b = (y[..., f:e:2], y[..., f + 1:e:2]) if c["pairs"] else (y[..., f:f + half], y[..., f + half:e])
        ra, rb = a * cos - b * sin, a * sin + b * cos
        z = torch.stack((ra, rb), -1).flatten(-2) if c["pairs"] else torch.cat((ra, rb), -1)
        return torch.cat((y[..., :f], z, y[..., e:]), -1).to(s["q"].dtype)
    return one(s["q"], s["wq"]), one(s["k"], s["wk"])


def _cache_rows(s, b, pos):
    """Rows of the token cache that hold the given positions of sequences b (positions of no row give any row)."""
    c = s["case"]
    pos = pos.clamp(min=0)
    if c["page_tokens"]:
        lp = (pos // c["page_tokens"]).clamp(max=s["table"].shape[1] - 1)
        return s["table"][b, lp].long().clamp(min=0) * c["page_tokens"] + pos % c["page_tokens"]
    ns, w = c["sinks"], c["window"]
    return b * (ns + w) + torch.where(pos < ns, pos, ns + (pos - ns) % w)


def _plain_attn(s):
    c, dev = s["case"], s["L"].device
    ns, w, H, Hk, d = c["sinks"], c["window"], c["H"], c["Hk"], c["d"]
    Q = max(1, min(c["n_max"], 32 if c["tree"] else 64))                           # tokens of a block of queries
    blocks = [(b, i) for b in range(c["B"]) for i in range(0, s["n_host"][b], Q)]
    out = torch.empty_like(s["q"])
    if not blocks:
        return out
    b = torch.tensor([x[0] for x in blocks], device=dev)
    i0 = torch.tensor([x[1] for x in blocks], device=dev)
    L, n, row0 = s["L"].long()[b], s["n"].long()[b], s["row0"][b]
    at = i0[:, None] + torch.arange(Q, device=dev)                                  # [blocks, Q] tokens
    live = at < n[:, None]
    sink, back = torch.arange(ns, device=dev).expand(len(blocks), ns), torch.arange(1 - w, 0 if c["tree"] else Q, device=dev)
    low = (L + i0 + 1 - w).clamp(min=0)
    kp = torch.cat((sink, (L + i0)[:, None] + back), 1)                             # key positions: sinks, window, (chain) the block itself
    new = torch.full_like(kp, 0)
    ok = (kp >= 0) & (kp < (L if c["tree"] else L + n)[:, None])
    ok[:, :ns] &= sink < low[:, None]
    if c["tree"]:
        depth, kin = _family(s)
        node = torch.arange(c["n_max"], device=dev).expand(len(blocks), c["n_max"])
        qp = L[:, None] + depth[b][:, :Q]
        kp, new = torch.cat((kp, L[:, None] + depth[b]), 1), torch.cat((new, node), 1)
        ok = torch.cat((ok, node < n[:, None]), 1)
        seen = torch.cat((torch.ones(len(blocks), Q, ns + w - 1, dtype=torch.bool, device=dev), kin[b][:, :Q]), 2)
    else:
        qp, new, seen = L[:, None] + at, kp - L[:, None], True
    see = ok[:, None] & live[..., None] & seen & (kp[:, None] <= qp[..., None]) & ((kp[:, None] > qp[..., None] - w) | (kp[:, None] < ns))
    fresh = (kp >= L[:, None])[..., None, None]
    crow, nrow = _cache_rows(s, b[:, None], kp), (row0[:, None] + new).clamp(0, s["T"] - 1)
    K = torch.where(fresh, s["k"][nrow], s["ck"][crow]).float()                     # [blocks, keys, Hk, d]
    V = K if s["v"] is None else torch.where(fresh, s["v"][nrow], s["cv"][crow]).float()
    qrow = (row0[:, None] + at).clamp(max=s["T"] - 1)
    q = s["q"][qrow].float().view(len(blocks), Q, Hk, H // Hk, d).permute(0, 2, 1, 3, 4).reshape(len(blocks), Hk, -1, d)
    S = torch.matmul(q, K.permute(0, 2, 3, 1)).view(len(blocks), Hk, Q, H // Hk, -1) / math.sqrt(d)
    S = S.masked_fill_(~see[:, None, :, None], -math.inf)
    S = torch.exp_(S.sub_(S.amax(-1, keepdim=True).clamp_(min=-1e30)))
    total = S.sum(-1, keepdim=True).flatten(2, 3)
    O = torch.matmul(S.flatten(2, 3), V.permute(0, 2, 1, 3)) / total.clamp(min=1e-30)
    O = O.view(len(blocks), Hk, Q, H // Hk, d).permute(0, 2, 1, 3, 4).reshape(len(blocks), Q, H, d)
    pick = (qrow + torch.where(live, 0, s["T"])).flatten()                          # rows of no token go behind the last one
    full = torch.empty(2 * s["T"], H, d, dtype=out.dtype, device=dev)
    full[pick] = O.flatten(0, 1).to(out.dtype)
    return full[:s["T"]]


def _plain_commit(s):
    c, dev = s["case"], s["L"].device
    s["L"].copy_(s["L0"])
    count = s["n"] if s["count"] is None else s["count"]
    seq = torch.repeat_interleave(torch.arange(c["B"], device=dev), count.long(), output_size=sum(s["count_host"]))
    i = torch.arange(seq.numel(), device=dev) - (count.long().cumsum(0) - count)[seq]
    pos = s["L"][seq].long() + i
    row = s["row0"][seq] + (i if s["path"] is None else s["path"][seq, i].long())
    at = _cache_rows(s, seq, pos)
    if not c["page_tokens"]:            # of a ring's slot the last writer stays: the others go where nothing is read
        stays = (pos < c["sinks"]) | (i >= count[seq] - c["window"])
        at, row = at[stays], row[stays]
    s["ck"][at] = s["k"][row]
    if s["cv"] is not None:
        s["cv"][at] = s["v"][row]
    s["L"] += count
    return (s["ck"], s["L"]) if s["cv"] is None else (s["ck"], s["cv"], s["L"])


def _plain_fork(s):
    c, table, ref = s["case"], s["table"], s["ref"]
    src, dst, page = s["src"].long(), s["dst"].long(), c["page_tokens"]
    held = table[dst].long()                                                        # the children of the last pass go
    ref.index_add_(0, held.clamp(min=0).flatten(), -(held >= 0).int().flatten())
    mine = table[src]
    lp = torch.arange(table.shape[1], device=table.device)
    whole = lp < (s["L"][src] // page)[:, None]
    fresh = (mine >= 0) & ~whole
    free = torch.sort((ref != 0).int(), stable=True).indices                        # free pages first, ascending
    rank = fresh.flatten().long().cumsum(0).view_as(fresh) - 1
    got = torch.where(fresh, free[rank.clamp(min=0)].int(), mine)
    ref.index_add_(0, got.clamp(min=0).long().flatten(), (got >= 0).int().flatten())
    table[dst] = got
    part = [k for k, b in enumerate(s["src_host"]) if s["L_host"][b] % page]
    if part:
        k = torch.tensor(part, device=table.device)
        at = (s["L"][src[k]] // page).long()
        a, z = mine[k, at].long(), got[k, at].long()
        for plane in s["planes"]:
            plane[z] = plane[a]
    for row in s["rows"]:
        row[dst] = row[src]
    s["L"][dst] = s["L"][src]
    return {"table": table, "ref": ref, "planes": s["planes"], "rows": s["rows"][:4], "L": s["L"]}


def _plain_compact(s):
    table, ref = s["table"], s["ref"]
    table.copy_(s["table0"])
    ref.copy_(s["ref0"])
    N = ref.numel()
    used = sum(-(-a // s["case"]["page_tokens"]) for a in s["L_host"])              # (no page is shared in these pools)
    where = torch.arange(N, device=ref.device)
    m = s["moves_host"]
    src = torch.sort(((ref == 0) | (where < used)).int(), stable=True).indices[:m]
    dst = torch.sort(((ref != 0) | (where >= used)).int(), stable=True).indices[:m]
    to = where.clone()
    to[src] = dst
    for plane in s["planes"]:
        plane[dst] = plane[src]
    table.copy_(torch.where(table >= 0, to[table.long().clamp(min=0)].int(), table))
    ref.copy_((where < used).int())
    return {"table": table, "ref": ref, "planes": s["planes"], "used": torch.full((1,), used, dtype=torch.int32, device=ref.device)}


# ------------------------------------------------------------------------------------------------ work and 64-bit values
def _visible(c):
    """(token, visible key) pairs, and rows of keys that a sequence's new tokens read in all."""
    pairs = rows = 0
    for L, n in zip(*_lengths(c)):
        if not n:
            continue
        w, ns = c["window"], c["sinks"]
        mean_depth = (n - 1) / 2 if not c["tree"] else min(n - 1, math.log(n + 1))
        low = max(0, L - w + 1)
        rows += min(low, ns) + (L - low) + n
        if c["tree"]:
            pairs += n * (min(low, ns) + min(L, w - 1) + 1 + mean_depth)
        else:
            a = max(0, min(n, w - 1 - L))                                           # tokens whose window starts at position 0
            pairs += a * (L + 1) + a * (a - 1) // 2 + (n - a) * w + sum(min(ns, max(0, L + i - w + 1)) for i in range(a, min(n, a + ns))) + max(0, n - a - ns) * min(
                ns, max(0, L + a + ns - w + 1))
    return pairs, rows


def work(case):
    c = case
    if c["kind"] in ("fork", "compact"):
        L, _ = _lengths(c)
        page = sum(a * w * 2 for a, w in _planes(c)) * c["layers"]
        need = [-(-a // c["page_tokens"]) for a in L]
        if c["kind"] == "fork":
            copied = sum(1 for a in L if a % c["page_tokens"]) * c["children"]
            row = 4 + c["layers"] * 4 * (4 + D_KV + D_IK + D_KV)
            return {"bytes": 2 * copied * page + 2 * c["B"] * c["children"] * row, "flops": 0}
        N = max(sum(need) + 1, int(sum(need) / c["used"]))
        return {"bytes": 2 * page * sum(need) * (N - sum(need)) / N + 12 * N, "flops": 0}
    es, T = 2 if c["dtype"] == "bf16" else 4, sum(_lengths(c)[1])
    kv = c["Hk"] * c["d"] * es * (1 if c["shared"] else 2)
    if c["kind"] == "rope":
        return {"bytes": 2 * T * (c["H"] + c["Hk"]) * c["d"] * es, "flops": 8 * T * (c["H"] + c["Hk"]) * c["d"]}
    if c["kind"] == "commit":
        t = T
        if c["tree"]:
            t = c["B"] * 2.5
        elif not c["page_tokens"]:
            t = sum(min(n, c["sinks"] + c["window"]) for n in _lengths(c)[1])
        return {"bytes": 2 * t * kv + 8 * c["B"], "flops": 0}
    pairs, rows = _visible(c)
    return {"bytes": 2 * T * c["H"] * c["d"] * es + rows * kv, "flops": 4 * pairs * c["H"] * c["d"]}


def exact(case, seed):
    if case["kind"] not in ("rope", "attn"):
        return None                     # copies and whole numbers
    s = prepare(case, seed)
    c, dev = case, s["L"].device
    up = s["parent"].tolist() if s["parent"] is not None else None
    outs = [torch.zeros(s["T"], c["H"], c["d"], dtype=torch.float64, device=dev)]
    if c["kind"] == "rope":
        outs.append(torch.zeros(s["T"], c["Hk"], c["d"], dtype=torch.float64, device=dev))
    for b in range(c["B"]):
        L, n, r0 = s["L_host"][b], s["n_host"][b], s["row0_host"][b]
        kin = []
        for i in range(n):
            kin.append({i} | (kin[up[r0 + i]] if up and up[r0 + i] >= 0 else set())) if up else None
        depth = [len(k) - 1 for k in kin] if up else list(range(n))
        if c["kind"] == "rope":
            _exact_rope(s, outs, r0, [L + x for x in depth])
            continue
        step = 32 if up else 128
        for i in range(0, n, step):
            e = min(n, i + step)
            qp = torch.tensor([L + x for x in depth[i:e]], device=dev)
            low = max(0, int(qp.min()) - c["window"] + 1)
            old = [p for p in range(min(c["sinks"], low, L))] + list(range(low, L))
            fresh = list(range(0, n if up else e))
            fresh = [j for j in fresh if L + depth[j] >= low or L + depth[j] < c["sinks"]]
            kp = torch.tensor(old + [L + depth[j] for j in fresh], device=dev)
            nr = torch.tensor([r0 + j for j in fresh], dtype=torch.long, device=dev)
            if c["page_tokens"]:
                P = c["page_tokens"]
                own_pages = s["table"][b].tolist()
                cr = [own_pages[p // P] * P + p % P for p in old]
            else:
                cr = [b * (c["sinks"] + c["window"]) + (p if p < c["sinks"] else c["sinks"] + (p - c["sinks"]) % c["window"]) for p in old]
            cr = torch.tensor(cr, dtype=torch.long, device=dev)
            K = torch.cat((s["ck"][cr], s["k"][nr])).double()
            V = K if c["shared"] else torch.cat((s["cv"][cr], s["v"][nr])).double()
            see = (kp <= qp[:, None]) & ((kp > qp[:, None] - c["window"]) | (kp < c["sinks"]))
            if up:
                kinship = torch.zeros(e - i, len(kp), dtype=torch.bool)
                kinship[:, :len(old)] = True
                for a in range(i, e):
                    for k, j in enumerate(fresh):
                        kinship[a - i, len(old) + k] = j in kin[a]
                see &= kinship.to(dev)
            K, V = (x.repeat_interleave(c["H"] // c["Hk"], 1) for x in (K, V))
            q = s["q"][r0 + i:r0 + e].double()
            score = torch.einsum("thd,khd->thk", q, K) / math.sqrt(c["d"])
            score = torch.where(see[:, None], score, torch.full_like(score, -math.inf))
            outs[0][r0 + i:r0 + e] = torch.einsum("thk,khd->thd", torch.softmax(score, -1), V)
    return outs[0] if c["kind"] == "attn" else tuple(outs)


def _exact_rope(s, outs, r0, pos):
    c, n = s["case"], len(pos)
    if not n:
        return
    turn = torch.tensor(pos, dtype=torch.float64, device=s["L"].device)[:, None, None] * s["inv_freq"].double()
    turn = torch.polar(torch.ones_like(turn), turn)
    for out, x, w in ((outs[0], s["q"], s["wq"]), (outs[1], s["k"], s["wk"])):
        x = x[r0:r0 + n].double()
        y = x / torch.sqrt((x ** 2).mean(-1, keepdim=True) + EPS) * w.double()
        part = y[..., c["first"]:c["first"] + c["rot"]]
        if c["pairs"]:
            z = torch.view_as_real(torch.view_as_complex(part.unflatten(-1, (-1, 2)).contiguous()) * turn).flatten(-2)
        else:
            z = torch.complex(*part.chunk(2, -1)) * turn
            z = torch.cat((z.real, z.imag), -1)
        y[..., c["first"]:c["first"] + c["rot"]] = z
        out[r0:r0 + n] = y


if __name__ == "__main__":
    for case in listed():
        print(json.dumps({**case, **work(case)}))
