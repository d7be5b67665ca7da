"""Performance cases of speculative decoding over linked paged caches.

After a cache hit a serving program keeps decoding on the linked context.  It
attends several drafted tokens of a request at once (a chain, or a tree of
candidates), verifies them against the target's probabilities, keeps the
accepted path in the paged cache, and forks, frees, copies and compacts the
cache's pages.  Each case is one such call (or the two that belong together),
with ``own`` through the package's ``pic_attend_draft``, ``pic_verify_draft``
and ``pic_page_*``, else in elementary torch operations.

Sizes are those of workloads.py, cases.py and the parity tests, or lie between
them; vocabularies are generic (a power of two, an odd number).  A case is a
dict of plain values; lengths, trees and page counts follow from the case
alone, values, choices and page placement from the seed.
"""
from __future__ import annotations

import math
from types import SimpleNamespace

import numpy as np
import torch

own = False
DEV = "cuda"
PAGE = 16

# (query heads, kv heads, head dim, RoPE base), as in cases.py
GEOMS = {
    "32/8/128": (32, 8, 128, 5e5),
    "28/4/128": (28, 4, 128, 1e6),
    "8/2/128": (8, 2, 128, 5e5),
    "32/2/128": (32, 2, 128, 5e5),
    "16/2/64": (16, 2, 64, 1e4),
    "4/1/64": (4, 1, 64, 1e4),
}


# ---------------------------------------------------------------------- cases
def _attend(geom, batch, ctx, draft, tree=False, style=0, q_scale=1.0):
    return dict(kind="attend", geom=geom, batch=batch, ctx_lo=ctx[0], ctx_hi=ctx[1], draft=draft,
                tree=tree, style=style, q_scale=q_scale)


def _verify(batch, draft, vocab, tree, agree=1.0):
    return dict(kind="verify", batch=batch, draft=draft, vocab=vocab, tree=tree, agree=agree)


def _fork(geom, layers, parents, children, ctx, reserve):
    return dict(kind="fork", geom=geom, layers=layers, parents=parents, children=children,
                ctx_lo=ctx[0], ctx_hi=ctx[1], reserve=reserve)


def _compact(geom, layers, rows, start, window, keep, rotate):
    return dict(kind="compact", geom=geom, layers=layers, rows=rows, start=start, window=window,
                keep=keep, rotate=rotate)


def _copy(geom, layers, pages, within):
    return dict(kind="copy", geom=geom, layers=layers, pages=pages, within=within)


def listed():
    c = []

    def add(name, case):
        c.append(dict(case, name=name))

    # The smallest call: one request on the "tiny" workload's context with a
    # chain of three drafts behind the last token.  Launches and round trips.
    add("draft_tiny", _attend("4/1/64", 1, (160, 160), 4, q_scale=2.0))
    # A ragged batch with wide candidate trees, a 64-wide head, GQA groups of
    # 8 and interleaved RoPE: 320 query rows per kv head in three row tiles.
    add("draft_tree_ragged_d64", _attend("16/2/64", 5, (37, 9001), 40, tree=True, style=1))
    # An ordinary batch: sixteen ~33k contexts of the decode workload, each
    # with a tree of 16 candidates (112 query rows per kv head).
    add("draft_tree_b16", _attend("28/4/128", 16, (32500, 33100), 16, tree=True))
    # The longest contexts, four of ~139k tokens, a chain of seven drafts.
    add("draft_128k_b4", _attend("32/8/128", 4, (138000, 140000), 8))
    # One request's tree of 16 candidates over an odd vocabulary, sampled
    # level by level: latency of the walk down the tree.
    add("verify_tree_1req", _verify(1, 16, 50001, True, agree=3.0))
    # A batch of 64 requests, chains of seven sampled drafts, a vocabulary of
    # 2^17: acceptance tests, then one row (or two) per request.
    add("verify_chain_b64", _verify(64, 8, 131072, False, agree=2.0))
    # Best-of-4 sampling off one linked context: free the last four branches,
    # fork four new ones, room for 32 tokens each.
    add("fork_1req", _fork("8/2/128", 4, 1, 4, (4290, 4290), 32))
    # The same for 16 contexts of the 28-layer decode workload, four branches
    # of each.
    add("fork_b16", _fork("28/4/128", 28, 16, 4, (2000, 2100), 32))
    # After verification of a batch of 8: the accepted path (five of a tree of
    # 16 tokens) moves together and the pages behind it go back, 32 layers.
    add("compact_drafts_b8", _compact("32/8/128", 32, 8, 1003, 16, 5, False))
    # Eviction: a request keeps three fifths of 15k positions, the kept keys
    # re-rotated to their new positions, 4 layers.
    add("compact_evict", _compact("32/8/128", 4, 1, 64, 15001, 9001, True))
    # A few pages between places of one cache (a request's tail, 2 layers).
    add("copy_few", _copy("8/2/128", 2, 5, True))
    # 512 pages (8k tokens) of a 32-layer cache into another one.
    add("copy_swap", _copy("32/8/128", 32, 512, False))
    return c


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 0.49)))))))


def draw(rng):
    """One more case of the listed ranges: any kind, sizes log-uniform."""
    top = [work(x) for x in listed()]
    top = (max(x["bytes"] for x in top), max(x["flops"] for x in top))
    while True:
        kind = rng.choice(["attend", "attend", "attend", "verify", "verify", "fork", "compact",
                           "compact", "copy"])
        geom = rng.choice(list(GEOMS))
        if kind == "attend":
            hi = _log_int(rng, 30, 140000)
            c = _attend(geom, _log_int(rng, 1, 24), (rng.choice([hi, hi // rng.randint(2, 20)]), hi),
                        _log_int(rng, 1, 64), tree=rng.random() < 0.5, style=rng.randint(0, 1),
                        q_scale=rng.choice([1.0, 1.0, 2.0]))
            # the plain form's scores in 32 bits stay within a few GB
            if c["batch"] * hi * c["draft"] * GEOMS[geom][0] > 4e8:
                continue
        elif kind == "verify":
            c = _verify(_log_int(rng, 1, 64), _log_int(rng, 1, 32), _log_int(rng, 8000, 160000),
                        rng.random() < 0.5, agree=rng.choice([1.0, 2.0, 3.0]))
            if c["batch"] * c["draft"] * c["vocab"] > 64 * 8 * 131072:
                continue
        elif kind == "fork":
            hi = _log_int(rng, 40, 16000)
            c = _fork(geom, _log_int(rng, 1, 32), _log_int(rng, 1, 24), _log_int(rng, 1, 8),
                      (max(1, hi - rng.randint(0, 200)), hi), rng.choice([0, 1, 16, 50]))
        elif kind == "compact":
            if rng.random() < 0.6:  # drafts
                t = _log_int(rng, 2, 64)
                c = _compact(geom, _log_int(rng, 1, 32), _log_int(rng, 1, 32), rng.randint(0, 3000),
                             t, rng.randint(1, t), False)
            else:  # eviction
                t = _log_int(rng, 100, 15001)
                c = _compact(geom, _log_int(rng, 1, 8), _log_int(rng, 1, 3), rng.randint(0, 100), t,
                             rng.randint(t // 4, t), rng.random() < 0.7)
        else:
            c = _copy(geom, _log_int(rng, 1, 32), _log_int(rng, 1, 512), rng.random() < 0.5)
        if kind in ("fork", "compact"):  # cache held on the device
            _, hkv, d, _ = GEOMS[geom]
            if _num_pages(c) * c["layers"] * hkv * PAGE * d * 4 > 5e9:
                continue
        w = work(c)
        if w["bytes"] < top[0] and w["flops"] <= top[1]:
            return c


# --------------------------------------------- what follows from a case alone
def _rng(c):
    return np.random.default_rng(sum((i + 1) * int(v) for i, v in enumerate(c.values())
                                     if isinstance(v, (int, float))) % (1 << 31))


def _ctx(c):
    n = c["batch"] if c["kind"] == "attend" else c["parents"]
    lens = _rng(c).integers(c["ctx_lo"], c["ctx_hi"] + 1, size=n)
    lens[0] = c["ctx_hi"]
    return lens.astype(np.int64)


def _draft_len(c):
    """Drafted tokens of each request: all of them for the first, from a half
    up for the others (ragged batches)."""
    n = c["batch"]
    lens = _rng(c).integers((c["draft"] + 1) // 2, c["draft"] + 1, size=n)
    lens[0] = c["draft"]
    return lens.astype(np.int64)


def _parents(c):
    """Topology of the candidate trees [batch][draft]: a root, then every
    token under one of the last few before it (-1: the root)."""
    r, n, t = _rng(c), c["batch"], c["draft"]
    par = np.full((n, t), -1, np.int64)
    for i in range(1, t):
        par[:, i] = np.maximum(0, i - 1 - r.integers(0, 4, size=n))
    return par


def _depths(par):
    dep = np.zeros_like(par)
    for i in range(1, par.shape[1]):
        dep[:, i] = np.take_along_axis(dep, np.maximum(par[:, i:i + 1], 0), 1)[:, 0] + 1
    return dep


def _kept(c):
    """Kept entries of each row's window: the listed number for the first row,
    from a half up for the others."""
    lens = _rng(c).integers((c["keep"] + 1) // 2, c["keep"] + 1, size=c["rows"])
    lens[0] = c["keep"]
    return lens.astype(np.int64)


def _num_pages(c):
    if c["kind"] == "fork":
        full = int((_ctx(c) // PAGE + 1).sum())
        return full + c["parents"] * c["children"] * (c["reserve"] // PAGE + 3)
    if c["kind"] == "compact":
        return c["rows"] * ((c["start"] + c["keep"] + c["window"]) // PAGE + 3)
    return 2 * c["pages"]


def _row_bytes(c):  # K and V of one position, every layer and kv head
    _, hkv, d, _ = GEOMS[c["geom"]]
    return c["layers"] * hkv * d * 4


def work(case):
    c = case
    if c["kind"] == "attend":
        hq, hkv, d, _ = GEOMS[c["geom"]]
        ctx, t = _ctx(c), _draft_len(c)
        par = _parents(c) if c["tree"] else np.tile(np.arange(c["draft"]) - 1, (c["batch"], 1))
        seen = _depths(par) + 1  # of the drafts themselves
        live = np.arange(c["draft"])[None] < t[:, None]
        pairs = int((ctx[:, None] * live).sum() + (seen * live).sum())
        kv = int((ctx + t).sum()) * hkv * d * 4
        rows = int(t.sum())
        return {"bytes": kv + rows * d * (4 * hq + 8 * hkv), "flops": 4.0 * d * hq * pairs}
    if c["kind"] == "verify":
        # one row of the target's per request and, where a draft is refused,
        # the draft's; a tree one row per level walked (at least the first)
        rows = c["batch"] * (1 if c["tree"] else 2 if c["draft"] > 1 else 1)
        b = rows * c["vocab"] * 4 + c["batch"] * c["draft"] * 24
        return {"bytes": b, "flops": rows * c["vocab"] * 2}
    if c["kind"] == "fork":
        ctx, n = _ctx(c), c["children"]
        full = int((ctx // PAGE).sum())
        return {"bytes": int((ctx % PAGE).sum()) * n * _row_bytes(c) * 2 + full * n * 16,
                "flops": 0}
    if c["kind"] == "compact":
        moved = int(_kept(c).sum())
        return {"bytes": moved * (_row_bytes(c) * 2 + 4),
                "flops": moved * _row_bytes(c) // 2 * 3 if c["rotate"] else 0}
    return {"bytes": c["pages"] * PAGE * _row_bytes(c) * 2, "flops": 0}


# ------------------------------------------------------------- input building
def _i32(x):
    return torch.as_tensor(np.ascontiguousarray(x), dtype=torch.int32).to(DEV)


def _cache(layers, pages, hkv, d, gen):
    return torch.randn((layers, pages, hkv, PAGE, d), generator=gen, device=DEV,
                       dtype=torch.bfloat16)


def _tables(lens, max_pages, num_pages, rows, r):
    """Block tables of the first len(lens) of `rows` rows over randomly placed
    pages, and the pages' use counts."""
    perm = r.permutation(num_pages)
    bt = np.full((rows, max_pages), -1, np.int64)
    o = 0
    for b, n in enumerate(lens):
        k = -(-int(n) // PAGE)
        bt[b, :k] = perm[o:o + k]
        o += k
    refs = np.zeros(num_pages, np.int64)
    refs[perm[:o]] = 1
    return _i32(bt), _i32(refs)


def prepare(case, seed):
    c = case
    gen = torch.Generator(device=DEV).manual_seed(seed)
    r = np.random.default_rng(seed)
    s = SimpleNamespace(c=c, kind=c["kind"])
    if c["kind"] == "verify":
        _prepare_verify(s, gen)
        return s
    hq, hkv, d, base = GEOMS[c["geom"]]
    s.hq, s.hkv, s.d, s.base = hq, hkv, d, base
    layers = c.get("layers", 1)
    if own:
        import paper_2607_28069_gb300 as pic
        s.geom = pic.Geometry(layers, hq, hkv, d, base, rope_style=c.get("style", 0))
    if c["kind"] == "attend":
        ctx, t = _ctx(c), _draft_len(c)
        B, T = c["batch"], c["draft"]
        need = [int(n) + T for n in ctx]
        s.max_pages = max(-(-n // PAGE) for n in need)
        s.num_pages = sum(-(-n // PAGE) for n in need) + 3
        s.block_table, _ = _tables(need, s.max_pages, s.num_pages, B, r)
        s.k_cache = _cache(1, s.num_pages, hkv, d, gen)
        s.v_cache = _cache(1, s.num_pages, hkv, d, gen)
        rnd = lambda h: torch.randn((B, T, h, d), generator=gen, device=DEV).bfloat16()  # noqa: E731
        s.q, s.k_new, s.v_new = rnd(hq) * c["q_scale"], rnd(hkv), rnd(hkv)
        s.ctx_len, s.draft_len = _i32(ctx), _i32(t)
        s.parent = _i32(_parents(c)) if c["tree"] else None
        s.out = torch.zeros((B, T, hq, d), dtype=torch.bfloat16, device=DEV)
        s.lse = torch.zeros((B, T, hq), dtype=torch.float32, device=DEV)
        if own:
            s.ws = torch.empty(pic.pic_draft_workspace_size(s.geom, B, T), dtype=torch.uint8,
                               device=DEV)
    elif c["kind"] == "fork":
        P, n = c["parents"], c["parents"] * c["children"]
        ctx = _ctx(c)
        s.max_pages = -(-(int(ctx.max()) + c["reserve"]) // PAGE) + 1
        s.num_pages = _num_pages(c)
        s.block_table, s.refs = _tables(ctx, s.max_pages, s.num_pages, P + n, r)
        s.ctx_len = _i32(np.concatenate([ctx, np.zeros(n, np.int64)]))
        s.src = _i32(np.repeat(np.arange(P), c["children"]))
        s.dst = _i32(P + r.permutation(n))
        s.result = torch.zeros(n, dtype=torch.int32, device=DEV)
        s.k_cache = _cache(layers, s.num_pages, hkv, d, gen)
        s.v_cache = _cache(layers, s.num_pages, hkv, d, gen)
    elif c["kind"] == "compact":
        n, kept = c["rows"], _kept(c)
        s.max_pages = -(-(c["start"] + c["keep"] + c["window"]) // PAGE) + 1
        s.num_pages = _num_pages(c)
        s.block_table, s.refs = _tables(c["start"] + kept, s.max_pages, s.num_pages, n, r)
        s.ctx_len = _i32(c["start"] + kept)
        s.row = _i32(r.permutation(n))
        s.start = _i32(np.full(n, c["start"]))
        keep = np.full((n, c["keep"]), -1, np.int64)
        for j, row in enumerate(s.row.tolist()):
            k = int(kept[row])
            keep[j, :k] = np.concatenate([[0], 1 + np.sort(r.choice(c["window"] - 1, k - 1,
                                                                    replace=False))])
        s.keep, s.keep_len = _i32(keep), _i32(kept[s.row.cpu().numpy()])
        s.pages = torch.zeros(n, dtype=torch.int32, device=DEV)
        s.result = torch.zeros(n, dtype=torch.int32, device=DEV)
        s.k_cache = _cache(layers, s.num_pages, hkv, d, gen)
        s.v_cache = _cache(layers, s.num_pages, hkv, d, gen)
        if own:
            s.ws = torch.empty(pic.pic_page_compact_workspace_size(s.geom, n, c["keep"]),
                               dtype=torch.uint8, device=DEV)
    else:
        n = c["pages"]
        s.num_pages = 2 * n
        s.k_cache = _cache(layers, 2 * n if c["within"] else n, hkv, d, gen)
        s.v_cache = _cache(layers, 2 * n if c["within"] else n, hkv, d, gen)
        if c["within"]:  # between the places of one cache
            perm = r.permutation(2 * n)
            s.src, s.dst = _i32(perm[:n]), _i32(perm[n:])
            s.k_to, s.v_to = s.k_cache, s.v_cache
        else:  # into another cache
            s.src, s.dst = _i32(r.permutation(n)), _i32(r.permutation(n))
            s.k_to, s.v_to = torch.zeros_like(s.k_cache), torch.zeros_like(s.v_cache)
    return s


def _prepare_verify(s, gen):
    """Probabilities of logits with four likely tokens a row; the draft's are those of disturbed
    logits (less so the larger `agree`).  A chain's tokens are sampled from
    the draft's rows, a tree's are its most likely ones, siblings distinct."""
    c = s.c
    B, T, V = c["batch"], c["draft"], c["vocab"]
    logits = 4.0 * torch.randn((B, T, V), generator=gen, device=DEV)
    likely = torch.randint(0, V, (B, T, 4), generator=gen, device=DEV)
    logits.scatter_(2, likely, torch.tensor([21.0, 20.5, 20.0, 19.0], device=DEV).expand(B, T, 4))
    s.target = torch.softmax(logits, -1)
    logits.add_(torch.randn((B, T, V), generator=gen, device=DEV), alpha=1.0 / c["agree"])
    s.draft_len = _i32(_draft_len(c))
    s.uniform = torch.rand((B, T), generator=gen, device=DEV)
    s.parent = s.draft = None
    s.tokens = torch.zeros((B, T), dtype=torch.int32, device=DEV)
    if c["tree"]:
        par = _parents(c)
        order = logits.topk(min(T, V), dim=-1).indices  # [B][T][T]
        rank = np.zeros_like(par)
        for i in range(1, T):
            rank[:, i] = (par[:, 1:i] == par[:, i:i + 1]).sum(1)
        p, k = torch.as_tensor(par, device=DEV).clamp(min=0), torch.as_tensor(rank, device=DEV)
        b = torch.arange(B, device=DEV)[:, None]
        s.tokens = order[b, p, k].int().contiguous()
        s.parent = _i32(par)
    elif T > 1:
        s.draft = torch.softmax(logits, -1)[:, :-1].contiguous()
        noise = torch.empty((B, T - 1, V), device=DEV).exponential_(generator=gen)
        s.tokens[:, 1:] = (s.draft / noise).argmax(-1).int()
    s.path = torch.zeros((B, T), dtype=torch.int32, device=DEV)
    s.path_len = torch.zeros(B, dtype=torch.int32, device=DEV)
    s.next = torch.zeros(B, dtype=torch.int32, device=DEV)


# ------------------------------------------------------------------ one pass
def run(s):
    if s.kind == "attend":
        (_attend_own if own else _attend_plain)(s)
        return {"out": s.out, "lse": s.lse, "k_cache": s.k_cache, "v_cache": s.v_cache}
    if s.kind == "verify":
        (_verify_own if own else _verify_plain)(s)
        return {"path": s.path, "path_len": s.path_len, "next": s.next}
    if s.kind == "fork":
        (_fork_own if own else _fork_plain)(s)
        return {"block_table": s.block_table, "refs": s.refs, "ctx_len": s.ctx_len,
                "result": s.result, "k_cache": s.k_cache, "v_cache": s.v_cache}
    if s.kind == "compact":
        (_compact_own if own else _compact_plain)(s)
        return {"block_table": s.block_table, "refs": s.refs, "ctx_len": s.ctx_len,
                "pages": s.pages, "result": s.result, "k_cache": s.k_cache,
                "v_cache": s.v_cache}
    (_copy_own if own else _copy_plain)(s)
    return {"k": s.k_to, "v": s.v_to}


def _attend_own(s):
    import paper_2607_28069_gb300 as pic
    pic.pic_attend_draft(s.geom, 0, s.q, s.k_new, s.v_new, s.ctx_len, s.draft_len, s.block_table,
                         s.num_pages, s.k_cache, s.v_cache, s.out, parent=s.parent, lse=s.lse,
                         workspace=s.ws)


def _verify_own(s):
    import paper_2607_28069_gb300 as pic
    pic.pic_verify_draft(s.tokens, s.draft_len, s.target, s.uniform, s.path, s.path_len, s.next,
                         draft_prob=s.draft, parent=s.parent)


def _fork_own(s):
    import paper_2607_28069_gb300 as pic
    pic.pic_page_free(s.dst, s.block_table, s.num_pages, s.refs, s.ctx_len)
    pic.pic_page_fork(s.geom, s.src, s.dst, s.ctx_len, s.block_table, s.num_pages, s.refs,
                      s.k_cache, s.v_cache, s.result, reserve=s.c["reserve"])


def _compact_own(s):
    import paper_2607_28069_gb300 as pic
    pic.pic_page_reserve(s.row, s.c["window"], s.ctx_len, s.block_table, s.num_pages, s.refs,
                         s.pages)
    pic.pic_page_compact(s.geom, s.row, s.keep, s.keep_len, s.ctx_len, s.block_table, s.num_pages,
                         s.refs, s.k_cache, s.v_cache, s.result, start=s.start,
                         rotate=s.c["rotate"], workspace=s.ws)


def _copy_own(s):
    import paper_2607_28069_gb300 as pic
    pic.pic_page_copy(s.geom, s.src, s.dst, s.k_cache, s.v_cache, s.k_to, s.v_to)


# ------------------------------------------------------------ the plain forms
def _rotate(x, pos, base, style):
    """RoPE of x [..., d] (32 bits) at pos [...]; the angle is formed in 64."""
    d = x.shape[-1]
    theta = torch.pow(torch.tensor(base, dtype=torch.float64, device=x.device),
                      -2.0 * torch.arange(d // 2, device=x.device, dtype=torch.float64) / d)
    a = pos.double()[..., None] * theta
    cs, sn = torch.cos(a).to(x.dtype), torch.sin(a).to(x.dtype)
    if style == 0:
        u, w = x[..., :d // 2], x[..., d // 2:]
        return torch.cat([u * cs - w * sn, u * sn + w * cs], -1)
    u, w = x[..., 0::2], x[..., 1::2]
    return torch.stack([u * cs - w * sn, u * sn + w * cs], -1).flatten(-2)


def _closure(parent, T):
    """[B][T][T]: token j is token i or one of its ancestors."""
    j = torch.arange(T, device=DEV)
    step = torch.eye(T, device=DEV) + (parent[..., None] == j).float()
    return torch.matrix_power(step, 64) > 0


def _attend_plain(s):
    c = s.c
    B, T, d, G = c["batch"], c["draft"], s.d, s.hq // s.hkv
    t = torch.arange(T, device=DEV)
    parent = s.parent if s.parent is not None else (t - 1).expand(B, T)
    sees = _closure(parent, T)
    pos = s.ctx_len[:, None] + sees.sum(-1) - 1
    live = t < s.draft_len[:, None]
    b = torch.arange(B, device=DEV)[:, None]
    # the new keys and values into their slots
    slot = s.ctx_len[:, None].long() + t
    page, at = s.block_table[b, slot // PAGE].long(), slot % PAGE
    kr = _rotate(s.k_new.float(), pos[..., None].expand(B, T, s.hkv), s.base, c["style"]).bfloat16()
    kc, vc = s.k_cache[0], s.v_cache[0]
    old = live[..., None, None]
    kc[page, :, at] = torch.where(old, kr, kc[page, :, at])
    vc[page, :, at] = torch.where(old, s.v_new, vc[page, :, at])
    # attention over the stitched context: the keys before the drafts, then
    # the drafts that a token descends from
    n = s.max_pages * PAGE
    K = kc[s.block_table.clamp(min=0).long()].transpose(1, 2).reshape(B, s.hkv, n, d).float()
    q = _rotate(s.q.float(), pos[..., None].expand(B, T, s.hq), s.base, c["style"])
    q = q.bfloat16().float().view(B, T, s.hkv, G, d).permute(0, 2, 1, 3, 4).reshape(
        B, s.hkv, T * G, d)
    sc = (q @ K.transpose(-1, -2)).view(B, s.hkv, T, G, n) / math.sqrt(d)
    del K
    at = torch.arange(n, device=DEV) - s.ctx_len[:, None]  # [B][n]: which draft a key is
    own_key = sees.gather(2, at.clamp(0, T - 1)[:, None].expand(B, T, n))
    vis = (at < 0)[:, None] | ((at >= 0) & (at < s.draft_len[:, None]))[:, None] & own_key
    sc = sc.masked_fill(~vis[:, None, :, None], -math.inf)
    m = sc.amax(-1, keepdim=True)
    p = torch.exp(sc - m)
    del sc
    l = p.sum(-1, keepdim=True)
    V = vc[s.block_table.clamp(min=0).long()].transpose(1, 2).reshape(B, s.hkv, n, d).float()
    o = (p.view(B, s.hkv, T * G, n) @ V).view(B, s.hkv, T, G, d) / l
    o = o.permute(0, 2, 1, 3, 4).reshape(B, T, s.hq, d).bfloat16()
    lse = (m + torch.log(l)).view(B, s.hkv, T, G).permute(0, 2, 1, 3).reshape(B, T, s.hq)
    s.out.copy_(torch.where(old, o, s.out))
    s.lse.copy_(torch.where(live[..., None], lse, s.lse))


def _weights(p):
    """Probabilities as whole numbers of 2^-36 (sums of them have no order)."""
    return (p.clamp(0.0, 1.0) * 2.0 ** 36).long()


def _sample(w, u):
    """The first entry whose running sum of w exceeds the share u of the total."""
    cum = w.cumsum(-1)
    r = (cum[..., -1] * (u * 2.0 ** 24).long().clamp(0, 2 ** 24 - 1)) >> 24
    x = (cum > r[..., None]).int().argmax(-1)
    return torch.where(cum[..., -1] > 0, x, -1)


def _verify_plain(s):
    c = s.c
    B, T = c["batch"], c["draft"]
    t = torch.arange(T, device=DEV)
    live = t < s.draft_len[:, None]
    if s.parent is None:
        b = torch.arange(B, device=DEV)
        tok = s.tokens[:, 1:, None].long()
        if T > 1:
            p = s.target[:, :-1].gather(2, tok)[..., 0]
            q = s.draft.gather(2, tok)[..., 0]
            ok = (s.uniform[:, :-1] * q < p) & live[:, 1:]
            acc = ok.int().cumprod(-1).sum(-1)
        else:
            acc = torch.zeros(B, dtype=torch.long, device=DEV)
        p = s.target[b, acc]
        w = _weights(p)
        if T > 1:  # refused somewhere: what the draft had too little of
            rest = _weights((p - s.draft[b, acc.clamp(max=T - 2)]).clamp(min=0.0))
            take = (acc < s.draft_len - 1) & (rest.sum(-1) > 0)
            w = torch.where(take[:, None], rest, w)
        u = s.uniform[b, s.draft_len.long() - 1]
        s.next.copy_(_sample(w, u))
        s.path.copy_(torch.where(t <= acc[:, None], t, -1))
        s.path_len.copy_(acc + 1)
        return
    sees = _closure(s.parent, T)
    depth = sees.sum(-1) - 1
    x = _sample(_weights(s.target), s.uniform.gather(1, depth))  # [B][T]: a draw at every node
    child = (s.parent[:, None] == t[:, None]) & (s.tokens[:, None] == x[..., None]) & live[:, None]
    first = torch.where(child.any(-1), child.int().argmax(-1), -1)  # [B][T]
    taken = (first.gather(1, s.parent.clamp(min=0).long()) == t) | (t == 0)
    on = (sees & ~taken[:, None]).sum(-1) == 0  # every step from the root to here was taken
    k = on.sum(-1)
    order = torch.where(on, depth, T + t).sort(-1).indices
    path = torch.where(t < k[:, None], order, -1)
    s.path.copy_(path)
    s.path_len.copy_(k)
    s.next.copy_(x.gather(1, path.gather(1, k[:, None] - 1))[:, 0])


def _free_pages(refs):
    """Every page, the unused ones first, lowest numbers first."""
    return torch.argsort((refs != 0).int(), stable=True)


def _release(s, table, cut):
    """Gives back the pages of `table`'s entries where `cut`."""
    cut = cut & (table >= 0)
    s.refs.index_add_(0, table.clamp(min=0).long().flatten(), -cut.int().flatten())
    return torch.where(cut, -1, table)


def _fork_plain(s):
    reserve = s.c["reserve"]
    src, dst = s.src.long(), s.dst.long()
    col = torch.arange(s.max_pages, device=DEV)
    s.block_table[dst] = _release(s, s.block_table[dst], torch.ones_like(s.block_table[dst],
                                                                         dtype=torch.bool))
    ctx = s.ctx_len[src].long()
    full = ctx // PAGE
    need = (ctx + reserve + PAGE - 1) // PAGE - full
    first = need.cumsum(0) - need
    free = _free_pages(s.refs)
    new = free[(first[:, None] + col - full[:, None]).clamp(0, s.num_pages - 1)].int()
    old = s.block_table[src]
    shared, fresh = col < full[:, None], (col >= full[:, None]) & (col < (full + need)[:, None])
    table = torch.where(shared, old, torch.where(fresh, new, -1))
    s.refs.index_add_(0, table.clamp(min=0).long().flatten(), (shared | fresh).int().flatten())
    s.block_table[dst] = table
    s.ctx_len[dst] = ctx.int()
    s.result.copy_(ctx)
    # the rows of the page that the context ends in, where it ends inside one
    # (elsewhere the context's first page is written back to itself)
    part = ctx % PAGE > 0
    a = torch.where(part, old.gather(1, full[:, None])[:, 0], old[:, 0]).long()
    z = torch.where(part, table.gather(1, full[:, None])[:, 0], old[:, 0]).long()
    row = (torch.arange(PAGE, device=DEV) < (ctx % PAGE)[:, None])[None, :, None, :, None]
    for cache in (s.k_cache, s.v_cache):
        cache[:, z] = torch.where(row, cache[:, a], cache[:, z])


def _compact_plain(s):
    c = s.c
    row = s.row.long()
    col = torch.arange(s.max_pages, device=DEV)
    # room for the window behind the present length
    ctx = s.ctx_len[row].long()
    have, want = (ctx + PAGE - 1) // PAGE, (ctx + c["window"] + PAGE - 1) // PAGE
    table = s.block_table[row]
    lack = (col >= have[:, None]) & (col < want[:, None]) & (table < 0)
    n = lack.sum(-1)
    free = _free_pages(s.refs)
    at = (n.cumsum(0) - n)[:, None] + lack.cumsum(-1) - 1
    table = torch.where(lack, free[at.clamp(0, s.num_pages - 1)].int(), table)
    s.refs.index_add_(0, table.clamp(min=0).long().flatten(), lack.int().flatten())
    s.pages.copy_(want)
    # the kept positions move together
    keep = s.keep.long()
    i = torch.arange(c["keep"], device=DEV)
    start = s.start.long()[:, None]
    src, dst = start + keep.clamp(min=0), start + i
    a, z = table.gather(1, src // PAGE).long(), table.gather(1, dst // PAGE).long()
    live = i < s.keep_len[:, None]
    # an entry past the kept ones moves nothing: one write of what is there
    # already, at the row's first kept position
    first = live.long() * 0 + 0
    a = torch.where(live, a, a.gather(1, first))
    z = torch.where(live, z, z.gather(1, first))
    ra = torch.where(live, src % PAGE, (src % PAGE).gather(1, first))
    rz = torch.where(live, dst % PAGE, (dst % PAGE).gather(1, first))
    by = torch.where(live, dst - src, 0)
    k, v = s.k_cache[:, a, :, ra], s.v_cache[:, a, :, ra]  # [n][keep][layers][hkv][d]
    if c["rotate"]:
        turned = _rotate(k.float(), by[..., None, None].expand(k.shape[:-1]), s.base, 0).bfloat16()
        k = torch.where((by != 0)[..., None, None, None], turned, k)
    s.k_cache[:, z, :, rz] = k
    s.v_cache[:, z, :, rz] = v
    # the pages behind them go back
    length = s.start.long() + s.keep_len.long()
    s.block_table[row] = _release(s, table, col >= ((length + PAGE - 1) // PAGE)[:, None])
    s.ctx_len[row] = length.int()
    s.result.copy_(length)


def _copy_plain(s):
    src, dst = s.src.long(), s.dst.long()
    s.k_to[:, dst] = s.k_cache[:, src]
    s.v_to[:, dst] = s.v_cache[:, src]


# ---------------------------------------------------------------- in 64 bits
def _turn64(x, pos, base, style):
    """RoPE of the numpy vectors x [..., d] at pos [...], as complex numbers."""
    d = x.shape[-1]
    w = np.exp(1j * np.asarray(pos, np.float64)[..., None] * base ** (-2.0 * np.arange(d // 2) / d))
    if style == 0:
        z = (x[..., :d // 2] + 1j * x[..., d // 2:]) * w
        return np.concatenate([z.real, z.imag], -1)
    z = (x[..., 0::2] + 1j * x[..., 1::2]) * w
    return np.stack([z.real, z.imag], -1).reshape(x.shape)


def exact(case, seed):
    c = case
    if c["kind"] == "verify":
        return None  # whole numbers alone
    s = prepare(c, seed)
    host = lambda x: x.cpu().numpy()  # noqa: E731
    if c["kind"] == "copy":
        k, v = s.k_to.double(), s.v_to.double()
        for i, j in zip(host(s.src).tolist(), host(s.dst).tolist()):
            k[:, j] = s.k_cache[:, i].double()
            v[:, j] = s.v_cache[:, i].double()
        return {"k": k, "v": v}
    if c["kind"] == "fork":
        k, v = s.k_cache.double(), s.v_cache.double()
        bt, ctx = host(s.block_table), host(s.ctx_len)
        free = [p for p, n in enumerate(host(s.refs).tolist()) if n == 0]
        for a in host(s.src).tolist():
            n, rows = -(-(int(ctx[a]) + c["reserve"]) // PAGE) - int(ctx[a]) // PAGE, int(ctx[a]) % PAGE
            mine, free = free[:n], free[n:]
            if rows:
                page = int(bt[a, int(ctx[a]) // PAGE])
                k[:, mine[0], :, :rows] = k[:, page, :, :rows]
                v[:, mine[0], :, :rows] = v[:, page, :, :rows]
        return {"block_table": None, "refs": None, "ctx_len": None, "result": None, "k_cache": k,
                "v_cache": v}
    if c["kind"] == "compact":
        return _exact_compact(s, c, host)
    out = torch.zeros(s.out.shape, dtype=torch.float64, device=DEV)
    lse = torch.zeros(s.lse.shape, dtype=torch.float64, device=DEV)
    k_all, v_all = s.k_cache.double(), s.v_cache.double()
    par = _parents(c) if c["tree"] else np.tile(np.arange(c["draft"]) - 1, (c["batch"], 1))
    G, rt = s.hq // s.hkv, math.sqrt(s.d)
    for b in range(c["batch"]):
        n, t = int(s.ctx_len[b]), int(s.draft_len[b])
        line = [[] for _ in range(t)]
        for i in range(t):
            line[i] = (line[par[b, i]] if par[b, i] >= 0 else []) + [i]
        pos = np.array([n + len(x) - 1 for x in line])
        f64 = lambda x: x[b, :t].double().cpu().numpy()  # noqa: E731,B023
        kn = torch.as_tensor(_turn64(f64(s.k_new), pos[:, None], s.base, c["style"]), device=DEV)
        qn = torch.as_tensor(_turn64(f64(s.q), pos[:, None], s.base, c["style"]), device=DEV)
        at = torch.arange(n + t, device=DEV)
        page = s.block_table[b].long()[at // PAGE]
        k_all[0, page[n:], :, at[n:] % PAGE] = kn
        v_all[0, page[n:], :, at[n:] % PAGE] = s.v_new[b, :t].double()
        vis = torch.zeros((t, n + t), dtype=torch.bool, device=DEV)
        vis[:, :n] = True
        for i in range(t):
            vis[i, [n + j for j in line[i]]] = True
        for g in range(s.hkv):
            K, V = k_all[0, page, g, at % PAGE], v_all[0, page, g, at % PAGE]
            for h in range(g * G, (g + 1) * G):
                z = torch.where(vis, qn[:, h] @ K.T / rt, -math.inf)
                lse[b, :t, h] = torch.logsumexp(z, -1)
                out[b, :t, h] = torch.exp(z - lse[b, :t, h, None]) @ V
    return {"out": out, "lse": lse, "k_cache": k_all, "v_cache": v_all}


def _exact_compact(s, c, host):
    k, v = s.k_cache.double(), s.v_cache.double()
    bt, ctx = host(s.block_table), host(s.ctx_len)
    free = [p for p, n in enumerate(host(s.refs).tolist()) if n == 0]
    for j, row in enumerate(host(s.row).tolist()):
        have, want = -(-int(ctx[row]) // PAGE), -(-(int(ctx[row]) + c["window"]) // PAGE)
        table = bt[row, :have].tolist() + free[:want - have]
        free = free[want - have:]
        m = int(s.keep_len[j])
        old = c["start"] + host(s.keep)[j, :m].astype(np.int64)
        new = c["start"] + np.arange(m)
        table = torch.as_tensor(table, device=DEV)
        o, w = torch.as_tensor(old, device=DEV), torch.as_tensor(new, device=DEV)
        x, y = k[:, table[o // PAGE], :, o % PAGE], v[:, table[o // PAGE], :, o % PAGE]
        if c["rotate"]:
            x = torch.as_tensor(_turn64(x.cpu().numpy(), (new - old)[:, None, None], s.base, 0),
                                device=DEV)
        k[:, table[w // PAGE], :, w % PAGE] = x
        v[:, table[w // PAGE], :, w % PAGE] = y
    return {"block_table": None, "refs": None, "ctx_len": None, "pages": None, "result": None,
            "k_cache": k, "v_cache": v}
