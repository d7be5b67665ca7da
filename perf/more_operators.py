"""Performance cases of decoding many branches of linked contexts.

After a cache hit a serving program forks a linked context (best-of-n sampling,
agents that continue one conversation) and decodes the branches together.  One
step plans the batch from its block tables (which rows share which pages), and
per layer norms and rotates the new queries and keys, appends keys and values to
the paged cache and attends, every shared key read once; then the next tokens are
sampled from the logits.  Each case is one such call, or the whole step, with
``own`` through the package's ``pic_append_normed``, ``pic_share_plan``,
``pic_attend_shared`` and ``pic_sample``, else in elementary torch operations.

Sizes are those of workloads.py, cases.py and the parity tests, or lie between
them; vocabularies are generic.  A case is a dict of plain values; lengths and the
way contexts branch follow from the case alone, values, random numbers and page
placement from the seed.
"""
from __future__ import annotations

import math
from types import SimpleNamespace

import numpy as np
import torch

own = False
DEV = "cuda"
PAGE = 16
TILE = 128    # positions of a tile of the plan
LEVELS = 4    # shared nodes above a branch, at most
EPS = 1e-6
LOG2E = 1.4426950408889634
# 2^f on [-1/2, 1/2] within 2e-7, of the sampling rule
EXP2 = (0.6931470036506653, 0.24022242426872253, 0.05550733581185341, 0.009671512991189957,
        0.001326472731307149)

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
def _append(geom, batch, tokens, ctx, style=0, fused=True):
    return dict(kind="append", geom=geom, batch=batch, tokens=tokens, ctx=ctx, style=style,
                fused=fused)


def _branches(kind, geom, contexts, children, root, ctx, tail, q_scale=1.0, **more):
    """`contexts` contexts of ctx positions, the first `root` of them common to all, each with
    `children` branches that have grown by a tail of their own."""
    return dict(kind=kind, geom=geom, contexts=contexts, children=children, root=root,
                ctx_lo=ctx[0], ctx_hi=ctx[1], tail_lo=tail[0], tail_hi=tail[1], q_scale=q_scale,
                **more)


def _sample(batch, vocab, dtype, mix):
    return dict(kind="sample", batch=batch, vocab=vocab, dtype=dtype, mix=mix)


def listed():
    c = []

    def add(name, case):
        c.append(dict(case, name=name))

    # The new token of one request on the "tiny" workload: launches and round trips.
    add("append_tiny", _append("4/1/64", 1, 1, 160))
    # Ragged prefills of eight requests, up to 1067 inline tokens, projections
    # that are views of one fused product.
    add("append_prefill_b8", _append("32/8/128", 8, 1067, 16000))
    # Best-of-4 off one small linked context.
    add("plan_4", _branches("plan", "8/2/128", 1, 4, 0, (4290, 4290), (1, 60)))
    # The largest plan: 64 branches each of four ~139k contexts.
    add("plan_256_128k", _branches("plan", "32/8/128", 4, 64, 2000, (138000, 140000), (1, 500)))
    # The smallest attention: four branches of the "tiny" workload's context.
    add("attend_tiny", _branches("attend", "4/1/64", 1, 4, 0, (160, 160), (1, 9), q_scale=2.0))
    # Eight contexts with a common beginning, six ragged branches of each, 64-wide
    # heads in GQA groups of 8.
    add("attend_nested_d64", _branches("attend", "16/2/64", 8, 6, 1100, (3000, 9001), (1, 700)))
    # Best-of-64 off one ~33k context of the decode workload, GQA groups of 7.
    add("attend_best_of_64", _branches("attend", "28/4/128", 1, 64, 0, (33000, 33000), (1, 400)))
    # Sixteen branches of one ~139k context.
    add("attend_128k_x16", _branches("attend", "32/8/128", 1, 16, 0, (139000, 139000), (1, 900)))
    # One request's next token over an odd vocabulary: temperature and top-p.
    add("sample_1req", _sample(1, 50001, "float32", "top_p"))
    # Temperature alone: every entry is a candidate.
    add("sample_plain_b64", _sample(64, 131072, "float32", "plain"))
    # A batch whose requests each bring their own settings (some greedy, top-k,
    # top-p, min-p, all of them), bf16 logits of an odd vocabulary.
    add("sample_mixed_b48", _sample(48, 100003, "bfloat16", "mixed"))
    # A whole step of 32 branches of two contexts, two layers.
    add("step_2x16", _branches("step", "32/8/128", 2, 16, 500, (9000, 16000), (1, 300), layers=2,
                               vocab=131072))
    return c


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 0.49)))))))


def draw(rng):
    """One more case of the listed ranges: any kind, sizes log-uniform."""
    top = [work(x) for x in listed()]
    top = (max(x["bytes"] for x in top), max(x["flops"] for x in top))
    while True:
        kind = rng.choice(["append", "append", "plan", "attend", "attend", "attend", "sample",
                           "sample", "step"])
        geom = rng.choice(list(GEOMS))
        if kind == "append":
            c = _append(geom, _log_int(rng, 1, 256), rng.choice([1, _log_int(rng, 1, 1067)]),
                        _log_int(rng, 1, 120000), style=rng.randint(0, 1), fused=rng.random() < 0.6)
            if c["batch"] * (c["ctx"] + c["tokens"]) > 2e6:
                continue
        elif kind == "sample":
            c = _sample(_log_int(rng, 1, 64), _log_int(rng, 8000, 160000),
                        rng.choice(["float32", "bfloat16"]), rng.choice(["plain", "top_p", "mixed"]))
        else:
            hi = _log_int(rng, 30, 140000)
            lo = rng.choice([hi, hi // rng.randint(2, 9)])
            more = {} if kind != "step" else dict(layers=rng.randint(1, 3),
                                                  vocab=_log_int(rng, 8000, 160000))
            c = _branches(kind, geom, _log_int(rng, 1, 24), _log_int(rng, 1, 64),
                          rng.choice([0, 0, rng.randint(0, lo)]), (lo, hi),
                          (1, _log_int(rng, 1, 900)), q_scale=rng.choice([1.0, 1.0, 2.0]), **more)
            n = c["contexts"] * c["children"]
            # the plain form's gathered keys in 32 bits stay within a few GB
            if n > 256 or (kind != "plan" and n * (hi + 900) * GEOMS[geom][1] * GEOMS[geom][2] > 2.4e9):
                continue
            if kind != "plan" and n * (hi + 900) * GEOMS[geom][0] > 3e8:
                continue
            if kind == "step" and n * c["vocab"] > 64 * 131072:
                continue
        w = work(c)
        if w["bytes"] < top[0] and w["flops"] <= top[1]:
            return c


# --------------------------------------------- what follows from a case alone
def _rng(c):
    return np.random.default_rng(sum((i + 1) * int(v) for i, v in enumerate(c.values())
                                     if isinstance(v, (int, float))) % (1 << 31))


def _token_counts(c):
    """Tokens of each request: all of them for the first, from a third up for the others."""
    t = c["tokens"]
    lens = _rng(c).integers((t + 2) // 3, t + 1, size=c["batch"])
    lens[0] = t
    return lens.astype(np.int64)


def _tree(c):
    """(context lengths, tails [contexts][children])."""
    r = _rng(c)
    ctx = r.integers(c["ctx_lo"], c["ctx_hi"] + 1, size=c["contexts"])
    ctx[0] = c["ctx_hi"]
    tail = r.integers(c["tail_lo"], c["tail_hi"] + 1, size=(c["contexts"], c["children"]))
    return ctx.astype(np.int64), tail.astype(np.int64)


def _unique_positions(c):
    """Positions that have a place of their own: shared pages once."""
    ctx, tail = _tree(c)
    root = min(c["root"], int(ctx.min())) // PAGE * PAGE if c["contexts"] > 1 else 0
    return root + int(((ctx // PAGE * PAGE - root)[:, None] * 1).sum() +
                      (ctx % PAGE)[:, None].repeat(c["children"], 1).sum() + tail.sum())


def work(case):
    c = case
    if c["kind"] == "sample":
        n = c["batch"] * c["vocab"]
        return {"bytes": n * (4 if c["dtype"] == "float32" else 2) + c["batch"] * 32,
                "flops": 20.0 * n}
    hq, hkv, d, _ = GEOMS[c["geom"]]
    if c["kind"] == "append":
        tok = int(_token_counts(c).sum())
        return {"bytes": tok * (hq + 2 * hkv) * d * 4, "flops": 9.0 * tok * (hq + hkv) * d}
    ctx, tail = _tree(c)
    keys = ctx[:, None] + tail
    if c["kind"] == "plan":
        return {"bytes": int(((keys + PAGE - 1) // PAGE).sum()) * 4 + keys.size * 68, "flops": 0}
    layers = c.get("layers", 1)
    b = layers * (_unique_positions(c) * hkv * d * 4 + keys.size * hq * d * 4)
    f = layers * 4.0 * d * hq * int(keys.sum())
    if c["kind"] == "step":
        tok = keys.size * layers
        b += tok * (hq + 2 * hkv) * d * 4 + keys.size * c["vocab"] * 4
        f += 9.0 * tok * (hq + hkv) * d + 20.0 * keys.size * c["vocab"]
    return {"bytes": b, "flops": f}


# ------------------------------------------------------------- input building
def _i32(x):
    return torch.as_tensor(np.ascontiguousarray(x), dtype=torch.int32).to(DEV)


def _projections(s, shape, gen, fused):
    """q, k, v of heads `s.hq`, `s.hkv`, `s.hkv`: views of one product's rows, or of their own."""
    heads = (s.hq, s.hkv, s.hkv)
    if fused:
        x = torch.randn((*shape, sum(heads), s.d), generator=gen, device=DEV).bfloat16()
        return x.split(heads, dim=-2)
    return [torch.randn((*shape, h, s.d), generator=gen, device=DEV).bfloat16() for h in heads]


def _norm_weights(s, gen):
    return [(1 + 0.3 * torch.randn(s.d, generator=gen, device=DEV)).bfloat16() for _ in range(2)]


def prepare(case, seed):
    c = case
    gen = torch.Generator(device=DEV).manual_seed(seed)
    r = np.random.default_rng(seed)
    s = SimpleNamespace(c=c, kind=c["kind"])
    if c["kind"] == "sample":
        _prepare_sample(s, gen, r, c["batch"], c["vocab"], c["dtype"], c["mix"])
        return s
    s.hq, s.hkv, s.d, s.base = GEOMS[c["geom"]]
    s.style = c.get("style", 0)
    layers = c.get("layers", 1)
    if own:
        import paper_2607_28069_gb300 as pic
        s.geom = pic.Geometry(layers, s.hq, s.hkv, s.d, s.base, rope_style=s.style)
    if c["kind"] == "append":
        lens, B, T = _token_counts(c), c["batch"], c["tokens"]
        start = r.integers(max(1, c["ctx"] // 2), c["ctx"] + 1, size=B)
        s.max_pages = -(-(c["ctx"] + T) // PAGE)
        # only the pages that get a token exist
        s.num_pages = B * (-(-T // PAGE) + 2)
        bt = np.full((B, s.max_pages), -1, np.int64)
        perm, o = r.permutation(s.num_pages), 0
        for b in range(B):
            lo, hi = int(start[b]) // PAGE, -(-int(start[b] + lens[b]) // PAGE)
            bt[b, lo:hi] = perm[o:o + hi - lo]
            o += hi - lo
        s.block_table, s.count = _i32(bt), _i32(lens)
        s.pos = _i32(start[:, None] + np.arange(T))
        s.q, s.k, s.v = _projections(s, (B, T), gen, c["fused"])
        s.wq, s.wk = _norm_weights(s, gen)
        shape = (1, s.num_pages, s.hkv, PAGE, s.d)
        s.k_cache = torch.zeros(shape, dtype=torch.bfloat16, device=DEV)
        s.v_cache = torch.zeros(shape, dtype=torch.bfloat16, device=DEV)
        s.q_out = torch.zeros((B, T, s.hq, s.d), dtype=torch.bfloat16, device=DEV)
        return s
    _prepare_branches(s, c, gen, r, layers)
    if c["kind"] == "step":
        n = s.n
        s.q, s.k, s.v = [x.unbind(0) for x in _projections(s, (layers, n, 1), gen, True)]
        s.wq, s.wk = _norm_weights(s, gen)
        s.q_rot = torch.zeros((n, 1, s.hq, s.d), dtype=torch.bfloat16, device=DEV)
        s.sampling = SimpleNamespace()
        _prepare_sample(s.sampling, gen, r, n, c["vocab"], "float32", "top_p")
    elif c["kind"] == "attend":
        s.q = (torch.randn((s.n, s.hq, s.d), generator=gen, device=DEV) * c["q_scale"]).bfloat16()
    if own:
        s.plan = torch.zeros(pic.pic_share_plan_size(s.n) // 4, dtype=torch.int32, device=DEV)
        s.ws = torch.empty(pic.pic_shared_workspace_size(s.geom, s.n), dtype=torch.uint8, device=DEV)
        if c["kind"] == "attend":  # the step's plan, made before its layers
            _plan_own(s)
    return s


def _prepare_branches(s, c, gen, r, layers):
    """Block tables as forks leave them: a branch shares its context's full pages, and has the
    last, partly filled one and its tail's to itself.  Rows of the table in any order; the list
    names branches of one context side by side."""
    ctx, tail = _tree(c)
    P, m = tail.shape
    s.n = P * m
    grow = 1 if c["kind"] == "step" else 0  # the position that the step appends
    full = ctx // PAGE
    root = min(c["root"], int(ctx.min())) // PAGE if P > 1 else 0
    need = -(-(ctx[:, None] + tail + grow) // PAGE) - full[:, None]
    s.num_pages = int(root + (full - root).sum() + need.sum()) + 3
    s.max_pages = int((full[:, None] + need).max()) + 1
    perm = r.permutation(s.num_pages)
    bt = np.full((s.n, s.max_pages), -1, np.int64)
    row = r.permutation(s.n)
    first, o = perm[:root], root
    for p in range(P):
        mine = perm[o:o + int(full[p]) - root]
        o += len(mine)
        for j in range(m):
            k, at = int(need[p, j]), row[p * m + j]
            bt[at, :int(full[p]) + k] = np.concatenate([first, mine, perm[o:o + k]])
            o += k
    s.row, s.block_table = _i32(row), _i32(bt)
    lens = np.zeros(s.n, np.int64)
    lens[row] = (ctx[:, None] + tail).reshape(-1)
    s.ctx_len = _i32(lens)
    # the last position that a branch sees: its context's, or the one a step appends behind it
    s.pos_offset = 0 if c["kind"] == "step" else -1
    if c["kind"] == "plan":
        return
    shape = (layers, s.num_pages, s.hkv, PAGE, s.d)
    s.k_cache = torch.randn(shape, generator=gen, device=DEV, dtype=torch.bfloat16)
    s.v_cache = torch.randn(shape, generator=gen, device=DEV, dtype=torch.bfloat16)
    s.out = torch.zeros((layers, s.n, s.hq, s.d), dtype=torch.bfloat16, device=DEV)
    s.lse = torch.zeros((layers, s.n, s.hq), dtype=torch.float32, device=DEV)


def _prepare_sample(s, gen, r, n, vocab, dtype, mix):
    """Logits with a few likely tokens a row, as a model's are, and each request's settings."""
    x = 3.0 * torch.randn((n, vocab), generator=gen, device=DEV)
    likely = torch.randint(0, vocab, (n, 6), generator=gen, device=DEV)
    x.scatter_(1, likely, torch.tensor([17.0, 16.5, 16.0, 15.5, 14.5, 13.0], device=DEV).expand(n, 6))
    s.logits = x if dtype == "float32" else x.bfloat16()
    f32 = lambda a: torch.as_tensor(a, dtype=torch.float32).to(DEV)  # noqa: E731
    s.uniform = torch.rand(n, generator=gen, device=DEV)
    s.temperature = f32(r.uniform(0.5, 1.3, n))
    s.top_k = s.top_p = s.min_p = None
    if mix == "top_p":
        s.top_p = f32(np.full(n, 0.9))
    elif mix == "mixed":
        use = r.random((4, n)) < 0.5
        s.temperature = torch.where(torch.as_tensor(use[0] & use[1] & use[2], device=DEV), 0.0, s.temperature)
        s.top_k = _i32(np.where(use[1], np.exp(r.uniform(0, np.log(2000), n)).astype(np.int64), 0))
        s.top_p = f32(np.where(use[2], r.uniform(0.3, 1.0, n), 1.0))
        s.min_p = f32(np.where(use[3], r.uniform(0.0, 0.2, n), 0.0))
    s.token = torch.zeros(n, dtype=torch.int32, device=DEV)
    s.kept = torch.zeros(n, dtype=torch.int32, device=DEV)
    s.logprob = torch.zeros(n, dtype=torch.float32, device=DEV)


# ------------------------------------------------------------------ one pass
def run(s):
    if s.kind == "append":
        (_append_own if own else _append_plain)(s, 0, s.q, s.k, s.v, s.q_out, s.count, s.pos)
        return {"q": s.q_out, "k_cache": s.k_cache, "v_cache": s.v_cache}
    if s.kind == "plan":
        return {"nodes": (_plan_own if own else _plan_plain)(s)}
    if s.kind == "attend":
        (_attend_own if own else _attend_plain)(s, 0, s.q)
        return {"out": s.out, "lse": s.lse}
    if s.kind == "sample":
        (_sample_own if own else _sample_plain)(s)
        return {"token": s.token, "kept": s.kept, "logprob": s.logprob}
    (_step_own if own else _step_plain)(s)
    t = s.sampling
    return {"out": s.out, "k_cache": s.k_cache, "v_cache": s.v_cache, "token": t.token,
            "kept": t.kept, "logprob": t.logprob}


def _append_own(s, layer, q, k, v, q_out, count, pos):
    import paper_2607_28069_gb300 as pic
    pic.pic_append_normed(s.geom, layer, q, k, v, s.block_table, s.num_pages, s.k_cache, s.v_cache,
                          q_out, q_weight=s.wq, k_weight=s.wk, eps=EPS, num_tokens=count, pos=pos)


def _plan_own(s):
    import paper_2607_28069_gb300 as pic
    pic.pic_share_plan(s.geom, s.ctx_len, s.block_table, s.num_pages, s.plan, row=s.row,
                       pos_offset=s.pos_offset)
    return pic.share_nodes(s.plan, s.n)


def _attend_own(s, layer, q):
    import paper_2607_28069_gb300 as pic
    pic.pic_attend_shared(s.geom, layer, q, s.block_table, s.num_pages, s.k_cache, s.v_cache, s.plan,
                          (s.out, layer), lse=(s.lse, layer) if s.kind == "attend" else None,
                          workspace=s.ws)


def _sample_own(s):
    import paper_2607_28069_gb300 as pic
    pic.pic_sample(s.logits, s.uniform, s.token, temperature=s.temperature, top_k=s.top_k,
                   top_p=s.top_p, min_p=s.min_p, logprob=s.logprob, kept=s.kept)


def _step_own(s):
    import paper_2607_28069_gb300 as pic
    _plan_own(s)
    for layer in range(s.c["layers"]):
        pic.pic_append_normed(s.geom, layer, s.q[layer], s.k[layer], s.v[layer], s.block_table,
                              s.num_pages, s.k_cache, s.v_cache, s.q_rot, q_weight=s.wq,
                              k_weight=s.wk, eps=EPS, row=s.row, ctx_len=s.ctx_len)
        _attend_own(s, layer, s.q_rot)
    _sample_own(s.sampling)


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


def _normed(x, weight):
    x = x.float()
    return x * torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS) * weight.float()


def _append_plain(s, layer, q, k, v, q_out, count, pos, table=None):
    table = s.block_table if table is None else table
    B, T = q.shape[:2]
    live = torch.arange(T, device=DEV) < count[:, None]
    b, t = live.nonzero(as_tuple=True)
    p = pos[b, t].long()
    page, at = table[b, p // PAGE].long(), p % PAGE
    turn = lambda x, w, h: _rotate(_normed(x[b, t], w), p[:, None].expand(-1, h), s.base,  # noqa: E731
                                   s.style).bfloat16()
    q_out[b, t] = turn(q, s.wq, s.hq)
    s.k_cache[layer, page, :, at] = turn(k, s.wk, s.hkv)
    s.v_cache[layer, page, :, at] = v[b, t]


def _plan_plain(s):
    """The nodes [2 n][8]: begin, end (of the list's entries), tile_begin, tile_end, row, keys,
    parent, level.  Node j < n: entry j's own tiles; node n + i: the run of entries around i that
    share more than the entries beyond it."""
    n = s.n
    row = s.row.long()
    keys = s.ctx_len[row].long() + s.pos_offset + 1
    bt = s.block_table[row]
    i = torch.arange(n, device=DEV)
    nodes = torch.zeros((2 * n, 8), dtype=torch.int64, device=DEV)
    nodes[:, 4], nodes[:, 6], nodes[:, 7] = -1, -1, -1
    common = torch.zeros(n + 1, dtype=torch.int64, device=DEV)  # of entries i - 1 and i; 0 at both ends
    if n > 1:
        same = (bt[1:] == bt[:-1]) & (bt[1:] >= 0) & (bt[1:] < s.num_pages)
        lcp = same.int().cumprod(1).sum(1).long()
        common[1:n] = torch.minimum(lcp // (TILE // PAGE), torch.minimum(keys[1:], keys[:-1]) // TILE)
    L = common[1:n + 1]  # of boundary i, between entries i and i + 1; 0 for the last
    big = n + 1
    # nearest boundaries on either side that share less
    less = common[None, :] < L[:, None]          # [boundary][0..n]; boundary i is column i + 1
    col = torch.arange(n + 1, device=DEV)
    left = torch.where(less & (col < i[:, None] + 1), col, -1).amax(1)           # column, -1 never
    right = torch.where(less & (col > i[:, None] + 1), col, big).amin(1)
    same_before = ((common[None, :] == L[:, None]) & (col > left[:, None]) & (col < i[:, None] + 1)).any(1)
    there = (L > 0) & ~same_before
    # the node a boundary belongs to: the first boundary of its run with the same count
    rep = torch.where((common[None, :] == L[:, None]) & (col > left[:, None]) & (col < right[:, None]),
                      col, big).amin(1) - 1
    up_l, up_r = common[left.clamp(min=0)], common[right.clamp(max=n)]
    up = torch.where(up_l >= up_r, left, right) - 1  # boundary of the parent's run
    up = torch.where(torch.maximum(up_l, up_r) > 0, rep[up.clamp(0, n - 1)], -1)
    level, at = torch.zeros_like(i), up
    chain = [i]
    while bool((at >= 0).any()):
        level = level + (at >= 0)
        chain.append(at)
        at = torch.where(at >= 0, up[at.clamp(min=0)], -1)
    kept = there & (level < LEVELS)
    # a node's nearest kept ancestor
    anc = torch.full_like(i, -1)
    for at in reversed(chain[1:]):
        anc = torch.where((at >= 0) & kept[at.clamp(min=0)], at, anc)
    end = L
    begin = torch.where(anc >= 0, L[anc.clamp(min=0)], 0)
    inner = torch.stack([left.clamp(min=0), right.clamp(max=n), begin, end, row[left.clamp(min=0, max=n - 1)],
                         end * TILE, torch.where(anc >= 0, anc + n, -1), level], 1)
    nodes[n:] = torch.where(kept[:, None], inner, nodes[n:])
    # an entry's own tiles: below the deeper of the two boundaries beside it
    cl, cr = common[:n], common[1:n + 1]
    leaf = torch.where(cl >= cr, i - 1, i)
    leaf = torch.where(torch.maximum(cl, cr) > 0, rep[leaf.clamp(min=0)], -1)
    own_up = torch.where((leaf >= 0) & kept[leaf.clamp(min=0)], leaf, -1)
    own_up = torch.where((leaf >= 0) & (own_up < 0), anc[leaf.clamp(min=0)], own_up)
    tb = torch.where(own_up >= 0, L[own_up.clamp(min=0)], 0)
    lvl = torch.where(own_up >= 0, level[own_up.clamp(min=0)] + 1, 0)
    nodes[:n] = torch.stack([i, i + 1, tb, (keys + TILE - 1) // TILE, row, keys,
                             torch.where(own_up >= 0, own_up + n, -1), lvl], 1)
    return nodes.int()


def _attend_plain(s, layer, q):
    n, d, G = s.n, s.d, s.hq // s.hkv
    keys = s.ctx_len[s.row.long()].long() + s.pos_offset + 1
    table = s.block_table[s.row.long()].clamp(min=0).long()
    length = s.max_pages * PAGE
    gather = lambda cache: cache[layer][table].transpose(1, 2).reshape(  # noqa: E731
        n, s.hkv, length, d).float()
    qg = q.reshape(n, s.hkv, G, d).float()
    sc = (qg @ gather(s.k_cache).transpose(-1, -2)) / math.sqrt(d)
    sc = sc.masked_fill(torch.arange(length, device=DEV) >= keys[:, None, None, None], -math.inf)
    m = sc.amax(-1, keepdim=True)
    p = torch.exp(sc - m)
    l = p.sum(-1, keepdim=True)
    o = (p @ gather(s.v_cache)) / l
    s.out[layer] = o.reshape(n, s.hq, d).bfloat16()
    s.lse[layer] = (m + torch.log(l)).reshape(n, s.hq)


def _weights(x, temperature):
    """(logits in 32 bits, the weights as whole numbers of 2^-36)."""
    x = x.float()
    x = torch.where(torch.isnan(x), -math.inf, x)
    top = x.amax(-1, keepdim=True)
    f32 = lambda a: torch.tensor(a, dtype=torch.float32, device=x.device)  # noqa: E731
    scale = torch.minimum(f32(LOG2E) / temperature, f32(1e30))[:, None]
    z = torch.where(x == top, 0.0, x - top) * scale
    z = torch.where(z >= -37.0, z, -38.0)
    k = torch.round(z)
    f = z - k
    p = f * EXP2[4] + EXP2[3]
    p = p * f + EXP2[2]
    p = p * f + EXP2[1]
    p = p * f + EXP2[0]
    p = p * f + 1.0
    w = ((p * 2.0 ** 24).long() << 12) >> (-k).long()
    return x, torch.where((z < -37.0) | (x == -math.inf), 0, w)


def _share(total, u):
    """floor(total floor(2^24 u) / 2^24)"""
    a = (u * 2.0 ** 24).long()
    hi, lo = total >> 24, total & (2 ** 24 - 1)
    return hi * a + ((lo * a) >> 24)


def _sample_plain(s):
    n, vocab = s.logits.shape
    greedy = ~(s.temperature > 0)
    x, w = _weights(s.logits, torch.where(greedy, 1.0, s.temperature))
    order = torch.sort(torch.where(w > 0, x, -math.inf), dim=-1, descending=True, stable=True).indices
    ws = w.gather(1, order)
    rank = torch.arange(vocab, device=DEV)
    live = ws > 0
    if s.top_k is not None:
        live &= (rank < s.top_k[:, None]) | (s.top_k[:, None] <= 0)
    live &= (rank < 1) | ~greedy[:, None]
    ws = torch.where(live, ws, 0)
    if s.top_p is not None:
        cum = ws.cumsum(1)
        cut = _share(cum[:, -1:], s.top_p.clamp(0.0, 1.0)[:, None])
        live &= (cum - ws < cut) | (rank < 1) | (s.top_p[:, None] >= 1.0)
    if s.min_p is not None:
        live &= ws >= (s.min_p.clamp(0.0, 1.0)[:, None] * 2.0 ** 36).long()
    keep = torch.zeros_like(live).scatter_(1, order, live)
    w = torch.where(keep, w, 0)
    cum = w.cumsum(1)
    total = cum[:, -1]
    token = (cum > _share(total, s.uniform.clamp(0.0, 1.0 - 2.0 ** -24))[:, None]).int().argmax(1)
    s.token.copy_(torch.where(total > 0, token, -1))
    s.kept.copy_(keep.sum(1))
    mine = w.gather(1, token[:, None])[:, 0].double()
    s.logprob.copy_(torch.log(mine / total.double()))


def _step_plain(s):
    # (the plain form has no use for a plan)
    pos = s.ctx_len[s.row.long()][:, None]
    one = torch.ones(s.n, dtype=torch.int32, device=DEV)
    for layer in range(s.c["layers"]):
        _append_plain(s, layer, s.q[layer], s.k[layer], s.v[layer], s.q_rot, one, pos,
                      table=s.block_table[s.row.long()])
        _attend_plain(s, layer, s.q_rot)
    _sample_plain(s.sampling)


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


def _host(x):
    return x.double().cpu().numpy()


def _turned64(x, weight, pos, s):
    x, w = _host(x), _host(weight)
    x = x / np.sqrt((x ** 2).mean(-1, keepdims=True) + EPS) * w
    return torch.as_tensor(_turn64(x, np.asarray(pos)[..., None], s.base, s.style), device=DEV)


def exact(case, seed):
    c = case
    if c["kind"] == "plan":
        return None  # whole numbers alone
    s = prepare(c, seed)
    if c["kind"] == "sample":
        return {"token": None, "kept": None, "logprob": _logprob64(s)}
    if c["kind"] == "append":
        q = torch.zeros(s.q_out.shape, dtype=torch.float64, device=DEV)
        k, v = s.k_cache.double(), s.v_cache.double()
        for b, m in enumerate(s.count.tolist()):
            p = s.pos[b, :m].cpu().numpy()
            page, at = s.block_table[b].long()[p // PAGE], p % PAGE
            q[b, :m] = _turned64(s.q[b, :m], s.wq, p, s)
            k[0, page, :, at] = _turned64(s.k[b, :m], s.wk, p, s)
            v[0, page, :, at] = s.v[b, :m].double()
        return {"q": q, "k_cache": k, "v_cache": v}
    out = torch.zeros(s.out.shape, dtype=torch.float64, device=DEV)
    lse = torch.zeros(s.lse.shape, dtype=torch.float64, device=DEV)
    G, rt = s.hq // s.hkv, math.sqrt(s.d)
    keys = (s.ctx_len[s.row.long()] + s.pos_offset + 1).tolist()
    k_all, v_all = s.k_cache, s.v_cache
    if c["kind"] == "step":
        k_all, v_all = k_all.double(), v_all.double()
    for layer in range(c.get("layers", 1)):
        if c["kind"] == "step":  # the new position's key and value
            # what the cache and the attention get is rounded to bf16
            q = _turned64(s.q[layer][:, 0], s.wq, np.asarray(keys) - 1, s).bfloat16().double()
            kn = _turned64(s.k[layer][:, 0], s.wk, np.asarray(keys) - 1, s).bfloat16().double()
        else:
            q = s.q.double()
        for e in range(s.n):
            at = torch.arange(keys[e], device=DEV)
            page = s.block_table[int(s.row[e])].long()[at // PAGE]
            if c["kind"] == "step":
                k_all[layer, page[-1], :, at[-1] % PAGE] = kn[e]
                v_all[layer, page[-1], :, at[-1] % PAGE] = s.v[layer][e, 0].double()
            K = k_all[layer, page, :, at % PAGE].transpose(0, 1).double()
            V = v_all[layer, page, :, at % PAGE].transpose(0, 1).double()
            z = q[e].view(s.hkv, G, s.d) @ K.transpose(1, 2) / rt
            lse[layer, e] = torch.logsumexp(z, -1).view(-1)
            out[layer, e] = (torch.softmax(z, -1) @ V).view(s.hq, s.d)
    if c["kind"] == "attend":
        return {"out": out, "lse": lse}
    return {"out": out, "k_cache": k_all, "v_cache": v_all, "token": None, "kept": None,
            "logprob": _logprob64(s.sampling)}


def _logprob64(s):
    """The drawn token's log-probability among the kept ones, from the softmax in 64 bits."""
    n, vocab = s.logits.shape
    got = np.zeros(n)
    host = lambda t, default: np.full(n, default) if t is None else _host(t)  # noqa: E731
    T, K, P, M = host(s.temperature, 1.0), host(s.top_k, 0), host(s.top_p, 1.0), host(s.min_p, 0.0)
    u = np.floor(_host(s.uniform) * 2.0 ** 24) / 2.0 ** 24
    for b in range(n):
        x = s.logits[b].double().cpu().numpy()
        if T[b] <= 0:
            continue  # certain: 0
        order = np.argsort(-x, kind="stable")
        w = np.exp((x[order] - x[order[0]]) / T[b])
        live = w >= 2.0 ** -36
        if K[b] > 0:
            live[int(K[b]):] = False
        w = np.where(live, w, 0.0)
        if P[b] < 1.0:
            before = np.cumsum(w) - w
            live &= before < P[b] * w.sum()
            live[0] = True
        live &= w >= M[b]
        kept = np.zeros(vocab)
        kept[order[live]] = w[live]
        cum = np.cumsum(kept)
        token = min(vocab - 1, int(np.searchsorted(cum, u[b] * cum[-1], side="right")))
        got[b] = np.log(kept[token] / cum[-1])
    return torch.as_tensor(got)
