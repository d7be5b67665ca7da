"""pic_share_plan and pic_attend_shared: the nodes against their definition, the attention
against 64 bits over forests of every shape."""
import numpy as np
import pytest
import torch

from tests import branch_reference as R

pytestmark = pytest.mark.gpu
BF = dict(dtype=torch.bfloat16, device="cuda")


def i32(x):
    return torch.tensor(np.asarray(x), dtype=torch.int32, device="cuda")


class Pool:
    """Rows of a block table that share pages; a row is [(pages, ...)] given by the test."""

    def __init__(self, lists, lens, max_pages=None, spare=3):
        self.num_pages = max((max(x, default=-1) for x in lists), default=-1) + 1 + spare
        width = max_pages or max(1, max(len(x) for x in lists))
        self.table = np.full((len(lists), width), -1, np.int64)
        for r, x in enumerate(lists):
            self.table[r, :len(x)] = x
        self.lens = list(lens)


def forest(rng, n, depth=3, span=60, tail=30, scatter=True):
    """Rows that share beginnings in a random tree, pages in any order."""
    fresh = iter(range(10 ** 9))
    lists, lens = [], []

    def grow(have, count, level):
        mine = have + [next(fresh) for _ in range(int(rng.integers(0, span)))]
        while count:
            k = int(rng.integers(1, count + 1)) if level < depth else 1
            if k == 1:
                own = mine[:len(mine) - int(rng.integers(0, min(4, len(mine)) + 1))] if rng.random() < 0.3 else list(mine)
                own += [next(fresh) for _ in range(int(rng.integers(0, tail)))]
                lists.append(own)
                lens.append(int(rng.integers(max(0, 16 * len(own) - 40), 16 * len(own) + 1)))
            else:
                grow(mine, k, level + 1)
            count -= k

    grow([], n, 0)
    if scatter:
        total = max((max(x, default=0) for x in lists), default=0) + 1
        perm = rng.permutation(total)
        lists = [[int(perm[i]) for i in x] for x in lists]
    return Pool(lists, lens)


def make_plan(pic, geom, pool, row=None, pos_offset=-1, table=None):
    n = len(row) if row is not None else len(pool.table)
    plan = torch.full((pic.pic_share_plan_size(n) // 4,), 12345, dtype=torch.int32, device="cuda")
    bt = i32(pool.table) if table is None else table
    pic.pic_share_plan(geom, i32(pool.lens), bt, pool.num_pages, plan, row=None if row is None else i32(row),
                       pos_offset=pos_offset)
    torch.cuda.synchronize()
    return plan, bt, n


def expected(pool, row=None, pos_offset=-1):
    row = list(range(len(pool.table))) if row is None else row
    keys = []
    for r in row:
        ok = 0 <= r < len(pool.table) and pool.lens[r] >= 0
        k = pool.lens[r] + pos_offset + 1 if ok else -1
        keys.append(k if ok and 0 <= k <= pool.table.shape[1] * 16 else -1)
    return row, keys, R.plan_nodes(row, keys, pool.table, pool.num_pages)


GEOM = dict(num_layers=1, num_q_heads=8, num_kv_heads=2, head_dim=64, rope_base=1e4)


@pytest.mark.parametrize("seed", range(12))
def test_nodes_of_random_forests(cuda_lib, seed):
    rng = np.random.default_rng(seed)
    n = [1, 2, 3, 5, 9, 17, 33, 64, 100, 150, 31, 200][seed]
    pool = forest(rng, n, depth=1 + seed % 6, span=[20, 60, 100][seed % 3])
    plan, _, _ = make_plan(cuda_lib, cuda_lib.Geometry(**GEOM), pool)
    _, _, want = expected(pool)
    assert (cuda_lib.share_nodes(plan, n).cpu().numpy() == want).all()
    assert cuda_lib.pic_device_status() == (0, 0)


def test_nodes_of_lists_with_repeats_bad_rows_and_lengths(cuda_lib):
    a = list(range(40))
    pool = Pool([a, a[:24] + [50, 51], a, [60] * 9 + [61]], [640, 410, 300, 160])
    for row in ([0, 1, 2, 3], [2, 2, 2], [0, 7, 1, -1, 2], [3, 3, 0, 0], [1]):
        plan, _, n = make_plan(cuda_lib, cuda_lib.Geometry(**GEOM), pool, row)
        _, _, want = expected(pool, row)
        assert (cuda_lib.share_nodes(plan, n).cpu().numpy() == want).all(), row
        assert cuda_lib.pic_device_status()[0] == (3 if 7 in row else 0)
    # lengths: negative, beyond the table, zero keys
    pool.lens = [-1, 16 * 40 + 1, 0, 127]
    plan, _, n = make_plan(cuda_lib, cuda_lib.Geometry(**GEOM), pool)
    _, keys, want = expected(pool)
    assert keys == [-1, -1, 0, 127] and (cuda_lib.share_nodes(plan, n).cpu().numpy() == want).all()
    assert cuda_lib.pic_device_status()[0] in (3, 5)
    # invalid page ids are not shared
    pool = Pool([a, a], [640, 640])
    pool.table[:, 17] = pool.num_pages
    plan, _, n = make_plan(cuda_lib, cuda_lib.Geometry(**GEOM), pool)
    _, _, want = expected(pool)
    assert want[2][3] == 2 and (cuda_lib.share_nodes(plan, n).cpu().numpy() == want).all()


def test_nodes_of_staircases_deeper_than_the_levels(cuda_lib):
    """Entry i shares i tiles more: every boundary is a node above the next."""
    for n in (7, 300):
        a = list(range(8 * n))
        up = [a[:8 * (i + 1)] + [10 ** 6 + i] for i in range(n)]
        for lists in (up, up[::-1], up[::2] + up[1::2][::-1]):
            lists = [[x if x < 10 ** 6 else 8 * n + x - 10 ** 6 for x in y] for y in lists]
            pool = Pool(lists, [16 * len(x) for x in lists])
            plan, _, _ = make_plan(cuda_lib, cuda_lib.Geometry(**GEOM), pool)
            _, _, want = expected(pool)
            assert (cuda_lib.share_nodes(plan, n).cpu().numpy() == want).all()


def test_the_largest_plan(cuda_lib):
    """4096 entries in runs of 64: sizes beyond one round of the plan's threads."""
    a = [list(range(r * 40, r * 40 + 40)) for r in range(64)]
    pool = Pool([a[i // 64][:32] + [2560 + i] for i in range(4096)], [16 * 33 - 5] * 4096)
    plan, _, n = make_plan(cuda_lib, cuda_lib.Geometry(**GEOM), pool)
    got = cuda_lib.share_nodes(plan, n).cpu().numpy()
    inner = got[n:][got[n:, 7] >= 0]
    assert len(inner) == 64 and (inner[:, 1] - inner[:, 0] == 64).all() and (inner[:, 3] == 4).all()
    assert (got[:n, 2] == 4).all() and (got[:n, 3] == 5).all() and (got[:n, 6] == n + got[:n, 0] // 64 * 64).all()
    assert cuda_lib.pic_share_plan_size(4097) == 0


# ---------------------------------------------------------------- attention
def attend(pic, geom, pool, row=None, pos_offset=-1, layer=0, q_scale=1.0, seed=0, fill=None, checks=None):
    g = torch.Generator(device="cuda").manual_seed(seed)
    plan, bt, n = make_plan(pic, geom, pool, row, pos_offset)
    shape = (geom.num_layers, pool.num_pages, geom.num_kv_heads, 16, geom.head_dim)
    kc, vc = (torch.randn(shape, generator=g, device="cuda").bfloat16() for _ in range(2))
    row, keys, _ = expected(pool, row, pos_offset)
    if fill is not None:  # every slot that no entry sees
        seen = torch.zeros((pool.num_pages, 16), dtype=torch.bool, device="cuda")
        for r, k in zip(row, keys):
            for j in range(-(-max(k, 0) // 16)):
                if 0 <= pool.table[r][j] < pool.num_pages:
                    seen[int(pool.table[r][j]), :min(16, k - 16 * j)] = True
        for c in (kc, vc):
            c.permute(0, 1, 3, 2, 4)[:, ~seen] = fill
    q = (torch.randn((n, geom.num_q_heads, geom.head_dim), generator=g, device="cuda") * q_scale).bfloat16()
    if checks:
        checks(q, kc, vc)
    out = torch.full_like(q, 7.0)
    lse = torch.full(q.shape[:2], 7.0, device="cuda")
    ws = torch.full((pic.pic_shared_workspace_size(geom, n),), 255, dtype=torch.uint8, device="cuda")
    pic.pic_attend_shared(geom, layer, q, bt, pool.num_pages, kc, vc, plan, out, lse=lse, workspace=ws)
    torch.cuda.synchronize()
    return q, kc, vc, out, lse, keys, row


def verify(geom, pool, res, layer=0, some=None):
    q, kc, vc, out, lse, keys, row = res
    K, V, Q = kc[layer], vc[layer], R.f64(q)
    out, lse = R.f64(out), R.f64(lse)
    for e in range(len(row)) if some is None else some:
        if keys[e] < 0:
            assert (out[e] == 7).all() and (lse[e] == 7).all()
            continue
        at = np.arange(keys[e])
        page = torch.tensor(pool.table[row[e]][at // 16], device="cuda")
        bad = ((page < 0) | (page >= pool.num_pages)).cpu().numpy()
        sel = page.clamp(0, pool.num_pages - 1), slice(None), torch.tensor(at % 16, device="cuda")
        k, v = R.f64(K[sel]), R.f64(V[sel])
        k[bad], v[bad] = 0, 0
        ref, lse_ref, A, S = R.attention(Q[e], k, v)
        ok, same = R.attention_close(out[e], lse[e], ref, S, A, lse_ref)
        assert ok and same, (e, keys[e], np.abs(out[e] - ref).max(), np.abs(lse[e] - lse_ref).max())


HEADS = [(8, 2, 64), (4, 1, 128), (7, 1, 128), (2, 2, 64), (16, 1, 128), (40, 1, 64), (48, 1, 128), (128, 1, 64), (20, 4, 128)]


@pytest.mark.parametrize("heads", HEADS)
@pytest.mark.parametrize("seed", range(3))
def test_random_forests(cuda_lib, heads, seed):
    rng = np.random.default_rng(100 * seed + heads[0])
    geom = cuda_lib.Geometry(2, *heads, 1e4)
    pool = forest(rng, [3, 12, 40][seed], depth=3, span=50, tail=20)
    res = attend(cuda_lib, geom, pool, layer=1, q_scale=[1.0, 3.0, 1.0][seed], seed=seed, fill=float("nan"))
    verify(geom, pool, res, layer=1)
    assert cuda_lib.pic_device_status() == (0, 0)


@pytest.mark.parametrize("d", [64, 128])
def test_lengths_around_tiles_and_pages(cuda_lib, d):
    geom = cuda_lib.Geometry(1, 4, 1, d, 1e4)
    a = list(range(40))
    lens = [0, 1, 15, 16, 17, 127, 128, 129, 255, 256, 257, 271, 640, 639, 384]
    pool = Pool([a] * len(lens), lens)
    verify(geom, pool, attend(cuda_lib, geom, pool, fill=float("inf")))
    verify(geom, pool, attend(cuda_lib, geom, pool, pos_offset=-1, row=[9, 9, 12, 12, 0, 5]))
    assert cuda_lib.pic_device_status() == (0, 0)
    pool = Pool([a[:3]], [17])
    verify(geom, pool, attend(cuda_lib, geom, pool, pos_offset=0))
    pool = Pool([a[:1], a[:1]], [0, 0])  # the first token: one key
    verify(geom, pool, attend(cuda_lib, geom, pool, pos_offset=0))
    pool = Pool([a[:1], a[:1]], [0, 0])  # no keys at all: no work anywhere
    verify(geom, pool, attend(cuda_lib, geom, pool, pos_offset=-1))


@pytest.mark.parametrize("heads,n,tiles", [((28, 4, 128), 40, 90), ((16, 2, 64), 60, 60), ((32, 8, 128), 3, 150), ((4, 1, 64), 70, 1)])
def test_wide_nodes_split_over_many_ctas(cuda_lib, heads, n, tiles):
    geom = cuda_lib.Geometry(1, *heads, 1e4)
    a = list(range(8 * tiles))
    lists = [a + list(range(8 * tiles + 20 * i, 8 * tiles + 20 * i + 1 + i % 19)) for i in range(n)]
    pool = Pool(lists, [16 * len(x) - i % 16 for i, x in enumerate(lists)])
    res = attend(cuda_lib, geom, pool, fill=float("nan"))
    verify(geom, pool, res, some=range(0, n, max(1, n // 9)))
    assert cuda_lib.pic_device_status() == (0, 0)


@pytest.mark.parametrize("tails", [1, 2, 3, 5])
def test_many_short_entries_in_a_row(cuda_lib, tails):
    """Shares of many units of few tiles each, in runs of equal and of mixed lengths."""
    geom = cuda_lib.Geometry(1, 14, 2, 128, 1e4)
    n, rng = 230, np.random.default_rng(tails)
    lists = [list(range(40 * i, 40 * i + 8 * int(rng.integers(1, tails + 1)))) for i in range(n)]
    pool = Pool(lists, [16 * len(x) - int(rng.integers(0, 100)) for x in lists])
    res = attend(cuda_lib, geom, pool, fill=float("nan"), seed=tails)
    verify(geom, pool, res, some=range(0, n, 11))
    assert cuda_lib.pic_device_status() == (0, 0)


def test_duplicates_bad_rows_and_pages(cuda_lib):
    geom = cuda_lib.Geometry(1, 8, 2, 64, 1e4)
    a = list(range(40))
    pool = Pool([a, a[:24] + [50, 51], a, [60] * 9 + [61]], [640, 410, 300, 160])
    for row in ([2, 2, 2, 2], [0, 9, 1, -1, 2]):
        verify(geom, pool, attend(cuda_lib, geom, pool, row))
    assert cuda_lib.pic_device_status()[0] == 3
    pool.table[1, 3], pool.table[2, 5], pool.table[0, 39] = pool.num_pages, -7, 1 << 30
    verify(geom, pool, attend(cuda_lib, geom, pool))
    assert cuda_lib.pic_device_status()[0] == 6


def test_underflow_and_infinities(cuda_lib):
    """Scores far apart (weights of whole parts underflow); an infinite value shows in the
    entries that see it, and no others."""
    geom = cuda_lib.Geometry(1, 4, 2, 128, 1e4)
    a = list(range(64))
    lists = [a + [64 + i] for i in range(5)]
    pool = Pool(lists, [16 * 65 - 3] * 5)

    def far(q, kc, vc):
        kc[0, 8:16] *= 30
        q *= 4

    verify(geom, pool, attend(cuda_lib, geom, pool, checks=far))

    def wild(q, kc, vc):
        vc[0, 65, 1, 4, 7] = float("inf")     # entry 1's own page
        vc[0, 66, 0, 12, 9] = float("nan")    # entry 2's, the last key's
        kc[0, 67, 1, 2, 3] = float("nan")     # entry 3's

    q, kc, vc, out, lse, keys, _ = attend(cuda_lib, geom, pool, checks=wild)
    fine = torch.isfinite(out.float())
    where = {tuple(x) for x in (~fine).nonzero().tolist()}
    assert where == {(1, h, 7) for h in (2, 3)} | {(2, h, 9) for h in (0, 1)} | {(3, h, i) for h in (2, 3) for i in range(128)}
    assert torch.isfinite(lse).logical_not().nonzero().tolist() == [[3, 2], [3, 3]]
    # a shared one shows in all
    q, kc, vc, out, *_ = attend(cuda_lib, geom, pool, checks=lambda q, k, v: v[0, 3, 0, 0, 5].fill_(float("-inf")))
    assert (~torch.isfinite(out.float())).nonzero().tolist() == [[e, h, 5] for e in range(5) for h in (0, 1)]


def test_other_forms_of_the_same_call(cuda_lib):
    """[n][1][Hq][d] queries, no lse, another stream, a captured graph with new lengths, two graphs
    on one workspace."""
    pic = cuda_lib
    geom = pic.Geometry(1, 8, 2, 64, 1e4)
    rng = np.random.default_rng(3)
    pool = forest(rng, 9, span=40)
    q, kc, vc, out, lse, keys, row = res = attend(pic, geom, pool)
    verify(geom, pool, res)
    bt, ctx = i32(pool.table), i32(pool.lens)
    plan = torch.zeros(pic.pic_share_plan_size(9) // 4, dtype=torch.int32, device="cuda")
    ws = torch.empty(pic.pic_shared_workspace_size(geom, 9), dtype=torch.uint8, device="cuda")
    outs = [torch.zeros((9, 1, 8, 64), **BF) for _ in range(2)]
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    graphs = []
    with torch.cuda.stream(s):
        for o in outs:
            g = torch.cuda.CUDAGraph()
            with torch.cuda.graph(g, stream=s):
                pic.pic_share_plan(geom, ctx, bt, pool.num_pages, plan, pos_offset=-1)
                pic.pic_attend_shared(geom, 0, q.view(9, 1, 8, 64), bt, pool.num_pages, kc, vc, plan, o, workspace=ws)
            graphs.append(g)
        for lens in (pool.lens, [max(0, x - 37 * i) for i, x in enumerate(pool.lens)]):
            ctx.copy_(i32(lens))
            for g in graphs:
                g.replay()
            s.synchronize()
            pool.lens = lens
            _, keys, _ = expected(pool)
            assert torch.equal(outs[0], outs[1])
            verify(geom, pool, (q, kc, vc, outs[0][:, 0], None, keys, row)[:4] + (ref_lse(geom, pool, q, kc, vc, keys), keys, row))


def ref_lse(geom, pool, q, kc, vc, keys):
    lse = np.zeros((len(keys), geom.num_q_heads))
    for e, k in enumerate(keys):
        at = np.arange(k)
        page = torch.tensor(pool.table[e][at // 16], device="cuda")
        sel = page, slice(None), torch.tensor(at % 16, device="cuda")
        lse[e] = R.attention(R.f64(q[e]), R.f64(kc[0][sel]), R.f64(vc[0][sel]))[1]
    return torch.tensor(lse)


def test_a_plan_of_other_sizes_is_refused(cuda_lib):
    pic = cuda_lib
    geom = pic.Geometry(1, 8, 2, 64, 1e4)
    pool = forest(np.random.default_rng(1), 6, span=40)
    plan, bt, n = make_plan(pic, geom, pool)
    other = pic.Geometry(1, 16, 2, 64, 1e4)
    kc = torch.zeros((1, pool.num_pages, 2, 16, 64), **BF)
    for g, table, m in ((other, bt, 6), (geom, bt[:5].contiguous(), 6), (geom, bt[:, :-1].contiguous(), 6), (geom, bt, 5)):
        q = torch.zeros((m, g.num_q_heads, 64), **BF)
        out = torch.full_like(q, 7.0)
        ws = torch.empty(pic.pic_shared_workspace_size(g, m), dtype=torch.uint8, device="cuda")
        pic.pic_attend_shared(g, 0, q, table, pool.num_pages, kc, kc, plan, out, workspace=ws)
        assert pic.pic_device_status() == (3, -1) and (out == 7).all()
    garbage = torch.randint(-2 ** 31, 2 ** 31 - 1, (plan.numel(),), dtype=torch.int32, device="cuda")
    out = torch.full((6, 8, 64), 7.0, **BF)
    ws = torch.empty(pic.pic_shared_workspace_size(geom, 6), dtype=torch.uint8, device="cuda")
    pic.pic_attend_shared(geom, 0, torch.zeros_like(out), bt, pool.num_pages, kc, kc, garbage, out, workspace=ws)
    assert pic.pic_device_status() == (3, -1) and (out == 7).all()


def test_pages_beyond_31_bits_of_elements(cuda_lib):
    pic = cuda_lib
    geom = pic.Geometry(1, 8, 8, 128, 1e4)
    pages = 140000
    kc, vc = (torch.empty((1, pages, 8, 16, 128), **BF) for _ in range(2))
    ids = [pages - 1 - 7 * i for i in range(20)]
    for c in (kc, vc):
        c[0, ids] = torch.randn((20, 8, 16, 128), device="cuda").bfloat16()
    pool = Pool([ids[:16] + [x] for x in ids[16:]], [260, 257, 265, 272], spare=1)
    pool.num_pages = pages
    plan, bt, n = make_plan(pic, geom, pool)
    q = torch.randn((n, 8, 128), device="cuda").bfloat16()
    out, lse = torch.zeros_like(q), torch.zeros((n, 8), device="cuda")
    ws = torch.empty(pic.pic_shared_workspace_size(geom, n), dtype=torch.uint8, device="cuda")
    pic.pic_attend_shared(geom, 0, q, bt, pages, kc, vc, plan, out, lse=lse, workspace=ws)
    torch.cuda.synchronize()
    row, keys, _ = expected(pool)
    verify(geom, pool, (q, kc, vc, out, lse, keys, row))
    assert pic.pic_device_status() == (0, 0)
