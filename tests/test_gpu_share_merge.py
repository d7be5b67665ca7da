"""The merge of pic_attend_shared with four warps a row, which calls take whose block table is wide
and whose kv heads and pairs of row tiles are at most two: many parts a row, fewer parts than
warps, none, weights that underflow, infinities and NaN."""
import numpy as np
import pytest
import torch

from tests.test_gpu_share import BF, Pool, attend, i32, make_plan, verify

pytestmark = pytest.mark.gpu
ONE, TWO = 2440, 1224  # pages of a table from which a call of one unit, of two, takes this form
# query heads, kv heads, head dim, entries, pages of the table
FORMS = [(4, 1, 64, 3, ONE), (4, 1, 128, 3, ONE), (8, 1, 128, 36, TWO), (7, 1, 128, 40, TWO), (8, 2, 64, 5, TWO),
         (8, 2, 128, 2, TWO), (14, 2, 128, 9, TWO)]
IDS = ["x".join(map(str, f)) for f in FORMS]


def four_warps(geom, n, pages):
    """The rule of the launch, written again."""
    ept = 128 // (geom.num_q_heads // geom.num_kv_heads)
    units = geom.num_kv_heads * (-(-(-(-n // ept)) // 2))
    return units <= 2 and units * (pages // 8) >= 2 * 152


def setup(pic, form, layers=1):
    hq, hkv, d, n, pages = form
    geom = pic.Geometry(layers, hq, hkv, d, 1e4)
    assert four_warps(geom, n, pages)
    return geom, n, pages


@pytest.mark.parametrize("form", FORMS, ids=IDS)
def test_many_parts_a_row(cuda_lib, form):
    """A context over most of the table, split over all CTAs, and tails of 0 to 5 pages."""
    geom, n, pages = setup(cuda_lib, form, layers=2)
    a = list(range(pages - 40))
    lists = [a[:len(a) - i % 3] + list(range(pages + 8 * i, pages + 8 * i + i % 6)) for i in range(n)]
    pool = Pool(lists, [16 * len(x) - (5 * i) % 16 for i, x in enumerate(lists)], max_pages=pages)
    res = attend(cuda_lib, geom, pool, layer=1, fill=float("nan"), seed=n)
    verify(geom, pool, res, layer=1, some=range(0, n, max(1, n // 5)))
    assert cuda_lib.pic_device_status() == (0, 0)
    again = attend(cuda_lib, geom, pool, layer=1, fill=float("nan"), seed=n)
    assert torch.equal(res[3], again[3]) and torch.equal(res[4], again[4])


@pytest.mark.parametrize("form", FORMS, ids=IDS)
def test_short_rows_in_a_wide_table(cuda_lib, form):
    """None, one, two and a few parts: warps that have nothing to add.  No keys at all, a row
    that is none, a length beyond the table, rows listed twice."""
    geom, n, pages = setup(cuda_lib, form)
    a = list(range(60))
    pool = Pool([a, a[:40] + [70, 71], a[:16] + list(range(80, 120)), a[:1], a], [960, 660, 890, 3, 0], max_pages=pages)
    rows = {0: [0, 1, 2], 1: [4, 3, 0], 2: [0, 0, 4], 3: [3, 3], 4: [4], 5: [9, 0, -1], 6: [2, 1, 0, 3, 4, 0]}
    for row in rows.values():
        row = row[:n] + [row[-1]] * max(0, n - len(row)) if n > 3 else row[:n]
        verify(geom, pool, attend(cuda_lib, geom, pool, row, fill=float("nan")))
    assert cuda_lib.pic_device_status()[0] == 3
    pool.lens[1] = 16 * pages + 1
    verify(geom, pool, attend(cuda_lib, geom, pool, ([0, 1] * n)[:n], fill=float("nan")))
    assert cuda_lib.pic_device_status()[0] == 5


@pytest.mark.parametrize("form", [FORMS[0], FORMS[1], FORMS[5]], ids=[IDS[0], IDS[1], IDS[5]])
def test_weights_that_underflow(cuda_lib, form):
    """Scores of one tile far above all others, in the first part, in a middle and in the last: the
    other parts' weights are 0.  An infinity in their values shows all the same, a part of NaN
    alone as NaN, and neither in a column or head that does not hold it."""
    geom, n, pages = setup(cuda_lib, form)
    shared = pages - 100
    a = list(range(shared))
    lists = [a + list(range(shared + 8 * i, shared + 8 * i + 8)) for i in range(n)]
    pool = Pool(lists, [16 * len(x) - 3 for x in lists], max_pages=pages)
    G = geom.num_q_heads // geom.num_kv_heads
    last = geom.num_kv_heads - 1
    for at in (0, shared // 16 * 8, shared - 8):
        def far(q, kc, vc):
            kc[0, at:at + 8] *= 30
            q *= 4

        verify(geom, pool, attend(cuda_lib, geom, pool, checks=far), some=[0, n - 1])
        other = (at + shared // 2) % shared  # a page of a part half the context away

        def wild(q, kc, vc):
            far(q, kc, vc)
            vc[0, other, last, 3, 5] = float("inf")
            vc[0, shared + 8 * 1, 0, 2, 9] = float("-inf")  # entry 1's own first page

        _, _, _, out, lse, _, _ = attend(cuda_lib, geom, pool, checks=wild)
        bad = {tuple(x) for x in (~torch.isfinite(out.float())).nonzero().tolist()}
        assert bad == ({(e, h, 5) for e in range(n) for h in range(last * G, (last + 1) * G)} |
                       {(1, h, 9) for h in range(G)})
        assert torch.isfinite(lse).all()

        def nans(q, kc, vc):
            far(q, kc, vc)
            kc[0, other // 8 * 8:other // 8 * 8 + 8, last] = float("nan")  # a tile of its own

        _, _, _, out, lse, _, _ = attend(cuda_lib, geom, pool, checks=nans)
        heads = torch.zeros(geom.num_q_heads, dtype=torch.bool, device="cuda")
        heads[last * G:] = True
        assert torch.isnan(out[:, heads].float()).all() and torch.isnan(lse[:, heads]).all()
        assert torch.isfinite(out[:, ~heads].float()).all() and torch.isfinite(lse[:, ~heads]).all()


def test_all_scores_minus_infinity_and_no_lse(cuda_lib):
    """Queries of infinities against keys of one sign: every weight is 0, zeros come out; the call
    without a log-sum-exp gives the same output."""
    pic = cuda_lib
    geom, n, pages = setup(pic, FORMS[1])
    a = list(range(900))
    pool = Pool([a + [900 + i] for i in range(n)], [16 * 901 - 2] * n, max_pages=pages)

    def minus(q, kc, vc):
        kc.abs_().clamp_(min=0.01)
        q[1] = float("-inf")

    q, kc, vc, out, lse, _, _ = attend(pic, geom, pool, checks=minus)
    assert (out[1] == 0).all() and (lse[1] == -float("inf")).all()
    assert torch.isfinite(out.float()).all() and torch.isfinite(lse[[0, 2]]).all()
    plan, bt, n = make_plan(pic, geom, pool)
    without = torch.empty_like(out)
    ws = torch.empty(pic.pic_shared_workspace_size(geom, n), dtype=torch.uint8, device="cuda")
    pic.pic_attend_shared(geom, 0, q, bt, pool.num_pages, kc, vc, plan, without, workspace=ws)
    assert torch.equal(out, without) and pic.pic_device_status() == (0, 0)


def test_a_plan_of_other_sizes_is_refused(cuda_lib):
    pic = cuda_lib
    geom, n, pages = setup(pic, FORMS[0])
    pool = Pool([list(range(40))] * n, [640] * n, max_pages=pages)
    plan, bt, n = make_plan(pic, geom, pool)
    kc = torch.zeros((1, pool.num_pages, 1, 16, 64), **BF)
    wider = i32(np.pad(pool.table, ((0, 0), (0, 1)), constant_values=-1))
    out = torch.full((n, 4, 64), 7.0, **BF)
    ws = torch.empty(pic.pic_shared_workspace_size(geom, n), dtype=torch.uint8, device="cuda")
    pic.pic_attend_shared(geom, 0, torch.zeros_like(out), wider, pool.num_pages, kc, kc, plan, out, workspace=ws)
    assert pic.pic_device_status() == (3, -1) and (out == 7).all()
