"""Long keep lists of pic_page_compact (several checking CTAs of 1024 entries): rows of
every length beside each other, and lists that are refused for an entry at either side
of a checking CTA's boundary beside rows that are served."""
import numpy as np
import pytest
import torch

from tests.test_gpu_pages import PAGE, Model

pytestmark = pytest.mark.gpu


def call(m, rows, lists, start, lens=None, reserve=0, rotate=False, refused=()):
    """The call and, for the rows that it serves, the plain model; their results."""
    n, width = len(rows), max(len(x) for x in lists)
    keep = np.full((n, width), -7, np.int64)
    for i, x in enumerate(lists):
        keep[i, :len(x)] = x
    lens = [len(x) for x in lists] if lens is None else lens
    res = m.i32([77] * n)
    ws = torch.full((m.pic.pic_page_compact_workspace_size(m.geom, n, width),), 255, dtype=torch.uint8,
                    device="cuda")
    m.pic.pic_page_compact(m.geom, m.i32(rows), m.i32(keep), m.i32(lens), m.dctx, m.dbt, m.pages, m.drefs,
                           m.dk, m.dv, res, workspace=ws, start=m.i32(start), reserve=reserve, rotate=rotate)
    out = []
    for i, r in enumerate(rows):
        if i in refused:
            out.append(-1)
            continue
        old = start[i] + np.asarray(lists[i], np.int64)
        new = start[i] + np.arange(len(old))
        t = m.bt[r]
        for c in (m.k, m.v):
            c[:, t[new // PAGE], :, new % PAGE] = c[:, t[old // PAGE], :, old % PAGE].clone()
        m.ctx[r] = start[i] + len(old)
        cut = -(-(int(m.ctx[r]) + reserve) // PAGE)
        m.refs[t[cut:][t[cut:] >= 0]] -= 1
        t[cut:] = -1
        out.append(int(m.ctx[r]))
    assert res.cpu().tolist() == out
    return out


def some(m, n, of):
    return np.sort(m.rng.choice(of, n, replace=False)).tolist()


@pytest.mark.parametrize("dim,hkv", [(64, 1), (128, 5)])
def test_lists_of_several_checking_ctas(cuda_lib, dim, hkv):
    m = Model(6, 1000, 3800, layers=2, heads=(hkv, hkv), dim=dim)
    for r, n in enumerate([15000, 9500, 2200, 2100, 4000, 3000]):
        m.place(r, n)
    m.up()
    lists = [some(m, 9001, 14900), list(range(9001)), some(m, 2049, 2100), [],
             list(range(1024)) + list(range(1030, 1031)), list(range(7, 1031))]
    call(m, [0, 1, 2, 3, 4, 5], lists, [64, 0, 5, 17, 31, 16], reserve=30)
    m.check()
    call(m, [4, 1], [some(m, 1025, 1040), some(m, 1023, 8000)], [0, 3])  # (the longest: 1025)
    m.check()


# (entry, what stands there instead, the code); 2100 entries: three checking CTAs
BAD = [(at, v, 7) for at in (0, 1023, 1024, 2047, 2048, 2099) for v in (-1, -100, -(1 << 31))]
BAD += [(at, "before", 7) for at in (1, 1023, 1024, 1025, 2099)]  # the same as the entry before
BAD += [(at, "lower", 7) for at in (1023, 1024, 2099)]            # one less than its index
BAD += [(at, 1 << 30, 7) for at in (0, 1023, 1024, 2098)] + [(2099, (1 << 31) - 1, 5), (2099, 4000 * 16, 5)]


@pytest.mark.parametrize("at,value,code", BAD)
@pytest.mark.parametrize("place", [0, 1, 2])
def test_a_bad_list_is_refused_and_its_neighbours_served(cuda_lib, at, value, code, place):
    m = Model(3, 300, 700, layers=2, heads=(2, 2), dim=64, seed=at)
    for r in range(3):
        m.place(r, 3000)
    m.up()
    lists = [some(m, n, 2900) for n in (2100, 2100, 1500)]
    lists[place] = some(m, 2100, 2900)
    lists[place][at] = {"before": lists[place][at - 1], "lower": at - 1}.get(value, value)
    call(m, [2, 0, 1], lists, [20, 40, 33], refused=(place,))
    got = cuda_lib.pic_device_status()
    assert got[1] == place and (got[0] == code or (value == 1 << 30 and got[0] == 5))
    m.check()


@pytest.mark.parametrize("row", [0, 1])
def test_other_refusals_of_long_lists(cuda_lib, row):
    """A length beyond the list's, a start below 0, a row that is none, pages outside the
    cache and pages with another user, behind the first checking CTA."""
    for name, code in (("length", 3), ("start", 3), ("row", 3), ("page", 6), ("shared", 9), ("table", 5)):
        m = Model(5, 400, 900, layers=2, heads=(2, 2), dim=64)
        for r in range(2):
            m.place(r, 4000)
        rows, start = [0, 1], [10, 10]
        lists = [some(m, 2100, 2900), some(m, 2000, 2900)]
        lens = [len(x) for x in lists]
        if name == "length":
            lens[row] = 2101
        elif name == "start":
            start[row] = -1
        elif name == "row":
            rows[row] = 5
        elif name == "table":
            start[row] = 400 * 16 - 1900
        elif name == "shared":
            m.bt[2, 0] = m.bt[row, (10 + 1990) // PAGE]  # of the list's last positions
            m.refs[m.bt[2, 0]] = 2
        elif name == "page":
            m.refs[m.bt[row, 100]] = 0
            m.bt[row, 100] = -1
        m.up()
        call(m, rows, lists, start, lens=lens, refused=(row,))
        assert cuda_lib.pic_device_status() == (code, row), name
        m.check()
