"""Branches that share pages: room for further positions is never given in a page that
another row reads, wherever a row was cut, so an append into the room that was given leaves
the other rows' keys and values as they are."""
import numpy as np
import pytest
import torch

from tests.test_gpu_pages import PAGE, Model

pytestmark = pytest.mark.gpu


def branches(length, spare=0):
    """Row 0 with a context, row 1 its branch."""
    m = Model(4, 40, 120, layers=2, heads=(4, 2), dim=64)
    m.place(0, length, spare)
    m.up()
    m.fork([0], [1])
    m.check()
    return m


def context(m, row):
    """Keys and values of a row's positions, on the device."""
    t = np.arange(int(m.dctx[row]))
    page = m.dbt[row].long().cpu()[t // PAGE]
    return torch.stack([c[:, page, :, t % PAGE] for c in (m.dk, m.dv)]).clone()


def append(m, row, n=3):
    """Room for n tokens behind the row and, whatever came of it, their append."""
    pic, B = m.pic, m.rows
    res = m.i32([77])
    pic.pic_page_reserve(m.i32([row]), n, m.dctx, m.dbt, m.pages, m.drefs, res)
    if res.item() < 0:
        return -1
    q, kv = (torch.full((B, n, h, 64), 9.0, dtype=torch.bfloat16, device="cuda") for h in (4, 2))
    lens = torch.zeros(B, dtype=torch.int32, device="cuda")
    lens[row] = n
    ws = torch.empty(pic.pic_draft_workspace_size(m.geom, B, n), dtype=torch.uint8, device="cuda")
    for layer in range(2):
        pic.pic_attend_draft(m.geom, layer, q, kv, kv, m.dctx, lens, m.dbt, m.pages, m.dk, m.dv,
                             torch.empty_like(q), workspace=ws)
    return res.item()


def compact(m, row, start, keep, reserve=0, width=None):
    """The call alone: the row's new length or -1."""
    lists = np.full((1, width or max(1, len(keep))), -3, np.int64)
    lists[0, :len(keep)] = keep
    res = m.i32([77])
    ws = torch.empty(m.pic.pic_page_compact_workspace_size(m.geom, 1, lists.shape[1]), dtype=torch.uint8,
                     device="cuda")
    m.pic.pic_page_compact(m.geom, m.i32([row]), m.i32(lists), m.i32([len(keep)]), m.dctx, m.dbt, m.pages,
                           m.drefs, m.dk, m.dv, res, start=m.i32([start]), reserve=reserve, workspace=ws)
    return res.item()


WIDTHS = [None, 65, 1500]  # the short form, the long one, two checking CTAs


@pytest.mark.parametrize("width", WIDTHS)
@pytest.mark.parametrize("row", [0, 1])  # the context and its branch
@pytest.mark.parametrize("start,keep,reserve", [(20, 0, 1), (0, 20, 16), (17, 30, 8), (16, 0, 8), (0, 47, 1)])
def test_a_cut_with_room_in_a_shared_page(cuda_lib, row, start, keep, reserve, width):
    """Refused, and the row left as it is."""
    m = branches(64)
    other = context(m, 1 - row)
    assert compact(m, row, start, list(range(keep)), reserve, width) == -1
    assert cuda_lib.pic_device_status() == (9, 0)
    m.check()
    assert append(m, row) == 5
    assert cuda_lib.pic_device_status() == (0, 0)
    assert torch.equal(context(m, 1 - row), other)


@pytest.mark.parametrize("width", WIDTHS)
@pytest.mark.parametrize("row", [0, 1])
@pytest.mark.parametrize("start,keep", [(20, 0), (0, 20), (17, 30)])
def test_a_cut_in_a_shared_page(cuda_lib, row, start, keep, width):
    """Served, but the row gets no room; a branch of it does."""
    m = branches(64)
    other = context(m, 1 - row)
    n = start + keep
    assert compact(m, row, start, list(range(keep)), 0, width) == n
    m.refs[m.bt[row, -(-n // PAGE):4]] -= 1
    m.bt[row, -(-n // PAGE):] = -1
    m.ctx[row] = n
    m.check()
    assert append(m, row) == -1
    assert cuda_lib.pic_device_status() == (9, 0)
    m.check()
    m.fork([row], [3], reserve=3)
    m.free([row])
    m.check()
    assert append(m, 3) == -(-(n + 3) // PAGE)
    assert cuda_lib.pic_device_status() == (0, 0)
    assert torch.equal(context(m, 1 - row), other)


@pytest.mark.parametrize("row", [0, 1])
def test_a_cut_between_shared_pages(cuda_lib, row):
    """A cut at a page's end gives the pages behind back; room comes in new pages."""
    m = branches(64)
    other = context(m, 1 - row)
    m.compact([row], [[]], start=[32])
    m.check()
    assert append(m, row, 20) == 4
    assert cuda_lib.pic_device_status() == (0, 0)
    assert torch.equal(context(m, 1 - row), other)


@pytest.mark.parametrize("length,cut", [(64, 20), (64, 32), (70, 31), (70, 65)])
@pytest.mark.parametrize("row", [0, 1])
def test_a_length_set_by_the_caller(cuda_lib, row, length, cut):
    """A row whose ctx_len was lowered gets no room in a page that another row reads; a branch
    of it does, with its own copy of the last page."""
    m = branches(length)
    shared = cut < 64
    other = context(m, 1 - row)
    m.dctx[row] = m.ctx[row] = cut
    if shared:
        assert append(m, row) == -1
        assert cuda_lib.pic_device_status() == (9, 0)
        m.check()
    assert m.reserve([row], 0) == [-(-cut // PAGE)]
    m.fork([row], [3], reserve=3)
    m.check()
    assert append(m, 3) == -(-(cut + 3) // PAGE)
    assert torch.equal(context(m, 1 - row), other)
    if not shared:
        assert append(m, row) == -(-(cut + 3) // PAGE)
    assert torch.equal(context(m, 1 - row), other)
    assert cuda_lib.pic_device_status() == (0, 0)


def test_reserve_serves_the_rows_beside(cuda_lib):
    m = branches(64)
    m.place(2, 5)
    m.up()
    m.dctx[1] = 20
    res = m.i32([77] * 3)
    m.pic.pic_page_reserve(m.i32([1, 2, 0]), 20, m.dctx, m.dbt, m.pages, m.drefs, res)
    assert res.tolist() == [-1, 2, 6] and cuda_lib.pic_device_status() == (9, 0)
    free = np.flatnonzero(m.refs == 0)
    m.bt[2, 1], m.bt[0, 4:6], m.ctx[1] = free[0], free[1:3], 20
    m.refs[free[:3]] = 1
    m.check()


def test_the_last_user_may_cut_anywhere(cuda_lib):
    for row in (0, 1):
        m = branches(64)
        m.free([1 - row])
        m.compact([row], [list(range(9))], start=[11])
        m.check()
        assert append(m, row) == 2
        assert cuda_lib.pic_device_status() == (0, 0)
