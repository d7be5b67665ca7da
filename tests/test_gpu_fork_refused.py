"""DraftDecoder.fork where the pool serves only some of the branches: the others' rows stay
empty and out of use, and the steps that follow leave them alone."""
import numpy as np
import pytest
import torch

from tests.test_gpu_speculative import inputs, linked, step

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("left,served", [(0, [False, False, False]), (2, [True, False, False]),
                                         (4, [True, True, False]), (6, [True, True, True])])
def test_only_served_branches_are_in_use(cuda_lib, left, served):
    from paper_2607_28069_gb300.pipeline import DraftDecoder
    T = 17  # a branch needs two pages: the rest of its last one, and room
    wl, path = linked(1, spare=40)
    dec = DraftDecoder(path, T, rows=5, max_new=64)
    dec.begin()
    for b in range(2):  # contexts that end in the middle of a page
        dec.ctx_len[b] = dec.ctx_len[b] // 16 * 16 - 10
    assert cuda_lib.pic_device_status() == (0, 0)
    free = torch.nonzero(dec.page_refs == 0)[:, 0]
    dec.page_refs[free[left:]] = 1  # pages that something else holds
    ctx = dec.ctx_len.tolist()
    got = dec.fork([0, 1, 0], [3, 2, 4])
    assert got == [ctx[a] if ok else -1 for a, ok in zip([0, 1, 0], served)]
    status = cuda_lib.pic_device_status()
    assert status == (0, 0) if all(served) else status[0] == 10
    live = [0, 1] + [z for z, ok in zip([3, 2, 4], served) if ok]
    assert dec.in_use == sorted(live)
    for z in {2, 3, 4} - set(live):
        assert int(dec.ctx_len[z]) == 0 and bool((dec.block_table[z] == -1).all())
    # a step: room, drafts and acceptance for the rows in use, nothing for the others
    on = np.isin(np.arange(5), live)
    s = inputs(np.random.default_rng(left), 5, T, 1, 30, True, on)
    before = dec.ctx_len.clone()
    step(dec, s, 1)
    assert cuda_lib.pic_device_status() == (0, 0)
    assert torch.equal(dec.ctx_len, before + dec.path_len)
    for z in set(range(5)) - set(live):
        assert int(dec.ctx_len[z]) == 0 and bool((dec.block_table[z] == -1).all())
    if not all(served):  # the rows serve once there are pages again
        dec.page_refs[free[left:]] = 0
        rest = sorted({2, 3, 4} - set(live))
        assert dec.fork([0] * len(rest), rest) == [int(dec.ctx_len[0])] * len(rest)
        assert dec.in_use == [0, 1, 2, 3, 4] and cuda_lib.pic_device_status() == (0, 0)


def test_a_table_too_short(cuda_lib):
    from paper_2607_28069_gb300.pipeline import DraftDecoder
    wl, path = linked(1, spare=40)
    dec = DraftDecoder(path, 4, rows=4, max_new=0)
    dec.ctx_len[0] = dec.block_table.shape[1] * 16 - 1
    dec.block_table[0] = dec.block_table[0].clamp_min(0)
    got = dec.fork([0, 1], [2, 3])
    assert got == [-1, int(dec.ctx_len[1])] and dec.in_use == [0, 1, 3]
    assert cuda_lib.pic_device_status() == (5, 0)
    assert int(dec.ctx_len[2]) == 0 and bool((dec.block_table[2] == -1).all())
