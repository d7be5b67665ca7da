"""A step of BranchDecoder in which `begin` refuses a row: nothing of that row's reaches the cache,
whose pages other branches may be reading, and the other rows' step is the one they take without it."""
import pytest
import torch

from tests.test_gpu_branches import run, step_inputs
from tests.test_gpu_speculative import linked

pytestmark = pytest.mark.gpu
LAYERS, VOCAB = 2, 700


def decoder():
    """Two contexts, two branches of the first; rows in the order 0, 3, 2, 1."""
    from paper_2607_28069_gb300.pipeline import BranchDecoder
    wl, path = linked(LAYERS, spare=60)
    w = torch.full((64,), 1.5, dtype=torch.bfloat16, device="cuda")
    dec = BranchDecoder(path, rows=5, max_new=64, q_weight=w, k_weight=w)
    dec.fork([0, 0], [2, 3])
    assert dec.in_use == [0, 3, 2, 1]
    return dec


def state(dec):
    """Lengths, and the caches' bits as [layer][page][slot]..."""
    return [dec.ctx_len.clone()] + [c.view(torch.int16).permute(0, 1, 3, 2, 4).clone()
                                    for c in (dec.path.k_cache, dec.path.v_cache)]


@pytest.mark.parametrize("captured", [False, True])
@pytest.mark.parametrize("where", ["first", "middle", "last"])
def test_a_row_cut_inside_a_page_of_others_writes_nothing(cuda_lib, captured, where):
    """Row 2 is taken back to a length inside its context's shared pages."""
    from paper_2607_28069_gb300 import DEVICE_CODES
    got = []
    for cut in (False, True):
        dec = decoder()
        g = torch.Generator(device="cuda").manual_seed(7)
        qkv, logits, u = step_inputs(g, LAYERS, 4, VOCAB)
        full = int(dec.ctx_len[2]) // 16
        if cut:
            dec.ctx_len[2] = {"first": 0, "middle": full // 2 * 16 + 5, "last": full * 16 - 1}[where]
        before = state(dec)
        if captured:
            graph = torch.cuda.CUDAGraph()
            torch.cuda.synchronize()
            with torch.cuda.graph(graph):
                run(dec, LAYERS, qkv, logits, u, 0.8)
            graph.replay()
        else:
            run(dec, LAYERS, qkv, logits, u, 0.8)
        code, detail = cuda_lib.pic_device_status()
        assert (DEVICE_CODES[code], detail) == (("shared page", 2) if cut else ("ok", 0))
        grown = torch.zeros_like(dec.ctx_len)
        grown[[0, 1, 3] if cut else [0, 1, 2, 3]] = 1
        assert torch.equal(dec.ctx_len, before[0] + grown)
        # the slots that the step may write: behind the rows that were given room
        ours = torch.zeros(dec.num_pages, 16, dtype=torch.bool, device="cuda")
        for r in (0, 1, 3) if cut else (0, 1, 2, 3):
            at = int(before[0][r])
            ours[int(dec.block_table[r, at // 16]), at % 16] = True
        for old, new in zip(before[1:], state(dec)[1:]):
            assert torch.equal(old[:, ~ours], new[:, ~ours])
            assert not torch.equal(old[:, ours], new[:, ours])
        keep = [e for e, r in enumerate(dec.in_use) if r != 2]
        largest = dec.path.v_cache.float().abs().max()
        got.append((dec.out[:, keep].float(), dec.token[keep].tolist(), dec.kept[keep].tolist()))
    # The forest of the pages differs, and with it what a row's weights are relative to.  Of each
    # side, as in attention_close: 2^-8 of the output, at most the largest value, and of A, at most
    # that too; and 2 e with e = 2^-15 S + 2^-19, S < 18 by the lengths of the heads (12 for the
    # normed queries and keys, below 12 for the context's keys; their product over 8).
    assert (got[0][0] - got[1][0]).abs().max() <= largest * (2.0 ** -6 + 2.0 ** -8)
    assert got[0][1:] == got[1][1:]


def test_rows_without_room_in_table_or_pool_write_nothing(cuda_lib):
    """No free page for one row, a block table that ends for another."""
    dec = decoder()
    g = torch.Generator(device="cuda").manual_seed(9)
    dec.begin()  # (room for rows 1 and 2)
    at = int(dec.ctx_len[0]) // 16  # row 0 to a page's end, the page behind it given back
    dec.page_refs[int(dec.block_table[0, at])] = 0
    dec.block_table[0, at] = -1
    dec.ctx_len[0] = at * 16
    dec.ctx_len[3] = dec.block_table.shape[1] * 16
    dec.page_refs[dec.page_refs == 0] = 1
    assert cuda_lib.pic_device_status() == (0, 0)
    qkv, logits, u = step_inputs(g, LAYERS, 4, VOCAB)
    before = state(dec)
    run(dec, LAYERS, qkv, logits, u, 0.8)
    assert cuda_lib.pic_device_status()[0] in (5, 10)
    after = state(dec)
    assert (after[0] - before[0]).tolist() == [0, 1, 1, 0, 0]
    ours = torch.zeros(dec.num_pages, 16, dtype=torch.bool, device="cuda")
    for r in (1, 2):
        at = int(before[0][r])
        ours[int(dec.block_table[r, at // 16]), at % 16] = True
    for old, new in zip(before[1:], after[1:]):
        assert torch.equal(old[:, ~ours], new[:, ~ours])
