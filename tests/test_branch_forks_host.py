"""Forks that BranchDecoder refuses, on the host: before anything reaches the device, and without
a trace in its state (no GPU: the page calls are replaced by a record of themselves)."""
import os
from types import SimpleNamespace

import pytest
import torch

import paper_2607_28069_gb300 as pic
from paper_2607_28069_gb300 import pipeline


@pytest.fixture
def decoder(monkeypatch):
    if not os.path.exists(pic.lib_path()):
        from paper_2607_28069_gb300.build import build
        build()
    calls = []

    def fork(geom, src, dst, ctx_len, block_table, num_pages, page_refs, k_cache, v_cache, result, reserve=0):
        calls.append((src.tolist(), dst.tolist()))
        result.copy_(ctx_len[src.long()])
        ctx_len[dst.long()] = result

    monkeypatch.setattr(pipeline, "pic_page_fork", fork)
    monkeypatch.setattr(pipeline, "pic_page_free", lambda *a: None)
    table = torch.arange(8, dtype=torch.int32).view(2, 4)
    geom = pic.Geometry(1, 4, 2, 64, 1e4)
    path = SimpleNamespace(
        wl=SimpleNamespace(block_table=table, num_pages=20, spec=SimpleNamespace(page_size=16)), geom=geom, max_ctx=60,
        ctx_len=torch.tensor([50, 60], dtype=torch.int32), k_cache=torch.zeros(1), v_cache=torch.zeros(1))
    return pipeline.BranchDecoder(path, rows=6, max_new=16), calls


@pytest.mark.parametrize("src,dst", [([2], [3]), ([0, 4], [2, 3]), ([0, 2], [2, 3]), ([-1], [2]), ([99], [2])])
def test_a_source_that_is_not_in_use(decoder, src, dst):
    """Never used, a branch that the same call makes, no row at all."""
    dec, calls = decoder
    state = [x.clone() for x in (dec.ctx_len, dec.block_table, dec.page_refs)]
    with pytest.raises(ValueError, match="source"):
        dec.fork(src, dst)
    assert not calls and dec.in_use == [0, 1]
    assert all(torch.equal(a, b) for a, b in zip(state, (dec.ctx_len, dec.block_table, dec.page_refs)))
    assert dec.fork([0], [2]) == [50] and dec.in_use == [0, 2, 1]  # the row serves on


def test_a_released_source(decoder):
    dec, calls = decoder
    dec.fork([0, 0], [2, 3])
    dec.release([0])
    with pytest.raises(ValueError, match="source"):
        dec.fork([0], [4])
    assert len(calls) == 1 and dec.in_use == [3, 2, 1]
    assert dec.fork([2], [0]) == [50] and dec.in_use == [3, 2, 0, 1]


def test_destinations_as_before(decoder):
    dec, calls = decoder
    for src, dst in (([0], [1]), ([0, 0], [2, 2]), ([0], [2, 3])):
        with pytest.raises(ValueError, match="a row of its own"):
            dec.fork(src, dst)
    assert not calls
