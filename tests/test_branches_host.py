"""Host-side refusals of the entry points that decode branches together (no GPU): every argument
check comes before anything reaches the device."""
import ctypes
import os

import pytest
import torch

import paper_2607_28069_gb300 as pic
from tests import branch_reference as R

FAKE, NULL = ctypes.c_void_p(256), ctypes.c_void_p(0)   # never dereferenced


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(pic.lib_path()):
        from paper_2607_28069_gb300.build import build
        build()
    return pic.load()


def geom(**kw):
    g = dict(num_layers=2, num_q_heads=32, num_kv_heads=8, head_dim=128, rope_base=5e5)
    g.update(kw)
    return pic.Geometry(**g)


def error():
    return pic.load().pic_last_error().decode()


def append(g, layer=0, batch=2, tokens=4, q=FAKE, stride=(1024, 256, 128), weight=NULL, eps=1e-6, pos=FAKE, row=NULL,
           ctx=NULL, rows=2, max_pages=4, pages=9, out=FAKE, ws=NULL, ws_bytes=0):
    c, st = g._c(), (ctypes.c_int64 * 3)(*stride)
    return pic.load().pic_append_normed(ctypes.byref(c), layer, batch, tokens, q, st, FAKE, st, FAKE, st, weight, NULL,
                                        eps, NULL, pos, row, ctx, rows, FAKE, max_pages, pages, FAKE, FAKE, out, ws,
                                        ws_bytes, NULL)


def test_append_normed(lib):
    g = geom()
    for kw, status, text in (
            (dict(layer=2), 1, "layer 2"), (dict(batch=0), 1, "positive"), (dict(rows=0), 1, "positive"),
            (dict(q=NULL), 1, "NULL"), (dict(pos=NULL), 1, "neither positions nor lengths"),
            (dict(batch=3), 1, "block table of 2 rows"), (dict(out=NULL), 1, "one of q_out and workspace"),
            (dict(ws=FAKE), 1, "one of q_out and workspace"), (dict(eps=-1.0), 1, "eps"),
            (dict(eps=float("nan")), 1, "eps"), (dict(eps=float("inf")), 1, "eps"),
            (dict(stride=(-8, 0, 0)), 1, "negative stride"), (dict(stride=(1024, 4, 128)), 1, "16 bytes"),
            (dict(weight=ctypes.c_void_p(8)), 1, "16 bytes"), (dict(q=ctypes.c_void_p(264)), 1, "16 bytes"),
            (dict(batch=4097, row=FAKE), 2, "list of 4097 rows"),
            (dict(batch=1 << 20, tokens=1 << 12, rows=1 << 20), 2, "2^31"), (dict(max_pages=1 << 27), 2, "2^31"),
            (dict(out=NULL, ws=FAKE, ws_bytes=64), 4, "workspace needs"),
            (dict(out=NULL, ws=ctypes.c_void_p(64), ws_bytes=1 << 30), 4, "workspace needs")):
        assert append(g, **kw) == status and text in error(), (kw, error())
    assert append(geom(head_dim=96)) == 2 and "head_dim" in error()


def plan(g, n=2, rows=2, row=NULL, ctx=FAKE, max_pages=4, pages=9, buf=FAKE, nbytes=1 << 30):
    c = g._c()
    return pic.load().pic_share_plan(ctypes.byref(c), n, row, rows, ctx, 0, FAKE, max_pages, pages, buf, nbytes, NULL)


def test_share_plan(lib):
    g = geom()
    for kw, status, text in (
            (dict(n=0), 1, "positive"), (dict(n=4097, row=FAKE), 2, "4097"), (dict(n=3), 1, "block table of 2 rows"),
            (dict(ctx=NULL), 1, "NULL"), (dict(max_pages=1 << 27), 2, "32 bits"), (dict(buf=NULL), 4, "plan needs"),
            (dict(nbytes=100), 4, "plan needs"), (dict(buf=ctypes.c_void_p(8)), 4, "plan needs")):
        assert plan(g, **kw) == status and text in error(), (kw, error())
    assert plan(geom(num_q_heads=129, num_kv_heads=1)) == 2 and "129 query heads" in error()
    sizes = [pic.pic_share_plan_size(n) for n in (-1, 0, 1, 2, 4096, 4097)]
    assert sizes[:2] == [0, 0] and sizes[-1] == 0 and 0 < sizes[2] < sizes[3] < sizes[4] and all(x % 16 == 0 for x in sizes)


def attend(g, layer=0, n=2, q=FAKE, rows=2, max_pages=4, pages=9, plan_bytes=1 << 30, buf=FAKE, out=FAKE, ws=FAKE,
           ws_bytes=1 << 40):
    c = g._c()
    return pic.load().pic_attend_shared(ctypes.byref(c), layer, n, q, rows, FAKE, max_pages, pages, FAKE, FAKE, buf,
                                        plan_bytes, out, NULL, ws, ws_bytes, NULL)


def test_attend_shared(lib):
    g = geom()
    for kw, status, text in (
            (dict(layer=-1), 1, "layer -1"), (dict(n=0), 1, "positive"), (dict(n=5000), 2, "5000"),
            (dict(q=NULL), 1, "NULL"), (dict(buf=NULL), 1, "NULL"), (dict(out=ctypes.c_void_p(264)), 1, "16-byte"),
            (dict(pages=1 << 31), 2, "2^31 rows"), (dict(max_pages=1 << 27), 2, "32 bits"),
            (dict(plan_bytes=64), 4, "plan needs"), (dict(ws=NULL), 4, "workspace needs"),
            (dict(ws_bytes=100), 4, "workspace needs"), (dict(ws=ctypes.c_void_p(64)), 4, "workspace needs")):
        assert attend(g, **kw) == status and text in error(), (kw, error())
    assert attend(geom(num_q_heads=129, num_kv_heads=1)) == 2 and "129 query heads" in error()
    assert pic.pic_shared_workspace_size(g, 64) > pic.pic_shared_workspace_size(g, 8) > 0
    assert pic.pic_shared_workspace_size(g, 0) == pic.pic_shared_workspace_size(geom(head_dim=80), 8) == 0


def sample(batch=1, vocab=10, logits=FAKE, bf16=0, stride=10, uniform=FAKE, token=FAKE):
    return pic.load().pic_sample(batch, vocab, logits, bf16, stride, NULL, NULL, NULL, NULL, uniform, token, NULL, NULL,
                                 NULL)


def test_sample(lib):
    for kw, status, text in (
            (dict(batch=0), 1, "positive"), (dict(vocab=0), 1, "positive"), (dict(vocab=(1 << 24) + 1), 2, "vocab"),
            (dict(batch=1 << 28), 2, "batch"), (dict(logits=NULL), 1, "NULL"), (dict(uniform=NULL), 1, "NULL"),
            (dict(token=NULL), 1, "NULL"), (dict(stride=-1), 1, "negative stride"),
            (dict(logits=ctypes.c_void_p(258)), 1, "misaligned"), (dict(logits=ctypes.c_void_p(257), bf16=1), 1, "misaligned")):
        assert sample(**kw) == status and text in error(), (kw, error())


def test_binding_refuses_wrong_tensors(lib):
    g = geom(num_q_heads=4, num_kv_heads=2, head_dim=64)
    x = torch.zeros(2, 1, 4, 64, dtype=torch.bfloat16)
    with pytest.raises(ValueError, match="q must be a CUDA tensor"):
        pic.pic_append_normed(g, 0, x, x, x, None, 9, x, x, x)
    with pytest.raises(ValueError, match="logits must be a CUDA tensor"):
        pic.pic_sample(torch.zeros(2, 10), None, None)
    with pytest.raises(ValueError, match="logits must have two dimensions"):
        pic.pic_sample(torch.zeros(10), None, None)
    with pytest.raises(ValueError, match="ctx_len is required"):
        pic.pic_share_plan(g, None, None, 9, None)


def test_the_reference_of_the_plan():
    """The tests' own definition on a list worked out by hand: 5 entries of 4, 4, 4, 2 and 1 tiles,
    the first two share 3, the next 2, the next 1, the last nothing."""
    import numpy as np
    t = np.full((5, 32), -1)
    t[0] = np.arange(32)
    t[1] = np.r_[t[0][:24], 100:108]
    t[2] = np.r_[t[0][:16], 200:216]
    t[3, :16] = np.r_[t[0][:8], 300:308]
    t[4, :8] = np.arange(400, 408)
    got = R.plan_nodes([0, 1, 2, 3, 4], [512, 511, 512, 256, 100], t, 1000).tolist()
    assert got[5:] == [[0, 2, 2, 3, 0, 384, 6, 2], [0, 3, 1, 2, 0, 256, 7, 1], [0, 4, 0, 1, 0, 128, -1, 0],
                       [0, 0, 0, 0, -1, 0, -1, -1], [0, 0, 0, 0, -1, 0, -1, -1]]
    assert got[:5] == [[0, 1, 3, 4, 0, 512, 5, 3], [1, 2, 3, 4, 1, 511, 5, 3], [2, 3, 2, 4, 2, 512, 6, 2],
                       [3, 4, 1, 2, 3, 256, 7, 1], [4, 5, 0, 1, 4, 100, -1, 0]]


def test_the_reference_of_sampling():
    import math
    x = [0.0, math.log(2.0), math.log(4.0), -100.0]
    assert [R.sample(x, u)[0] for u in (0.0, 0.14, 0.15, 0.42, 0.43, 0.99)] == [0, 0, 1, 1, 2, 2]
    token, kept, lp = R.sample(x, 0.99)
    assert (token, kept) == (2, 3) and abs(lp - math.log(4 / 7)) < 1e-6
    assert R.sample(x, 0.0, k=2)[:2] == (1, 2) and R.sample(x, 0.0, p=0.5)[:2] == (2, 1)
    assert R.sample(x, 0.0, p=0.6)[:2] == (1, 2) and R.sample(x, 0.0, m=0.4)[:2] == (1, 2)
    assert R.sample(x, 0.99, T=0.0)[:2] == (2, 1) and R.sample([-math.inf] * 3, 0.5)[0] == -1
