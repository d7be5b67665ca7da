"""Host-side refusals of the speculative-decoding entry points (no GPU): every
argument check comes before anything reaches the device."""
import ctypes

import pytest

import paper_2607_28069_gb300 as pic

FAKE, NULL = ctypes.c_void_p(256), ctypes.c_void_p(0)   # never dereferenced


@pytest.fixture(scope="module")
def lib():
    import os
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


def attend(g, layer=0, batch=2, max_draft=4, q=FAKE, max_pages=4, num_pages=9, ws=FAKE, ws_bytes=1 << 40,
           out=FAKE):
    c = g._c()
    return pic.load().pic_attend_draft(ctypes.byref(c), layer, batch, max_draft, q, FAKE, FAKE, FAKE,
                                       FAKE, NULL, FAKE, max_pages, num_pages, FAKE, FAKE, out, NULL,
                                       ws, ws_bytes, NULL)


def test_attend_draft(lib):
    g = geom()
    for kw, status, text in ((dict(layer=2), 1, "layer 2"), (dict(batch=0), 1, "positive"),
                             (dict(max_draft=65), 2, "max_draft 65"), (dict(q=NULL), 1, "NULL"),
                             (dict(out=ctypes.c_void_p(264)), 1, "16-byte"),
                             (dict(ws=NULL), 4, "workspace needs"), (dict(ws_bytes=100), 4, "workspace needs"),
                             (dict(num_pages=1 << 31), 2, "2^31 rows"),
                             (dict(batch=65536, max_draft=1), 2, "grid too large")):
        assert attend(g, **kw) == status and text in error(), (kw, error())
    assert attend(geom(head_dim=96)) == 2 and "head_dim" in error()
    # the workspace: packed queries of whole 128-row tiles, partial states of 152 CTAs
    size = pic.pic_draft_workspace_size(g, 2, 4)
    assert size >= 2 * 8 * 128 * 128 * 2 + 4 * 152 * 128 * (128 + 2) * 4
    assert pic.pic_draft_workspace_size(g, 2, 64) > size
    assert pic.pic_draft_workspace_size(g, 2, 65) == 0
    assert pic.pic_draft_workspace_size(geom(head_dim=80), 2, 4) == 0


def verify(batch=1, max_draft=4, vocab=10, target=FAKE, draft=NULL, parent=NULL, stride=(40, 10)):
    st = (ctypes.c_int64 * 2)(*stride)
    ds = ctypes.cast(st, ctypes.c_void_p) if draft is not NULL else NULL
    return pic.load().pic_verify_draft(batch, max_draft, vocab, FAKE, parent, FAKE, target,
                                       ctypes.cast(st, ctypes.c_void_p), draft, ds, FAKE, FAKE, FAKE,
                                       FAKE, NULL)


def test_verify_draft(lib):
    for kw, status, text in ((dict(batch=0), 1, "positive"), (dict(vocab=0), 1, "positive"),
                             (dict(max_draft=65), 2, "max_draft 65"),
                             (dict(vocab=(1 << 24) + 1), 2, "vocab 16777217"),
                             (dict(target=NULL), 1, "NULL"), (dict(stride=(-1, 10)), 1, "stride"),
                             (dict(draft=FAKE, parent=FAKE), 1, "needs a chain")):
        assert verify(**kw) == status and text in error(), (kw, error())


def test_pages(lib):
    c = geom()._c()
    g = ctypes.byref(c)

    def reserve(n=1, row=FAKE, extra=1, rows=4, max_pages=4, num_pages=9, res=FAKE):
        return lib.pic_page_reserve(n, row, extra, rows, FAKE, FAKE, max_pages, num_pages, FAKE, res, NULL)

    for kw, status, text in ((dict(n=-1), 1, "-1 rows"), (dict(n=4097), 2, "4097 rows"),
                             (dict(row=NULL), 1, "NULL"), (dict(extra=-3), 1, "extra -3"),
                             (dict(num_pages=0), 1, "positive"), (dict(num_pages=1 << 31), 2, "32 bits"),
                             (dict(n=4096, max_pages=1 << 20), 2, "32 bits"), (dict(res=NULL), 1, "NULL")):
        assert reserve(**kw) == status and text in error(), (kw, error())
    assert reserve(n=0, row=NULL, res=NULL) == 0

    def fork(n=1, reserve=0, lb=0, le=2, src=FAKE, k=FAKE):
        return lib.pic_page_fork(g, n, src, FAKE, reserve, 4, FAKE, FAKE, 4, 9, FAKE, k, FAKE, lb, le,
                                 FAKE, NULL)

    for kw, status, text in ((dict(reserve=-1), 1, "reserve -1"), (dict(lb=1, le=3), 1, "[1, 3)"),
                             (dict(lb=-1), 1, "[-1, 2)"), (dict(src=NULL), 1, "NULL"),
                             (dict(k=ctypes.c_void_p(8)), 1, "16-byte")):
        assert fork(**kw) == status and text in error(), (kw, error())
    assert fork(n=0) == 0

    def compact(n=1, keep=FAKE, max_keep=4, reserve=0, lb=0, le=2, ws=NULL, ws_bytes=0):
        return lib.pic_page_compact(g, n, FAKE, NULL, keep, max_keep, FAKE, reserve, 0, 4, FAKE, FAKE, 4,
                                    9, FAKE, FAKE, FAKE, lb, le, FAKE, ws, ws_bytes, NULL)

    for kw, status, text in ((dict(max_keep=0), 1, "max_keep 0"), (dict(reserve=-1), 1, "reserve -1"),
                             (dict(keep=NULL), 1, "NULL"), (dict(le=0), 1, "no layers"),
                             (dict(max_keep=65), 4, "workspace needs"),
                             (dict(max_keep=65, ws=ctypes.c_void_p(264), ws_bytes=1 << 30), 4, "256-aligned")):
        assert compact(**kw) == status and text in error(), (kw, error())
    assert compact(n=0) == 0
    assert pic.pic_page_compact_workspace_size(geom(), 3, 64) == 0
    assert pic.pic_page_compact_workspace_size(geom(), 3, 65) >= 3 * 65 * 16 + 3 * 2 * 2 * 5 * 4

    def copy(n=1, src=FAKE, sp=9, dp=9, lb=0, le=2):
        return lib.pic_page_copy(g, n, src, FAKE, FAKE, FAKE, sp, FAKE, FAKE, dp, lb, le, NULL)

    for kw, status, text in ((dict(n=-1), 1, "n -1"), (dict(sp=0), 1, "positive"), (dict(src=NULL), 1, "NULL"),
                             (dict(le=3), 1, "[0, 3)")):
        assert copy(**kw) == status and text in error(), (kw, error())
    assert copy(n=0) == 0 and copy(lb=1, le=1) == 0

    def free(n=1, row=FAKE):
        return lib.pic_page_free(n, row, 4, FAKE, FAKE, 4, 9, FAKE, NULL)

    assert free(row=NULL) == 1 and free(n=4097) == 2 and free(n=0) == 0


def test_attend_draft_positions_stay_within_32_bits(lib):
    g = geom(num_q_heads=4, num_kv_heads=1)
    assert attend(g, batch=1, max_pages=(2 ** 31 - 1) // 16 - 15) == 2 and "beyond 32 bits" in error()
    assert attend(g, batch=1, max_pages=2 ** 31 - 1) == 2 and "beyond 32 bits" in error()
